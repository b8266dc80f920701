"""Plain references of the residual block's operators, on the CPU in 64 bits."""
import numpy as np
import torch

F64 = torch.float64
#: largest value, fraction bits, least exponent of a normal number
FORM = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


def scale_of(most, form):
    """The least 2^e, e >= -127, with most <= largest 2^e; 2^-127 for zeros."""
    largest = FORM[form][0]
    s = torch.exp2(torch.floor(torch.log2(most.clamp(min=1e-300) / largest)))
    s = torch.where(most > largest * s, 2 * s, s)
    s = torch.where(most > largest * s, 2 * s, s)
    s = torch.where(most <= largest * s / 2, s / 2, s)
    return s.clamp(min=2.0 ** -127)


def step_of(v, scale, form):
    """The distance of the format's numbers at v, under a scale."""
    _, bits, least = FORM[form]
    e = torch.floor(torch.log2((v / scale).abs().clamp(min=2.0 ** least)))
    return torch.exp2(e - bits) * scale


def spread(s, k):
    return s.repeat_interleave(128, -1)[..., :k]


def row_scales(x, form):
    k = x.shape[-1]
    pad = torch.zeros(*x.shape[:-1], (k + 127) // 128 * 128, dtype=F64)
    pad[..., :k] = x
    return scale_of(pad.view(*x.shape[:-1], -1, 128).abs().amax(-1), form)


def quantize(x, form):
    """Values (64 bits) and scales; a block with an infinity or NaN is NaN, with the scale of the rest."""
    x = x.to(F64)
    k, bad = x.shape[-1], ~torch.isfinite(x)
    s = row_scales(torch.where(bad, 0, x), form)
    step = step_of(x, spread(s, k), form)
    blocks = torch.stack([bad[..., at:at + 128].any(-1) for at in range(0, k, 128)], -1)
    return torch.where(spread(blocks, k), float("nan"), torch.round(x / step) * step), s


def quantize_weights(w):
    w = w.to(F64)
    g, k, m = w.shape
    out, scales = torch.zeros_like(w), torch.zeros(g, (k + 127) // 128, (m + 127) // 128, dtype=F64)
    for i in range(0, k, 128):
        for j in range(0, m, 128):
            b = w[:, i:i + 128, j:j + 128]
            s = scale_of(b.abs().amax((1, 2)), "e4m3")
            scales[:, i // 128, j // 128] = s
            step = step_of(b, s[:, None, None], "e4m3")
            out[:, i:i + 128, j:j + 128] = torch.round(b / step) * step
    return out, scales


def product(a, w, ids):
    """Rows of a times the matrix of their group, [groups, k, m]; rows of no group give zeros."""
    out = torch.zeros(a.shape[0], w.shape[2], dtype=F64)
    for t in range(w.shape[0]):
        at = (ids == t).nonzero().flatten()
        if len(at):
            out[at] = a[at] @ w[t]
    return out


def outer(a, b, ids, groups):
    out = torch.zeros(groups, a.shape[1], b.shape[1], dtype=F64)
    for t in range(groups):
        at = (ids == t).nonzero().flatten()
        if len(at):
            out[t] = a[at].T @ b[at]
    return out


def group_sum(a, ids, groups):
    return torch.zeros(groups, a.shape[1], dtype=F64).index_add_(
        0, torch.where((ids < 0) | (ids >= groups), 0, ids).long(),
        torch.where(((ids >= 0) & (ids < groups))[:, None], a, 0))


def philox(c, key, rounds=10):
    """Philox4x32 of counters uint64 [.., 4] below 2^32 and a key of two words."""
    low = np.uint64(0xffffffff)
    c = [c[..., i].astype(np.uint64) for i in range(4)]
    k = [np.uint64(key[0]), np.uint64(key[1])]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return np.stack(c, -1)


def keep_mask(n, k, p, seed, offset):
    offset %= 2 ** 64
    c = np.zeros((n, (k + 3) // 4, 4), dtype=np.uint64)
    c[..., 0] = np.arange((k + 3) // 4)
    c[..., 1] = np.arange(n)[:, None]
    c[..., 2], c[..., 3] = offset % 2 ** 32, offset // 2 ** 32
    u = philox(c, (seed % 2 ** 32, seed // 2 ** 32)).reshape(n, -1)[:, :k]
    return torch.tensor(u >= np.uint64(int(np.floor(p * 2.0 ** 32 + 0.5))))
