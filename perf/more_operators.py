"""The operators of a residual block of an energy head in 8 bits, as measurable cases.

  norm          ``rms_norm``: residual's addition and root-mean-square norm, gains of each type
  norm8         the same, its output in 8 bits with a scale for each block of 128
  norm_back     ``rms_norm_backward``: gradients of the rows and of the gains
  quantize      ``quantize_rows`` or ``quantize_weights``, and the values they stand for
  layer8        ``grouped_linear8``: a layer of 8-bit rows and weights of each element type
  layer8_back   ``grouped_linear8_backward``: its gradients of input, weights and bias
  dropout       ``dropout``: a mask from a counter-based generator, with the residual's addition

Rows are atoms; a row's group is its element type, of 118.  ``kind`` says how many types a
frame holds and how evenly: "one" (a crystal), "few" (a five-component alloy or a liquid,
unevenly), "all" (a batch of many small frames over the whole periodic table); a few rows in
a thousand are padding (no type).  Widths are those of the DPA4C variants, descriptors of 70 to
557 entries and MLP widths of 96 to 384, and up to 1,024 for wider heads.

``own`` selects the framework's calls; otherwise the operators run in elementary torch operations
in 32 bits, in 64 where a value is rounded to 8 bits.  ``exact`` is the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = 118
BLOCK = 128
EPS = 1e-6
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
#: largest value as (mantissa in [0.5, 1), exponent); fraction bits; least exponent
FORM = {"e4m3": (0.875, 9, 3, -6), "e5m2": (0.875, 16, 2, -14)}


def rows_case(name, op, rows, k, kind, dtype, **more):
    return dict({"name": name, "op": op, "rows": rows, "k": k, "groups": TYPES, "kind": kind,
                 "dtype": dtype}, **more)


def listed():
    return [
        # serving: the norm of the small model's descriptors of the 108-atom cell, latency
        rows_case("norm_108", "norm", 108, 144, "few", "fp32", residual=False),
        # the residual stream of a million atoms of an alloy, its norm for an 8-bit layer
        rows_case("norm8_1m", "norm8", 1000188, 384, "few", "bf16", residual=True, format="e4m3"),
        # a training step on a small frame of the alloy
        rows_case("norm_back_4000", "norm_back", 4000, 384, "few", "fp32", residual=True),
        # the gradients of a million descriptors' norm
        rows_case("norm_back_1m", "norm_back", 1000188, 541, "few", "bf16", residual=False),
        # a million descriptors to 8 bits and back
        rows_case("quantize_rows_1m", "quantize", 1000188, 541, "few", "bf16", what="rows",
                  format="e4m3"),
        # the descriptor layer's weights of every type, after an update
        rows_case("quantize_weights", "quantize", 0, 541, "all", "fp32", n=384, what="weights",
                  format="e4m3"),
        # serving: a layer of the small model for the 108-atom cell, latency
        rows_case("layer8_108", "layer8", 108, 144, "few", "bf16", n=192, silu=True,
                  residual=False, format="e4m3"),
        # the descriptor's layer on a million atoms of an alloy, with what its gradients need
        rows_case("layer8_1m", "layer8", 1000188, 541, "few", "bf16", n=384, silu=True,
                  residual=False, format="e4m3"),
        # the descriptor's layer of a training batch over the whole periodic table
        rows_case("layer8_back_31250", "layer8_back", 31250, 541, "all", "bf16", n=384, silu=True,
                  format="e4m3"),
        # a hidden layer of a wide head, where the products weigh most
        rows_case("layer8_back_wide", "layer8_back", 65536, 1024, "few", "bf16", n=1024, silu=True,
                  format="e4m3"),
        # a training step's dropout on a small frame
        rows_case("dropout_4000", "dropout", 4000, 384, "few", "fp32", residual=True, p=0.1),
        # a million atoms, joined to the residual stream
        rows_case("dropout_1m", "dropout", 1000188, 384, "few", "bf16", residual=True, p=0.1),
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5))))))

    op = rng.choice(("norm", "norm8", "norm_back", "quantize", "layer8", "layer8", "layer8_back",
                     "layer8_back", "dropout"))
    half = op in ("layer8", "layer8_back")
    c = rows_case("", op, 0, size(8, 1024 if half else 557), rng.choice(("one", "few", "all")),
                  rng.choice(("bf16", "fp16") if half else ("fp32", "bf16", "fp16")),
                  groups=size(1, TYPES))
    # no more than the largest listed case of the kind: entries, or products
    most = {"norm8": 384, "quantize": 541, "dropout": 384}.get(op, 541) * 1000188 // c["k"]
    if op == "quantize":
        c["what"] = rng.choice(("rows", "weights"))
        if c["what"] == "weights":
            c["n"], most = size(8, 1024), 1
    if half:
        c["n"], c["silu"] = size(8, 1024), rng.random() < 0.7
        most = int(2e11 if op == "layer8" else 6.8e10) // (c["k"] * c["n"])
    if op in ("norm", "norm8", "norm_back", "layer8", "dropout"):
        c["residual"] = rng.random() < 0.5
    if op in ("norm8", "quantize", "layer8", "layer8_back"):
        c["format"] = "e4m3" if c.get("what") == "weights" else rng.choice(("e4m3", "e4m3", "e5m2"))
    if op == "dropout":
        c["p"] = round(rng.uniform(0.01, 0.6), 3)
    c["rows"] = 0 if c.get("what") == "weights" else size(1, min(most, 1000188))
    over = work(c)["bytes"] / 3.2e9   # nor bytes
    if over > 1:
        c["rows"] = int(c["rows"] / over)
    del c["name"]
    return c


# ----------------------------------------------------------------------------------- inputs

def types_of(case, g):
    """Element type of every row: int64 [rows]; ``groups`` is padding."""
    n, groups, kind = case["rows"], case["groups"], case["kind"]
    u = torch.rand(n, generator=g, device="cuda")
    if kind == "all":
        t = (u * groups).long().clamp_(max=groups - 1)
    else:
        present = torch.randperm(groups, generator=g, device="cuda")[:1 if kind == "one" else 5]
        m = present.numel()
        t = present[(u * u * m).long().clamp_(max=m - 1)]   # uneven: the first types hold most
    if n > 1000:
        t = torch.where(torch.rand(n, generator=g, device="cuda") < 0.002, groups, t)
    return t


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def padded(q, to):
    """``q`` [.., k] as a view of rows whose starts are multiples of ``to`` bytes."""
    k = q.shape[-1]
    full = torch.zeros(*q.shape[:-1], (k + to - 1) // to * to, dtype=torch.uint8, device=q.device)
    full[..., :k] = q.view(torch.uint8)
    return full.view(q.dtype)[..., :k]


def in_pieces(fn, x, rows=1 << 17):
    """``fn`` of the rows in turn; it returns a tuple of tensors."""
    parts = [fn(x[at:at + rows]) for at in range(0, max(1, x.shape[0]), rows)]
    return tuple(torch.cat(p) for p in zip(*parts))


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 11)
    op, k, rows, groups, dt = case["op"], case["k"], case["rows"], case["groups"], DT[case["dtype"]]
    state = {"op": op, "dtype": dt, "format": case.get("format")}
    if op == "quantize":
        state["what"] = case["what"]
        if case["what"] == "weights":
            state["w"] = (normal(g, groups, k, case["n"]) * k ** -0.5).to(dt)
            return state
    if op == "dropout":
        state["p"], state["seed"], state["offset"] = case["p"], 0x9e3779b97f4a7c15 ^ int(seed), int(seed) + 5
    else:
        # what a program keeps with its frames: the rows by type
        types = types_of(case, g)
        count = torch.bincount(types, minlength=groups + 1)[:groups]
        ptr = torch.zeros(groups + 1, dtype=torch.int64, device="cuda")
        ptr[1:] = count.cumsum(0)
        state["types"], state["ptr"], state["sizes"] = types, ptr, count.tolist()
        state["order"] = torch.argsort(types, stable=True).to(torch.int32)
    # descriptors are calibrated to order one, entry by entry, with outliers
    x = normal(g, rows, k).mul_(torch.exp(0.5 * normal(g, k))).to(dt)
    if case.get("residual"):
        state["res"] = normal(g, rows, case["n"] if op == "layer8" else k).to(dt)
    if op == "layer8" or op == "layer8_back":
        # rows in 8 bits, as the norm before the layer leaves them, and the weights as laid out
        # once for serving or once after an update
        n = case["n"]
        q, s = in_pieces(lambda part: quantize_plain(part, case["format"]), x)
        state["x8"] = padded(q, 16), padded(s, 4)
        w = (normal(g, groups, k, n) * k ** -0.5).to(dt)
        if own:
            import paper_2608_19041_amd as dp
            state["x8"] = dp.Rows8(*state["x8"])
            state["w8"] = dp.quantize_weights(w, backward=op == "layer8_back")
        else:
            state["w8"] = quantize_weights_plain(w)
        state["b"], state["silu"] = (normal(g, groups, n) * 0.1).to(dt), case["silu"]
        if op == "layer8_back":
            state["z"] = normal(g, rows, n).to(dt) if case["silu"] else None
            # gradients of a mean over atoms: small, and of another size from atom to atom
            state["dy"] = normal(g, rows, n).mul_(torch.exp(normal(g, rows, 1)) * 1e-3).to(dt)
        return state
    state["x"] = x
    if op in ("norm", "norm8", "norm_back"):
        state["gain"] = (1 + 0.1 * normal(g, groups, k)).to(dt)
    if op == "norm_back":
        state["rstd"] = 1 / (x.double().square().mean(1) + EPS).sqrt()
        state["rstd"] = torch.where(types < groups, state["rstd"], 0.0).float()
        state["dy"] = normal(g, rows, k).mul_(torch.exp(normal(g, rows, 1)) * 1e-3).to(dt)
    return state


# ------------------------------------------------------------------------------ the plain form

def exponents(most, form):
    """The least e with most <= largest 2^e; 0 for a block of zeros."""
    mantissa, top = FORM[form][:2]
    m, e = torch.frexp(most)
    e = e - top + (m > mantissa).to(e.dtype)
    return torch.where(most > 0, e.clamp(-127, 127), 0)


def blocks_of(x):
    """[.., k] as [.., blocks, 128], padded with zeros."""
    k = x.shape[-1]
    full = x.new_zeros(*x.shape[:-1], (k + BLOCK - 1) // BLOCK * BLOCK)
    full[..., :k] = x
    return full.view(*x.shape[:-1], -1, BLOCK)


def quantize_plain(x, form):
    """8-bit values [.., k] and scale bytes [.., blocks], of float32 or float64 rows."""
    x = x if x.dtype == torch.float64 else x.float()
    b = blocks_of(x)
    e = exponents(b.abs().amax(-1), form)
    q = torch.ldexp(b, -e[..., None]).flatten(-2)[..., :x.shape[-1]]
    if x.dtype == torch.float64:
        # to 24 bits by truncation with a sticky last bit, which no rounding to 8 bits can see
        m, f = torch.frexp(q)
        m = m * 2.0 ** 24
        t = m.trunc()
        q = torch.ldexp(t + torch.where((m != t) & (t.remainder(2) == 0), m.sign(), 0), f - 24)
    return q.float().to(F8[form]).contiguous(), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def values_of(q, s):
    """What 8-bit rows stand for, in float32."""
    scale = torch.repeat_interleave(s.float(), BLOCK, dim=-1)[..., :q.shape[-1]]
    return q.float() * scale


def quantize_weights_plain(w):
    g, k, n = w.shape
    kb, nb = (k + BLOCK - 1) // BLOCK, (n + BLOCK - 1) // BLOCK
    full = w.new_zeros(g, kb * BLOCK, nb * BLOCK, dtype=torch.float32)
    full[:, :k, :n] = w
    b = full.view(g, kb, BLOCK, nb, BLOCK)
    e = exponents(b.abs().amax((2, 4)), "e4m3")
    q = torch.ldexp(b, -e[:, :, None, :, None]).view(g, kb * BLOCK, nb * BLOCK)[:, :k, :n]
    return q.to(F8["e4m3"]), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def weight_values(w8):
    q, s = w8
    scale = s.float().repeat_interleave(BLOCK, 1)[:, :q.shape[1]].repeat_interleave(BLOCK, 2)[:, :, :q.shape[2]]
    return q.float() * scale


def grouped_product(a, b, sizes):
    """Rows of ``a`` (in group order) times the matrix of their group, ``b`` [G, k, n]."""
    live = [i for i, s in enumerate(sizes) if s]
    most = max((sizes[i] for i in live), default=0)
    if len(live) > 4 and most * len(live) <= 2 * a.shape[0]:
        where = places(sizes, live, most, a.device)
        pad = a.new_zeros(len(live) * most, a.shape[1])
        pad[where] = a
        full = torch.bmm(pad.view(len(live), most, -1), b[live])
        return full.view(len(live) * most, -1)[where]
    out = a.new_empty(a.shape[0], b.shape[2])
    at = 0
    for i in live:
        torch.mm(a[at:at + sizes[i]], b[i], out=out[at:at + sizes[i]])
        at += sizes[i]
    return out


def places(sizes, live, most, device):
    n = torch.tensor([sizes[i] for i in live], device=device)
    first = torch.arange(len(live), device=device) * most - (n.cumsum(0) - n)
    total = sum(sizes)
    return torch.arange(total, device=device) + torch.repeat_interleave(first, n, output_size=total)


def grouped_outer(a, b, sizes):
    """sums over each group's rows of a^T b, [G, k, n], and of b, [G, n]."""
    out = a.new_zeros(len(sizes), a.shape[1], b.shape[1])
    total = a.new_zeros(len(sizes), b.shape[1])
    at = 0
    for i, s in enumerate(sizes):
        if s:
            torch.mm(a[at:at + s].t(), b[at:at + s], out=out[i])
            torch.sum(b[at:at + s], 0, out=total[i])
            at += s
    return out, total


def plain_norm(s):
    x, types, groups = s["x"], s["types"], s["gain"].shape[0]
    wide = torch.float64 if s["op"] == "norm8" else torch.float32
    gain = torch.cat([s["gain"], s["gain"].new_zeros(1, x.shape[1])])
    out = {}
    if "res" in s:
        out["h"] = (x.float() + s["res"].float()).to(x.dtype)

    def norm(at):
        h = x[at].to(wide)
        if "res" in s:
            h = h + s["res"][at].to(wide)
        r = 1 / torch.sqrt((h * h).mean(1) + EPS)
        r = torch.where(types[at] < groups, r, 0.0)
        y = h * r[:, None] * gain[types[at]].to(wide)
        if s["op"] == "norm8":
            y = values_of(*quantize_plain(y, s["format"]))
        return y.to(x.dtype), r.float()

    out["y"], out["rstd"] = in_pieces(norm, torch.arange(x.shape[0], device=x.device))
    return out


def plain_norm_back(s):
    x, types, k = s["x"], s["types"], s["x"].shape[1]
    groups = s["gain"].shape[0]
    gain = torch.cat([s["gain"], s["gain"].new_zeros(1, k)]).float()
    h, dy, r = x.float(), s["dy"].float(), s["rstd"][:, None]
    hat = h * r
    dh = dy * gain[types]
    dx = r * (dh - hat * (dh * hat).mean(1, keepdim=True))
    if "res" in s:
        dx = dx + s["res"].float()
    at = s["order"].long()[:sum(s["sizes"])]
    terms = (dy * hat)[at]
    dgain = terms.new_zeros(groups, k)
    start = 0
    for t, n in enumerate(s["sizes"]):
        if n:
            dgain[t] = terms[start:start + n].sum(0)
            start += n
    return {"dx": dx.to(x.dtype), "dgain": dgain.to(x.dtype)}


def plain_layer(s):
    total, dt = sum(s["sizes"]), s["dtype"]
    at = s["order"].long()[:total]
    q, scale = s["x8"]
    xs = values_of(q[at], scale[at])
    z = grouped_product(xs, weight_values(s["w8"]), s["sizes"])
    z += s["b"].float()[s["types"][at]]
    y = z * (1 / (1 + torch.exp(-z))) if s["silu"] else z
    if "res" in s:
        y = y + s["res"][at].float()
    out = torch.zeros(q.shape[0], z.shape[1], dtype=dt, device=z.device)
    out[at] = y.to(dt)
    if not s["silu"]:
        return {"y": out}
    pre = torch.zeros_like(out)
    pre[at] = z.to(dt)
    return {"y": out, "z": pre}


def plain_layer_back(s):
    total, dt = sum(s["sizes"]), s["dtype"]
    at = s["order"].long()[:total]
    q, scale = s["x8"]
    xs = values_of(q[at], scale[at])
    dz = s["dy"][at].double()
    if s["silu"]:
        z = s["z"][at].double()
        p = 1 / (1 + torch.exp(-z))
        dz = dz * (p * (1 + z * (1 - p)))
    dz8 = values_of(*in_pieces(lambda part: quantize_plain(part, s["format"]), dz))
    dx = torch.zeros(q.shape, dtype=dt, device=dz.device)
    dx[at] = grouped_product(dz8, weight_values(s["w8"]).transpose(1, 2).contiguous(), s["sizes"]).to(dt)
    dw, db = grouped_outer(xs, dz.float(), s["sizes"])
    return {"dx": dx, "dw": dw.to(dt), "db": db.to(dt)}


def philox_plain(rows, calls, seed, offset, device):
    """Philox4x32-10 (J. Salmon et al., 2011) of counters (call, row, offset): [rows, calls, 4]."""
    low = 0xffffffff
    c = [torch.arange(calls, device=device).expand(rows, calls),
         torch.arange(rows, device=device)[:, None].expand(rows, calls),
         torch.full((1, 1), offset & low, device=device).expand(rows, calls),
         torch.full((1, 1), offset >> 32 & low, device=device).expand(rows, calls)]
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57   # of 64 bits, wrapped: the bits are right
        c = [(b >> 32 & low) ^ c[1] ^ k0, b & low, (a >> 32 & low) ^ c[3] ^ k1, a & low]
        k0, k1 = k0 + 0x9E3779B9 & low, k1 + 0xBB67AE85 & low
    return torch.stack(c, -1)


def plain_dropout(s):
    x = s["x"]
    n, k = x.shape
    u = philox_plain(n, (k + 3) // 4, s["seed"], s["offset"], x.device).view(n, -1)[:, :k]
    y = torch.where(u >= int(s["p"] * 2.0 ** 32 + 0.5), x.float() * (1 / (1 - s["p"])), 0.0)
    if "res" in s:
        y = y + s["res"].float()
    return y.to(x.dtype)


def plain(s):
    op = s["op"]
    if op in ("norm", "norm8"):
        return plain_norm(s)
    if op == "norm_back":
        return plain_norm_back(s)
    if op == "quantize":
        if s["what"] == "weights":
            return weight_values(quantize_weights_plain(s["w"]))
        return values_of(*quantize_plain(s["x"], s["format"])).to(s["x"].dtype)
    if op == "layer8":
        return plain_layer(s)
    if op == "layer8_back":
        return plain_layer_back(s)
    return plain_dropout(s)


# ------------------------------------------------------------------------- the framework's calls

def run(state):
    if not own:
        return plain(state)
    import paper_2608_19041_amd as dp
    s, op = state, state["op"]
    if op in ("norm", "norm8"):
        got = dp.rms_norm(s["x"], s["gain"], s["ptr"], s["order"], residual=s.get("res"), eps=EPS,
                          quantize=s["format"])
        out = {"y": got[0] if op == "norm" else dp.dequantize(got[0], s["dtype"]), "rstd": got[1]}
        if "res" in s:
            out["h"] = got[2]
        return out
    if op == "norm_back":
        dx, dgain = dp.rms_norm_backward(s["dy"], s["x"], s["gain"], s["rstd"], s["ptr"], s["order"],
                                         dh=s.get("res"))
        return {"dx": dx, "dgain": dgain}
    if op == "quantize":
        if s["what"] == "weights":
            return dp.dequantize(dp.quantize_weights(s["w"]), torch.float32)
        return dp.dequantize(dp.quantize_rows(s["x"], s["format"]), s["dtype"])
    if op == "layer8":
        got = dp.grouped_linear8(s["x8"], s["w8"], s["ptr"], s["order"], bias=s["b"],
                                 activation="silu" if s["silu"] else None, residual=s.get("res"),
                                 preact=s["silu"], dtype=s["dtype"])
        return {"y": got[0], "z": got[1]} if s["silu"] else {"y": got}
    if op == "layer8_back":
        dx, dw, db = dp.grouped_linear8_backward(s["dy"], s["x8"], s["w8"], s["ptr"], s["order"],
                                                 preact=s["z"], format=s["format"])
        return {"dx": dx, "dw": dw, "db": db}
    return dp.dropout(s["x"], s["p"], s["seed"], s["offset"], residual=s.get("res"))


# ------------------------------------------------------------------------------------- the work

def live_groups(case):
    return min({"one": 1, "few": 5, "all": case["groups"]}[case["kind"]], case["groups"], case["rows"])


def work(case):
    op, n, k, groups = case["op"], case["rows"], case["k"], case["groups"]
    size, live = 4 if case["dtype"] == "fp32" else 2, live_groups(case)
    kb = (k + BLOCK - 1) // BLOCK
    res = 1 if case.get("residual") else 0
    if op in ("norm", "norm8"):
        # the output as it is returned; a residual is read and the sum written
        return {"bytes": n * (k * size * (2 + 2 * res) + 8) + live * k * size, "flops": 4 * n * k}
    if op == "norm_back":
        return {"bytes": n * (k * size * (3 + res) + 8) + (live + groups) * k * size, "flops": 8 * n * k}
    if op == "quantize":
        # read, and the values written
        if case["what"] == "weights":
            return {"bytes": groups * k * case["n"] * (size + 4), "flops": 0}
        return {"bytes": n * k * 2 * size, "flops": 0}
    if op == "dropout":
        # ten rounds of two products and four exclusive ors for four entries
        return {"bytes": n * k * size * (2 + res), "flops": n * k * 17}
    m = case["n"]
    weights = live * (k * m + 2 * m)
    if op == "layer8":
        wide = n * (k + kb + m * 2 * ((2 if case["silu"] else 1) + res))
        return {"bytes": wide + weights + 4 * n, "flops": 2 * n * k * m}
    wide = n * (k + kb + 2 * k + m * 2 * (2 if case["silu"] else 1))
    return {"bytes": wide + weights + groups * (k + 1) * m * 2 + 4 * n, "flops": 4 * n * k * m}


# ----------------------------------------------------------------------------- 64 bits, for ab

def exact(case, seed):
    global own
    kept, own = own, False   # the weights in the plain layout
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    f64, op = torch.float64, case["op"]

    def round8(v, form):
        """Blocks of 128 along the last axis, by the grid of the format's numbers."""
        mantissa, top, bits, least = FORM[form]
        out = torch.empty_like(v)
        for at in range(0, v.shape[-1], BLOCK):
            b = v[..., at:at + BLOCK]
            out[..., at:at + BLOCK] = on_grid(b, b.abs().amax(-1, keepdim=True), mantissa * 2.0 ** top, bits, least)
        return out

    def on_grid(b, most, largest, bits, least):
        scale = torch.exp2(torch.ceil(torch.log2(torch.where(most > 0, most / largest, 1.0))))
        scale = torch.where(most > largest * scale, 2 * scale, torch.where(most <= largest * scale / 2, scale / 2, scale))
        scale = torch.where(most > 0, scale, 1.0)
        u = b / scale
        p = torch.exp2(torch.floor(torch.log2(u.abs().clamp(min=2.0 ** least))) - bits)
        return torch.round(u / p) * p * scale

    if op in ("norm", "norm8"):
        x, types = s["x"], s["types"]
        out = {"rstd": torch.zeros(x.shape[0], dtype=f64, device=x.device),
               "y": torch.zeros(x.shape, dtype=f64, device=x.device)}
        h = x.to(f64) + (s["res"].to(f64) if "res" in s else 0)
        for t in range(case["groups"]):
            at = (types == t).nonzero().flatten()
            if at.numel():
                r = torch.rsqrt(torch.linalg.vector_norm(h[at], dim=1) ** 2 / case["k"] + EPS)
                y = s["gain"][t].to(f64) * h[at] * r[:, None]
                out["rstd"][at] = r
                out["y"][at] = round8(y, case["format"]) if op == "norm8" else y
        if "res" in s:
            out["h"] = h
        return out
    if op == "norm_back":
        x, types, k = s["x"], s["types"], case["k"]
        dx = s["res"].to(f64) if "res" in s else torch.zeros(x.shape, dtype=f64, device=x.device)
        dgain = torch.zeros(s["gain"].shape, dtype=f64, device=x.device)
        for t in range(case["groups"]):
            at = (types == t).nonzero().flatten()
            if at.numel():
                h, dy, r = x[at].to(f64), s["dy"][at].to(f64), s["rstd"][at].to(f64)[:, None]
                dgain[t] = torch.einsum("rc,rc->c", dy, h * r)
                up = dy * s["gain"][t].to(f64)
                inner = torch.einsum("rc,rc->r", up, h)[:, None]
                dx[at] += up * r - h * inner * r ** 3 / k
        return {"dx": dx, "dgain": dgain}
    if op == "quantize":
        if case["what"] == "rows":
            return torch.cat([round8(p.to(f64), case["format"]) for p in s["x"].split(1 << 17)])
        w, out = s["w"].to(f64), torch.empty(s["w"].shape, dtype=f64, device=s["w"].device)
        mantissa, top, bits, least = FORM["e4m3"]
        for i in range(0, w.shape[1], BLOCK):
            for j in range(0, w.shape[2], BLOCK):
                b = w[:, i:i + BLOCK, j:j + BLOCK]
                out[:, i:i + BLOCK, j:j + BLOCK] = on_grid(b, b.abs().amax((1, 2), keepdim=True),
                                                           mantissa * 2.0 ** top, bits, least)
        return out
    if op == "dropout":
        x = s["x"].to(f64)
        n, k = x.shape
        y = s["res"].to(f64) if "res" in s else torch.zeros_like(x)
        word = 0xffff

        def times(m, v):
            """High and low words of 32-bit numbers' products, by halves of 16 bits."""
            a, b = v & word, v >> 16
            p, q = a * (m & word), b * (m & word) + a * (m >> 16)
            q += p >> 16
            return (b * (m >> 16) + (q >> 16)) & 0xffffffff, ((q & word) << 16) | (p & word)

        for at in range(0, k, 4):
            c0 = torch.full((n,), at // 4, device=x.device)
            c1, c2 = torch.arange(n, device=x.device), torch.full_like(c0, s["offset"] % 2 ** 32)
            c3 = torch.full_like(c0, s["offset"] // 2 ** 32)
            for i in range(10):
                key = [(s["seed"] % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32,
                       (s["seed"] // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32]
                (h0, l0), (h1, l1) = times(0xD2511F53, c0), times(0xCD9E8D57, c2)
                c0, c1, c2, c3 = h1 ^ c1 ^ key[0], l1, h0 ^ c3 ^ key[1], l0
            for j, u in enumerate((c0, c1, c2, c3)):
                if at + j < k:
                    y[:, at + j] += torch.where(u >= round(s["p"] * 2 ** 32), x[:, at + j] / (1 - s["p"]), 0)
        return y
    (q, scale), (wq, ws) = s["x8"], s["w8"]
    n, k, m = q.shape[0], q.shape[1], wq.shape[2]

    def spread(v, e, axis, size):
        return v * torch.index_select(e, axis, torch.arange(size, device=v.device) // BLOCK)

    x = spread(q.to(torch.float32).to(f64), scale.to(torch.float32).to(f64), 1, k)
    rows_of = [(t, (s["types"] == t).nonzero().flatten()) for t in range(case["groups"])]

    def weights(t):
        e = spread(torch.ones(k, ws.shape[2], dtype=f64, device=q.device), ws[t].to(torch.float32).to(f64), 0, k)
        return spread(wq[t].to(torch.float32).to(f64), e, 1, m)

    if op == "layer8":
        y = torch.zeros(n, m, dtype=f64, device=q.device)
        z = torch.zeros_like(y)
        for t, at in rows_of:
            if at.numel():
                z[at] = x[at] @ weights(t) + s["b"][t].to(f64)
                y[at] = torch.nn.functional.silu(z[at]) if case["silu"] else z[at]
                if "res" in s:
                    y[at] += s["res"][at].to(f64)
        return {"y": y, "z": z} if case["silu"] else {"y": y}
    dx = torch.zeros(n, k, dtype=f64, device=q.device)
    dw = torch.zeros(wq.shape, dtype=f64, device=q.device)
    db = torch.zeros(s["b"].shape, dtype=f64, device=q.device)
    for t, at in rows_of:
        if at.numel():
            d = s["dy"][at].to(f64)
            if case["silu"]:
                v = s["z"][at].to(f64)
                e = torch.sigmoid(v)
                d = d * e * (1 + v * (1 - e))
            dx[at] = round8(d, case["format"]) @ weights(t).mT
            dw[t] = x[at].mT @ d
            db[t] = d.sum(0)
    return {"dx": dx, "dw": dw, "db": db}
