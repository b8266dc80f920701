// Newton-Schulz orthogonalisation of stacks of matrices, and the Muon update.
//
// Per step and matrix (lo x hi, the shorter side first):
//   A = X X^T                  lo lo hi flops (half of a product: A is symmetric)
//   B = a I + A (b I + c A)    lo lo lo       (half of one)
//   X <- B X                   2 lo lo hi
// each a product of float16 pairs on the matrix cores (tile.h), three times
// the above.  The identities go into the factors as they are written, C = b I +
// c A beside A, so no product has to read another operand at its end.  The iterates keep to fixed scales, since the norms are known:
// |X| <= 1 at the start and the iteration bounds it afterwards.  So the planes
// are written as the next product reads them: rows of 64 reduction entries.  X
// is the operand of A along its rows and of B X along its columns and is
// kept in both orders; A and B, symmetric, in one.
//
// All matrices of a call go through a phase in one launch: one for the
// momentum and the norms, one for the start, three for each step, of which the
// last writes the result or the weights itself.
#include <hip/hip_runtime.h>

#include "tile.h"

namespace dpa4c {

namespace {

constexpr int kThreads = kTileThreads;
constexpr int64_t kChunk = 8192;   // entries of a partial sum of squares

// fixed scales of the planes: entries of X, A and B (and C) below 4, 16 and 64
constexpr float kScaleX = 8192.0f, kScaleA = 2048.0f, kScaleB = 512.0f;

// One stack.  A plane set is [matrix][step of 64][hi, lo][rows padded to
// 128][64 entries].
struct Stack {
  const void* grad;
  void* out;
  float* momentum;
  char* xr[2];    // rows lo, entries along hi; read and written in turn
  char* xt[2];    // rows hi, entries along lo
  char *a, *b, *c;   // rows lo, entries along lo
  double* squares;   // [matrix][chunks]
  int64_t batch;
  int rows, cols;
  int lo, hi;
  int lo_pad, hi_pad;   // to 128
  int lo_steps, hi_steps;
  int chunks;
  int turned;   // X is the transpose of the matrix
};
struct Stacks {
  Stack s[kMaxStacks];
  int count;
};
// first work item of every stack in a phase
struct Shares {
  int64_t first[kMaxStacks + 1];
};

__device__ inline int stack_of(const Shares& sh, int count, int64_t item) {
  int i = 0;
  while (i + 1 < count && item >= sh.first[i + 1]) ++i;
  return i;
}

__host__ __device__ inline int64_t set_bytes(int steps, int rows_pad) {
  return int64_t(steps) * 2 * rows_pad * 128;
}

// U of the update: the gradient, or with momentum (already updated) its mix
template <class T, bool Muon>
__device__ inline float update_of(const Stack& s, int64_t at, float beta, int nesterov) {
  const float g = to_f32(static_cast<const T*>(s.grad)[at]);
  if constexpr (!Muon) return g;
  const float m = s.momentum[at];
  return nesterov ? g + beta * m : m;
}

// the momentum update and the sums of squares of U, a chunk a workgroup
template <class T, bool Muon>
__global__ void __launch_bounds__(kThreads) newton_norm_kernel(Stacks all, Shares sh, float beta,
                                                               int nesterov) {
  const int i = stack_of(sh, all.count, blockIdx.x);
  const Stack& s = all.s[i];
  const int64_t item = blockIdx.x - sh.first[i], m = item / s.chunks;
  const int64_t size = int64_t(s.rows) * s.cols, base = m * size;
  const int64_t begin = (item - m * s.chunks) * kChunk;
  const int64_t end = begin + kChunk < size ? begin + kChunk : size;
  double sum = 0.0;
  for (int64_t j = begin + threadIdx.x; j < end; j += kThreads) {
    if constexpr (Muon)
      s.momentum[base + j] = beta * s.momentum[base + j] + to_f32(static_cast<const T*>(s.grad)[base + j]);
    const double u = update_of<T, Muon>(s, base + j, beta, nesterov);
    sum += u * u;
  }
  __shared__ double part[kThreads];
  part[threadIdx.x] = sum;
  __syncthreads();
  for (int d = kThreads / 2; d > 0; d /= 2) {
    if (threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
    __syncthreads();
  }
  if (threadIdx.x == 0) s.squares[item] = part[0];
}

// ---------------------------------------------------------------------------
// Results in LDS (stage_at), and where they go
// ---------------------------------------------------------------------------

// eight values as one slot of each plane of a set
__device__ inline void write_slot(char* set, int rows_pad, int row, int entry, const float* f, float scale) {
  u4 hi, lo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    unsigned h, l;
    split2(f[2 * j] * scale, f[2 * j + 1] * scale, &h, &l);
    hi[j] = h;
    lo[j] = l;
  }
  char* to = set + int64_t(entry / kDepth) * 2 * rows_pad * 128 + slot_at(row, entry % kDepth / 8);
  *reinterpret_cast<u4*>(to) = hi;
  *reinterpret_cast<u4*>(to + int64_t(rows_pad) * 128) = lo;
}

// mul x the stage (+ diag on the matrix's diagonal) as rows r0 .. of a plane
// set, entries from c0; Rows: the stage's rows
template <int Rows>
__device__ inline void write_rows(char* set, int rows_pad, int steps, int r0, int c0,
                                  const float* stage, float scale, float mul = 1.0f, float diag = 0.0f) {
#pragma unroll 4
  for (int i = 0; i < Rows * 16 / kThreads; ++i) {
    const int slot = threadIdx.x % 16, r = threadIdx.x / 16 + i * (kThreads / 16), c = slot * 8;
    if ((c0 + c) / kDepth >= steps) continue;
    float f[8];
    *reinterpret_cast<v4f*>(f) = *reinterpret_cast<const v4f*>(stage + stage_at(r, c));
    *reinterpret_cast<v4f*>(f + 4) = *reinterpret_cast<const v4f*>(stage + stage_at(r, c + 4));
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = f[j] * mul + (r0 + r == c0 + c + j ? diag : 0.0f);
    write_slot(set, rows_pad, r0 + r, c0 + c, f, scale);
  }
}
// the stage's columns as rows c0 .., entries from r0
template <int Rows>
__device__ inline void write_columns(char* set, int rows_pad, int steps, int r0, int c0,
                                     const float* stage, float scale, float mul = 1.0f) {
#pragma unroll 4
  for (int i = 0; i < Rows * 16 / kThreads; ++i) {
    const int c = threadIdx.x % kTileCols, slot = threadIdx.x / kTileCols + 2 * i;
    if ((r0 + slot * 8) / kDepth >= steps) continue;
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = stage[stage_at(slot * 8 + j, c)] * mul;
    write_slot(set, rows_pad, c0 + c, r0 + slot * 8, f, scale);
  }
}

struct Finish {
  float keep, step;   // W <- keep W - step O (Muon)
};

// the stage as the result: out = O, or the weights' update
template <class T, bool Muon, int Rows>
__device__ inline void write_result(const Stack& s, int64_t m, int r0, int c0, const float* stage,
                                    const Finish& f) {
  T* out = static_cast<T*>(s.out) + m * s.rows * s.cols;
  const float step = Muon ? f.step * sqrtf(fmaxf(1.0f, float(s.cols) / float(s.rows))) : 0.0f;
#pragma unroll 8
  for (int i = threadIdx.x; i < Rows * kTileCols; i += kThreads) {
    const int r = s.turned ? i % Rows : i / kTileCols;
    const int c = s.turned ? i / Rows : i % kTileCols;
    if (r0 + r >= s.lo || c0 + c >= s.hi) continue;
    const int64_t at = s.turned ? int64_t(c0 + c) * s.cols + r0 + r : int64_t(r0 + r) * s.cols + c0 + c;
    const float o = stage[stage_at(r, c)];
    out[at] = from_f32<T>(Muon ? f.keep * to_f32(out[at]) - step * o : o);
  }
}

constexpr int kStartRows = 64;

// X = U / (|U| + eps), 64 x 128 a workgroup
template <class T, bool Muon, bool Last>
__global__ void __launch_bounds__(kThreads) newton_start_kernel(Stacks all, Shares sh, float beta,
                                                                int nesterov, float eps, Finish f) {
  __shared__ __attribute__((aligned(16))) float stage[kStartRows * kTileCols];
  __shared__ double norm;
  const int i = stack_of(sh, all.count, blockIdx.x);
  const Stack& s = all.s[i];
  const int64_t item = blockIdx.x - sh.first[i];
  const int tr = s.lo_pad / kStartRows, tc = s.hi_pad / kTileCols;
  const int64_t m = item / (tr * tc);
  const int r0 = static_cast<int>(item / tc % tr) * kStartRows, c0 = static_cast<int>(item % tc) * kTileCols;
  if (threadIdx.x < kWave) {
    double sum = 0.0;
    for (int j = threadIdx.x; j < s.chunks; j += kWave) sum += s.squares[m * s.chunks + j];
    for (int d = kWave / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x == 0) norm = 1.0 / (sqrt(sum) + double(eps));
  }
  __syncthreads();
  const double inv = norm;
  const int64_t base = m * s.rows * s.cols;
#pragma unroll 8
  for (int j = threadIdx.x; j < kStartRows * kTileCols; j += kThreads) {
    const int r = s.turned ? j % kStartRows : j / kTileCols;
    const int c = s.turned ? j / kStartRows : j % kTileCols;
    float v = 0.0f;
    if (r0 + r < s.lo && c0 + c < s.hi) {
      const int64_t at = s.turned ? int64_t(c0 + c) * s.cols + r0 + r : int64_t(r0 + r) * s.cols + c0 + c;
      v = static_cast<float>(update_of<T, Muon>(s, base + at, beta, nesterov) * inv);
    }
    stage[stage_at(r, c)] = v;
  }
  __syncthreads();
  if constexpr (Last) {
    write_result<T, Muon, kStartRows>(s, m, r0, c0, stage, f);
  } else {
    write_rows<kStartRows>(s.xr[0] + m * set_bytes(s.hi_steps, s.lo_pad), s.lo_pad, s.hi_steps, r0, c0, stage, kScaleX);
    write_columns<kStartRows>(s.xt[0] + m * set_bytes(s.lo_steps, s.hi_pad), s.hi_pad, s.lo_steps, r0, c0, stage, kScaleX);
  }
}

enum Phase { kGram, kPoly, kApply, kLast };

// one 128 x 128 tile of a phase
template <class T, bool Muon, Phase P>
__global__ void __launch_bounds__(kThreads, 2) newton_product_kernel(Stacks all, Shares sh, int from,
                                                                     float ca, float cb, float cc,
                                                                     Finish f) {
  __shared__ __attribute__((aligned(16))) char lds[4 * kPlane];
  char* la = lds;
  char* lb = lds + 2 * kPlane;
  const int64_t work = xcd_block(blockIdx.x, gridDim.x);
  const int is = stack_of(sh, all.count, work);
  const Stack& s = all.s[is];
  const int64_t item = work - sh.first[is];
  constexpr bool kWide = P == kApply || P == kLast;
  const int tr = s.lo_pad / kTileRows, tc = kWide ? s.hi_pad / kTileCols : tr;
  const int each = kWide ? tr * tc : tr * (tr + 1) / 2;
  const int64_t m = item / each;
  int ti, tj;
  if (kWide) {
    const int t = static_cast<int>(item - m * each);
    ti = t / tc;
    tj = t - ti * tc;
  } else {   // tiles (i, j <= i) of the lower triangle
    int t = static_cast<int>(item - m * each);
    ti = 0;
    while (t > ti) t -= ++ti;
    tj = t;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;

  const int64_t xr_bytes = set_bytes(s.hi_steps, s.lo_pad), xt_bytes = set_bytes(s.lo_steps, s.hi_pad);
  const int64_t sq_bytes = set_bytes(s.lo_steps, s.lo_pad);
  const char* xr = s.xr[from] + m * xr_bytes;
  const char* A = s.a + m * sq_bytes;
  const char* left = P == kGram ? xr : P == kPoly ? A : s.b + m * sq_bytes;
  const char* right = P == kGram ? xr : P == kPoly ? s.c + m * sq_bytes : s.xt[from] + m * xt_bytes;
  const int steps = P == kGram ? s.hi_steps : s.lo_steps;
  const int64_t lplane = int64_t(s.lo_pad) * 128, rplane = kWide ? int64_t(s.hi_pad) * 128 : lplane;
  left += int64_t(ti) * kPlane;
  right += int64_t(tj) * kPlane;

  u4 ra[2][4], rb[2][4];
  auto fetch = [&](int step) {
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ra[p][i] = *reinterpret_cast<const u4*>(left + (2 * step + p) * lplane + i * 4096 + tid * 16);
        rb[p][i] = *reinterpret_cast<const u4*>(right + (2 * step + p) * rplane + i * 4096 + tid * 16);
      }
  };
  Sums acc;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc.v[i][j] = v16f{};
  fetch(0);
  for (int step = 0; step < steps; ++step) {
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<u4*>(la + p * kPlane + i * 4096 + tid * 16) = ra[p][i];
        *reinterpret_cast<u4*>(lb + p * kPlane + i * 4096 + tid * 16) = rb[p][i];
      }
    __syncthreads();
    if (step + 1 < steps) fetch(step + 1);
    if (ti * kTileRows + 64 * wm < s.lo && tj * kTileCols + 64 * wn < (kWide ? s.hi : s.lo))
      tile_step<false, 2, 2>(acc, la + wm * 64 * 128, lb + wn * 64 * 128, lane);
  }

  float* stage = reinterpret_cast<float*>(lds);
  __syncthreads();
  stage_sums(stage, acc, wm, wn, lane,
             P == kGram   ? 1.0f / (kScaleX * kScaleX)
             : P == kPoly ? 1.0f / (kScaleA * kScaleB)
                          : 1.0f / (kScaleB * kScaleX));
  __syncthreads();
  const int r0 = ti * kTileRows, c0 = tj * kTileCols;
  if constexpr (P == kGram) {
    char* out = s.a + m * sq_bytes;
    char* mix = s.c + m * sq_bytes;
    write_rows<kTileRows>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleA);
    write_rows<kTileRows>(mix, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleB, cc, cb);
    if (ti != tj) {
      write_columns<kTileRows>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleA);
      write_columns<kTileRows>(mix, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleB, cc);
    }
  } else if constexpr (P == kPoly) {
    char* out = s.b + m * sq_bytes;
    write_rows<kTileRows>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleB, 1.0f, ca);
    if (ti != tj) write_columns<kTileRows>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleB);
  } else if constexpr (P == kApply) {
    write_rows<kTileRows>(s.xr[from ^ 1] + m * xr_bytes, s.lo_pad, s.hi_steps, r0, c0, stage, kScaleX);
    write_columns<kTileRows>(s.xt[from ^ 1] + m * xt_bytes, s.hi_pad, s.lo_steps, r0, c0, stage, kScaleX);
  } else {
    write_result<T, Muon, kTileRows>(s, m, r0, c0, stage, f);
  }
}

Stacks lay_out(int count, const NewtonStack* in, void* work, int64_t* bytes) {
  Stacks all{};
  Arena ar{static_cast<char*>(work)};
  for (int i = 0; i < count; ++i) {
    if (in[i].batch == 0) continue;
    Stack& s = all.s[all.count++];
    s.grad = in[i].grad;
    s.out = in[i].out;
    s.momentum = in[i].momentum;
    s.batch = in[i].batch;
    s.rows = in[i].rows;
    s.cols = in[i].cols;
    s.turned = s.rows > s.cols;
    s.lo = s.turned ? s.cols : s.rows;
    s.hi = s.turned ? s.rows : s.cols;
    s.lo_pad = static_cast<int>(align_up(s.lo, kTileRows));
    s.hi_pad = static_cast<int>(align_up(s.hi, kTileCols));
    s.lo_steps = (s.lo + kDepth - 1) / kDepth;
    s.hi_steps = (s.hi + kDepth - 1) / kDepth;
    s.chunks = static_cast<int>((int64_t(s.rows) * s.cols + kChunk - 1) / kChunk);
    for (int k = 0; k < 2; ++k) {
      s.xr[k] = ar.take<char>(s.batch * set_bytes(s.hi_steps, s.lo_pad));
      s.xt[k] = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.hi_pad));
    }
    s.a = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.lo_pad));
    s.b = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.lo_pad));
    s.c = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.lo_pad));
    s.squares = ar.take<double>(s.batch * s.chunks);
  }
  *bytes = ar.used;
  return all;
}

// the work items of a phase, ``of`` a matrix
template <class Fn>
Shares share(const Stacks& all, Fn&& of) {
  Shares sh{};
  for (int i = 0; i < all.count; ++i) sh.first[i + 1] = sh.first[i] + all.s[i].batch * of(all.s[i]);
  return sh;
}

template <class T, bool Muon>
int run(const Stacks& all, const dpa4c_newton& how, const MuonStep& mu, hipStream_t st) {
  const Shares norms = share(all, [](const Stack& s) { return int64_t(s.chunks); });
  const Shares starts = share(all, [](const Stack& s) {
    return int64_t(s.lo_pad / kStartRows) * (s.hi_pad / kTileCols);
  });
  const Shares squares = share(all, [](const Stack& s) {
    const int64_t t = s.lo_pad / kTileRows;
    return t * (t + 1) / 2;
  });
  const Shares wides = share(all, [](const Stack& s) {
    return int64_t(s.lo_pad / kTileRows) * (s.hi_pad / kTileCols);
  });
  const Finish f{1.0f - mu.lr * mu.decay, mu.lr};
  newton_norm_kernel<T, Muon><<<norms.first[all.count], kThreads, 0, st>>>(all, norms, mu.momentum, mu.nesterov);
  DPA4C_HIP_TRY(hipGetLastError());
  const int64_t tiles = starts.first[all.count];
  if (how.steps == 0)
    newton_start_kernel<T, Muon, true><<<tiles, kThreads, 0, st>>>(all, starts, mu.momentum, mu.nesterov, how.eps, f);
  else
    newton_start_kernel<T, Muon, false><<<tiles, kThreads, 0, st>>>(all, starts, mu.momentum, mu.nesterov, how.eps, f);
  DPA4C_HIP_TRY(hipGetLastError());
  const int64_t square = squares.first[all.count], wide = wides.first[all.count];
  for (int step = 0; step < how.steps; ++step) {
    const int from = step & 1;
    newton_product_kernel<float, false, kGram><<<square, kThreads, 0, st>>>(all, squares, from, how.a, how.b, how.c, f);
    newton_product_kernel<float, false, kPoly><<<square, kThreads, 0, st>>>(all, squares, from, how.a, how.b, how.c, f);
    if (step + 1 < how.steps)
      newton_product_kernel<float, false, kApply><<<wide, kThreads, 0, st>>>(all, wides, from, how.a, how.b, how.c, f);
    else
      newton_product_kernel<T, Muon, kLast><<<wide, kThreads, 0, st>>>(all, wides, from, how.a, how.b, how.c, f);
    DPA4C_HIP_TRY(hipGetLastError());
  }
  return 0;
}

}  // namespace

int64_t newton_work(int count, const NewtonStack* s) {
  int64_t bytes;
  lay_out(count, s, nullptr, &bytes);
  return bytes;
}

int launch_newton(int dtype, int count, const NewtonStack* in, const dpa4c_newton& how,
                  const MuonStep* muon, void* work, hipStream_t st) {
  int64_t bytes;
  const Stacks all = lay_out(count, in, work, &bytes);
  if (all.count == 0) return 0;
  return with_dtype(dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    return muon ? run<T, true>(all, how, *muon, st) : run<T, false>(all, how, MuonStep{}, st);
  });
}

}  // namespace dpa4c
