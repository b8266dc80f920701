// Newton-Schulz orthogonalisation of stacks of matrices, and the Muon update.
//
// Per step and matrix (lo x hi, the shorter side first):
//   A = X X^T                  lo lo hi flops (half of a product: A is symmetric)
//   B = a I + b A + c A A      lo lo lo       (half of one)
//   X <- B X                   2 lo lo hi
// each a product of float16 pairs on the matrix cores (tile.h), three times
// the above.  The iterates keep to fixed scales, since the norms are known:
// |X| <= 1 at the start and the iteration bounds it afterwards.  So each product
// writes its result as planes that the next one reads without converting: rows
// of 32 reduction entries.  X is written once, along its rows; B X reads it
// through transposing LDS reads.  A step moves 4 bytes an entry of
// X twice (and its write), A and B twice each (and theirs).
//
// All matrices of a call go through a phase in one launch: one for the
// momentum and the norms, one for the start, three for each step, of which the
// last writes the result or the weights itself.
//
// Measured, a step's three products and what they come to in float16 products:
// 118 matrices of 541 x 384 55 + 45 + 93 us (0.54 PFLOP/s), 236 of 384 x 384
// 81 + 94 + 125 us (0.54).  Matrix cores are busy 20 to 28 %, LDS 25 to 30 % (50 in tiles
// of 64 x 64) and 3.1 to 4.4 TB/s come past the L2s: the loads and barriers of a step,
// and the last workgroups of each launch.  Twelve matrices up to
// 688 x 768 17 + 12 + 16 us: too few tiles for the chip, each a chain of steps whose
// latencies nothing hides.  Eleven up to 192 x 192 take 6 to 7 us a launch.
#include <hip/hip_runtime.h>

#include "tile.h"

namespace dpa4c {

namespace {

constexpr int kThreads = kTileThreads;
constexpr int64_t kChunk = 4096;   // entries of a partial sum of squares

// fixed scales of the planes: entries of X, A and B below 4, 16 and 64
constexpr float kScaleX = 8192.0f, kScaleA = 2048.0f, kScaleB = 512.0f;

// One stack.  A plane set is [matrix][step of 32][hi, lo][rows padded to
// 128][32 entries].
struct Stack {
  const void* grad;
  void* out;
  float* momentum;
  char* x[2];     // rows lo, entries along hi; read and written in turn
  char *a, *b;    // rows lo, entries along lo
  double* squares;   // [matrix][chunks]
  int64_t batch;
  int rows, cols;
  int lo, hi;
  int lo_pad;     // to 128
  int lo_steps, hi_steps;
  int chunks;
  int turned;     // X is the transpose of the matrix
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
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t next = sh.first[lane < kMaxStacks ? lane + 1 : 0];
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(lane < count - 1 && item >= next)));
}

__host__ __device__ inline int64_t set_bytes(int steps, int rows_pad) {
  return int64_t(steps) * 2 * rows_pad * kRowBytes;
}

// U of the update: the gradient, or with momentum m (already updated) its mix
template <bool Muon>
__device__ inline float update_of(float g, float m, float beta, int nesterov) {
  if constexpr (!Muon) return g;
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
  const int count = static_cast<int>(begin + kChunk < size ? kChunk : size - begin);
  const T* __restrict__ grad = static_cast<const T*>(s.grad) + base + begin;
  constexpr int kEach = kChunk / kThreads;
  // past the chunk its last entry is read again, and counts as zero
  T g[kEach];
  float u[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) g[k] = grad[min(int(threadIdx.x) + k * kThreads, count - 1)];
  if constexpr (Muon) {
    float* momentum = s.momentum + base + begin;
    float v[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) v[k] = momentum[min(int(threadIdx.x) + k * kThreads, count - 1)];
    __syncthreads();   // read before the last entry is written
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const int j = threadIdx.x + k * kThreads;
      u[k] = to_f32(g[k]);
      v[k] = beta * v[k] + u[k];
      if (j < count) momentum[j] = v[k];
      u[k] = update_of<true>(u[k], v[k], beta, nesterov);
    }
  } else {
#pragma unroll
    for (int k = 0; k < kEach; ++k) u[k] = to_f32(g[k]);
  }
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    sum += threadIdx.x + k * kThreads < unsigned(count) ? double(u[k]) * double(u[k]) : 0.0;
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

// byte offset of the slot of entries entry .. entry + 7 of a row of a plane set
__device__ inline int64_t slot_of(int rows_pad, int row, int entry) {
  return int64_t(entry / kDepth) * 2 * rows_pad * kRowBytes + slot_at(row, entry % kDepth / 8);
}

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
  char* to = set + slot_of(rows_pad, row, entry);
  *reinterpret_cast<u4*>(to) = hi;
  *reinterpret_cast<u4*>(to + int64_t(rows_pad) * kRowBytes) = lo;
}

// What a slot of the result gets besides the stage: add x the same slot of a
// plane set, and diag on the matrix's diagonal.
struct Extra {
  const char* set;
  float add, diag;
};
struct Slot {
  v8h hi, lo;
};
__device__ inline Slot read_slot(const char* set, int rows_pad, int row, int entry) {
  const char* from = set + slot_of(rows_pad, row, entry);
  return {*reinterpret_cast<const v8h*>(from),
          *reinterpret_cast<const v8h*>(from + int64_t(rows_pad) * kRowBytes)};
}
__device__ inline void add_slot(const Extra& x, const Slot& s, int row, int entry, float* f) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f[j] += x.add * (static_cast<float>(s.hi[j]) + static_cast<float>(s.lo[j]));
    f[j] += row == entry + j ? x.diag : 0.0f;
  }
}
constexpr int kBatch = 4;   // slots of a thread in flight

// the stage (Rows of it) as rows r0 .. of a plane set, entries from c0
template <int NB, int Rows, bool Has = false>
__device__ inline void write_rows(char* set, int rows_pad, int steps, int r0, int c0,
                                  const float* stage, float scale, const Extra& x = {}) {
  constexpr int kSlots = kSide<NB> / 8, kEach = Rows * kSlots / kThreads;
  const int c = threadIdx.x % kSlots * 8;
  const int entry = c0 + c;
  if (entry / kDepth >= steps) return;
  constexpr int kGo = kEach < kBatch ? kEach : kBatch;
#pragma unroll
  for (int i0 = 0; i0 < kEach; i0 += kGo) {
    Slot old[kGo];
#pragma unroll
    for (int k = 0; k < kGo; ++k)
      if constexpr (Has)
        old[k] = read_slot(x.set, rows_pad, r0 + int(threadIdx.x) / kSlots + (i0 + k) * (kThreads / kSlots), entry);
#pragma unroll
    for (int k = 0; k < kGo; ++k) {
      const int r = threadIdx.x / kSlots + (i0 + k) * (kThreads / kSlots);
      float f[8];
      *reinterpret_cast<v4f*>(f) = *reinterpret_cast<const v4f*>(stage + stage_at<NB>(r, c));
      *reinterpret_cast<v4f*>(f + 4) = *reinterpret_cast<const v4f*>(stage + stage_at<NB>(r, c + 4));
      if constexpr (Has) add_slot(x, old[k], r0 + r, entry, f);
      write_slot(set, rows_pad, r0 + r, entry, f, scale);
    }
  }
}
// the stage's columns as rows c0 .., entries from r0: four lanes a row of a step;
// with ``mirror`` its rows are added (a tile on the diagonal)
template <int NB, bool Has = false>
__device__ inline void write_columns(char* set, int rows_pad, int steps, int r0, int c0, bool mirror,
                                     const float* stage, float scale, const Extra& x = {}) {
  constexpr int kEach = kSide<NB> * kSide<NB> / 8 / kThreads, kGo = kEach < kBatch ? kEach : kBatch;
#pragma unroll
  for (int i0 = 0; i0 < kEach; i0 += kGo) {
    Slot old[kGo];
#pragma unroll
    for (int k = 0; k < kGo; ++k) {
      const int i = i0 + k, c = threadIdx.x / 4 + i % NB * 64, slot = threadIdx.x % 4 + i / NB * 4;
      if constexpr (Has)
        if ((r0 + slot * 8) / kDepth < steps) old[k] = read_slot(x.set, rows_pad, c0 + c, r0 + slot * 8);
    }
#pragma unroll
    for (int k = 0; k < kGo; ++k) {
      const int i = i0 + k, c = threadIdx.x / 4 + i % NB * 64, slot = threadIdx.x % 4 + i / NB * 4;
      if ((r0 + slot * 8) / kDepth >= steps) continue;
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = stage[stage_at<NB>(slot * 8 + j, c)];
      if (mirror) {
        const v4f u = *reinterpret_cast<const v4f*>(stage + stage_at<NB>(c, slot * 8));
        const v4f v = *reinterpret_cast<const v4f*>(stage + stage_at<NB>(c, slot * 8 + 4));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          f[j] += u[j];
          f[4 + j] += v[j];
        }
      }
      if constexpr (Has) add_slot(x, old[k], c0 + c, r0 + slot * 8, f);
      write_slot(set, rows_pad, c0 + c, r0 + slot * 8, f, scale);
    }
  }
}

struct Finish {
  float keep, step;   // W <- keep W - step O (Muon)
};

// the stage as the result: out = O, or the weights' update
template <class T, bool Muon, int NB, int Rows>
__device__ inline void write_result(const Stack& s, int64_t m, int r0, int c0, const float* stage,
                                    const Finish& f) {
  T* out = static_cast<T*>(s.out) + m * s.rows * s.cols;
  const float step = Muon ? f.step * sqrtf(fmaxf(1.0f, float(s.cols) / float(s.rows))) : 0.0f;
  if (r0 + Rows <= s.lo && c0 + kSide<NB> <= s.hi) {   // inside: four entries a lane
    constexpr int kQuads = Rows * kSide<NB> / 4 / kThreads, kGo = 4;
#pragma unroll 1
    for (int k0 = 0; k0 < kQuads; k0 += kGo) {
      Pack<T, 4> w[kGo];
      int64_t at[kGo];
#pragma unroll
      for (int k = 0; k < kGo; ++k) {
        const int i = threadIdx.x + (k0 + k) * kThreads;
        const int r = s.turned ? i % (Rows / 4) * 4 : i / (kSide<NB> / 4);
        const int c = s.turned ? i / (Rows / 4) : i % (kSide<NB> / 4) * 4;
        at[k] = s.turned ? int64_t(c0 + c) * s.cols + r0 + r : int64_t(r0 + r) * s.cols + c0 + c;
        if constexpr (Muon) w[k] = *reinterpret_cast<const Pack<T, 4>*>(out + at[k]);
      }
#pragma unroll
      for (int k = 0; k < kGo; ++k) {
        const int i = threadIdx.x + (k0 + k) * kThreads;
        Pack<T, 4> p;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float o = s.turned ? stage[stage_at<NB>(i % (Rows / 4) * 4 + j, i / (Rows / 4))]
                                   : stage[stage_at<NB>(i / (kSide<NB> / 4), i % (kSide<NB> / 4) * 4 + j)];
          p.v[j] = from_f32<T>(Muon ? f.keep * to_f32(w[k].v[j]) - step * o : o);
        }
        *reinterpret_cast<Pack<T, 4>*>(out + at[k]) = p;
      }
    }
    return;
  }
  constexpr int kEach = Rows * kSide<NB> / kThreads, kGo = 8;
#pragma unroll 1
  for (int k0 = 0; k0 < kEach; k0 += kGo) {
    // the weights of the place, or past the matrix of its last row or column
    T w[kGo];
    int64_t at[kGo];
#pragma unroll
    for (int k = 0; k < kGo; ++k) {
      const int i = threadIdx.x + (k0 + k) * kThreads;
      const int r = min(r0 + (s.turned ? i % Rows : i / kSide<NB>), s.lo - 1);
      const int c = min(c0 + (s.turned ? i / Rows : i % kSide<NB>), s.hi - 1);
      at[k] = s.turned ? int64_t(c) * s.cols + r : int64_t(r) * s.cols + c;
      if constexpr (Muon) w[k] = out[at[k]];
    }
#pragma unroll
    for (int k = 0; k < kGo; ++k) {
      const int i = threadIdx.x + (k0 + k) * kThreads;
      const int r = s.turned ? i % Rows : i / kSide<NB>, c = s.turned ? i / Rows : i % kSide<NB>;
      const float o = stage[stage_at<NB>(r, c)];
      if (r0 + r < s.lo && c0 + c < s.hi)
        out[at[k]] = from_f32<T>(Muon ? f.keep * to_f32(w[k]) - step * o : o);
    }
  }
}

constexpr int kStartRows = 64, kStartSide = 1;

// X = U / (|U| + eps), 64 x 64 a workgroup
template <class T, bool Muon, bool Last>
__global__ void __launch_bounds__(kThreads) newton_start_kernel(Stacks all, Shares sh, float beta,
                                                                int nesterov, float eps, Finish f) {
  constexpr int kCols = kSide<kStartSide>;
  __shared__ __attribute__((aligned(16))) float stage[kStartRows * kCols];
  __shared__ double norm;
  const int i = stack_of(sh, all.count, blockIdx.x);
  const Stack& s = all.s[i];
  const int64_t item = blockIdx.x - sh.first[i];
  const int tr = s.lo_pad / kStartRows, tc = (s.hi + kCols - 1) / kCols;
  const int64_t m = item / (tr * tc);
  const int r0 = static_cast<int>(item / tc % tr) * kStartRows, c0 = static_cast<int>(item % tc) * kCols;
  const int64_t base = m * s.rows * s.cols;
  constexpr int kEach = kStartRows * kCols / kThreads;
  // past the matrix the last entry is read again: no load waits for another's value
  T g[kEach];
  float mom[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int j = threadIdx.x + k * kThreads;
    const int r = min(r0 + (s.turned ? j % kStartRows : j / kCols), s.lo - 1);
    const int c = min(c0 + (s.turned ? j / kStartRows : j % kCols), s.hi - 1);
    const int64_t at = base + (s.turned ? int64_t(c) * s.cols + r : int64_t(r) * s.cols + c);
    g[k] = static_cast<const T*>(s.grad)[at];
    if constexpr (Muon) mom[k] = s.momentum[at];
  }
  if (threadIdx.x < kWave) {
    double sum = 0.0;
    for (int j = threadIdx.x; j < s.chunks; j += kWave) sum += s.squares[m * s.chunks + j];
    for (int d = kWave / 2; d > 0; d /= 2) sum += __shfl_xor(sum, d);
    if (threadIdx.x == 0) norm = 1.0 / (sqrt(sum) + double(eps));
  }
  __syncthreads();
  const double inv = norm;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int j = threadIdx.x + k * kThreads;
    const int r = s.turned ? j % kStartRows : j / kCols, c = s.turned ? j / kStartRows : j % kCols;
    const float u = update_of<Muon>(to_f32(g[k]), Muon ? mom[k] : 0.0f, beta, nesterov);
    // the padding stays zero also where the norm is not finite
    stage[stage_at<kStartSide>(r, c)] = r0 + r < s.lo && c0 + c < s.hi ? static_cast<float>(u * inv) : 0.0f;
  }
  __syncthreads();
  if constexpr (Last)
    write_result<T, Muon, kStartSide, kStartRows>(s, m, r0, c0, stage, f);
  else
    write_rows<kStartSide, kStartRows>(s.x[0] + m * set_bytes(s.hi_steps, s.lo_pad), s.lo_pad, s.hi_steps, r0, c0,
                              stage, kScaleX);
}

enum Phase { kGram, kPoly, kApply, kLast };

// One tile of a phase.  In a tile on the diagonal of A = X X^T (or of A A) both
// operands are the same rows, and with S = hi hi^T / 2 + hi lo^T the sum of its
// three products is S + S^T: two products, with lo doubled and the sums halved, which
// is exact, and the sum with the transpose on the way out.
template <class T, bool Muon, Phase P, int NB>
__global__ void __launch_bounds__(kThreads, 2) newton_product_kernel(Stacks all, Shares sh, int from,
                                                                     float ca, float cb, float cc,
                                                                     Finish f) {
  constexpr bool kWide = P == kApply || P == kLast;
  constexpr int kOne = kPlane<NB>, kTile = kSide<NB>;
  __shared__ __attribute__((aligned(16))) char lds[8 * kOne];
  const int64_t work = xcd_block(blockIdx.x, gridDim.x);
  const int is = stack_of(sh, all.count, work);
  const Stack& s = all.s[is];
  const int64_t item = work - sh.first[is];
  const int tr = (s.lo + kTile - 1) / kTile, tc = kWide ? (s.hi + kTile - 1) / kTile : tr;
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
  const int r0 = ti * kTile, c0 = tj * kTile;
  const bool same = !kWide && ti == tj;

  const int64_t x_bytes = set_bytes(s.hi_steps, s.lo_pad), sq_bytes = set_bytes(s.lo_steps, s.lo_pad);
  const char* X = s.x[from] + m * x_bytes;
  const char* A = s.a + m * sq_bytes;
  const int64_t plane = int64_t(s.lo_pad) * kRowBytes;
  const int steps = P == kGram ? s.hi_steps : s.lo_steps;
  // rows of a step follow each other, a 16-byte slot a thread
  const char* left = (P == kGram ? X : P == kPoly ? A : s.b + m * sq_bytes) + r0 * kRowBytes;
  const char* right = P == kGram ? X + c0 * kRowBytes : P == kPoly ? A + c0 * kRowBytes : X;

  // For float32 results, small tiles have registers for sums of their own of the
  // small products, so that the large ones' are rounded a third as often, and form
  // the fourth, lo lo, of tiles on the diagonal, where it only ever adds up.  (16
  // matrices of 3 x 179: off by 1.1e-6, by 1.5e-6 without.)  Large tiles serve large
  // matrices, whose errors are other terms'.
  constexpr bool kFull = NB == 1 && sizeof(T) == 4;
  Sums<NB> acc, low;
  acc.clear();
  if constexpr (kFull) low.clear();
  const bool live = r0 + kTile / 2 * wm < s.lo && c0 + kTile / 2 * wn < (kWide ? s.hi : s.lo);
  auto run = [&](auto diagonal) {   // a constant: no branch inside the steps
    constexpr bool kSame = decltype(diagonal)::value;
    u4 ra[2][2][NB], rb[2][2][NB];   // four steps ahead gain nothing: they are in L2
    Part<NB, 2> fa[2], fb[2];
    auto fetch = [&](auto turn, int step) {
      constexpr int q = decltype(turn)::value;
      const bool in = step < steps;   // past the end: one line
      const int st = in ? step : 0, at = in ? tid * 16 : 0;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          ra[q][p][i] = *reinterpret_cast<const u4*>(left + (2 * st + p) * plane + i * 4096 + at);
          if constexpr (kWide) {
            // 32 rows of X of each of the tile's blocks of 32 columns; blocks
            // past the last repeat it, and nothing of them is stored
            int block = c0 / 32 + i * 2 + tid / 128;
            block = block < s.hi_steps ? block : s.hi_steps - 1;
            rb[q][p][i] = *reinterpret_cast<const u4*>(right + (2 * block + p) * plane + st * 32 * kRowBytes +
                                                       (in ? tid % 128 * 16 : 0));
          } else if constexpr (!kSame) {
            rb[q][p][i] = *reinterpret_cast<const u4*>(right + (2 * st + p) * plane + i * 4096 + at);
          }
        }
    };
    auto put = [&](auto turn, auto, int) {
      constexpr int q = decltype(turn)::value;
      char* to = lds + q * 4 * kOne + tid * 16;
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          if constexpr (kSame) {
            const v8h x = __builtin_bit_cast(v8h, ra[q][p][i]);
            *reinterpret_cast<v8h*>(to + p * kOne + i * 4096) = p == 0 || kFull ? x : x + x;
          } else {
            *reinterpret_cast<u4*>(to + p * kOne + i * 4096) = ra[q][p][i];
            *reinterpret_cast<u4*>(to + (2 + p) * kOne + i * 4096) = rb[q][p][i];
          }
        }
    };
    auto read = [&](auto half, int step) {
      constexpr int ks = decltype(half)::value;
      if (!live) return;
      const char* a = lds + (step & 1) * 4 * kOne + wm * (kTile / 2) * kRowBytes;
      const char* b = lds + (step & 1) * 4 * kOne + (kSame ? 0 : 2 * kOne) + wn * (kTile / 2) * kRowBytes;
      load_part(fa[ks], a, kOne, lane, ks);
      if constexpr (kWide)
        load_part_turned(fb[ks], b, kOne, lane, ks);
      else
        load_part(fb[ks], b, kOne, lane, ks);
    };
    auto multiply = [&](auto half) {
      constexpr int ks = decltype(half)::value;
      if (!live) return;
      if constexpr (kFull) {
        const u4 ah = fa[ks].v[0][0], al = fa[ks].v[0][1], bh = fb[ks].v[0][0], bl = fb[ks].v[0][1];
        v16f &big = acc.v[0][0], &small = low.v[0][0];
        if constexpr (kSame)
          big = mfma<false>(al, bl, big);
        else
          small = mfma<false>(al, bh, small);
        small = mfma<false>(ah, bl, small);
        big = mfma<false>(ah, bh, big);
      } else if constexpr (kSame) {
#pragma unroll
        for (int p = 1; p >= 0; --p)
#pragma unroll
          for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < NB; ++j)
              acc.v[i][j] = mfma<false>(fa[ks].v[i][0], fb[ks].v[j][p], acc.v[i][j]);
      } else {
        multiply_parts<false>(acc, fa[ks], fb[ks]);
      }
    };
    run_steps<2, 2>(steps, fetch, [](auto, int) {}, put, read, [](int) {}, multiply);
  };
  if constexpr (kWide) {
    run(std::false_type{});
  } else {
    if (same)
      run(std::true_type{});
    else
      run(std::false_type{});
  }

  float* stage = reinterpret_cast<float*>(lds);
  if constexpr (kFull)
    for (int r = 0; r < 16; ++r) acc.v[0][0][r] += (same ? 2.0f : 1.0f) * low.v[0][0][r];
  stage_sums(stage, acc, kTile / 2 * wm, kTile / 2 * wn, lane,
             (same ? 0.5f : 1.0f) * (P == kGram   ? 1.0f / (kScaleX * kScaleX)
                                     : P == kPoly ? cc / (kScaleA * kScaleA)
                                                  : 1.0f / (kScaleB * kScaleX)));
  __syncthreads();
  if constexpr (P == kGram) {
    char* out = s.a + m * sq_bytes;
    if (!same) write_rows<NB, kTile>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleA);
    write_columns<NB>(out, s.lo_pad, s.lo_steps, r0, c0, same, stage, kScaleA);
  } else if constexpr (P == kPoly) {
    char* out = s.b + m * sq_bytes;
    const Extra x{A, cb / kScaleA, ca};
    if (!same) write_rows<NB, kTile, true>(out, s.lo_pad, s.lo_steps, r0, c0, stage, kScaleB, x);
    write_columns<NB, true>(out, s.lo_pad, s.lo_steps, r0, c0, same, stage, kScaleB, x);
  } else if constexpr (P == kApply) {
    write_rows<NB, kTile>(s.x[from ^ 1] + m * x_bytes, s.lo_pad, s.hi_steps, r0, c0, stage, kScaleX);
  } else {
    write_result<T, Muon, NB, kTile>(s, m, r0, c0, stage, f);
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
    s.lo_pad = static_cast<int>(align_up(s.lo, kPad));
    s.lo_steps = (s.lo + kDepth - 1) / kDepth;
    s.hi_steps = (s.hi + kDepth - 1) / kDepth;
    s.chunks = static_cast<int>((int64_t(s.rows) * s.cols + kChunk - 1) / kChunk);
    for (int k = 0; k < 2; ++k) s.x[k] = ar.take<char>(s.batch * set_bytes(s.hi_steps, s.lo_pad));
    s.a = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.lo_pad));
    s.b = ar.take<char>(s.batch * set_bytes(s.lo_steps, s.lo_pad));
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
Shares share_square(const Stacks& all, int side) {
  return share(all, [&](const Stack& s) {
    const int64_t t = (s.lo + side - 1) / side;
    return t * (t + 1) / 2;
  });
}
Shares share_wide(const Stacks& all, int side) {
  return share(all, [&](const Stack& s) {
    return int64_t((s.lo + side - 1) / side) * ((s.hi + side - 1) / side);
  });
}

Shares share_norms(const Stacks& all) {
  return share(all, [](const Stack& s) { return int64_t(s.chunks); });
}
Shares share_starts(const Stacks& all) {
  return share(all, [](const Stack& s) {
    return int64_t(s.lo_pad / kStartRows) * ((s.hi + kSide<kStartSide> - 1) / kSide<kStartSide>);
  });
}

template <class T, bool Muon, Phase P>
int product(const Stacks& all, const Shares (&sh)[2], int from, const dpa4c_newton& how, const Finish& f,
            hipStream_t st) {
  // Tiles of 128 x 128 once they make two rounds of the 512 workgroups that the
  // 256 compute units hold, and unless they cover a quarter more than tiles of
  // 64 x 64 do.  (Five steps, us: 118 matrices of 541 x 384, whose squares are
  // 708 large tiles, 1,030 with small ones for them, 1,070 without; 100 of 192 x 144
  // 167 with small tiles, 187 with large ones; products of 236 of 384 x 384,
  // A 90 with large tiles and 101 with small ones, B X 141 and 174.)
  const int64_t large = sh[1].first[all.count], small = sh[0].first[all.count];
  if (large >= 1024 && 16 * large <= 5 * small)
    newton_product_kernel<T, Muon, P, 2><<<large, kThreads, 0, st>>>(all, sh[1], from, how.a, how.b, how.c, f);
  else
    newton_product_kernel<T, Muon, P, 1>
        <<<small, kThreads, 0, st>>>(all, sh[0], from, how.a, how.b, how.c, f);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

template <class T, bool Muon>
int run(const Stacks& all, const dpa4c_newton& how, const MuonStep& mu, hipStream_t st) {
  const Shares norms = share_norms(all), starts = share_starts(all);
  const Shares squares[2] = {share_square(all, kSide<1>), share_square(all, kSide<2>)};
  const Shares wides[2] = {share_wide(all, kSide<1>), share_wide(all, kSide<2>)};
  const Finish f{1.0f - mu.lr * mu.decay, mu.lr};
  newton_norm_kernel<T, Muon><<<norms.first[all.count], kThreads, 0, st>>>(all, norms, mu.momentum, mu.nesterov);
  DPA4C_HIP_TRY(hipGetLastError());
  const int64_t tiles = starts.first[all.count];
  if (how.steps == 0)
    newton_start_kernel<T, Muon, true><<<tiles, kThreads, 0, st>>>(all, starts, mu.momentum, mu.nesterov, how.eps, f);
  else
    newton_start_kernel<T, Muon, false><<<tiles, kThreads, 0, st>>>(all, starts, mu.momentum, mu.nesterov, how.eps, f);
  DPA4C_HIP_TRY(hipGetLastError());
  using P = std::conditional_t<sizeof(T) == 4, float, _Float16>;   // of the phases between
  for (int step = 0; step < how.steps; ++step) {
    DPA4C_TRY((product<P, false, kGram>(all, squares, step & 1, how, f, st)));
    DPA4C_TRY((product<P, false, kPoly>(all, squares, step & 1, how, f, st)));
    if (step + 1 < how.steps)
      DPA4C_TRY((product<P, false, kApply>(all, wides, step & 1, how, f, st)));
    else
      DPA4C_TRY((product<T, Muon, kLast>(all, wides, step & 1, how, f, st)));
  }
  return 0;
}

}  // namespace

bool newton_fits(int count, const NewtonStack* s) {
  int64_t bytes;
  const Stacks all = lay_out(count, s, nullptr, &bytes);
  // the most workgroups: a product's small tiles are no more than the start's
  return grid_fits(share_norms(all).first[all.count], kThreads) &&
         grid_fits(share_starts(all).first[all.count], kThreads);
}

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
