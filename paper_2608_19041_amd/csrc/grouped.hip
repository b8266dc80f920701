// Grouped layers: rows of each group times the weights of the group, and the
// gradients of that.
//
//   forward   y = act(x W_g + b_g) (+ x)          one product of depth k
//   dx        dz W_g^T (+ dy), dz = dy act'(z)    one product of depth n_out
//   dW, db    x^T dz, sum of dz over a group      products of depth rows
//
// Rows are addressed by place in the group order; a tile of 128 places belongs
// to one group.  A first launch lists the tiles (group_ptr lives on the
// device, so the launch's grid is an upper bound, and the workgroups past the
// last tile leave at once) and lays the weights of the groups that have rows
// out as the product tile reads them: the reduction entries of a column
// together, in steps of 64, padded with zeros, float32 as scaled float16 pairs.
// Per float32 weight that is 8 bytes written and read again once per row tile.
#include <hip/hip_runtime.h>

#include "tile.h"

namespace dpa4c {

namespace {

constexpr int kThreads = kTileThreads;

__device__ inline float logistic(float z) { return 1.0f / (1.0f + __expf(-z)); }
// act'(z) for SiLU
__device__ inline float silu_slope(float z) {
  const float p = logistic(z);
  return p * (1.0f + z * (1.0f - p));
}

// bounds of group g's places, whatever group_ptr holds; group n_groups is the
// rest, the rows of no group
struct Span {
  int64_t begin, end;
};
__device__ inline int64_t clamp_place(int64_t p, int64_t n) { return p < 0 ? 0 : p > n ? n : p; }
__device__ inline Span span_of(const int64_t* ptr, int g, int n_groups, int64_t n) {
  Span s;
  s.begin = clamp_place(ptr[g], n);
  s.end = g < n_groups ? clamp_place(ptr[g + 1], n) : n;
  s.end = s.end < s.begin ? s.begin : s.end;
  return s;
}

__device__ inline int64_t row_at(const int32_t* order, int64_t place, int64_t n) {
  const int64_t r = order ? order[place] : place;
  return r >= 0 && r < n ? r : -1;
}

// A stretch of places of one group; ``part`` of ``parts`` of the group.
struct RowTile {
  int64_t first;
  int32_t group;
  int32_t count;
  int32_t part, parts;
};

// Tiles of at most ``rows`` places of all groups, in group order, into list;
// *count of them, first_of[g] the first of group g.  With ``rest`` group
// n_groups stands for the rows of no group.  The work of one workgroup of
// ``blocks``; starts: LDS of n_groups + 2 words.
struct TileList {
  RowTile* list;
  int32_t* first_of;   // [n_groups + 2]
  int32_t* count;
  int rows;
  int rest;
};
__device__ inline void list_tiles(const TileList& tl, const int64_t* ptr, int n_groups, int64_t n,
                                  int block, int blocks, int32_t* starts) {
  const int groups = n_groups + (tl.rest ? 1 : 0);
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    int run = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {
      const int g = g0 + lane;
      int mine = 0;
      if (g < groups) {
        const Span s = span_of(ptr, g, n_groups, n);
        mine = static_cast<int>((s.end - s.begin + tl.rows - 1) / tl.rows);
      }
      int sum = mine;
      for (int d = 1; d < kWave; d *= 2) {
        const int v = __shfl_up(sum, d);
        sum += lane >= d ? v : 0;
      }
      if (g < groups) starts[g] = run + sum - mine;
      run += __shfl(sum, kWave - 1);
    }
    if (lane == 0) starts[groups] = run;
  }
  __syncthreads();
  const int total = starts[groups];
  if (block == 0) {
    for (int g = threadIdx.x; g <= groups; g += blockDim.x) tl.first_of[g] = starts[g];
    if (threadIdx.x == 0) *tl.count = total;
  }
  for (int t = block * blockDim.x + threadIdx.x; t < total; t += blocks * blockDim.x) {
    int lo = 0, hi = groups;   // starts[lo] <= t < starts[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (starts[mid] <= t) lo = mid; else hi = mid;
    }
    const Span s = span_of(ptr, lo, n_groups, n);
    RowTile r;
    r.group = lo;
    r.part = t - starts[lo];
    r.parts = starts[lo + 1] - starts[lo];
    r.first = s.begin + int64_t(r.part) * tl.rows;
    r.count = static_cast<int32_t>(s.end - r.first < tl.rows ? s.end - r.first : tl.rows);
    tl.list[t] = r;
  }
}

// ---------------------------------------------------------------------------
// Weights as the product tile reads them
// ---------------------------------------------------------------------------

// [group][step of 64][plane][columns padded to 128][64 entries], and for
// float32 the exponent of each column
struct Weights {
  char* planes;
  int32_t* exps;
  int steps, cols_pad, planes_n;
  __host__ __device__ int64_t step_bytes() const { return int64_t(planes_n) * cols_pad * 128; }
};

struct PrepArgs {
  const int64_t* ptr;
  int n_groups;
  int64_t n;
  const void* w;
  int depth, cols;   // entries of a column and columns; W is [depth][cols], or [cols][depth]
  Weights out;
  TileList tiles, blocks;   // the row tiles; the row blocks of dW (list = null: none)
  int list_blocks;          // workgroups that list tiles, after those of the weights
};

// 32 columns of one group's weights by a workgroup of 512 threads.  The entries
// of the columns are read along the rows of W: 32 columns of one entry, or (Back,
// a column is a row of W) 64 entries of one column a wave.  float32 columns
// are read twice, for the largest entry and for the planes (from L2).
constexpr int kPrepThreads = 512, kPrepCols = 32;

template <class T, bool Back>
__device__ inline void lay_weights(const PrepArgs& a, int g, int c0) {
  const Span s = span_of(a.ptr, g, a.n_groups, a.n);
  if (s.begin == s.end) return;
  const T* w = static_cast<const T*>(a.w) + int64_t(g) * a.depth * a.cols;
  constexpr bool kSplit = sizeof(T) == 4;
  __shared__ float most[kPrepThreads / kPrepCols][kPrepCols];
  __shared__ int32_t exps[kPrepCols];
  auto at = [&](int c, int k) {
    return to_f32(Back ? w[int64_t(c) * a.depth + k] : w[int64_t(k) * a.cols + c]);
  };
  if (kSplit) {
    // column c0 + r, entries q, q + 16, ..; Back: eight neighbours q a lane
    const int r = Back ? threadIdx.x / 16 : threadIdx.x % kPrepCols;
    const int q = Back ? threadIdx.x % 16 : threadIdx.x / kPrepCols;
    float m = 0.0f;
    if (c0 + r < a.cols) {
#pragma unroll 8
      for (int k = q; k < a.depth; k += 16) m = fmaxf(m, fabsf(at(c0 + r, k)));
    }
    most[q][r] = m;
    __syncthreads();
    if (threadIdx.x < kPrepCols) {
      for (int i = 0; i < 16; ++i) m = fmaxf(m, most[i][threadIdx.x]);
      const int e = m > 0.0f ? exp_for(m) : 0;
      exps[threadIdx.x] = e;
      a.out.exps[int64_t(g) * a.out.cols_pad + c0 + threadIdx.x] = e;
    }
    __syncthreads();
  }
  // slots (column, 8 entries)
  const int r = Back ? threadIdx.x / 8 % kPrepCols : threadIdx.x % kPrepCols;
  const int first = Back ? threadIdx.x % 8 + threadIdx.x / 256 * 8 : threadIdx.x / kPrepCols;
  const int c = c0 + r;
  const float scale = kSplit ? exp2_of(exps[r]) : 1.0f;
#pragma unroll 2
  for (int sl = first; sl < a.out.steps * 8; sl += 16) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = c < a.cols && sl * 8 + j < a.depth ? at(c, sl * 8 + j) : 0.0f;
    u4 hi, lo;
    if constexpr (kSplit) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unsigned h, l;
        split2(f[2 * j] * scale, f[2 * j + 1] * scale, &h, &l);
        hi[j] = h;
        lo[j] = l;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const T x = from_f32<T>(f[2 * j]), y = from_f32<T>(f[2 * j + 1]);
        hi[j] = unsigned(__builtin_bit_cast(unsigned short, x)) |
                unsigned(__builtin_bit_cast(unsigned short, y)) << 16;
      }
    }
    char* to = a.out.planes + (int64_t(g) * a.out.steps + sl / 8) * a.out.step_bytes() + slot_at(c, sl % 8);
    *reinterpret_cast<u4*>(to) = hi;
    if (kSplit) *reinterpret_cast<u4*>(to + int64_t(a.out.cols_pad) * 128) = lo;
  }
}

template <class T, bool Back>
__global__ void __launch_bounds__(kPrepThreads) grouped_prepare_kernel(PrepArgs a) {
  extern __shared__ int32_t starts[];
  // the lists first: the other workgroups' work hides theirs
  if (blockIdx.x < unsigned(a.list_blocks)) {
    if (a.tiles.list) list_tiles(a.tiles, a.ptr, a.n_groups, a.n, blockIdx.x, a.list_blocks, starts);
    __syncthreads();
    if (a.blocks.list) list_tiles(a.blocks, a.ptr, a.n_groups, a.n, blockIdx.x, a.list_blocks, starts);
    return;
  }
  const int col_blocks = a.out.cols_pad / kPrepCols;
  const int64_t b = int64_t(blockIdx.x) - a.list_blocks;
  lay_weights<T, Back>(a, static_cast<int>(b / col_blocks), static_cast<int>(b % col_blocks) * kPrepCols);
}

// dz = dy act'(z) by place: float32 as it is, half types as a pair of their own
// type, hi + lo (16 or 22 bits: dz is an intermediate, rounded to its 8 or 11 bits
// it would add as much error to dx and dW as their own rounding does)
template <class T>
__device__ inline unsigned pair_of(float x) {
  const T hi = from_f32<T>(x), lo = from_f32<T>(x - to_f32(hi));
  return unsigned(__builtin_bit_cast(unsigned short, hi)) |
         unsigned(__builtin_bit_cast(unsigned short, lo)) << 16;
}

template <class T>
__global__ void __launch_bounds__(kThreads) grouped_dz_kernel(
    const int64_t* __restrict__ ptr, const int32_t* __restrict__ order, int n_groups, int64_t n,
    int cols, int pitch, const T* __restrict__ dy, int64_t ldy, const T* __restrict__ z, int64_t ldz,
    unsigned* __restrict__ dz) {
  const int64_t live = clamp_place(ptr[n_groups], n);
  const int quads = pitch / 4;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < live * quads;
       i += int64_t(gridDim.x) * kThreads) {
    const int64_t place = i / quads;
    const int c = static_cast<int>(i - place * quads) * 4;
    const int64_t row = row_at(order, place, n);
    u4 out = {0, 0, 0, 0};
    if (row >= 0) {
      T a[4], b[4];
      if (c + 4 <= cols) {
        const Pack<T, 4> pa = *reinterpret_cast<const Pack<T, 4>*>(dy + row * ldy + c);
        const Pack<T, 4> pb = *reinterpret_cast<const Pack<T, 4>*>(z + row * ldz + c);
        for (int j = 0; j < 4; ++j) a[j] = pa.v[j], b[j] = pb.v[j];
      } else {
        for (int j = 0; j < 4; ++j) {
          a[j] = c + j < cols ? dy[row * ldy + c + j] : from_f32<T>(0.0f);
          b[j] = c + j < cols ? z[row * ldz + c + j] : from_f32<T>(0.0f);
        }
      }
      for (int j = 0; j < 4; ++j) {
        const float v = to_f32(a[j]) * silu_slope(to_f32(b[j]));
        if constexpr (sizeof(T) == 4)
          out[j] = __builtin_bit_cast(unsigned, v);
        else
          out[j] = pair_of<T>(v);
      }
    }
    *reinterpret_cast<u4*>(dz + place * pitch + c) = out;
  }
}

// ---------------------------------------------------------------------------
// Rows times weights
// ---------------------------------------------------------------------------

// How an operand's entries come: float32, a half type, or pairs of one
enum Source { kFloat, kHalf, kPair };
template <Source S>
constexpr int planes_of() { return S == kHalf ? 1 : 2; }

struct RowsArgs {
  const int32_t* order;
  int n_groups;
  int64_t n;
  const RowTile* tiles;
  const int32_t* n_tiles;
  int kin, kout;
  const void* in;   // rows of kin entries, ldin apart
  int64_t ldin;
  int by_place;     // ``in`` is in group order
  Weights w;
  const void* bias;
  int silu;
  const void* residual;   // rows of kout entries, ldres apart, or null
  int64_t ldres;
  void* out;
  void* zout;
};

// eight entries of a row as they come
template <Source S>
struct Raw {
  u4 v[S == kHalf ? 1 : 2];
};

template <Source S>
__device__ inline void load_raw(Raw<S>& r, const char* row, int k, int kin) {
  constexpr int kSize = S == kHalf ? 2 : 4;
  if (k + 8 <= kin) {
    // rows start at multiples of the entry's size only
    typedef typename std::conditional<S == kHalf, unsigned short, unsigned>::type W;
    const Pack<W, 8> p = *reinterpret_cast<const Pack<W, 8>*>(row + int64_t(k) * kSize);
    __builtin_memcpy(&r, &p, sizeof(r));
  } else {
    const u4 none = {0, 0, 0, 0};
    for (unsigned i = 0; i < sizeof(r) / 16; ++i) r.v[i] = none;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (k + j < kin) {
        if constexpr (S == kHalf)
          r.v[0][j / 2] |= unsigned(reinterpret_cast<const unsigned short*>(row)[k + j]) << (16 * (j & 1));
        else
          r.v[j / 4][j % 4] = reinterpret_cast<const unsigned*>(row)[k + j];
      }
  }
}

template <class T, Source S>
__global__ void __launch_bounds__(kThreads, 2) grouped_rows_kernel(RowsArgs a) {
  constexpr int PA = planes_of<S>(), PB = S == kFloat ? 2 : 1;
  constexpr bool kBf = std::is_same<T, __bf16>::value;
  constexpr int kOperands = (PA + PB) * kPlane;
  __shared__ __attribute__((aligned(16))) char lds[kOperands > kStageBytes ? kOperands : kStageBytes];
  __shared__ int32_t row_of[kTileRows];   // -1: nothing is stored
  __shared__ int32_t change[kTileRows];   // exponent that a row's sums are to move by
  __shared__ int32_t row_exp[kTileRows];
  __shared__ int32_t flag[2];
  char* la = lds;
  char* lb = lds + PA * kPlane;

  const int col_tiles = a.w.cols_pad / kTileCols;
  const int64_t total = int64_t(*a.n_tiles) * col_tiles;
  if (blockIdx.x >= total) return;
  // the column tiles of a row tile follow each other on one XCD
  const int64_t work = xcd_block(blockIdx.x, total);
  const RowTile t = a.tiles[work / col_tiles];
  const int c0 = static_cast<int>(work % col_tiles) * kTileCols;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  T* out = static_cast<T*>(a.out);
  T* zout = static_cast<T*>(a.zout);

  if (t.group == a.n_groups) {   // rows of no group
    const int width = a.kout - c0 < kTileCols ? a.kout - c0 : kTileCols;
    for (int i = tid; i < t.count * width; i += kThreads) {
      const int64_t row = row_at(a.order, t.first + i / width, a.n);
      if (row < 0) continue;
      out[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
      if (zout) zout[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
    }
    return;
  }

  // this thread's four rows (32 i + tid / 8) and its eight entries of a step;
  // rows past the tile repeat its last one, and nothing of them is stored
  const int sub = tid & 7;
  constexpr int kSize = S == kHalf ? 2 : 4;
  const char* rows[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int r = 32 * i + tid / 8;
    r = r < t.count ? r : t.count - 1;
    int64_t row = a.by_place ? t.first + r : row_at(a.order, t.first + r, a.n);
    if (sub == 0) {
      const int64_t to = a.by_place ? row_at(a.order, t.first + r, a.n) : row;
      row_of[32 * i + tid / 8] = 32 * i + tid / 8 < t.count ? static_cast<int32_t>(to) : -1;
    }
    row = row < 0 ? 0 : row;
    rows[i] = static_cast<const char*>(a.in) + row * a.ldin * kSize;
  }
  const char* wsrc = a.w.planes + int64_t(t.group) * a.w.steps * a.w.step_bytes() + int64_t(c0) * 128;
  const int64_t wplane = int64_t(a.w.cols_pad) * 128;

  Raw<S> ra[4];
  u4 rb[PB][4];
  auto fetch = [&](int step) {
    const int k = step * kDepth + sub * 8;
    if ((step + 1) * kDepth <= a.kin) {
#pragma unroll
      for (int i = 0; i < 4; ++i) load_raw<S>(ra[i], rows[i], k, 1 << 30);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) load_raw<S>(ra[i], rows[i], k, a.kin);
    }
    const char* src = wsrc + step * a.w.step_bytes();
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        rb[p][i] = *reinterpret_cast<const u4*>(src + p * wplane + i * 4096 + tid * 16);
  };

  Sums acc;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc.v[i][j] = v16f{};
  int e[4] = {kFirstExp, kFirstExp, kFirstExp, kFirstExp};
  unsigned changed = 0;
  if (S == kFloat) {
    if (tid < kTileRows) change[tid] = 0;
    if (tid < 2) flag[tid] = 0;
  }

  fetch(0);
  for (int step = 0; step < a.w.steps; ++step) {
    __syncthreads();   // the step before has been read
    if constexpr (S == kFloat) {
      if (tid == 0) flag[(step + 1) & 1] = 0;
      if (changed) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (changed >> i & 1) change[32 * i + tid / 8] = 0;
        changed = 0;
      }
      float f[4][8];
      bool over = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unsigned bits = ra[i].v[j / 4][j % 4];
          f[i][j] = __builtin_bit_cast(float, bits);
          m = fmaxf(m, fabsf(f[i][j]));
        }
        over |= m * exp2_of(e[i]) > kLimit;
      }
      if (__ballot(over) != 0) {   // a row has outgrown its scale: rare past the first step
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float m = 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[i][j]));
          m = fmaxf(m, __shfl_xor(m, 1));
          m = fmaxf(m, __shfl_xor(m, 2));
          m = fmaxf(m, __shfl_xor(m, 4));
          if (m * exp2_of(e[i]) > kLimit) {
            const int now = exp_for(m);
            if (sub == 0) {
              change[32 * i + tid / 8] = now - e[i];
              changed |= 1u << i;
              flag[step & 1] = 1;
            }
            e[i] = now;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float scale = exp2_of(e[i]);
        u4 hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          unsigned h, l;
          split2(f[i][2 * j] * scale, f[i][2 * j + 1] * scale, &h, &l);
          hi[j] = h;
          lo[j] = l;
        }
        const int at = slot_at(32 * i + tid / 8, sub);
        *reinterpret_cast<u4*>(la + at) = hi;
        *reinterpret_cast<u4*>(la + kPlane + at) = lo;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = slot_at(32 * i + tid / 8, sub);
        if constexpr (S == kHalf) {
          *reinterpret_cast<u4*>(la + at) = ra[i].v[0];
        } else {
          u4 hi, lo;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const unsigned x = ra[i].v[j / 2][2 * j % 4], y = ra[i].v[j / 2][2 * j % 4 + 1];
            hi[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
            lo[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
          }
          *reinterpret_cast<u4*>(la + at) = hi;
          *reinterpret_cast<u4*>(la + kPlane + at) = lo;
        }
      }
    }
#pragma unroll
    for (int p = 0; p < PB; ++p)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<u4*>(lb + p * kPlane + i * 4096 + tid * 16) = rb[p][i];
    __syncthreads();
    if (step + 1 < a.w.steps) fetch(step + 1);
    if constexpr (S == kFloat) {
      if (flag[step & 1]) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int d = change[64 * wm + 32 * i + sum_row(lane, r)];
#pragma unroll
            for (int j = 0; j < 2; ++j) acc.v[i][j][r] = ldexpf(acc.v[i][j][r], d);
          }
      }
    }
    if (c0 + 64 * wn < a.kout)
      tile_step<kBf, PA, PB>(acc, la + wm * 64 * 128, lb + wn * 64 * 128, lane);
  }

  // outputs through LDS, so that rows are written in one piece: 32 lanes a row
  if (S == kFloat && sub == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) row_exp[32 * i + tid / 8] = e[i];
  float* stage = reinterpret_cast<float*>(lds);
  const int quad = tid & 31, c = c0 + quad * 4;
  const T* bias = a.bias ? static_cast<const T*>(a.bias) + int64_t(t.group) * a.kout : nullptr;
  float bq[4];
  int eq[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bq[j] = bias && c + j < a.kout ? to_f32(bias[c + j]) : 0.0f;
    if (S == kFloat) eq[j] = a.w.exps[int64_t(t.group) * a.w.cols_pad + c + j];
  }
  __syncthreads();
  stage_sums(stage, acc, wm, wn, lane, 1.0f);
  __syncthreads();
  if (c >= a.kout) return;
  const bool whole = c + 4 <= a.kout;
  constexpr int kBatch = 4;   // rows in flight
#pragma unroll 1
  for (int r0 = tid / 32; r0 < t.count; r0 += 8 * kBatch) {
    int64_t row[kBatch];
    Pack<T, 4> res[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      row[k] = row_of[r0 + 8 * k];
      if (a.residual && row[k] >= 0) {
        const T* src = static_cast<const T*>(a.residual) + row[k] * a.ldres + c;
        if (whole)
          res[k] = *reinterpret_cast<const Pack<T, 4>*>(src);
        else
          for (int j = 0; j < 4; ++j) res[k].v[j] = c + j < a.kout ? src[j] : from_f32<T>(0.0f);
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + 8 * k;
      const v4f s = *reinterpret_cast<const v4f*>(stage + stage_at(r, quad * 4));
      const int er = S == kFloat ? row_exp[r] : 0;
      Pack<T, 4> py, pz;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float z = S == kFloat ? ldexpf(s[j], -er - eq[j]) : s[j];
        z += bq[j];
        float y = a.silu ? z * logistic(z) : z;
        if (a.residual) y += to_f32(res[k].v[j]);
        py.v[j] = from_f32<T>(y);
        pz.v[j] = from_f32<T>(z);
      }
      if (row[k] < 0) continue;
      const int64_t to = row[k] * a.kout + c;
      if (whole) {
        *reinterpret_cast<Pack<T, 4>*>(out + to) = py;
        if (zout) *reinterpret_cast<Pack<T, 4>*>(zout + to) = pz;
      } else {
        for (int j = 0; j < 4; ++j)
          if (c + j < a.kout) {
            out[to + j] = py.v[j];
            if (zout) zout[to + j] = pz.v[j];
          }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradients of the weights
// ---------------------------------------------------------------------------

struct OuterArgs {
  const int32_t* order;
  int64_t n;
  const RowTile* blocks;
  const int32_t* n_blocks;
  int k, m;
  const void* x;      // by row
  int64_t ldx;
  const void* dz;     // by row, or by place
  int64_t lddz;
  int by_place;
  void* dw;           // null: not formed
  void* db;
  float* parts;       // [block][k][m] where a group has several blocks
  float* db_parts;    // [block][m]
};

// 32 places x 64 columns of an operand, a column a lane, as they come
struct Column {
  unsigned v[32];
};

// Column ``col`` of the places first .. first + 31 (zeros from ``end`` on).  The
// row is the same for all lanes, so its address is scalar work: a lane holds the
// row of one place, and each load takes its own from there.
template <Source S>
__device__ inline void load_columns(Column& r, const void* base, int64_t ld, const int32_t* order,
                                    int64_t n, int64_t first, int64_t end, int col) {
  constexpr int kSize = S == kHalf ? 2 : 4;
  const int64_t place = first + (threadIdx.x & 31);
  int64_t mine = -1;
  if (place < end) mine = row_at(order, place, n);
  const bool whole = __ballot(mine < 0) == 0;
  const int row = static_cast<int>(mine < 0 ? 0 : mine);
  const int64_t pitch = ld * kSize;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const char* p = static_cast<const char*>(base) + __builtin_amdgcn_readlane(row, i) * pitch;
    r.v[i] = S == kHalf ? reinterpret_cast<const unsigned short*>(p)[col]
                        : reinterpret_cast<const unsigned*>(p)[col];
  }
  if (!whole)
#pragma unroll
    for (int i = 0; i < 32; ++i)
      r.v[i] = __builtin_amdgcn_readlane(static_cast<int>(mine < 0), i) ? 0 : r.v[i];
}

template <class T, Source S>
__device__ inline float value_of(unsigned v) {
  if constexpr (S == kFloat) {
    return __builtin_bit_cast(float, v);
  } else {
    const T hi = __builtin_bit_cast(T, static_cast<unsigned short>(v & 0xffff));
    if constexpr (S == kHalf) return to_f32(hi);
    return to_f32(hi) + to_f32(__builtin_bit_cast(T, static_cast<unsigned short>(v >> 16)));
  }
}

// the column's 32 entries into slots 4 half .. 4 half + 3 of its row in LDS
template <Source S>
__device__ inline void store_columns(const Column& r, char* lds, int row, int half, float scale) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    u4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const unsigned x = r.v[8 * s + 2 * j], y = r.v[8 * s + 2 * j + 1];
      if constexpr (S == kFloat) {
        unsigned h, l;
        split2(__builtin_bit_cast(float, x) * scale, __builtin_bit_cast(float, y) * scale, &h, &l);
        hi[j] = h;
        lo[j] = l;
      } else {
        hi[j] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        if (S == kPair) lo[j] = __builtin_amdgcn_perm(y, x, 0x07060302u);
      }
    }
    const int at = slot_at(row, 4 * half + s);
    *reinterpret_cast<u4*>(lds + at) = hi;
    if (S != kHalf) *reinterpret_cast<u4*>(lds + kPlane + at) = lo;
  }
}

template <class T, Source SX, Source SZ>
__global__ void __launch_bounds__(kThreads, 2) grouped_outer_kernel(OuterArgs a) {
  constexpr int PA = planes_of<SX>(), PB = planes_of<SZ>();
  constexpr bool kBf = std::is_same<T, __bf16>::value;
  __shared__ __attribute__((aligned(16))) char lds[(PA + PB) * kPlane];
  __shared__ unsigned most[kTileRows + kTileCols];   // largest magnitude of a column, as bits
  __shared__ int32_t exps[kTileRows + kTileCols], change[kTileRows + kTileCols];
  __shared__ int32_t flag[2];
  __shared__ float bias_part[2][kTileCols];
  char* la = lds;
  char* lb = lds + PA * kPlane;

  const int row_tiles = a.dw ? (a.k + kTileRows - 1) / kTileRows : 1;
  const int col_tiles = (a.m + kTileCols - 1) / kTileCols;
  const int64_t total = int64_t(*a.n_blocks) * row_tiles * col_tiles;
  if (blockIdx.x >= total) return;
  // the tiles of a block of rows follow each other on one XCD
  const int64_t work = xcd_block(blockIdx.x, total);
  const int64_t block = work / (row_tiles * col_tiles);
  const RowTile t = a.blocks[block];
  const int r0 = static_cast<int>(work / col_tiles % row_tiles) * kTileRows;
  const int c0 = static_cast<int>(work % col_tiles) * kTileCols;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int side = wave & 1, half = wave >> 1;   // the columns and places that this wave fetches
  const int mine = 64 * side + lane;
  // columns past the last repeat it, and nothing of them is stored
  const int xcol = r0 + mine < a.k ? r0 + mine : a.k - 1;
  const int zcol = c0 + mine < a.m ? c0 + mine : a.m - 1;
  const int64_t end = t.first + t.count;
  const bool sums_bias = a.db && r0 == 0;

  Column cx, cz;
  auto fetch = [&](int64_t first) {
    load_columns<SX>(cx, a.x, a.ldx, a.order, a.n, first + 32 * half, end, xcol);
    load_columns<SZ>(cz, a.dz, a.lddz, a.by_place ? nullptr : a.order, a.n, first + 32 * half, end,
                     zcol);
  };
  Sums acc;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc.v[i][j] = v16f{};
  float ex = exp2_of(kFirstExp), ez = ex, bias = 0.0f;
  if (SX == kFloat) {
    most[tid] = 0;
    exps[tid] = kFirstExp;
    if (tid < 2) flag[tid] = 0;
    __syncthreads();
  }

  fetch(t.first);
  int turn = 0;
  for (int64_t p = t.first; p < end; p += kDepth, turn ^= 1) {
    float mx = 0.0f, mz = 0.0f;
    if constexpr (SX == kFloat) {
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        mx = fmaxf(mx, fabsf(__builtin_bit_cast(float, cx.v[i])));
        mz = fmaxf(mz, fabsf(__builtin_bit_cast(float, cz.v[i])));
      }
      if (mx * ex > kLimit || mz * ez > kLimit) flag[turn] = 1;
    }
    if (sums_bias)
#pragma unroll
      for (int i = 0; i < 32; ++i) bias += value_of<T, SZ>(cz.v[i]);
    __syncthreads();   // the step before has been read; the flag is set
    if constexpr (SX == kFloat) {
      if (flag[turn]) {   // a column has outgrown its scale: rare past the first step
        atomicMax(&most[mine], __builtin_bit_cast(unsigned, mx));
        atomicMax(&most[kTileRows + mine], __builtin_bit_cast(unsigned, mz));
        __syncthreads();
        {
          const float m = __builtin_bit_cast(float, most[tid]);
          const int e = exps[tid];
          const int now = m * exp2_of(e) > kLimit ? exp_for(m) : e;
          change[tid] = now - e;
          exps[tid] = now;
        }
        __syncthreads();
        most[tid] = 0;
        ex = exp2_of(exps[mine]);
        ez = exp2_of(exps[kTileRows + mine]);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int d = change[64 * wm + 32 * i + sum_row(lane, r)];
#pragma unroll
            for (int j = 0; j < 2; ++j)
              acc.v[i][j][r] = ldexpf(acc.v[i][j][r],
                                      d + change[kTileRows + 64 * wn + 32 * j + (lane & 31)]);
          }
      }
      if (tid == 0) flag[turn ^ 1] = 0;
    }
    if (a.dw) {
      store_columns<SX>(cx, la, mine, half, ex);
      store_columns<SZ>(cz, lb, mine, half, ez);
    }
    __syncthreads();
    if (p + kDepth < end) fetch(p + kDepth);
    if (a.dw && r0 + 64 * wm < a.k && c0 + 64 * wn < a.m)
      tile_step<kBf, PA, PB>(acc, la + wm * 64 * 128, lb + wn * 64 * 128, lane);
  }

  const bool whole = t.parts == 1;   // no other block adds to this group
  if (a.dw) {
    T* dw = static_cast<T*>(a.dw) + int64_t(t.group) * a.k * a.m;
    float* part = a.parts + block * a.k * a.m;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int cl = 64 * wn + 32 * j + (lane & 31), c = c0 + cl;
        const int ec = SX == kFloat ? exps[kTileRows + cl] : 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int rl = 64 * wm + 32 * i + sum_row(lane, r), row = r0 + rl;
          if (row >= a.k || c >= a.m) continue;
          float v = acc.v[i][j][r];
          if (SX == kFloat) v = ldexpf(v, -exps[rl] - ec);
          if (whole)
            dw[int64_t(row) * a.m + c] = from_f32<T>(v);
          else
            part[int64_t(row) * a.m + c] = v;
        }
      }
  }
  if (sums_bias) {
    bias_part[half][mine] = bias;
    __syncthreads();
    if (tid < kTileCols && c0 + tid < a.m) {
      const float v = bias_part[0][tid] + bias_part[1][tid];
      if (whole)
        static_cast<T*>(a.db)[int64_t(t.group) * a.m + c0 + tid] = from_f32<T>(v);
      else
        a.db_parts[block * a.m + c0 + tid] = v;
    }
  }
}

// the blocks of a group added up in their order; zeros for groups without rows
template <class T>
__global__ void __launch_bounds__(kThreads) grouped_join_kernel(const int32_t* __restrict__ first_of,
                                                                int64_t each,
                                                                const float* __restrict__ parts,
                                                                T* __restrict__ out) {
  const int g = blockIdx.y;
  const int64_t first = first_of[g], count = first_of[g + 1] - first;
  if (count == 1) return;
  const int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= each) return;
  float s = 0.0f;
  for (int64_t b = 0; b < count; ++b) s += parts[(first + b) * each + i];
  out[g * each + i] = from_f32<T>(s);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

int64_t tiles_at_most(int64_t n, int n_groups, int64_t rows) {
  return n / rows + (n < n_groups + 1 ? n : n_groups + 1);
}

// Rows of a block of dW: 4,096 workgroups in all, some rounds of the chip's 512
// resident ones, but no fewer than 512 rows, so that a block's sums are small
// beside its rows, and groups of a few hundred rows are one block, whose sums go
// straight to dW.  Where even that gives fewer than 512 workgroups, 256.
int outer_rows(const dpa4c_grouped& l) {
  const int64_t tiles = ((l.k + kTileRows - 1) / kTileRows) * int64_t((l.n_out + kTileCols - 1) / kTileCols);
  if (l.n * tiles < 512 * 512) return 256;
  const int64_t rows = align_up((l.n * tiles + 4095) / 4096, kDepth);
  return static_cast<int>(rows < 512 ? 512 : rows > 16384 ? 16384 : rows);
}

Weights weights_of(Arena& ar, const dpa4c_grouped& l, bool back) {
  Weights w;
  const int depth = back ? l.n_out : l.k, cols = back ? l.k : l.n_out;
  w.steps = (depth + kDepth - 1) / kDepth;
  w.cols_pad = static_cast<int>(align_up(cols, kTileCols));
  w.planes_n = l.dtype == DPA4C_F32 ? 2 : 1;
  w.planes = ar.take<char>(int64_t(l.n_groups) * w.steps * w.step_bytes());
  w.exps = ar.take<int32_t>(l.dtype == DPA4C_F32 ? int64_t(l.n_groups) * w.cols_pad : 0);
  return w;
}

TileList list_of(Arena& ar, const dpa4c_grouped& l, int rows, bool rest) {
  TileList t;
  t.list = ar.take<RowTile>(tiles_at_most(l.n, l.n_groups, rows));
  t.first_of = ar.take<int32_t>(l.n_groups + 2);
  t.count = ar.take<int32_t>(1);
  t.rows = rows;
  t.rest = rest;
  return t;
}

int pitch_of(int cols) { return static_cast<int>(align_up(cols, 4)); }

struct ForwardPlan {
  Weights w;
  TileList tiles;
};
ForwardPlan plan_forward(const dpa4c_grouped& l, void* work, int64_t* bytes) {
  Arena ar{static_cast<char*>(work)};
  ForwardPlan p;
  p.w = weights_of(ar, l, false);
  p.tiles = list_of(ar, l, kTileRows, true);
  *bytes = ar.used;
  return p;
}

struct BackwardPlan {
  Weights w;
  TileList tiles, blocks;
  unsigned* dz;
  float *parts, *db_parts;
};
BackwardPlan plan_backward(const dpa4c_grouped& l, void* work, int64_t* bytes) {
  Arena ar{static_cast<char*>(work)};
  BackwardPlan p;
  p.w = weights_of(ar, l, true);
  p.tiles = list_of(ar, l, kTileRows, true);
  const int rows = outer_rows(l);
  p.blocks = list_of(ar, l, rows, false);
  p.dz = ar.take<unsigned>(l.n * pitch_of(l.n_out));
  const int64_t blocks = tiles_at_most(l.n, l.n_groups, rows);
  p.parts = ar.take<float>(blocks * l.k * l.n_out);
  p.db_parts = ar.take<float>(blocks * l.n_out);
  *bytes = ar.used;
  return p;
}

template <class T, bool Back>
int prepare(const dpa4c_grouped& l, const Weights* w, const TileList* tiles, const TileList* blocks,
            hipStream_t st) {
  PrepArgs a{};
  a.ptr = l.group_ptr;
  a.n_groups = l.n_groups;
  a.n = l.n;
  a.depth = Back ? l.n_out : l.k;
  a.cols = Back ? l.k : l.n_out;
  int64_t grid = 0, list = 0;
  if (w) {
    a.w = l.weight;
    a.out = *w;
    grid = int64_t(l.n_groups) * (w->cols_pad / kPrepCols);
  }
  if (tiles) {
    a.tiles = *tiles;
    list = tiles_at_most(l.n, l.n_groups, tiles->rows);
  }
  if (blocks) {
    a.blocks = *blocks;
    list = std::max(list, tiles_at_most(l.n, l.n_groups, blocks->rows));
  }
  a.list_blocks = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(64, list / kPrepThreads)));
  grouped_prepare_kernel<T, Back>
      <<<grid + a.list_blocks, kPrepThreads, (l.n_groups + 2) * sizeof(int32_t), st>>>(a);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

template <class T, Source S>
int run_rows(const RowsArgs& a, const TileList& tiles, hipStream_t st) {
  const int64_t grid = tiles_at_most(a.n, a.n_groups, tiles.rows) * (a.w.cols_pad / kTileCols);
  grouped_rows_kernel<T, S><<<grid, kThreads, 0, st>>>(a);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

template <class T, Source SX, Source SZ>
int run_outer(const dpa4c_grouped& l, const OuterArgs& a, const TileList& blocks, hipStream_t st) {
  const int64_t tiles = (a.dw ? (l.k + kTileRows - 1) / kTileRows : 1) *
                        int64_t((l.n_out + kTileCols - 1) / kTileCols);
  if (l.n > 0) {
    const int64_t grid = tiles_at_most(l.n, l.n_groups, blocks.rows) * tiles;
    grouped_outer_kernel<T, SX, SZ><<<grid, kThreads, 0, st>>>(a);
    DPA4C_HIP_TRY(hipGetLastError());
  }
  auto join = [&](int64_t each, const float* parts, void* out) {
    const dim3 grid((each + kThreads - 1) / kThreads, l.n_groups);
    grouped_join_kernel<T><<<grid, kThreads, 0, st>>>(blocks.first_of, each, parts, static_cast<T*>(out));
  };
  if (a.dw) join(int64_t(l.k) * l.n_out, a.parts, a.dw);
  if (a.db) join(l.n_out, a.db_parts, a.db);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

}  // namespace

int64_t grouped_forward_work(const dpa4c_grouped& l) {
  int64_t bytes;
  plan_forward(l, nullptr, &bytes);
  return bytes;
}

int64_t grouped_backward_work(const dpa4c_grouped& l) {
  int64_t bytes;
  plan_backward(l, nullptr, &bytes);
  return bytes;
}

int launch_grouped_forward(const dpa4c_grouped& l, const void* bias, bool silu, bool residual,
                           void* y, void* z, void* work, hipStream_t st) {
  if (l.n == 0) return 0;
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    int64_t bytes;
    const ForwardPlan p = plan_forward(l, work, &bytes);
    DPA4C_TRY((prepare<T, false>(l, &p.w, &p.tiles, nullptr, st)));
    RowsArgs a{};
    a.order = l.order;
    a.n_groups = l.n_groups;
    a.n = l.n;
    a.tiles = p.tiles.list;
    a.n_tiles = p.tiles.count;
    a.kin = l.k;
    a.kout = l.n_out;
    a.in = l.x;
    a.ldin = l.ldx;
    a.w = p.w;
    a.bias = bias;
    a.silu = silu;
    a.residual = residual ? l.x : nullptr;
    a.ldres = l.ldx;
    a.out = y;
    a.zout = z;
    return run_rows<T, sizeof(T) == 4 ? kFloat : kHalf>(a, p.tiles, st);
  });
}

int launch_grouped_backward(const dpa4c_grouped& l, const void* dy, int64_t ldy, const void* z,
                            int64_t ldz, bool residual, void* dx, void* dw, void* db, void* work,
                            hipStream_t st) {
  const bool rows = dx && l.n > 0, outer = dw || db;
  if (!rows && !outer) return 0;
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    constexpr Source kOwn = sizeof(T) == 4 ? kFloat : kHalf, kMade = sizeof(T) == 4 ? kFloat : kPair;
    int64_t bytes;
    const BackwardPlan p = plan_backward(l, work, &bytes);
    DPA4C_TRY((prepare<T, true>(l, rows ? &p.w : nullptr, rows ? &p.tiles : nullptr,
                                outer ? &p.blocks : nullptr, st)));
    const int pitch = pitch_of(l.n_out);
    if (z && l.n > 0) {
      const int64_t quads = l.n * (pitch / 4);
      const int64_t grid = std::min<int64_t>((quads + kThreads - 1) / kThreads, 8192);
      grouped_dz_kernel<T><<<grid, kThreads, 0, st>>>(
          l.group_ptr, l.order, l.n_groups, l.n, l.n_out, pitch, static_cast<const T*>(dy), ldy,
          static_cast<const T*>(z), ldz, p.dz);
      DPA4C_HIP_TRY(hipGetLastError());
    }
    if (rows) {
      RowsArgs a{};
      a.order = l.order;
      a.n_groups = l.n_groups;
      a.n = l.n;
      a.tiles = p.tiles.list;
      a.n_tiles = p.tiles.count;
      a.kin = l.n_out;
      a.kout = l.k;
      a.in = z ? static_cast<const void*>(p.dz) : dy;
      a.ldin = z ? pitch : ldy;
      a.by_place = z != nullptr;
      a.w = p.w;
      a.residual = residual ? dy : nullptr;
      a.ldres = ldy;
      a.out = dx;
      if (z)
        DPA4C_TRY((run_rows<T, kMade>(a, p.tiles, st)));
      else
        DPA4C_TRY((run_rows<T, kOwn>(a, p.tiles, st)));
    }
    if (outer) {
      OuterArgs a{};
      a.order = l.order;
      a.n = l.n;
      a.blocks = p.blocks.list;
      a.n_blocks = p.blocks.count;
      a.k = l.k;
      a.m = l.n_out;
      a.x = l.x;
      a.ldx = l.ldx;
      a.dz = z ? static_cast<const void*>(p.dz) : dy;
      a.lddz = z ? pitch : ldy;
      a.by_place = z != nullptr;
      a.dw = dw;
      a.db = db;
      a.parts = p.parts;
      a.db_parts = p.db_parts;
      if (z)
        DPA4C_TRY((run_outer<T, kOwn, kMade>(l, a, p.blocks, st)));
      else
        DPA4C_TRY((run_outer<T, kOwn, kOwn>(l, a, p.blocks, st)));
    }
    return 0;
  });
}

}  // namespace dpa4c
