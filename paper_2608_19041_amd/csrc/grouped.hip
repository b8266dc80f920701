// Grouped layers: rows of each group times the weights of the group, and the
// gradients of that.
//
//   forward   y = act(x W_g + b_g) (+ x)          one product of depth k
//   dx        dz W_g^T (+ dy), dz = dy act'(z)    one product of depth n_out
//   dW, db    x^T dz, sum of dz over a group      products of depth rows
//
// Rows are addressed by place in the group order; a tile of 64 or 128 places
// belongs to one group.  A first launch lists the tiles (group_ptr lives on the
// device, so a launch's grid is an upper bound, and the workgroups past the
// last tile leave at once), lays the weights of the groups that have rows out as
// the product tile reads them where that pays (WeightForm), forms dz by place and
// clears the gradients of the groups without rows.  dx and dW then read dz with
// plain rows.  Sums are float32 and every output rounds once; dz of a half type is
// kept as a pair of them (16 bits of bfloat16, 22 of float16 under a scale of its row),
// not rounded to one.
//
// The launches of a call depend on each other, so a call of few rows is bound by
// the latencies of two (forward) or four (backward) kernels: 108 rows of 144 -> 192
// take 5 + 10 us, 4,000 rows of 384 -> 384 backward 17 + 18 + 27 + 8.
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
// n_groups stands for the rows of no group.  No more than ``room`` tiles are listed,
// the most that a group_ptr can have that does not decrease: what one that does
// would add is left out.  The work of one workgroup of ``blocks``; starts: LDS of
// n_groups + 2 words.
struct TileList {
  RowTile* list;
  int32_t* first_of;   // [n_groups + 2]
  int32_t* count;
  int rows;
  int rest;
  int room;
};
__device__ inline void list_tiles(const TileList& tl, const int64_t* ptr, int n_groups, int64_t n,
                                  int block, int blocks, int32_t* starts) {
  const int groups = n_groups + (tl.rest ? 1 : 0);
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    const int64_t room = tl.room;
    int64_t run = 0;
    for (int g0 = 0; g0 < groups; g0 += kWave) {
      const int g = g0 + lane;
      int64_t mine = 0;
      if (g < groups) {
        const Span s = span_of(ptr, g, n_groups, n);
        mine = (s.end - s.begin + tl.rows - 1) / tl.rows;
      }
      int64_t sum = mine;
      for (int d = 1; d < kWave; d *= 2) {
        const int64_t v = __shfl_up(sum, d);
        sum += lane >= d ? v : 0;
      }
      if (g < groups) starts[g] = static_cast<int>(run + sum - mine < room ? run + sum - mine : room);
      run += __shfl(sum, kWave - 1);
    }
    if (lane == 0) starts[groups] = static_cast<int>(run < room ? run : room);
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

// [set][step of 32][plane][columns padded to 128][32 entries], and for float32 the
// exponent of each column.  A set for every group or, with fewer rows than groups, for
// every row: that of a group with rows is then the place of its first one.
struct Weights {
  char* planes;
  int32_t* exps;
  int steps, cols_pad, planes_n, by_start;
  __host__ __device__ int64_t step_bytes() const { return int64_t(planes_n) * cols_pad * kRowBytes; }
  __device__ int64_t set_of(int group, int64_t begin) const { return by_start ? begin : group; }
};

struct PrepArgs {
  const int64_t* ptr;
  int n_groups;
  int64_t n;
  const void* w;
  int depth, cols;   // entries of a column and columns; W is [depth][cols], or [cols][depth]
  Weights out;
  TileList tiles, blocks;   // the row tiles; the row blocks of dW (list = null: none)
  // gradients: zeros for the groups without rows (null: not formed), and dz
  void *dw, *db;
  const int32_t* order;
  const void *dy, *z;       // dy = null: dz is not formed
  int64_t ldy, ldz;
  int pitch;
  void* dz;
  int32_t* dz_exps;   // float16: the exponent of each place's row
  // the workgroups of each kind, in this order
  int64_t list_blocks, weight_blocks, clear_blocks, dz_blocks;
};

// 32 columns of one group's weights by a workgroup of 512 threads, which holds them
// in registers between finding the largest entry and writing the planes (columns
// of more than kHeld x 128 entries are read twice, from L2).  The entries are
// read along the rows of W: 32 columns of one entry, or (Back, a column is a row of
// W) eight entries a lane.
constexpr int kPrepThreads = 512, kPrepCols = 32, kHeld = 6;

template <class T, bool Back>
__device__ inline void lay_weights(const PrepArgs& a, int g, int c0) {
  const Span s = span_of(a.ptr, g, a.n_groups, a.n);
  if (s.begin == s.end) return;
  const T* w = static_cast<const T*>(a.w) + int64_t(g) * a.depth * a.cols;
  const int64_t set = a.out.set_of(g, s.begin);
  constexpr bool kSplit = sizeof(T) == 4;
  __shared__ float most[kPrepThreads / kPrepCols][kPrepCols];
  __shared__ int32_t exps[kPrepCols];
  // slots (column c0 + r, entries 8 sl ..), sl = first, first + 16, ..
  constexpr int kSlots = kDepth / 8;
  const int r = Back ? threadIdx.x / 16 : threadIdx.x % kPrepCols;
  const int first = Back ? threadIdx.x % 16 : threadIdx.x / kPrepCols;
  const int c = c0 + r, slots = a.out.steps * kSlots;
  auto load = [&](int sl, T* f) {
    const int k = sl * 8;
    if (Back && c < a.cols && k + 8 <= a.depth) {
      *reinterpret_cast<Pack<T, 8>*>(f) = *reinterpret_cast<const Pack<T, 8>*>(w + int64_t(c) * a.depth + k);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        f[j] = c < a.cols && k + j < a.depth ? w[Back ? int64_t(c) * a.depth + k + j : int64_t(k + j) * a.cols + c]
                                             : from_f32<T>(0.0f);
    }
  };
  auto write = [&](int sl, const T* f, float scale) {
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
      for (int j = 0; j < 4; ++j)
        hi[j] = unsigned(__builtin_bit_cast(unsigned short, f[2 * j])) |
                unsigned(__builtin_bit_cast(unsigned short, f[2 * j + 1])) << 16;
    }
    char* to = a.out.planes + (set * a.out.steps + sl / kSlots) * a.out.step_bytes() +
               slot_at(c, sl % kSlots);
    *reinterpret_cast<u4*>(to) = hi;
    if (kSplit) *reinterpret_cast<u4*>(to + int64_t(a.out.cols_pad) * kRowBytes) = lo;
  };
  const bool held = slots <= kHeld * 16;
  T f[kHeld][8];
  if (held) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (first + 16 * i < slots) load(first + 16 * i, f[i]);
  }
  float scale = 1.0f;
  if constexpr (kSplit) {
    float m = 0.0f;
    if (held) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (first + 16 * i < slots)
#pragma unroll
          for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[i][j]));
    } else {
      for (int sl = first; sl < slots; sl += 16) {
        load(sl, f[0]);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(f[0][j]));
      }
    }
    most[first][r] = m;
    __syncthreads();
    if (threadIdx.x < kPrepCols) {
      float top = 0.0f;
      for (int i = 0; i < 16; ++i) top = fmaxf(top, most[i][threadIdx.x]);
      const int e = top > 0.0f ? exp_for(top) : 0;
      exps[threadIdx.x] = e;
      a.out.exps[set * a.out.cols_pad + c0 + threadIdx.x] = e;
    }
    __syncthreads();
    scale = exp2_of(exps[r]);
  }
  if (held) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (first + 16 * i < slots) write(first + 16 * i, f[i], scale);
  } else {
    for (int sl = first; sl < slots; sl += 16) {
      load(sl, f[0]);
      write(sl, f[0], scale);
    }
  }
}

// a part of the zeros of one group without rows
constexpr int64_t kClear = 1 << 16;   // entries of a workgroup
template <class T>
__device__ inline void clear_gradients(const PrepArgs& a, int g, int64_t part) {
  const Span s = span_of(a.ptr, g, a.n_groups, a.n);
  if (s.begin != s.end) return;
  constexpr int kEach = 16 / sizeof(T);
  const Pack<T, kEach> none = {};
  const int64_t each = int64_t(a.depth) * a.cols;   // k n_out either way
  if (a.dw) {
    T* out = static_cast<T*>(a.dw) + g * each;
    const int64_t end = (part + 1) * kClear < each ? (part + 1) * kClear : each;
    for (int64_t i = part * kClear + threadIdx.x * kEach; i < end; i += kPrepThreads * kEach) {
      if (i + kEach <= end)
        *reinterpret_cast<Pack<T, kEach>*>(out + i) = none;
      else
        for (int64_t j = i; j < end; ++j) out[j] = none.v[0];
    }
  }
  if (a.db && part == 0)
    for (int i = threadIdx.x; i < a.depth; i += kPrepThreads)
      static_cast<T*>(a.db)[int64_t(g) * a.depth + i] = none.v[0];   // Back: depth = n_out
}

// Rows of fewer than eight entries, eight entries apart, so that loads of eight
// stay inside.
constexpr int kLeastWidth = 8;
template <class T>
__global__ void __launch_bounds__(kThreads) grouped_widen_kernel(int64_t n, int width, const T* __restrict__ in,
                                                                 int64_t ld, T* __restrict__ out) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n * kLeastWidth;
       i += int64_t(gridDim.x) * kThreads) {
    const int c = static_cast<int>(i % kLeastWidth);
    out[i] = c < width ? in[i / kLeastWidth * ld + c] : from_f32<T>(0.0f);
  }
}

// dz = dy act'(z) (z = null: dy) by place: float32 as it is, half types as a plane of their own
// type and one of what that leaves, hi + lo (16 or, of float16 below, 22 bits: dz is an
// intermediate; rounded to its 8 or 11 bits it would add as much error to dx and dW as their
// own rounding does)
template <class T>
__device__ inline void form_dz(const PrepArgs& p, int64_t block, int64_t blocks) {
  constexpr int kEach = 16 / sizeof(T);
  const int64_t n = p.n, ldy = p.ldy, ldz = p.ldz;
  const int cols = p.depth, pitch = p.pitch;   // Back: depth = n_out
  const T* dy = static_cast<const T*>(p.dy);
  const T* z = static_cast<const T*>(p.z);
  T* dz = static_cast<T*>(p.dz);
  const int64_t live = clamp_place(p.ptr[p.n_groups], n);
  const int each = pitch / kEach;
  for (int64_t i = block * kPrepThreads + threadIdx.x; i < live * each; i += blocks * kPrepThreads) {
    const int64_t place = i / each;
    const int c = static_cast<int>(i - place * each) * kEach;
    const int64_t row = row_at(p.order, place, n);
    Pack<T, kEach> a = {}, b = {}, hi, lo;
    if (row >= 0) {
      if (c + kEach <= cols) {
        a = *reinterpret_cast<const Pack<T, kEach>*>(dy + row * ldy + c);
        if (z) b = *reinterpret_cast<const Pack<T, kEach>*>(z + row * ldz + c);
      } else {
        for (int j = 0; j < kEach; ++j)
          if (c + j < cols) {
            a.v[j] = dy[row * ldy + c + j];
            if (z) b.v[j] = z[row * ldz + c + j];
          }
      }
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      float v = to_f32(a.v[j]);
      if (z) v *= silu_slope(to_f32(b.v[j]));
      // v as one value: fused with the product, the two conversions below could
      // round it to neighbouring hi at a tie
      asm("" : "+v"(v));
      hi.v[j] = from_f32<T>(v);
      if (sizeof(T) == 2) lo.v[j] = from_f32<T>(v - to_f32(hi.v[j]));
    }
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
    *reinterpret_cast<V*>(dz + place * pitch + c) = __builtin_bit_cast(V, hi);
    if (sizeof(T) == 2) *reinterpret_cast<V*>(dz + (n + place) * pitch + c) = __builtin_bit_cast(V, lo);
  }
}

// The same of float16, whose exponents end too early for what a gradient can be: a
// row is multiplied by 2^e first, so that its largest finite entry lies in [2^14, 2^15).
// hi + lo then holds an entry to 2^-22 of itself or 2^-39 of that largest one, and
// nothing overflows.  A row of zeros has kNoExp.  lanes_of_dz(pitch) lanes take a row,
// eight entries each; longer rows are formed twice.  (1,000,188 rows of 384: the
// launch 710 us, of bfloat16 640 on the same card, and dW of 541 columns 1,975 against 1,715.)
constexpr int kDzTop = 14, kNoExp = 100;
__host__ __device__ inline int lanes_of_dz(int pitch) {
  int lanes = 1;
  while (lanes < kWave && lanes * 8 < pitch) lanes *= 2;
  return lanes;
}
__device__ inline void form_dz_scaled(const PrepArgs& p, int64_t block, int64_t blocks) {
  using T = _Float16;
  const int64_t n = p.n;
  const int cols = p.depth, pitch = p.pitch;   // Back: depth = n_out
  const T* dy = static_cast<const T*>(p.dy);
  const T* z = static_cast<const T*>(p.z);
  T* dz = static_cast<T*>(p.dz);
  const int64_t live = clamp_place(p.ptr[p.n_groups], n);
  const int lanes = lanes_of_dz(pitch), sub = threadIdx.x & (lanes - 1);
  const int rows = kPrepThreads / lanes;
  for (int64_t place = block * rows + int(threadIdx.x) / lanes; place < live; place += blocks * rows) {
    const int64_t row = row_at(p.order, place, n);
    float v[8];
    auto form = [&](int c) {
      Pack<T, 8> a = {}, b = {};
      if (row >= 0) {
        if (c + 8 <= cols) {
          a = *reinterpret_cast<const Pack<T, 8>*>(dy + row * p.ldy + c);
          if (z) b = *reinterpret_cast<const Pack<T, 8>*>(z + row * p.ldz + c);
        } else {
          for (int j = 0; j < 8; ++j)
            if (c + j < cols) {
              a.v[j] = dy[row * p.ldy + c + j];
              if (z) b.v[j] = z[row * p.ldz + c + j];
            }
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = to_f32(a.v[j]);
        if (z) v[j] *= silu_slope(to_f32(b.v[j]));
      }
    };
    float m = 0.0f;
    for (int c = sub * 8; c < pitch; c += lanes * 8) {
      form(c);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float size = fabsf(v[j]);
        m = size < INFINITY ? fmaxf(m, size) : m;   // neither infinities nor NaN
      }
    }
    for (int d = lanes / 2; d > 0; d /= 2) m = fmaxf(m, __shfl_xor(m, d));
    const int top = kDzTop - (static_cast<int>(__builtin_bit_cast(unsigned, m) >> 23) - 127);
    const int e = top < kNoExp ? top : kNoExp;   // m = 0 too
    if (sub == 0) p.dz_exps[place] = e;
    const float scale = exp2_of(e);
    for (int c = sub * 8; c < pitch; c += lanes * 8) {
      if (pitch > lanes * 8) form(c);
      u4 hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // one value each: as in form_dz
        float x = v[2 * j] * scale, y = v[2 * j + 1] * scale;
        asm("" : "+v"(x), "+v"(y));
        unsigned h, l;
        split2(x, y, &h, &l);
        hi[j] = h;
        lo[j] = l;
      }
      *reinterpret_cast<u4*>(dz + place * pitch + c) = hi;
      *reinterpret_cast<u4*>(dz + (n + place) * pitch + c) = lo;
    }
  }
}

// What the products of a call need first, each piece by workgroups of its own, since
// all of it is bound by HBM: 31,250 rows of 541 -> 384 in 118 groups move 340 MB in
// 65 us (5.2 TB/s, reads of dy and z that the last-level cache holds among them), dz
// of a million bfloat16 rows 3.1 GB in 624 us (5.0 TB/s).
template <class T, bool Back>
__global__ void __launch_bounds__(kPrepThreads) grouped_prepare_kernel(PrepArgs a) {
  extern __shared__ int32_t starts[];
  int64_t b = blockIdx.x;
  if (b < a.list_blocks) {
    const int block = static_cast<int>(b), blocks = static_cast<int>(a.list_blocks);
    if (a.tiles.list) list_tiles(a.tiles, a.ptr, a.n_groups, a.n, block, blocks, starts);
    __syncthreads();
    if (a.blocks.list) list_tiles(a.blocks, a.ptr, a.n_groups, a.n, block, blocks, starts);
    return;
  }
  b -= a.list_blocks;
  if (b < a.weight_blocks) {
    const int64_t each = a.weight_blocks / a.n_groups;
    lay_weights<T, Back>(a, static_cast<int>(b / each), static_cast<int>(b % each) * kPrepCols);
    return;
  }
  if constexpr (Back) {
    b -= a.weight_blocks;
    if (b < a.clear_blocks) {
      const int64_t each = a.clear_blocks / a.n_groups;
      clear_gradients<T>(a, static_cast<int>(b / each), b % each);
      return;
    }
    if constexpr (std::is_same<T, _Float16>::value)
      form_dz_scaled(a, b - a.clear_blocks, a.dz_blocks);
    else
      form_dz<T>(a, b - a.clear_blocks, a.dz_blocks);
  }
}

// ---------------------------------------------------------------------------
// Rows times weights
// ---------------------------------------------------------------------------

// How an operand's entries come: float32, a half type, or a plane of one and a
// plane of what that leaves
enum Source { kFloat, kHalf, kPair };
template <Source S>
constexpr int planes_of = S == kHalf ? 1 : 2;
template <Source S>
constexpr int bytes_of = S == kFloat ? 4 : 2;
// a pair of float16 has an exponent of its row
template <class T, Source S>
constexpr bool row_scaled = S == kPair && std::is_same<T, _Float16>::value;

// How a product reads the weights.  Half types take them as they are: the rows of W
// are the reduction entries of x W (read through transposing LDS reads) and the
// columns of dz W^T.  float32 weights are laid out as planes first, and so are
// rows of fewer than eight entries and, since the planes are quicker to fetch, the
// weights under kLaidRows rows and more for each group of the table: how many of its
// groups have rows only the device knows, and what laying out costs grows with them.
// (bfloat16, 541 -> 384, 118 groups, us, as they are and laid out.  Forward with z, all
// groups present: 31,250 rows 60, 80; 250,000 378, 405; 1,000,188 1,421, 1,435.  Five
// present: 58, 62; 366, 370; 1,408, 1,398.  dx of dy and z, all: 94, 105; 577, 586; 2,173,
// 2,158; five: 87, 85; 562, 555; 2,154, 2,118.  Of 144 -> 192 1,000,188 rows 588, 571.)
enum WeightForm { kLaid, kEntries, kColumns };
constexpr int kLaidRows = 4096;

struct RowsArgs {
  const int32_t* order;
  int n_groups;
  int64_t n;
  const RowTile* tiles;
  const int32_t* n_tiles;
  int kin, kout;
  const void* in;   // rows of kin entries, ldin apart
  int64_t ldin;
  int by_place;     // ``in`` is in group order; its second plane n ldin entries on
  const int32_t* in_exps;   // row_scaled: the rows' exponents, by place
  Weights w;
  const void* weight;   // as they are, unless kLaid
  const void* bias;
  int silu;
  const void* residual;   // rows of kout entries, ldres apart, or null
  int64_t ldres;
  void* out;
  void* zout;
};

// Eight entries of a row as they come.  A load takes eight entries whatever the
// row's length, without a condition (loads under one would make the compiler
// wait for all that are in flight): ``last`` is the largest k at which eight entries
// lie inside the array, and trim() puts the entries from there in their place
// and zeros in that of those past the row.
template <Source S>
struct Raw {
  u4 v[planes_of<S>];
};
// entries of an array of n rows of ``width``, ``ld`` apart, from row ``row`` to its end
__host__ __device__ inline int last_of(int64_t n, int64_t ld, int width, int64_t row) {
  const int64_t left = (n - 1 - row) * ld + width - 8;
  return left > (1 << 30) ? 1 << 30 : static_cast<int>(left);
}

// from ``row``, which starts at any multiple of an entry's size, at entry ``k``
template <Source S>
__device__ inline void load_raw(Raw<S>& r, const char* row, int64_t plane, int k) {
  if constexpr (S == kFloat) {
    const Pack<unsigned, 8> p = *reinterpret_cast<const Pack<unsigned, 8>*>(row + int64_t(k) * 4);
    __builtin_memcpy(&r, &p, sizeof(r));
  } else {
#pragma unroll
    for (int i = 0; i < planes_of<S>; ++i) {
      const Pack<unsigned short, 8> p =
          *reinterpret_cast<const Pack<unsigned short, 8>*>(row + i * plane + int64_t(k) * 2);
      __builtin_memcpy(&r.v[i], &p, 16);
    }
  }
}
// what was loaded at min(k, last) as the entries k .. k + 7 of a row of ``width``
template <Source S>
__device__ inline void trim(Raw<S>& r, int k, int last, int width) {
  const int off = k < last ? 0 : k - last, keep = width - k;
  if constexpr (S == kFloat) {
    unsigned e[8];
    __builtin_memcpy(e, &r, 32);
#pragma unroll
    for (int bit = 1; bit < 8; bit *= 2)
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = !(off & bit) ? e[j] : j + bit < 8 ? e[j + bit] : 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < keep && off < 8 ? e[j] : 0u;
    __builtin_memcpy(&r, e, 32);
  } else {
#pragma unroll
    for (int p = 0; p < planes_of<S>; ++p) {
      unsigned __int128 x;
      __builtin_memcpy(&x, &r.v[p], 16);
      x = off >= 8 || keep <= 0 ? 0 : x >> (16 * off);
      if (keep < 8 && keep > 0) x &= ((unsigned __int128)1 << (16 * keep)) - 1;
      __builtin_memcpy(&r.v[p], &x, 16);
    }
  }
}

// A tile of rows times weights, by run_steps(); rows and unlaid weights are the far
// operands, laid out weights (from L2) the near one.  A float32 row has a running
// scale, so it is read once.  31,250 rows of 541 -> 384 in 118 groups: bfloat16
// forward 55 to 57 us for 140 MB (2.5 TB/s, matrix cores busy 10 %: one step of loads is
// 0.3 us of products, so the tiles of a compute unit wait for them), float32 dx 123 us
// (0.32 PFLOP/s of float16 products, 16 %, with half of the row tiles short).  dx of
// 1,000,188 bfloat16 rows in two planes 1,640 us (0.51 PFLOP/s): matrix cores 22 %, LDS
// 29 %, 1.6 TB/s; a step's loads, LDS writes and barrier with two waves to a SIMD.
template <class T, Source S, int NB, WeightForm W>
__global__ void __launch_bounds__(kThreads, 2) grouped_rows_kernel(RowsArgs a) {
  static_assert(S != kFloat || W == kLaid, "float32 weights are split into planes first");
  constexpr int PA = planes_of<S>, PB = S == kFloat ? 2 : 1;
  constexpr bool kBf = std::is_same<T, __bf16>::value;
  constexpr int kTile = kSide<NB>, kOne = kPlane<NB>;
  constexpr int kHalfLds = (PA + PB) * kOne;   // one step's operands
  constexpr int kStageRows = kHalfLds * 2 >= kTile * kTile * 4 ? kTile : kTile / 2;
  constexpr int kStage = kStageRows * kTile * 4;
  __shared__ __attribute__((aligned(16))) char lds[2 * kHalfLds > kStage ? 2 * kHalfLds : kStage];
  __shared__ int32_t row_of[kTile];      // -1: nothing is stored
  __shared__ int32_t change[2][kTile];   // exponent that a row's sums are to move by
  __shared__ int32_t row_exp[kTile];
  __shared__ int32_t flag[3];

  const int col_tiles = (a.kout + kTile - 1) / kTile;
  const int64_t total = int64_t(*a.n_tiles) * col_tiles;
  if (blockIdx.x >= total) return;
  // the column tiles of a row tile follow each other on one XCD
  const int64_t work = xcd_block(blockIdx.x, total);
  const RowTile t = a.tiles[work / col_tiles];
  const int c0 = static_cast<int>(work % col_tiles) * kTile;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  T* out = static_cast<T*>(a.out);
  T* zout = static_cast<T*>(a.zout);

  if (t.group == a.n_groups) {   // rows of no group
    const int width = a.kout - c0 < kTile ? a.kout - c0 : kTile;
    for (int i = tid; i < t.count * width; i += kThreads) {
      const int64_t row = row_at(a.order, t.first + i / width, a.n);
      if (row < 0) continue;
      out[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
      if (zout) zout[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
    }
    return;
  }

  // this thread's NB rows (64 i + tid / 4) and its eight entries of a step; rows
  // past the tile repeat its last one, and nothing of them is stored
  const int sub = tid & 3, own = tid / 4;
  const char* rows[NB];
  int last[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    int r = 64 * i + own;
    r = r < t.count ? r : t.count - 1;
    const int64_t to = row_at(a.order, t.first + r, a.n);
    if (sub == 0) row_of[64 * i + own] = 64 * i + own < t.count ? static_cast<int32_t>(to) : -1;
    if (row_scaled<T, S> && sub == 0) row_exp[64 * i + own] = a.in_exps[t.first + r];
    const int64_t row = a.by_place ? t.first + r : to < 0 ? 0 : to;
    rows[i] = static_cast<const char*>(a.in) + row * a.ldin * bytes_of<S>;
    last[i] = last_of(a.n, a.ldin, a.by_place ? static_cast<int>(a.ldin) : a.kin, row);
  }
  const int64_t in_plane = a.n * a.ldin * bytes_of<S>;
  // laid out: from c0 of the first step; as they are: of the group
  const int64_t set = a.w.set_of(t.group, t.first - int64_t(t.part) * kTile);
  const char* wsrc =
      W == kLaid ? a.w.planes + set * a.w.steps * a.w.step_bytes() + int64_t(c0) * kRowBytes
                 : static_cast<const char*>(a.weight) + int64_t(t.group) * a.kin * a.kout * sizeof(T);
  const int64_t wplane = int64_t(a.w.cols_pad) * kRowBytes;
  // kColumns: this thread's NB columns (rows of W, as those of ``in``); columns past
  // the last repeat it
  const char* wrow[NB];
  int wlast[NB];
  if constexpr (W == kColumns) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int c = c0 + 64 * i + own < a.kout ? c0 + 64 * i + own : a.kout - 1;
      wrow[i] = wsrc + int64_t(c) * a.kin * sizeof(T);
      wlast[i] = last_of(int64_t(a.n_groups) * a.kout, a.kin, a.kin, int64_t(t.group) * a.kout + c);
    }
  }
  // kEntries: eight columns of entry tid / kTileSlots (+ 16) of a step; from ``wleft`` on, in
  // the group, eight entries would reach past the last group's end
  constexpr int kTileSlots = kTile / 8;
  const int wentry = tid / kTileSlots, wslot = tid % kTileSlots;
  const int64_t wleft = (int64_t(a.n_groups) - t.group) * a.kin * a.kout - 8;
  auto entry_at = [&](int step, int i) {
    const int k = step * kDepth + wentry + 16 * i;
    return int64_t(k < a.kin ? k : a.kin - 1) * a.kout + c0 + wslot * 8;
  };

  constexpr int kFar = S == kFloat && NB == 2 ? 2 : 4;   // what the registers hold
  // weights as they are come from HBM too
  constexpr int kNear = W == kLaid || S == kPair ? 2 : kFar;
  Raw<S> ra[kFar][NB];
  u4 rb[kNear][PB][NB];
  auto far = [&](auto turn, int step) {
    constexpr int q = decltype(turn)::value;
    const bool in = step < a.w.steps;   // past the end: one line of the weights
    const int k = step * kDepth + sub * 8;
#pragma unroll
    for (int i = 0; i < NB; ++i)
      load_raw<S>(ra[q][i], in ? rows[i] : wsrc, in ? in_plane : 0, !in ? 0 : k < last[i] ? k : last[i]);
  };
  auto near = [&](auto turn, int step) {
    constexpr int q = decltype(turn)::value;
    const bool in = step < a.w.steps;
    if constexpr (W == kLaid) {
      const char* src = in ? wsrc + step * a.w.step_bytes() + tid * 16 : wsrc;
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int i = 0; i < NB; ++i)
          rb[q][p][i] = *reinterpret_cast<const u4*>(src + (in ? p * wplane + i * 4096 : 0));
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        Raw<kHalf> r;
        if constexpr (W == kColumns) {
          const int k = step * kDepth + sub * 8;
          load_raw<kHalf>(r, in ? wrow[i] : wsrc, 0, !in ? 0 : k < wlast[i] ? k : wlast[i]);
        } else {
          const int64_t at = entry_at(step, i);
          load_raw<kHalf>(r, wsrc + (!in ? 0 : at < wleft ? at : wleft) * sizeof(T), 0, 0);
        }
        rb[q][0][i] = r.v[0];
      }
    }
  };

  Sums<NB> acc;
  acc.clear();
  int e[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) e[i] = kFirstExp;
  unsigned changed[2] = {0, 0};
  if (S == kFloat) {
    if (tid < 2 * kTile) change[tid / kTile][tid % kTile] = 0;
    if (tid < 3) flag[tid] = 0;
    __syncthreads();
  }

  auto put = [&](auto turn, auto far_turn, int step) {
    constexpr int n = decltype(turn)::value, f = decltype(far_turn)::value, q = f & 1;
    char* la = lds + q * kHalfLds;
    char* lb = la + PA * kOne;
    if constexpr (W == kLaid) {
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int i = 0; i < NB; ++i)
          *reinterpret_cast<u4*>(lb + p * kOne + i * 4096 + tid * 16) = rb[n][p][i];
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if ((step + 1) * kDepth >= a.kin) {   // the last step
          Raw<kHalf> r{{rb[n][0][i]}};
          if constexpr (W == kColumns) {
            trim<kHalf>(r, step * kDepth + sub * 8, wlast[i], a.kin);
          } else {
            const int64_t past = entry_at(step, i) - wleft;
            const int off = past > 0 ? static_cast<int>(past) : 0;
            trim<kHalf>(r, off, 0, step * kDepth + wentry + 16 * i < a.kin ? off + 8 : off);
          }
          rb[n][0][i] = r.v[0];
        }
        const int at = W == kColumns ? slot_at(64 * i + own, sub)
                                     : wslot / 4 * kDepth * kRowBytes + slot_at(wentry + 16 * i, wslot % 4);
        *reinterpret_cast<u4*>(lb + at) = rb[n][0][i];
      }
    }
    if ((step + 1) * kDepth > a.kin)
#pragma unroll
      for (int i = 0; i < NB; ++i) trim<S>(ra[f][i], step * kDepth + sub * 8, last[i], a.kin);
    if constexpr (S == kFloat) {
      if (tid == 0) flag[(step + 1) % 3] = 0;
      if (changed[q]) {   // two steps ago; its readers are past it
#pragma unroll
        for (int i = 0; i < NB; ++i)
          if (changed[q] >> i & 1) change[q][64 * i + own] = 0;
        changed[q] = 0;
      }
      float v[NB][8];
      bool over = false;
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const unsigned bits = ra[f][i].v[j / 4][j % 4];
          v[i][j] = __builtin_bit_cast(float, bits);
          m = fmaxf(m, fabsf(v[i][j]));
        }
        over |= m * exp2_of(e[i]) > kLimit;
      }
      if (__ballot(over) != 0) {   // a row has outgrown its scale: rare past the first step
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          float m = 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(v[i][j]));
          m = fmaxf(m, __shfl_xor(m, 1));
          m = fmaxf(m, __shfl_xor(m, 2));
          if (m * exp2_of(e[i]) > kLimit) {
            const int now = exp_for(m);
            if (sub == 0) {
              change[q][64 * i + own] = now - e[i];
              changed[q] |= 1u << i;
              flag[step % 3] = 1;
            }
            e[i] = now;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const float scale = exp2_of(e[i]);
        u4 hi, lo;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          unsigned h, l;
          split2(v[i][2 * j] * scale, v[i][2 * j + 1] * scale, &h, &l);
          hi[j] = h;
          lo[j] = l;
        }
        const int at = slot_at(64 * i + own, sub);
        *reinterpret_cast<u4*>(la + at) = hi;
        *reinterpret_cast<u4*>(la + kOne + at) = lo;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int p = 0; p < PA; ++p)
          *reinterpret_cast<u4*>(la + p * kOne + slot_at(64 * i + own, sub)) = ra[f][i].v[p];
    }
  };
  auto before = [&](int step) {
    if constexpr (S == kFloat) {
      if (flag[step % 3]) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int d = change[step & 1][kTile / 2 * wm + 32 * i + sum_row(lane, r)];
#pragma unroll
            for (int j = 0; j < NB; ++j) acc.v[i][j][r] = ldexpf(acc.v[i][j][r], d);
          }
      }
    }
  };
  const bool live = c0 + kTile / 2 * wn < a.kout && kTile / 2 * wm < t.count;
  Part<NB, PA> fa[2];
  Part<NB, PB> fb[2];
  auto read = [&](auto half, int step) {
    constexpr int ks = decltype(half)::value;
    if (!live) return;
    load_part(fa[ks], lds + (step & 1) * kHalfLds + wm * (kTile / 2) * kRowBytes, kOne, lane, ks);
    const char* lb = lds + (step & 1) * kHalfLds + PA * kOne + wn * (kTile / 2) * kRowBytes;
    if constexpr (W == kEntries)
      load_part_turned(fb[ks], lb, kOne, lane, ks);
    else
      load_part(fb[ks], lb, kOne, lane, ks);
  };
  auto multiply = [&](auto half) {
    constexpr int ks = decltype(half)::value;
    if (live) multiply_parts<kBf>(acc, fa[ks], fb[ks]);
  };
  run_steps<kNear, kFar>(a.w.steps, near, far, put, read, before, multiply);

  // outputs through LDS, so that rows are written in one piece
  if (S == kFloat && sub == 0)
#pragma unroll
    for (int i = 0; i < NB; ++i) row_exp[64 * i + own] = e[i];
  float* stage = reinterpret_cast<float*>(lds);
  constexpr int kLanes = kTile / 4, kRowsOnce = kThreads / kLanes;   // lanes a row, rows at a time
  const int quad = tid % kLanes, c = c0 + quad * 4;
  const T* bias = a.bias ? static_cast<const T*>(a.bias) + int64_t(t.group) * a.kout : nullptr;
  float bq[4];
  int eq[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    bq[j] = bias && c + j < a.kout ? to_f32(bias[c + j]) : 0.0f;
    if (S == kFloat) eq[j] = a.w.exps[set * a.w.cols_pad + c + j];
  }
  const bool whole = c + 4 <= a.kout;
#pragma unroll 1
  for (int h = 0; h < kTile; h += kStageRows) {
    if (h > 0) __syncthreads();
    if (kStageRows == kTile || kTile / 2 * wm == h)
      stage_sums(stage, acc, kStageRows == kTile ? kTile / 2 * wm : 0, kTile / 2 * wn, lane, 1.0f);
    __syncthreads();
    if (c >= a.kout) continue;
    constexpr int kBatch = 4;   // rows in flight
    const int last = t.count - h < kStageRows ? t.count - h : kStageRows;
#pragma unroll 1
    for (int r0 = tid / kLanes; r0 < last; r0 += kRowsOnce * kBatch) {
      int64_t row[kBatch];
      Pack<T, 4> res[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int r = r0 + kRowsOnce * k;
        row[k] = r < last ? row_of[h + r] : -1;
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
        if (row[k] < 0) continue;
        const int r = r0 + kRowsOnce * k;
        const v4f s = *reinterpret_cast<const v4f*>(stage + stage_at<NB>(r, quad * 4));
        const int er = S == kFloat || row_scaled<T, S> ? row_exp[h + r] : 0;
        Pack<T, 4> py, pz;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float z = S == kFloat || row_scaled<T, S> ? ldexpf(s[j], -er - eq[j]) : s[j];
          z += bq[j];
          float y = a.silu ? z * logistic(z) : z;
          if (a.residual) y += to_f32(res[k].v[j]);
          py.v[j] = from_f32<T>(y);
          pz.v[j] = from_f32<T>(z);
        }
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
}

// ---------------------------------------------------------------------------
// Many float32 rows times weights: 128 rows x up to 384 columns a workgroup
// ---------------------------------------------------------------------------

// Rows come from HBM with some 2 us of latency, and a compute unit needs 37 KB of
// them in flight for its share of the bandwidth.  Tiles of 128 columns each fetch
// the same rows; here a workgroup of eight waves, one a compute unit, fetches a row
// once for up to 384 columns.  A wave forms 64 x 96 outputs, so LDS is read 2/3 as
// often for a product too, and a float32 step is 1 us of the matrix cores, three
// of which cover the latency.  1,000,188 rows of 384 -> 384 with SiLU, z and a residual:
// 1,660 us (1,570 to 1,750), 0.53 PFLOP/s of float16 products, 6.3 GB at 3.6 TB/s, of
// which the residual's rows, read again from HBM, are 340 us.  Matrix cores are busy
// 25 %, LDS 24 %, vector instructions 40 %, and the clock is 1.92 GHz; on zeros, which
// draw less power, 1,300 us.
constexpr int kWideThreads = 512, kWideRows = 128, kWideBlocks = 12;   // blocks of 32 columns

__global__ void __launch_bounds__(kWideThreads, 2) grouped_wide_kernel(RowsArgs a) {
  constexpr int NT = kWideBlocks / 4;
  constexpr int kOneA = kWideRows * kRowBytes, kOneB = kWideBlocks * 32 * kRowBytes;
  constexpr int kHalfLds = 2 * kOneA + 2 * kOneB;
  __shared__ __attribute__((aligned(16))) char lds[2 * kHalfLds];
  __shared__ int32_t row_of[kWideRows];      // -1: nothing is stored
  __shared__ int32_t change[2][kWideRows];   // exponent that a row's sums are to move by
  __shared__ int32_t row_exp[kWideRows];
  __shared__ int32_t flag[3];

  const int all_blocks = (a.kout + 31) / 32;
  const int col_tiles = (all_blocks + kWideBlocks - 1) / kWideBlocks;
  const int each = (all_blocks + col_tiles - 1) / col_tiles;   // blocks of a tile
  const int64_t total = int64_t(*a.n_tiles) * col_tiles;
  if (blockIdx.x >= total) return;
  const int64_t work = xcd_block(blockIdx.x, total);
  const RowTile t = a.tiles[work / col_tiles];
  const int b0 = static_cast<int>(work % col_tiles) * each, c0 = b0 * 32;
  const int blocks = all_blocks - b0 < each ? all_blocks - b0 : each;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
  float* out = static_cast<float*>(a.out);
  float* zout = static_cast<float*>(a.zout);

  if (t.group == a.n_groups) {   // rows of no group
    const int width = a.kout - c0 < blocks * 32 ? a.kout - c0 : blocks * 32;
    for (int i = tid; i < t.count * width; i += kWideThreads) {
      const int64_t row = row_at(a.order, t.first + i / width, a.n);
      if (row < 0) continue;
      out[row * a.kout + c0 + i % width] = 0.0f;
      if (zout) zout[row * a.kout + c0 + i % width] = 0.0f;
    }
    return;
  }

  // this thread's row and its eight entries of a step; rows past the tile repeat
  // its last one, and nothing of them is stored
  const int sub = tid & 3, own = tid / 4;
  const char* row_p;
  int last;
  {
    const int r = own < t.count ? own : t.count - 1;
    const int64_t to = row_at(a.order, t.first + r, a.n);
    if (sub == 0) row_of[own] = own < t.count ? static_cast<int32_t>(to) : -1;
    const int64_t row = a.by_place ? t.first + r : to < 0 ? 0 : to;
    row_p = static_cast<const char*>(a.in) + row * a.ldin * 4;
    last = last_of(a.n, a.ldin, a.by_place ? static_cast<int>(a.ldin) : a.kin, row);
  }
  const int64_t set = a.w.set_of(t.group, t.first - int64_t(t.part) * kWideRows);
  const char* wsrc = a.w.planes + set * a.w.steps * a.w.step_bytes() + int64_t(c0) * kRowBytes;
  const int64_t wplane = int64_t(a.w.cols_pad) * kRowBytes;

  constexpr int kFar = 2;
  Raw<kFloat> ra[kFar];
  u4 rb[2][NT];
  auto far = [&](auto turn, int step) {
    constexpr int q = decltype(turn)::value;
    const bool in = step < a.w.steps;   // past the end: one line of the weights
    const int k = step * kDepth + sub * 8;
    load_raw<kFloat>(ra[q], in ? row_p : wsrc, 0, !in ? 0 : k < last ? k : last);
  };
  // slots i 512 + tid of the tile's columns; those past them: one line
  unsigned slot_of_b[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const unsigned idx = i * kWideThreads + tid;
    slot_of_b[i] = idx < unsigned(blocks) * 128 ? idx * 16 : 0;
  }
  auto near = [&](auto, int step) {
    const bool in = step < a.w.steps;
    const char* src = in ? wsrc + step * a.w.step_bytes() : wsrc;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < NT; ++i)
        rb[p][i] = *reinterpret_cast<const u4*>(src + p * wplane + size_t(in ? slot_of_b[i] : 0));
  };

  v16f acc[2][NT];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = v16f{};
  int e = kFirstExp;
  bool changed[2] = {false, false};
  if (tid < 2 * kWideRows) change[tid / kWideRows][tid % kWideRows] = 0;
  if (tid < 3) flag[tid] = 0;
  __syncthreads();

  auto put = [&](auto, auto far_turn, int step) {
    constexpr int f = decltype(far_turn)::value, q = f & 1;   // q: step % 2
    char* la = lds + q * kHalfLds;
    char* lb = la + 2 * kOneA;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < NT; ++i)
        *reinterpret_cast<u4*>(lb + p * kOneB + (i * kWideThreads + tid) * 16) = rb[p][i];
    if ((step + 1) * kDepth > a.kin) trim<kFloat>(ra[f], step * kDepth + sub * 8, last, a.kin);
    const int at = slot_at(own, sub);
    if (tid == 0) flag[(step + 1) % 3] = 0;
    if (changed[q]) {   // two steps ago; its readers are past it
      change[q][own] = 0;
      changed[q] = false;
    }
    float v[8];
    float m = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned bits = ra[f].v[j / 4][j % 4];
      v[j] = __builtin_bit_cast(float, bits);
      m = fmaxf(m, fabsf(v[j]));
    }
    if (__ballot(m * exp2_of(e) > kLimit) != 0) {   // a row has outgrown its scale: rare past the first step
      m = fmaxf(m, __shfl_xor(m, 1));
      m = fmaxf(m, __shfl_xor(m, 2));
      if (m * exp2_of(e) > kLimit) {
        const int now = exp_for(m);
        if (sub == 0) {
          change[q][own] = now - e;
          changed[q] = true;
          flag[step % 3] = 1;
        }
        e = now;
      }
    }
    const float scale = exp2_of(e);
    u4 hi, lo;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      unsigned h, l;
      split2(v[2 * j] * scale, v[2 * j + 1] * scale, &h, &l);
      hi[j] = h;
      lo[j] = l;
    }
    *reinterpret_cast<u4*>(la + at) = hi;
    *reinterpret_cast<u4*>(la + kOneA + at) = lo;
  };
  auto before = [&](int step) {
    if (!flag[step % 3]) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = change[step & 1][64 * wm + 32 * i + sum_row(lane, r)];
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j][r] = ldexpf(acc[i][j][r], d);
      }
  };
  // this wave's blocks wn, wn + 4, ..
  const int mine = 64 * wm >= t.count || wn >= blocks ? 0 : (blocks - wn + 3) / 4;
  Part<2, 2> fa[2];
  Part<1, 2> fb[2][NT];
  auto read = [&](auto half, int step) {
    constexpr int ks = decltype(half)::value;
    if (mine == 0) return;
    const char* la = lds + (step & 1) * kHalfLds + wm * 64 * kRowBytes;
    const char* lb = lds + (step & 1) * kHalfLds + 2 * kOneA + wn * 32 * kRowBytes;
    load_part(fa[ks], la, kOneA, lane, ks);
#pragma unroll
    for (int j = 0; j < NT; ++j) load_part(fb[ks][j], lb + j * 128 * kRowBytes, kOneB, lane, ks);
  };
  auto multiply = [&](auto half) {
    constexpr int ks = decltype(half)::value;
    if (mine == 0) return;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int p = 2; p >= 0; --p)   // the small products first
#pragma unroll
        for (int i = 0; i < 2; ++i)
          acc[i][j] = mfma<false>(fa[ks].v[i][p == 2], fb[ks][j].v[0][p == 1], acc[i][j]);
  };
  run_steps<1, kFar>(a.w.steps, near, far, put, read, before, multiply);

  if (sub == 0) row_exp[own] = e;
  __syncthreads();
  // outputs from the registers: a lane has a column, 32 of them are 128 bytes of a row
  const float* bias = a.bias ? static_cast<const float*>(a.bias) + int64_t(t.group) * a.kout : nullptr;
  const float* res = static_cast<const float*>(a.residual);
  if (mine == 0) return;
  // sixteen sums (i, j) at a time; the residual's entries one group ahead
  float rv[2][16];
  auto fetch_residual = [&](auto turn, int i, int j) {
    constexpr int q = decltype(turn)::value;
    if (!res) return;
    int c = c0 + (wn + 4 * (j < mine ? j : mine - 1)) * 32 + (lane & 31);
    c = c < a.kout ? c : a.kout - 1;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = row_of[64 * wm + 32 * i + sum_row(lane, r)];
      rv[q][r] = res[int64_t(row < 0 ? 0 : row) * a.ldres + c];
    }
  };
  auto store = [&](auto part, int j, const v16f& sums, float bv, int ec) {
    constexpr int i = decltype(part)::value;
    const int c = c0 + (wn + 4 * j) * 32 + (lane & 31);
    const bool in = c < a.kout;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      float y[2], z[2];
      int row[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int rl = 64 * wm + 32 * i + sum_row(lane, r + q);
        row[q] = row_of[rl];
        z[q] = ldexpf(sums[r + q], -row_exp[rl] - ec) + bv;
        y[q] = a.silu ? z[q] * logistic(z[q]) : z[q];
        if (res) y[q] += rv[i][r + q];
      }
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (in && row[q] >= 0) {
          out[int64_t(row[q]) * a.kout + c] = y[q];
          if (zout) zout[int64_t(row[q]) * a.kout + c] = z[q];
        }
    }
  };
  fetch_residual(Const<0>{}, 0, 0);
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    if (j >= mine) continue;
    const int c = c0 + (wn + 4 * j) * 32 + (lane & 31);
    const float bv = bias ? bias[c < a.kout ? c : a.kout - 1] : 0.0f;
    const int ec = a.w.exps[set * a.w.cols_pad + c];
    fetch_residual(Const<1>{}, 1, j);
    store(Const<0>{}, j, acc[0][j], bv, ec);
    fetch_residual(Const<0>{}, 0, j + 1);
    store(Const<1>{}, j, acc[1][j], bv, ec);
  }
}

// ---------------------------------------------------------------------------
// Gradients of the weights
// ---------------------------------------------------------------------------

// The slot of a block's sums: its number or, where that takes less room, the number that
// its group would start at in blocks of half as many rows, and on from there.  Groups of
// several blocks, P over more than (P - 1) ``rows`` places, then do not meet, and end
// below 2 n / rows.
struct Slots {
  int rows, by_start;
  __host__ __device__ int64_t of(int64_t begin, int part) const {
    return static_cast<uint32_t>(2 * begin) / static_cast<uint32_t>(rows) + int64_t(part);
  }
};

struct OuterArgs {
  const int32_t* order;
  int64_t n;
  const RowTile* blocks;
  const int32_t* n_blocks;
  int k, m;
  const void* x;      // by row
  int64_t ldx;
  const void* dz;     // by row, or by place (its second plane n lddz entries on)
  int64_t lddz;
  int by_place;
  const int32_t* dz_exps;   // row_scaled: the rows' exponents, by place
  void* dw;           // null: not formed
  void* db;
  float* parts;       // [slot][k][m] where a group has several blocks
  float* db_parts;    // [slot][m]
  Slots slots;
};

constexpr int kOuterTile = kSide<2>;

// this workgroup's tile: columns r0 .. of x and c0 .. of dz over a block of rows;
// false past the last
struct OuterTile {
  RowTile t;
  int64_t slot;
  int r0, c0;
};
__device__ inline bool outer_tile(const OuterArgs& a, OuterTile& o) {
  const int row_tiles = a.dw ? (a.k + kOuterTile - 1) / kOuterTile : 1;
  const int col_tiles = (a.m + kOuterTile - 1) / kOuterTile;
  const int64_t total = int64_t(*a.n_blocks) * row_tiles * col_tiles;
  if (blockIdx.x >= total) return false;
  // the tiles of a block of rows follow each other on one XCD
  const int64_t work = xcd_block(blockIdx.x, total);
  const int64_t block = work / (row_tiles * col_tiles);
  o.t = a.blocks[block];
  o.slot = a.slots.by_start ? a.slots.of(o.t.first - int64_t(o.t.part) * a.slots.rows, o.t.part) : block;
  o.r0 = static_cast<int>(work / col_tiles % row_tiles) * kOuterTile;
  o.c0 = static_cast<int>(work % col_tiles) * kOuterTile;
  return true;
}

// sums of a tile, scaled by 2^-(row exponent + column exponent) or by 2^-e_all, to dW
// where no other block adds to the group, else to the block's own sums
template <class T>
__device__ inline void store_outer(const OuterArgs& a, const OuterTile& o, const Sums<2>& acc,
                                   const int32_t* exps, int e_all = 0) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave >> 1, wn = wave & 1;
  const bool whole = o.t.parts == 1;
  T* dw = static_cast<T*>(a.dw) + int64_t(o.t.group) * a.k * a.m;
  float* part = a.parts + o.slot * a.k * a.m;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int cl = 64 * wn + 32 * j + (lane & 31), c = o.c0 + cl;
      const int ec = exps ? exps[kOuterTile + cl] : 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int rl = 64 * wm + 32 * i + sum_row(lane, r), row = o.r0 + rl;
        if (row >= a.k || c >= a.m) continue;
        float v = acc.v[i][j][r];
        v = ldexpf(v, exps ? -exps[rl] - ec : -e_all);
        if (whole)
          dw[int64_t(row) * a.m + c] = from_f32<T>(v);
        else
          part[int64_t(row) * a.m + c] = v;
      }
    }
}
template <class T>
__device__ inline void store_bias(const OuterArgs& a, const OuterTile& o, int col, float v) {
  if (o.c0 + col >= a.m) return;
  if (o.t.parts == 1)
    static_cast<T*>(a.db)[int64_t(o.t.group) * a.m + o.c0 + col] = from_f32<T>(v);
  else
    a.db_parts[o.slot * a.m + o.c0 + col] = v;
}

// float32.  A wave fetches 64 columns of one operand, so a lane has a column of a
// step, and its scale, to itself.
struct Column {
  float v[kDepth];
};

// the row of place first + lane % 32, -1 past ``end``
__device__ inline int look_up(const int32_t* order, int64_t n, int64_t first, int64_t end) {
  const int64_t place = first + (threadIdx.x & 31);
  const int64_t at = place < end ? place : end - 1;
  const int64_t row = order ? order[at] : at;   // without a condition
  return place < end && row >= 0 && row < n ? static_cast<int>(row) : -1;
}
// Column ``col`` of 32 rows, a lane holding the number of one.  The row of a load
// is the same for all lanes, so its address is scalar work.
__device__ inline void load_column(Column& r, const float* base, int64_t ld, int row, int col) {
  const int at = row < 0 ? 0 : row;
#pragma unroll
  for (int i = 0; i < kDepth; ++i) r.v[i] = (base + __builtin_amdgcn_readlane(at, i) * ld)[col];
}
// the sum of N entries as a tree
template <int N>
__device__ inline float tree_sum(const float* v) {
  if constexpr (N == 1)
    return v[0];
  else
    return tree_sum<N / 2>(v) + tree_sum<N / 2>(v + N / 2);
}
// zeros for the rows that are not there
__device__ inline void clear_column(Column& r, int row) {
  if (__ballot(row < 0) == 0) return;
#pragma unroll
  for (int i = 0; i < kDepth; ++i) r.v[i] = __builtin_amdgcn_readlane(row, i) < 0 ? 0.0f : r.v[i];
}

// float32: 31,250 rows of 541 x 384 in 118 groups 143 us (0.27 PFLOP/s of float16
// products, matrix cores busy 12 %; a block's 15 tiles read x three and dz five times, from L2), 4,000 rows in
// 5 groups 27 us for four steps a tile: the latencies of its start and end.
__global__ void __launch_bounds__(kThreads, 2) grouped_outer_kernel(OuterArgs a) {
  constexpr int kOne = kPlane<2>, kHalfLds = 4 * kOne;
  __shared__ __attribute__((aligned(16))) char lds[2 * kHalfLds];
  // by column, x's then dz's: the exponent, and what it is to move by
  __shared__ int32_t exps[2 * kOuterTile], change[2][2 * kOuterTile];
  __shared__ int32_t flag[3];
  OuterTile o;
  if (!outer_tile(a, o)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  // waves 0 and 1 fetch x, 2 and 3 dz; columns past the last repeat it, and
  // nothing of them is stored
  const bool of_x = wave < 2;
  const int mine = 64 * (wave & 1) + lane;
  const int width = of_x ? a.k : a.m, at0 = of_x ? o.r0 : o.c0;
  const int col = at0 + mine < width ? at0 + mine : width - 1;
  const float* base = static_cast<const float*>(of_x ? a.x : a.dz);
  const int64_t ld = of_x ? a.ldx : a.lddz;
  const int32_t* order = !of_x && a.by_place ? nullptr : a.order;
  const int64_t end = o.t.first + o.t.count;
  const int steps = (o.t.count + kDepth - 1) / kDepth;
  const bool sums_bias = a.db && o.r0 == 0 && !of_x;

  // The rows of a step are looked up one fetch before its loads, and before
  // that fetch's own: loads arrive in order, so they are there in time without
  // the columns having to be.
  Column c[2];
  int row[2], next = look_up(order, a.n, o.t.first, end);
  auto fetch = [&](auto turn, int step) {
    constexpr int q = decltype(turn)::value;
    row[q] = next;
    next = look_up(order, a.n, o.t.first + int64_t(step + 1) * kDepth, end);
    const bool in = step < steps;   // past the end: one entry
    load_column(c[q], base, in ? ld : 0, row[q], in ? col : 0);
  };
  Sums<2> acc;
  acc.clear();
  int e = kFirstExp;
  bool changed[2] = {false, false};
  double bias = 0.0;   // a step's sum at a time: roundings of many rows can all go one way
  change[0][tid] = change[1][tid] = 0;
  if (tid < 3) flag[tid] = 0;
  __syncthreads();
  auto put = [&](auto turn, auto, int step) {
    constexpr int q = decltype(turn)::value;
    clear_column(c[q], row[q]);
    if (sums_bias) bias += tree_sum<kDepth>(c[q].v);
    if (!a.dw) return;
    if (tid == 0) flag[(step + 1) % 3] = 0;
    if (changed[q]) {   // two steps ago; its readers are past it
      change[q][tid] = 0;
      changed[q] = false;
    }
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kDepth; ++i) m = fmaxf(m, fabsf(c[q].v[i]));
    if (m * exp2_of(e) > kLimit) {   // the column has outgrown its scale
      const int now = exp_for(m);
      change[q][tid] = now - e;
      changed[q] = true;
      flag[step % 3] = 1;
      e = now;
    }
    const float scale = exp2_of(e);
    char* to = lds + q * kHalfLds + (of_x ? 0 : 2 * kOne);
#pragma unroll
    for (int s = 0; s < kDepth / 8; ++s) {
      u4 hi, lo;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unsigned h, l;
        split2(c[q].v[8 * s + 2 * j] * scale, c[q].v[8 * s + 2 * j + 1] * scale, &h, &l);
        hi[j] = h;
        lo[j] = l;
      }
      *reinterpret_cast<u4*>(to + slot_at(mine, s)) = hi;
      *reinterpret_cast<u4*>(to + kOne + slot_at(mine, s)) = lo;
    }
  };
  auto before = [&](int step) {
    if (!flag[step % 3]) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = change[step & 1][64 * wm + 32 * i + sum_row(lane, r)];
#pragma unroll
        for (int j = 0; j < 2; ++j)
          acc.v[i][j][r] =
              ldexpf(acc.v[i][j][r], d + change[step & 1][kOuterTile + 64 * wn + 32 * j + (lane & 31)]);
      }
  };
  const bool live = a.dw && o.r0 + 64 * wm < a.k && o.c0 + 64 * wn < a.m;
  Part<2, 2> fa[2], fb[2];
  auto read = [&](auto half, int step) {
    constexpr int ks = decltype(half)::value;
    if (!live) return;
    load_part(fa[ks], lds + (step & 1) * kHalfLds + wm * 64 * kRowBytes, kOne, lane, ks);
    load_part(fb[ks], lds + (step & 1) * kHalfLds + 2 * kOne + wn * 64 * kRowBytes, kOne, lane, ks);
  };
  auto multiply = [&](auto half) {
    constexpr int ks = decltype(half)::value;
    if (live) multiply_parts<false>(acc, fa[ks], fb[ks]);
  };
  run_steps<2, 2>(steps, fetch, [](auto, int) {}, put, read, before, multiply);

  if (a.dw) {
    exps[tid] = e;
    __syncthreads();
    store_outer<float>(a, o, acc, exps);
  }
  if (sums_bias) store_bias<float>(a, o, mine, static_cast<float>(bias));
}

// Half types need no scale of their columns, so the rows go to LDS as they come, eight columns a
// lane, and transposing reads turn them: 6 loads a lane and step for dz in two
// planes, where a column a lane would take 64 loads of 2 or 4 bytes.  1,000,188
// bfloat16 rows of 541 x 384 in two planes: 1,690 us, 0.49 PFLOP/s, matrix cores busy
// 21 %, LDS 26 %, 7.7 GB past the L2s at 4.5 TB/s; five tiles across read dz
// five times and three x three times, from L2 as they run side by side.
//
// Rows of dz with exponents of their own are brought to the least one of the block on
// the way to LDS, by powers of two: exact, but for what falls below 2^-39 of the block's
// largest entry.
template <class T, Source SZ>
__global__ void __launch_bounds__(kThreads, 2) grouped_outer_half_kernel(OuterArgs a) {
  constexpr int PB = planes_of<SZ>, kOne = kPlane<2>, kHalfLds = (1 + PB) * kOne;
  constexpr bool kBf = std::is_same<T, __bf16>::value;
  __shared__ __attribute__((aligned(16))) char lds[2 * kHalfLds];
  __shared__ float bias_part[16][kOuterTile];
  OuterTile o;
  if (!outer_tile(a, o)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int64_t end = o.t.first + o.t.count;
  const int steps = (o.t.count + kDepth - 1) / kDepth;
  const bool sums_bias = a.db && o.r0 == 0;
  constexpr bool kScaled = row_scaled<T, SZ>;
  int e_all = 0;
  if constexpr (kScaled) {
    __shared__ int32_t least[kThreads / kWave];
    e_all = kNoExp;
    for (int i = tid; i < o.t.count; i += kThreads) e_all = min(e_all, a.dz_exps[o.t.first + i]);
    for (int d = kWave / 2; d > 0; d /= 2) e_all = min(e_all, __shfl_xor(e_all, d));
    if (lane == 0) least[wave] = e_all;
    __syncthreads();
    for (int i = 0; i < kThreads / kWave; ++i) e_all = min(e_all, least[i]);
  }
  // places tid / 16 and tid / 16 + 16 of a step, columns 8 (tid % 16) .. of both operands
  const int own = tid / 16, cg = tid % 16;
  const int xc = o.r0 + 8 * cg, zc = o.c0 + 8 * cg;
  const int64_t z_plane = a.n * a.lddz * 2;

  // the rows of a step, looked up one fetch before its loads, and before that
  // fetch's own (see above)
  int64_t next[2];
  int next_exp[2] = {}, exps[2][2];
  auto look = [&](int step) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t place = o.t.first + int64_t(step) * kDepth + 16 * i + own;
      const int64_t at = place < end ? place : end - 1;
      const int64_t row = a.order ? a.order[at] : at;   // without a condition
      next[i] = place < end && row >= 0 && row < a.n ? row : -1;
      if constexpr (kScaled) next_exp[i] = a.dz_exps[at];
    }
  };
  Raw<kHalf> rx[2][2];
  Raw<SZ> rz[2][2];
  int x_last[2][2], z_last[2][2];
  bool there[2][2];
  look(0);
  auto fetch = [&](auto turn, int step) {
    constexpr int q = decltype(turn)::value;
    int64_t row[2] = {next[0], next[1]};
    exps[q][0] = next_exp[0];
    exps[q][1] = next_exp[1];
    look(step + 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // places past the end: row 0, put as zeros
      there[q][i] = row[i] >= 0;
      const int64_t x_row = there[q][i] ? row[i] : 0;
      const int64_t z_row =
          !there[q][i] ? 0 : a.by_place ? o.t.first + int64_t(step) * kDepth + 16 * i + own : row[i];
      x_last[q][i] = last_of(a.n, a.ldx, a.k, x_row);
      z_last[q][i] = last_of(a.n, a.lddz, a.by_place ? static_cast<int>(a.lddz) : a.m, z_row);
      const char* px = static_cast<const char*>(a.x) + x_row * a.ldx * 2;
      const char* pz = static_cast<const char*>(a.dz) + z_row * a.lddz * 2;
      load_raw<kHalf>(rx[q][i], px, 0, xc < x_last[q][i] ? xc : x_last[q][i]);
      load_raw<SZ>(rz[q][i], pz, z_plane, zc < z_last[q][i] ? zc : z_last[q][i]);
    }
  };
  float bias[8] = {};
  auto put = [&](auto turn, auto, int) {
    constexpr int q = decltype(turn)::value;
    const u4 none = {0, 0, 0, 0};
    char* to = lds + q * kHalfLds + cg / 4 * 32 * kRowBytes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = slot_at(16 * i + own, cg % 4);
      if (o.r0 + kOuterTile > a.k) trim<kHalf>(rx[q][i], xc, x_last[q][i], a.k);
      if (o.c0 + kOuterTile > a.m) trim<SZ>(rz[q][i], zc, z_last[q][i], a.m);
      *reinterpret_cast<u4*>(to + at) = there[q][i] ? rx[q][i].v[0] : none;
      const int d = kScaled ? e_all - exps[q][i] : 0;   // never above 0
      const float own_scale = kScaled ? exp2_of(-exps[q][i]) : 1.0f;
#pragma unroll
      for (int p = 0; p < PB; ++p) {
        u4 v = there[q][i] ? rz[q][i].v[p] : none;
        if (sums_bias)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const unsigned w = v[j / 2];
            bias[j] += own_scale *
                       to_f32(__builtin_bit_cast(T, static_cast<unsigned short>(j & 1 ? w >> 16 : w & 0xffff)));
          }
        if constexpr (kScaled) {
          // 2^-24 is the least power that float16 has: the rest in a second product
          v8h f = __builtin_bit_cast(v8h, v) * static_cast<_Float16>(exp2_of(max(d, -24)));
          if (__ballot(d < -24) != 0)
            f *= static_cast<_Float16>(d < -48 ? 0.0f : exp2_of(min(d + 24, 0)));
          v = __builtin_bit_cast(u4, f);
        }
        *reinterpret_cast<u4*>(to + (1 + p) * kOne + at) = v;
      }
    }
  };
  Sums<2> acc;
  acc.clear();
  const bool live = a.dw && o.r0 + 64 * wm < a.k && o.c0 + 64 * wn < a.m;
  Part<2, 1> fa[2];
  Part<2, PB> fb[2];
  auto read = [&](auto half, int step) {
    constexpr int ks = decltype(half)::value;
    if (!live) return;
    load_part_turned(fa[ks], lds + (step & 1) * kHalfLds + wm * 64 * kRowBytes, kOne, lane, ks);
    load_part_turned(fb[ks], lds + (step & 1) * kHalfLds + kOne + wn * 64 * kRowBytes, kOne, lane, ks);
  };
  auto multiply = [&](auto half) {
    constexpr int ks = decltype(half)::value;
    if (live) multiply_parts<kBf>(acc, fa[ks], fb[ks]);
  };
  run_steps<2, 2>(steps, fetch, [](auto, int) {}, put, read, [](int) {}, multiply);

  if (a.dw) store_outer<T>(a, o, acc, nullptr, e_all);
  if (sums_bias) {
#pragma unroll
    for (int j = 0; j < 8; ++j) bias_part[own][8 * cg + j] = bias[j];
    __syncthreads();
    if (tid < kOuterTile) {
      float v = 0.0f;
      for (int i = 0; i < 16; ++i) v += bias_part[i][tid];
      store_bias<T>(a, o, tid, v);
    }
  }
}

// Entries i .. of the sum of a group's blocks in their order, kJoin a thread; in 64
// bits, since blocks can be thousands and of one sign.
constexpr int kJoin = 4;
template <class T>
__device__ inline void join_parts(const float* part, int count, int64_t each, int64_t i, T* out) {
  if (i + kJoin > each) {   // the last entries once more, as one vector (or each < kJoin)
    if (each < kJoin) {
      for (; i < each; ++i) {
        double s = 0.0;
        for (int b = 0; b < count; ++b) s += part[b * each + i];
        out[i] = from_f32<T>(static_cast<float>(s));
      }
      return;
    }
    i = each - kJoin;
  }
  part += i;
  double s[kJoin] = {};
  int b = 0;
  for (; b + 8 <= count; b += 8) {   // eight loads in flight
    Pack<float, kJoin> v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = *reinterpret_cast<const Pack<float, kJoin>*>(part + (b + k) * each);
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
      for (int j = 0; j < kJoin; ++j) s[j] += v[k].v[j];
  }
  for (; b < count; ++b) {
    const Pack<float, kJoin> v = *reinterpret_cast<const Pack<float, kJoin>*>(part + b * each);
#pragma unroll
    for (int j = 0; j < kJoin; ++j) s[j] += v.v[j];
  }
  Pack<T, kJoin> r;
#pragma unroll
  for (int j = 0; j < kJoin; ++j) r.v[j] = from_f32<T>(static_cast<float>(s[j]));
  *reinterpret_cast<Pack<T, kJoin>*>(out + i) = r;
}

// The blocks of the groups that have several, added up: dW, then db (null: not
// formed).  Bound by HBM where blocks are many (a million rows, 541 x 384: 244 blocks,
// 230 MB in 47 us), by its launch else (4,000 rows: 8 us).
template <class T>
__global__ void __launch_bounds__(kThreads) grouped_join_kernel(const int32_t* __restrict__ first_of,
                                                                const int64_t* __restrict__ ptr, int64_t n,
                                                                Slots slots, int64_t each_w, int64_t each_b,
                                                                const float* __restrict__ parts_w,
                                                                const float* __restrict__ parts_b,
                                                                T* __restrict__ dw, T* __restrict__ db) {
  const int g = blockIdx.y;
  const int64_t begin = clamp_place(ptr[g], n);   // beside the loads of first_of
  const int count = first_of[g + 1] - first_of[g];
  if (count < 2) return;
  const int64_t first = slots.by_start ? slots.of(begin, 0) : first_of[g];
  int64_t i = (int64_t(blockIdx.x) * kThreads + threadIdx.x) * kJoin;
  const int64_t of_w = dw ? align_up(each_w, kJoin) : 0;
  if (i < of_w)
    join_parts(parts_w + first * each_w, count, each_w, i, dw + g * each_w);
  else if (db && i - of_w < each_b)
    join_parts(parts_b + first * each_b, count, each_b, i - of_w, db + g * each_b);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

int64_t tiles_at_most(int64_t n, int n_groups, int64_t rows) {
  return n / rows + (n < n_groups + 1 ? n : n_groups + 1);
}

// whether products read planes of the weights, not the weights (WeightForm)
bool laid_out(const dpa4c_grouped& l) {
  return l.dtype == DPA4C_F32 || l.n_out < kLeastWidth || l.n >= int64_t(kLaidRows) * l.n_groups;
}

// The tile of rows times weights.  Wide: float32 with more than 256 columns,
// from two rounds of the 256 compute units on (1,000,188 x 384 -> 384: 1,600 us,
// 128 x 128 tiles 1,850; bfloat16 1,140 against 1,000, and 128 columns 3,600
// against 1,910: half types and few columns leave its columns or matrix cores
// idle).  Else 128 x 128 where such tiles fill the compute units, and 64 x 64.
enum TileKind { kSmallTile, kLargeTile, kWideTile };
TileKind tile_kind(const dpa4c_grouped& l, bool back) {
  const int cols = back ? l.k : l.n_out;
  if (l.dtype == DPA4C_F32 && cols > 256 && l.n >= 2 * 256 * kWideRows) return kWideTile;
  return cols > 64 && (l.n / 128) * ((cols + 127) / 128) >= 256 ? kLargeTile : kSmallTile;
}
int tile_rows(const dpa4c_grouped& l, bool back) {
  return tile_kind(l, back) == kSmallTile ? kSide<1> : kSide<2>;
}

// Rows of a block of dW: 4,096 workgroups in all, some rounds of the chip's 512
// resident ones, but no fewer than 512 rows, so that a block's sums are small
// beside its rows, and groups of a few hundred rows are one block, whose sums go
// straight to dW, and no more than 8,192, whose sums of one sign in float32 are off by
// 4e-5 at the most (70,000,000 equal rows: 8e-5 in blocks of 16,384).  Where even 512 give
// few workgroups 256, and 128.
int outer_rows(const dpa4c_grouped& l) {
  const int64_t tiles = ((l.k + kOuterTile - 1) / kOuterTile) * int64_t((l.n_out + kOuterTile - 1) / kOuterTile);
  if (l.n * tiles < 256 * 256) return 128;
  if (l.n * tiles < 512 * 512) return 256;
  const int64_t rows = align_up((l.n * tiles + 4095) / 4096, kDepth);
  return static_cast<int>(rows < 512 ? 512 : rows > 8192 ? 8192 : rows);
}

Weights weights_of(Arena& ar, const dpa4c_grouped& l, bool back) {
  Weights w{};
  const int depth = back ? l.n_out : l.k, cols = back ? l.k : l.n_out;
  w.steps = (depth + kDepth - 1) / kDepth;
  w.cols_pad = static_cast<int>(align_up(cols, kPad));
  w.planes_n = l.dtype == DPA4C_F32 ? 2 : 1;
  w.by_start = l.n < l.n_groups;
  if (!laid_out(l)) return w;
  const int64_t sets = std::min<int64_t>(l.n, l.n_groups);
  w.planes = ar.take<char>(sets * w.steps * w.step_bytes());
  w.exps = ar.take<int32_t>(l.dtype == DPA4C_F32 ? sets * w.cols_pad : 0);
  return w;
}

TileList list_of(Arena& ar, const dpa4c_grouped& l, int rows, bool rest) {
  TileList t;
  t.room = static_cast<int>(tiles_at_most(l.n, l.n_groups, rows));
  t.list = ar.take<RowTile>(t.room);
  t.first_of = ar.take<int32_t>(l.n_groups + 2);
  t.count = ar.take<int32_t>(1);
  t.rows = rows;
  t.rest = rest;
  return t;
}

// entries of a row of dz: rows start at multiples of 16 bytes
int pitch_of(const dpa4c_grouped& l) { return static_cast<int>(align_up(l.n_out, 8)); }

// x with rows of at least eight entries
struct Input {
  const void* at;
  int64_t ld;
};
int64_t wide_bytes(const dpa4c_grouped& l) {
  return l.k < kLeastWidth ? l.n * kLeastWidth * (l.dtype == DPA4C_F32 ? 4 : 2) : 0;
}
template <class T>
int widen(const dpa4c_grouped& l, void* room, Input* in, hipStream_t st) {
  *in = {l.x, l.ldx};
  if (l.k >= kLeastWidth) return 0;
  const int64_t grid = std::min<int64_t>((l.n * kLeastWidth + kThreads - 1) / kThreads, 1 << 20);
  grouped_widen_kernel<T><<<grid, kThreads, 0, st>>>(
      l.n, l.k, static_cast<const T*>(l.x), l.ldx, static_cast<T*>(room));
  DPA4C_HIP_TRY(hipGetLastError());
  *in = {room, kLeastWidth};
  return 0;
}

struct ForwardPlan {
  Weights w;
  TileList tiles;
  void* wide;
};
ForwardPlan plan_forward(const dpa4c_grouped& l, void* work, int64_t* bytes) {
  Arena ar{static_cast<char*>(work)};
  ForwardPlan p;
  p.w = weights_of(ar, l, false);
  p.tiles = list_of(ar, l, tile_rows(l, false), true);
  p.wide = ar.take<char>(wide_bytes(l));
  *bytes = ar.used;
  return p;
}

struct BackwardPlan {
  Weights w;
  TileList tiles, blocks;
  void *dz, *wide;
  int32_t* dz_exps;
  float *parts, *db_parts;
  Slots slots;
};
// dz is formed, by place
bool makes_dz(const dpa4c_grouped& l, bool z) { return l.n > 0 && (z || l.n_out < kLeastWidth); }
BackwardPlan plan_backward(const dpa4c_grouped& l, const Wanted& want, void* work, int64_t* bytes) {
  Arena ar{static_cast<char*>(work)};
  BackwardPlan p{};
  const bool outer = want.dw || want.db, made = makes_dz(l, want.z) && (want.dx || outer);
  if (want.dx) {
    p.w = weights_of(ar, l, true);
    p.tiles = list_of(ar, l, tile_rows(l, true), true);
  }
  const int rows = outer_rows(l);
  if (outer) p.blocks = list_of(ar, l, rows, false);
  p.dz = ar.take<float>(made ? l.n * pitch_of(l) : 0);   // or two planes of a half type
  p.dz_exps = ar.take<int32_t>(made && l.dtype == DPA4C_F16 ? l.n : 0);
  p.wide = ar.take<char>(outer ? wide_bytes(l) : 0);
  // only groups of more than ``rows`` rows have several blocks
  const int64_t blocks = tiles_at_most(l.n, l.n_groups, rows), ends = l.n > rows ? (2 * l.n + rows - 1) / rows : 0;
  p.slots = {rows, ends < blocks};
  p.parts = ar.take<float>(want.dw ? std::min(blocks, ends) * l.k * l.n_out : 0);
  p.db_parts = ar.take<float>(want.db ? std::min(blocks, ends) * l.n_out : 0);
  *bytes = ar.used;
  return p;
}

// the arguments of the preparing launch: the lists and, with ``w``, the weights
template <bool Back>
PrepArgs prepare_args(const dpa4c_grouped& l, const Weights* w, const TileList* tiles, const TileList* blocks) {
  PrepArgs a{};
  a.ptr = l.group_ptr;
  a.n_groups = l.n_groups;
  a.n = l.n;
  a.depth = Back ? l.n_out : l.k;
  a.cols = Back ? l.k : l.n_out;
  int64_t list = 0;
  if (w && laid_out(l)) {
    a.w = l.weight;
    a.out = *w;
    a.weight_blocks = int64_t(l.n_groups) * (w->cols_pad / kPrepCols);
  }
  if (tiles) {
    a.tiles = *tiles;
    list = tiles_at_most(l.n, l.n_groups, tiles->rows);
  }
  if (blocks) {
    a.blocks = *blocks;
    list = std::max(list, tiles_at_most(l.n, l.n_groups, blocks->rows));
  }
  a.list_blocks = std::max<int64_t>(1, std::min<int64_t>(64, list / kPrepThreads));
  return a;
}
template <class T, bool Back>
int prepare(const PrepArgs& a, hipStream_t st) {
  const int64_t grid = a.list_blocks + a.weight_blocks + a.clear_blocks + a.dz_blocks;
  grouped_prepare_kernel<T, Back>
      <<<grid, kPrepThreads, (a.n_groups + 2) * sizeof(int32_t), st>>>(a);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

template <class T, Source S, bool Back>
int run_rows(const dpa4c_grouped& l, const RowsArgs& a, const TileList& tiles, hipStream_t st) {
  constexpr WeightForm W = S == kFloat ? kLaid : Back ? kColumns : kEntries;
  const int64_t most = tiles_at_most(a.n, a.n_groups, tiles.rows);
  const int64_t small = most * ((a.kout + 63) / 64), large = most * ((a.kout + 127) / 128);
  const TileKind kind = tile_kind(l, Back);
  if (kind == kSmallTile && laid_out(l))
    grouped_rows_kernel<T, S, 1, kLaid><<<small, kThreads, 0, st>>>(a);
  else if (kind == kSmallTile)
    grouped_rows_kernel<T, S, 1, W><<<small, kThreads, 0, st>>>(a);
  else if (kind == kLargeTile && laid_out(l))
    grouped_rows_kernel<T, S, 2, kLaid><<<large, kThreads, 0, st>>>(a);
  else if (kind == kLargeTile)
    grouped_rows_kernel<T, S, 2, W><<<large, kThreads, 0, st>>>(a);
  else if constexpr (S == kFloat)
    grouped_wide_kernel<<<most * (((a.kout + 31) / 32 + kWideBlocks - 1) / kWideBlocks), kWideThreads, 0, st>>>(a);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

template <class T>
int run_outer(const dpa4c_grouped& l, const OuterArgs& a, const TileList& blocks, hipStream_t st) {
  const int64_t tiles = (a.dw ? (l.k + kOuterTile - 1) / kOuterTile : 1) *
                        int64_t((l.n_out + kOuterTile - 1) / kOuterTile);
  if (l.n > 0) {
    const int64_t grid = tiles_at_most(l.n, l.n_groups, blocks.rows) * tiles;
    if constexpr (sizeof(T) == 4)
      grouped_outer_kernel<<<grid, kThreads, 0, st>>>(a);
    else if (a.by_place)
      grouped_outer_half_kernel<T, kPair><<<grid, kThreads, 0, st>>>(a);
    else
      grouped_outer_half_kernel<T, kHalf><<<grid, kThreads, 0, st>>>(a);
    DPA4C_HIP_TRY(hipGetLastError());
  }
  const int64_t each_w = int64_t(l.k) * l.n_out;
  const int64_t all = (a.dw ? align_up(each_w, kJoin) : 0) + (a.db ? l.n_out : 0);
  const dim3 grid((all + kThreads * kJoin - 1) / (kThreads * kJoin), l.n_groups);
  grouped_join_kernel<T><<<grid, kThreads, 0, st>>>(blocks.first_of, l.group_ptr, l.n, a.slots, each_w, l.n_out, a.parts, a.db_parts,
                                                    static_cast<T*>(a.dw), static_cast<T*>(a.db));
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

}  // namespace

bool grouped_fits(const dpa4c_grouped& l) {
  auto up = [](int64_t x, int64_t by) { return (x + by - 1) / by; };
  const int64_t most = std::max(l.k, l.n_out);
  const int64_t prep = 64 + 4096 + l.n_groups * (up(most, kPad) * (kPad / kPrepCols) +
                                                 up(int64_t(l.k) * l.n_out, kClear));
  const int64_t rows = tiles_at_most(l.n, l.n_groups, kSide<1>) * up(most, kSide<1>);
  const int64_t outer = tiles_at_most(l.n, l.n_groups, outer_rows(l)) * up(l.k, kOuterTile) * up(l.n_out, kOuterTile);
  return grid_fits(prep, kPrepThreads) && grid_fits(rows, kThreads) && grid_fits(outer, kThreads);
}

int64_t grouped_forward_work(const dpa4c_grouped& l) {
  int64_t bytes;
  plan_forward(l, nullptr, &bytes);
  return bytes;
}

int64_t grouped_backward_work(const dpa4c_grouped& l, const Wanted& want) {
  int64_t bytes;
  plan_backward(l, want, nullptr, &bytes);
  return bytes;
}

int launch_grouped_forward(const dpa4c_grouped& l, const void* bias, bool silu, bool residual,
                           void* y, void* z, void* work, hipStream_t st) {
  if (l.n == 0) return 0;
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    int64_t bytes;
    const ForwardPlan p = plan_forward(l, work, &bytes);
    DPA4C_TRY((prepare<T, false>(prepare_args<false>(l, &p.w, &p.tiles, nullptr), st)));
    Input in;
    DPA4C_TRY(widen<T>(l, p.wide, &in, st));
    RowsArgs a{};
    a.order = l.order;
    a.n_groups = l.n_groups;
    a.n = l.n;
    a.tiles = p.tiles.list;
    a.n_tiles = p.tiles.count;
    a.kin = l.k;
    a.kout = l.n_out;
    a.in = in.at;
    a.ldin = in.ld;
    a.w = p.w;
    a.weight = l.weight;
    a.bias = bias;
    a.silu = silu;
    a.residual = residual ? l.x : nullptr;
    a.ldres = l.ldx;
    a.out = y;
    a.zout = z;
    return run_rows<T, sizeof(T) == 4 ? kFloat : kHalf, false>(l, a, p.tiles, st);
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
    const BackwardPlan p = plan_backward(l, {z != nullptr, dx != nullptr, dw != nullptr, db != nullptr}, work, &bytes);
    const int pitch = pitch_of(l);
    const bool made = makes_dz(l, z);
    PrepArgs pre = prepare_args<true>(l, rows ? &p.w : nullptr, rows ? &p.tiles : nullptr,
                                      outer ? &p.blocks : nullptr);
    if (outer) {
      pre.dw = dw;
      pre.db = db;
      const int64_t each = dw ? int64_t(l.k) * l.n_out : 1;
      pre.clear_blocks = int64_t(l.n_groups) * ((each + kClear - 1) / kClear);
    }
    if (made) {
      pre.order = l.order;
      pre.dy = dy;
      pre.ldy = ldy;
      pre.z = z;
      pre.ldz = ldz;
      pre.pitch = pitch;
      pre.dz = p.dz;
      pre.dz_exps = p.dz_exps;
      const int64_t each =
          l.n * (l.dtype == DPA4C_F16 ? lanes_of_dz(pitch) : pitch * int64_t(sizeof(T)) / 16);
      pre.dz_blocks = std::min<int64_t>((each + kPrepThreads - 1) / kPrepThreads, 4096);
    }
    DPA4C_TRY((prepare<T, true>(pre, st)));
    if (rows) {
      RowsArgs a{};
      a.order = l.order;
      a.n_groups = l.n_groups;
      a.n = l.n;
      a.tiles = p.tiles.list;
      a.n_tiles = p.tiles.count;
      a.kin = l.n_out;
      a.kout = l.k;
      a.in = made ? p.dz : dy;
      a.ldin = made ? pitch : ldy;
      a.by_place = made;
      a.in_exps = p.dz_exps;
      a.w = p.w;
      a.weight = l.weight;
      a.residual = residual ? dy : nullptr;
      a.ldres = ldy;
      a.out = dx;
      if (made)
        DPA4C_TRY((run_rows<T, kMade, true>(l, a, p.tiles, st)));
      else
        DPA4C_TRY((run_rows<T, kOwn, true>(l, a, p.tiles, st)));
    }
    if (outer) {
      OuterArgs a{};
      a.order = l.order;
      a.n = l.n;
      a.blocks = p.blocks.list;
      a.n_blocks = p.blocks.count;
      a.k = l.k;
      a.m = l.n_out;
      Input in{l.x, l.ldx};
      if (l.n > 0) DPA4C_TRY(widen<T>(l, p.wide, &in, st));
      a.x = in.at;
      a.ldx = in.ld;
      a.dz = made ? p.dz : dy;
      a.lddz = made ? pitch : ldy;
      a.by_place = made;
      a.dz_exps = p.dz_exps;
      a.dw = dw;
      a.db = db;
      a.parts = p.parts;
      a.db_parts = p.db_parts;
      a.slots = p.slots;
      DPA4C_TRY(run_outer<T>(l, a, p.blocks, st));
    }
    return 0;
  });
}

}  // namespace dpa4c
