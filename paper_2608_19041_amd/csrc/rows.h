// What the operators on grouped rows share: the rows of a group by place, tiles of
// them, and sums over a group's rows that are formed in blocks and then joined.
#pragma once

#include "tile.h"

namespace dpa4c {

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

namespace {

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
// Sums over the rows of a group
// ---------------------------------------------------------------------------

constexpr int kOuterTile = kSide<2>;

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
__global__ void __launch_bounds__(kTileThreads) grouped_join_kernel(const int32_t* __restrict__ first_of,
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
  int64_t i = (int64_t(blockIdx.x) * kTileThreads + threadIdx.x) * kJoin;
  const int64_t of_w = dw ? align_up(each_w, kJoin) : 0;
  if (i < of_w)
    join_parts(parts_w + first * each_w, count, each_w, i, dw + g * each_w);
  else if (db && i - of_w < each_b)
    join_parts(parts_b + first * each_b, count, each_b, i - of_w, db + g * each_b);
}

// ---------------------------------------------------------------------------
// Host
// ---------------------------------------------------------------------------

inline int64_t tiles_at_most(int64_t n, int n_groups, int64_t rows) {
  return n / rows + (n < n_groups + 1 ? n : n_groups + 1);
}

// Rows of a block of dW: 4,096 workgroups in all, some rounds of the chip's 512
// resident ones, but no fewer than 512 rows, so that a block's sums are small
// beside its rows, and groups of a few hundred rows are one block, whose sums go
// straight to dW, and no more than 8,192, whose sums of one sign in float32 are off by
// 4e-5 at the most (70,000,000 equal rows: 8e-5 in blocks of 16,384).  Where even 512 give
// few workgroups 256, and 128.
inline int outer_rows(int64_t n, int k, int m) {
  const int64_t tiles = ((k + kOuterTile - 1) / kOuterTile) * int64_t((m + kOuterTile - 1) / kOuterTile);
  if (n * tiles < 256 * 256) return 128;
  if (n * tiles < 512 * 512) return 256;
  const int64_t rows = align_up((n * tiles + 4095) / 4096, kDepth);
  return static_cast<int>(rows < 512 ? 512 : rows > 8192 ? 8192 : rows);
}

inline TileList list_of(Arena& ar, int64_t n, int n_groups, int rows, bool rest) {
  TileList t;
  t.room = static_cast<int>(tiles_at_most(n, n_groups, rows));
  t.list = ar.take<RowTile>(t.room);
  t.first_of = ar.take<int32_t>(n_groups + 2);
  t.count = ar.take<int32_t>(1);
  t.rows = rows;
  t.rest = rest;
  return t;
}

}  // namespace

}  // namespace dpa4c
