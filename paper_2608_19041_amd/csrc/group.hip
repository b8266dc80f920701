// Rows by group: a stable counting sort of small integer keys.
//
// place(r) = (rows of smaller groups) + (earlier rows of r's group).  Reads 4
// and writes 4 bytes a row; the counters stay in LDS, so the sort is bound by
// its launches up to some 10^5 rows and by memory latency beyond.
//
// A wave takes 64 rows at a time in row order.  Lanes with equal keys find each
// other by one ballot for each bit of the key, so a lane's rank among its peers
// is a population count, and no atomic's order enters the result.  A workgroup
// ranks its rows, a wave's stretch at a time, turns the counts into starts and
// places the rows, whose keys and ranks stay in registers in between (up to
// kMostBlocks workgroups; beyond, stretches grow and are read again from L2).
// More than one workgroup's rows are counted by a first launch; every workgroup
// of the second adds up the counts of those before it by itself, which costs the
// chip one more read of 4 (n_groups + 1) bytes a pair of workgroups but no third
// launch.
#include <hip/hip_runtime.h>

#include "train.h"

namespace dpa4c {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
// Rows of a workgroup.  Up to kOneBlock one workgroup takes all of them in one
// launch; beyond, as many as keep 256 compute units busy at a million rows, and
// more from kMostBlocks workgroups on: the pairs of workgroups grow as their square.
constexpr int64_t kBlockRows = 4096, kOneBlock = 8192, kMostBlocks = 1024;
constexpr int kStrips = static_cast<int>(kBlockRows / (kWaves * kWave));     // of a wave, in registers
constexpr int kOneStrips = static_cast<int>(kOneBlock / (kWaves * kWave));

int64_t rows_of_block(int64_t n) {
  if (n <= kOneBlock) return n;
  return kBlockRows * ((n + kBlockRows * kMostBlocks - 1) / (kBlockRows * kMostBlocks));
}
int64_t sort_blocks(int64_t n) { return n <= kOneBlock ? 1 : (n + rows_of_block(n) - 1) / rows_of_block(n); }

// lanes of this wave with the same key (bits: enough for every key)
__device__ inline uint64_t peers_of(int key, int bits) {
  uint64_t m = __ballot(key >= 0);
  for (int b = 0; b < bits; ++b) {
    const uint64_t v = __ballot((key >> b) & 1);
    m &= ((key >> b) & 1) ? v : ~v;
  }
  return m;
}

// the stretch of rows [first, last) of this wave
__device__ inline void wave_rows(int64_t n, int64_t per_block, int64_t block, int wave,
                                 int64_t* first, int64_t* last) {
  const int64_t begin = block * per_block, end = begin + per_block < n ? begin + per_block : n;
  const int64_t strips = (end - begin + kWave - 1) / kWave;
  const int64_t per = (strips + kWaves - 1) / kWaves * kWave;
  *first = begin + wave * per < end ? begin + wave * per : end;
  *last = *first + per < end ? *first + per : end;
}

// LDS written by one lane of a wave is read by another in the next pass
__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// S strips of rows from r0: their keys (the group; n_groups for ids outside the
// range; -1 past ``last``) and their ranks, counted on in cnt[key]
template <int S>
__device__ inline void rank_rows(const int32_t* group, int n_groups, int bits, int64_t r0, int64_t last,
                                 int32_t* cnt, int (&key)[S], int (&rank)[S]) {
  if (r0 >= last) {
#pragma unroll
    for (int i = 0; i < S; ++i) key[i] = -1;
    return;
  }
  const int lane = threadIdx.x & (kWave - 1);
#pragma unroll
  for (int i = 0; i < S; ++i) {   // all in flight; past the last row it is read again
    const int64_t r = r0 + i * kWave + lane;
    key[i] = group[r < last ? r : last - 1];
  }
#pragma unroll
  for (int i = 0; i < S; ++i) {
    if (r0 + i * kWave >= last) {
      key[i] = -1;
      continue;
    }
    key[i] = r0 + i * kWave + lane >= last ? -1 : key[i] >= 0 && key[i] < n_groups ? key[i] : n_groups;
    const uint64_t m = peers_of(key[i], bits);
    if (key[i] >= 0) {
      const int before = cnt[key[i]], mine = __popcll(m & ((uint64_t(1) << lane) - 1));
      rank[i] = before + mine;
      if (mine == 0) cnt[key[i]] = before + __popcll(m);
    }
    wave_sync();
  }
}

__global__ void __launch_bounds__(kThreads) group_count_kernel(const int32_t* __restrict__ group,
                                                               int64_t n, int n_groups, int bits,
                                                               int64_t per_block,
                                                               int32_t* __restrict__ counts) {
  extern __shared__ int32_t sh[];   // [kWaves][n_groups + 1]
  const int g1 = n_groups + 1, wave = threadIdx.x / kWave;
  for (int i = threadIdx.x; i < kWaves * g1; i += kThreads) sh[i] = 0;
  __syncthreads();
  int64_t first, last;
  wave_rows(n, per_block, blockIdx.x, wave, &first, &last);
  int key[kStrips], rank[kStrips];
  for (int64_t r = first; r < last; r += kStrips * kWave)
    rank_rows(group, n_groups, bits, r, last, sh + wave * g1, key, rank);
  __syncthreads();
  for (int g = threadIdx.x; g < g1; g += kThreads) {
    int c = 0;
    for (int w = 0; w < kWaves; ++w) c += sh[w * g1 + g];
    counts[int64_t(blockIdx.x) * g1 + g] = c;
  }
}

// places the rows of a workgroup; counts = null: there is one workgroup only,
// which counts its rows first
template <int S>
__global__ void __launch_bounds__(kThreads) group_place_kernel(
    const int32_t* __restrict__ group, int64_t n, int n_groups, int bits, int64_t per_block,
    const int32_t* __restrict__ counts, int64_t* __restrict__ group_ptr,
    int32_t* __restrict__ order) {
  // [kWaves][n_groups + 1] counts, then places; [g1] totals, then starts; [g1] rows before
  extern __shared__ int32_t sh[];
  const int g1 = n_groups + 1, wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  int32_t* total = sh + kWaves * g1;
  int32_t* before = total + g1;
  for (int i = threadIdx.x; i < (kWaves + 2) * g1; i += kThreads) sh[i] = 0;
  __syncthreads();
  int64_t first, last;
  wave_rows(n, per_block, blockIdx.x, wave, &first, &last);
  int32_t* at = sh + wave * g1;
  const bool held = per_block <= S * kWaves * kWave;
  int key[S], rank[S];
  rank_rows(group, n_groups, bits, first, last, at, key, rank);
  for (int64_t r = first + S * kWave; r < last; r += S * kWave)
    rank_rows(group, n_groups, bits, r, last, at, key, rank);
  __syncthreads();
  // the rows of each group before this workgroup and in all (whole numbers:
  // the order of the additions does not matter)
  if (counts)
    for (int g = lane; g < g1; g += kWave) {
      int bef = 0, all = 0;
      constexpr int kFlight = 16;
      for (int b0 = wave; b0 < int(gridDim.x); b0 += kFlight * kWaves) {
        int c[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
          c[k] = counts[int64_t(min(b0 + k * kWaves, int(gridDim.x) - 1)) * g1 + g];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) {
          const int b = b0 + k * kWaves;
          bef += b < int(blockIdx.x) ? c[k] : 0;
          all += b < int(gridDim.x) ? c[k] : 0;
        }
      }
      atomicAdd(&before[g], bef);
      atomicAdd(&total[g], all);
    }
  __syncthreads();
  // a wave's start inside its group
  for (int g = threadIdx.x; g < g1; g += kThreads) {
    int run = before[g];
    for (int w = 0; w < kWaves; ++w) {
      const int c = sh[w * g1 + g];
      sh[w * g1 + g] = run;
      run += c;
    }
    if (!counts) total[g] = run;
  }
  __syncthreads();
  // starts of the groups: a scan by the first wave
  if (wave == 0) {
    int run = 0;
    for (int g0 = 0; g0 < g1; g0 += kWave) {
      const int g = g0 + lane;
      const int c = g < g1 ? total[g] : 0;
      int s = c;
      for (int d = 1; d < kWave; d *= 2) {
        const int v = __shfl_up(s, d);
        s += lane >= d ? v : 0;
      }
      if (g < g1) total[g] = run + s - c;
      run += __shfl(s, kWave - 1);
    }
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int g = threadIdx.x; g < g1; g += kThreads) group_ptr[g] = total[g];
  // held: a row's rank in its wave's stretch; else its place in the group, in a
  // second pass over the stretch
  for (int64_t r = first; r < last; r += S * kWave) {
    if (!held) rank_rows(group, n_groups, bits, r, last, at, key, rank);
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (key[i] >= 0)
        order[total[key[i]] + (held ? at[key[i]] : 0) + rank[i]] = static_cast<int32_t>(r + i * kWave + lane);
  }
}

}  // namespace

int64_t group_rows_work(int64_t n, int n_groups) {
  const int64_t blocks = sort_blocks(n);
  return blocks > 1 ? align_up(blocks * (n_groups + 1) * 4, 256) : 0;
}

int launch_group_rows(const int32_t* group, int64_t n, int n_groups, int64_t* group_ptr,
                      int32_t* order, void* work, hipStream_t st) {
  int bits = 0;
  while ((n_groups >> bits) != 0) ++bits;   // keys 0 .. n_groups
  const int64_t blocks = sort_blocks(n);
  const size_t lds = size_t(kWaves + 2) * (n_groups + 1) * 4;
  int32_t* counts = nullptr;
  const int64_t rows = rows_of_block(n);
  if (blocks > 1) {
    counts = static_cast<int32_t*>(work);
    group_count_kernel<<<blocks, kThreads, lds, st>>>(group, n, n_groups, bits, rows, counts);
    DPA4C_HIP_TRY(hipGetLastError());
    group_place_kernel<kStrips><<<blocks, kThreads, lds, st>>>(group, n, n_groups, bits, rows, counts,
                                                               group_ptr, order);
  } else {
    group_place_kernel<kOneStrips><<<1, kThreads, lds, st>>>(group, n, n_groups, bits, rows, nullptr,
                                                             group_ptr, order);
  }
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

}  // namespace dpa4c
