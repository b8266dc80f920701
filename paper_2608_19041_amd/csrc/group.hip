// Rows by group: a stable counting sort of small integer keys.
//
// place(r) = (rows of smaller groups) + (earlier rows of r's group).  Reads 4
// and writes 4 bytes a row; the counters stay in LDS, so the sort is bound by
// its launches up to some 10^5 rows and by memory latency beyond.
//
// A wave takes 64 rows at a time in row order.  Lanes with equal keys find each
// other by one ballot for each bit of the key, so a lane's rank among its peers
// is a population count, and no atomic's order enters the result.  A workgroup
// counts the keys of its rows, a wave at a time, turns the counts into starts
// and places the rows in a second pass over them (from L2).  More than one
// workgroup's rows are counted by a first launch; every workgroup of the second
// adds up the counts of those before it by itself, which costs the chip one
// more read of 4 (n_groups + 1) bytes a workgroup but no third launch.
#include <hip/hip_runtime.h>

#include "train.h"

namespace dpa4c {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
// Rows of a workgroup.  Up to kOneBlock one workgroup takes all of them in one
// launch; beyond, as many as keep 256 compute units busy at a million rows.
constexpr int64_t kBlockRows = 4096, kOneBlock = 8192;

__host__ __device__ inline int64_t sort_blocks(int64_t n) {
  return n <= kOneBlock ? 1 : (n + kBlockRows - 1) / kBlockRows;
}

// the group of a row; n_groups for ids outside the range
__device__ inline int key_of(const int32_t* group, int64_t r, int64_t n, int n_groups) {
  if (r >= n) return -1;
  const int g = group[r];
  return g >= 0 && g < n_groups ? g : n_groups;
}

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

// counts of this wave's keys into cnt[key]
__device__ inline void count_rows(const int32_t* group, int64_t n, int n_groups, int bits,
                                  int64_t first, int64_t last, int32_t* cnt) {
  const int lane = threadIdx.x & (kWave - 1);
  for (int64_t r = first; r < last; r += kWave) {
    const int key = key_of(group, r + lane, last, n_groups);
    const uint64_t m = peers_of(key, bits);
    if (key >= 0 && lane == __builtin_ctzll(m)) cnt[key] += __popcll(m);
    wave_sync();
  }
}

__global__ void __launch_bounds__(kThreads) group_count_kernel(const int32_t* __restrict__ group,
                                                               int64_t n, int n_groups, int bits,
                                                               int32_t* __restrict__ counts) {
  extern __shared__ int32_t sh[];   // [kWaves][n_groups + 1]
  const int g1 = n_groups + 1, wave = threadIdx.x / kWave;
  for (int i = threadIdx.x; i < kWaves * g1; i += kThreads) sh[i] = 0;
  __syncthreads();
  int64_t first, last;
  wave_rows(n, kBlockRows, blockIdx.x, wave, &first, &last);
  count_rows(group, n, n_groups, bits, first, last, sh + wave * g1);
  __syncthreads();
  for (int g = threadIdx.x; g < g1; g += kThreads) {
    int c = 0;
    for (int w = 0; w < kWaves; ++w) c += sh[w * g1 + g];
    counts[int64_t(blockIdx.x) * g1 + g] = c;
  }
}

// places the rows of a workgroup; counts = null: there is one workgroup only,
// which counts its rows first
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
  count_rows(group, n, n_groups, bits, first, last, sh + wave * g1);
  __syncthreads();
  // the rows of each group before this workgroup and in all (whole numbers:
  // the order of the additions does not matter)
  if (counts)
    for (int g = lane; g < g1; g += kWave) {
      int bef = 0, all = 0;
      for (int64_t b = wave; b < gridDim.x; b += kWaves) {
        const int c = counts[b * g1 + g];
        bef += b < blockIdx.x ? c : 0;
        all += c;
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
  int32_t* at = sh + wave * g1;
  for (int64_t r = first; r < last; r += kWave) {
    const int key = key_of(group, r + lane, last, n_groups);
    const uint64_t m = peers_of(key, bits);
    if (key >= 0) {
      const int rank = __popcll(m & ((uint64_t(1) << lane) - 1));
      const int base = at[key];
      order[total[key] + base + rank] = static_cast<int32_t>(r + lane);
      if (rank == 0) at[key] = base + __popcll(m);
    }
    wave_sync();
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
  if (blocks > 1) {
    counts = static_cast<int32_t*>(work);
    group_count_kernel<<<blocks, kThreads, lds, st>>>(group, n, n_groups, bits, counts);
    DPA4C_HIP_TRY(hipGetLastError());
  }
  group_place_kernel<<<blocks, kThreads, lds, st>>>(group, n, n_groups, bits,
                                                    blocks > 1 ? kBlockRows : n, counts, group_ptr,
                                                    order);
  DPA4C_HIP_TRY(hipGetLastError());
  return 0;
}

}  // namespace dpa4c
