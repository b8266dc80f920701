// Grouped layers: rows of each group times the weights of the group, and the
// gradients of that.
#include <hip/hip_runtime.h>

#include "train.h"

namespace dpa4c {

namespace {

constexpr int kTile = 64, kStep = 16;   // a workgroup forms 64 x 64 outputs, 16 inputs at a time
constexpr int kThreads = 256;

__device__ inline float silu_factor(float z) { return 1.0f / (1.0f + __expf(-z)); }
// act'(z) for SiLU
__device__ inline float silu_slope(float z) {
  const float p = silu_factor(z);
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

// The tile ``t`` in the sequence of the tiles of ``rows`` places of all groups
// (and of the rest): its group, first place and count; count 0 past the last.
struct RowTile {
  int group;
  int64_t first;
  int count;
};
__device__ inline RowTile find_tile(const int64_t* ptr, int n_groups, int64_t n, int rows, int64_t t) {
  __shared__ RowTile found;
  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    if (lane == 0) found = {0, 0, 0};
    int64_t run = 0;
    for (int g0 = 0; g0 <= n_groups; g0 += kWave) {
      const int g = g0 + lane;
      Span s{0, 0};
      if (g <= n_groups) s = span_of(ptr, g, n_groups, n);
      const int64_t mine = (s.end - s.begin + rows - 1) / rows;
      int64_t sum = mine;
      for (int d = 1; d < kWave; d *= 2) {
        const int64_t v = __shfl_up(sum, d);
        sum += lane >= d ? v : 0;
      }
      const int64_t at = run + sum - mine;
      if (t >= at && t < at + mine) {
        found.group = g;
        found.first = s.begin + (t - at) * rows;
        found.count = static_cast<int>(s.end - found.first < rows ? s.end - found.first : rows);
      }
      run += __shfl(sum, kWave - 1);
    }
  }
  __syncthreads();
  return found;
}

__device__ inline int64_t row_at(const int32_t* order, int64_t place, int64_t n) {
  const int64_t r = order ? order[place] : place;
  return r >= 0 && r < n ? r : -1;
}

// 4 x 4 outputs a thread: acc += a[k][row]^T b[k][col]
__device__ inline void tile_product(const float (*a)[kTile + 4], const float (*b)[kTile + 4],
                                    float (*acc)[4]) {
  const int tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
#pragma unroll
  for (int k = 0; k < kStep; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] += a[k][tr + i] * b[k][tc + j];
}

// y = act(x W + b) (+ x), or dx = dz W^T (+ dy) with dz = dy act'(z): inputs
// are [n][kin] rows, outputs [n][kout]; W is [kin][kout], or [kout][kin] with
// Back.
template <class T, bool Back>
__global__ void __launch_bounds__(kThreads) grouped_rows_kernel(
    const int64_t* __restrict__ ptr, const int32_t* __restrict__ order, int n_groups, int64_t n,
    int kin, int kout, const T* __restrict__ in, int64_t ldin, const T* __restrict__ zin,
    int64_t ldz, const T* __restrict__ w, const T* __restrict__ bias, int silu, int residual,
    T* __restrict__ out, T* __restrict__ zout) {
  __shared__ float a[kStep][kTile + 4], b[kStep][kTile + 4];
  const RowTile t = find_tile(ptr, n_groups, n, kTile, blockIdx.x);
  if (t.count == 0) return;
  const int col0 = blockIdx.y * kTile;
  const bool live = t.group < n_groups;
  float acc[4][4] = {};
  if (live) {
    const T* wg = w + int64_t(t.group) * kin * kout;
    for (int k0 = 0; k0 < kin; k0 += kStep) {
      for (int i = threadIdx.x; i < kTile * kStep; i += kThreads) {
        const int r = i / kStep, k = k0 + i % kStep;
        const int64_t row = r < t.count ? row_at(order, t.first + r, n) : -1;
        float v = 0.0f;
        if (row >= 0 && k < kin) {
          v = to_f32(in[row * ldin + k]);
          if (Back && zin) v *= silu_slope(to_f32(zin[row * ldz + k]));
        }
        a[i % kStep][r] = v;
        const int kb = Back ? i % kStep : i / kTile, c = Back ? i / kStep : i % kTile;
        const int kk = k0 + kb, cc = col0 + c;
        b[kb][c] = kk < kin && cc < kout
                       ? to_f32(wg[Back ? int64_t(cc) * kin + kk : int64_t(kk) * kout + cc])
                       : 0.0f;
      }
      __syncthreads();
      tile_product(a, b, acc);
      __syncthreads();
    }
  }
  const int tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
  for (int i = 0; i < 4; ++i) {
    const int64_t row = tr + i < t.count ? row_at(order, t.first + tr + i, n) : -1;
    if (row < 0) continue;
    for (int j = 0; j < 4; ++j) {
      const int c = col0 + tc + j;
      if (c >= kout) continue;
      float v = 0.0f, z = 0.0f;
      if (live) {
        z = acc[i][j] + (bias ? to_f32(bias[int64_t(t.group) * kout + c]) : 0.0f);
        v = silu ? z * silu_factor(z) : z;
        if (residual) v += to_f32(in[row * ldin + c]);
      }
      out[row * kout + c] = from_f32<T>(v);
      if (zout) zout[row * kout + c] = from_f32<T>(z);
    }
  }
}

// dW_g = x^T dz and db_g = sum dz over the rows of a group
template <class T>
__global__ void __launch_bounds__(kThreads) grouped_outer_kernel(
    const int64_t* __restrict__ ptr, const int32_t* __restrict__ order, int n_groups, int64_t n,
    int k, int m, const T* __restrict__ x, int64_t ldx, const T* __restrict__ dy, int64_t ldy,
    const T* __restrict__ zin, int64_t ldz, T* __restrict__ dw, T* __restrict__ db) {
  __shared__ float a[kStep][kTile + 4], b[kStep][kTile + 4];
  const int g = blockIdx.z, k0 = blockIdx.x * kTile, c0 = blockIdx.y * kTile;
  const Span s = span_of(ptr, g, n_groups, n);
  float acc[4][4] = {};
  float sum = 0.0f;
  for (int64_t p = s.begin; p < s.end; p += kStep) {
    for (int i = threadIdx.x; i < kTile * kStep; i += kThreads) {
      const int r = i / kTile, c = i % kTile;
      const int64_t row = p + r < s.end ? row_at(order, p + r, n) : -1;
      a[r][c] = row >= 0 && k0 + c < k ? to_f32(x[row * ldx + k0 + c]) : 0.0f;
      float v = 0.0f;
      if (row >= 0 && c0 + c < m) {
        v = to_f32(dy[row * ldy + c0 + c]);
        if (zin) v *= silu_slope(to_f32(zin[row * ldz + c0 + c]));
      }
      b[r][c] = v;
    }
    __syncthreads();
    tile_product(a, b, acc);
    if (threadIdx.x < kTile)
      for (int r = 0; r < kStep; ++r) sum += b[r][threadIdx.x];
    __syncthreads();
  }
  const int tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
  if (dw)
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j)
        if (k0 + tr + i < k && c0 + tc + j < m)
          dw[(int64_t(g) * k + k0 + tr + i) * m + c0 + tc + j] = from_f32<T>(acc[i][j]);
  if (db && k0 == 0 && threadIdx.x < kTile && c0 + threadIdx.x < m)
    db[int64_t(g) * m + c0 + threadIdx.x] = from_f32<T>(sum);
}

int64_t tiles_at_most(int64_t n, int n_groups) {
  return n / kTile + (n < n_groups + 1 ? n : n_groups + 1);
}

}  // namespace

int64_t grouped_forward_work(const dpa4c_grouped&) { return 0; }
int64_t grouped_backward_work(const dpa4c_grouped&) { return 0; }

int launch_grouped_forward(const dpa4c_grouped& l, const void* bias, bool silu, bool residual,
                           void* y, void* z, void*, hipStream_t st) {
  if (l.n == 0) return 0;
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    const dim3 grid(tiles_at_most(l.n, l.n_groups), (l.n_out + kTile - 1) / kTile);
    grouped_rows_kernel<T, false><<<grid, kThreads, 0, st>>>(
        l.group_ptr, l.order, l.n_groups, l.n, l.k, l.n_out, static_cast<const T*>(l.x), l.ldx,
        nullptr, 0, static_cast<const T*>(l.weight), static_cast<const T*>(bias), silu, residual,
        static_cast<T*>(y), static_cast<T*>(z));
    DPA4C_HIP_TRY(hipGetLastError());
    return 0;
  });
}

int launch_grouped_backward(const dpa4c_grouped& l, const void* dy, int64_t ldy, const void* z,
                            int64_t ldz, bool residual, void* dx, void* dw, void* db, void*,
                            hipStream_t st) {
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    const T* dyt = static_cast<const T*>(dy);
    const T* zt = static_cast<const T*>(z);
    if (dx && l.n > 0) {
      const dim3 grid(tiles_at_most(l.n, l.n_groups), (l.k + kTile - 1) / kTile);
      grouped_rows_kernel<T, true><<<grid, kThreads, 0, st>>>(
          l.group_ptr, l.order, l.n_groups, l.n, l.n_out, l.k, dyt, ldy, zt, ldz,
          static_cast<const T*>(l.weight), nullptr, 0, residual, static_cast<T*>(dx), nullptr);
      DPA4C_HIP_TRY(hipGetLastError());
    }
    if (dw || db) {
      const dim3 grid(dw ? (l.k + kTile - 1) / kTile : 1, (l.n_out + kTile - 1) / kTile, l.n_groups);
      grouped_outer_kernel<T><<<grid, kThreads, 0, st>>>(
          l.group_ptr, l.order, l.n_groups, l.n, l.k, l.n_out, static_cast<const T*>(l.x), l.ldx,
          dyt, ldy, zt, ldz, static_cast<T*>(dw), static_cast<T*>(db));
      DPA4C_HIP_TRY(hipGetLastError());
    }
    return 0;
  });
}

}  // namespace dpa4c
