// Root-mean-square norm of rows with gains of each group, and its gradients.
//
//   h = x (+ residual),  s = 1 / sqrt(mean_c h_c^2 + eps),  y = h s gain_g
//   t = mean_c dy_c gain_c h_c,  dx = s dy gain - h s^3 t (+ dh),  dgain_g = sum_r dy h s
//
// Bound by HBM.  A few lanes, or all of a wave, hold a row in registers, so it is
// read once; a wave walks neighbouring places, so that it keeps its group's gains. Squares, and
// the sums over a row and over the rows of a group, are in 64 bits, which cost a few of the
// cycles that the memory leaves idle.
#include <hip/hip_runtime.h>

#include "block.h"

namespace dpa4c {

namespace {

constexpr int kThreads = 256;
constexpr int kPlain = -1;   // the output is of the rows' type

__device__ inline int64_t clamp_place(int64_t p, int64_t n) { return p < 0 ? 0 : p > n ? n : p; }
__device__ inline int64_t row_at(const int32_t* order, int64_t place, int64_t n) {
  const int64_t r = order ? order[place] : place;
  return r >= 0 && r < n ? r : -1;
}
__device__ inline double sum_lanes(double v, int lanes) {
  for (int d = lanes / 2; d > 0; d /= 2) v += __shfl_xor(v, d);
  return v;
}

struct NormArgs {
  const void* x;
  int64_t ldx;
  const void* res;   // or null, and then h is
  int64_t ldr;
  const void* gain;
  const int64_t* ptr;   // null: one group of all rows
  const int32_t* order;
  int n_groups;
  int64_t n;
  int k;
  float eps;
  void* y;
  int64_t ldy;        // of 8-bit rows
  uint8_t* scales;
  int64_t lds;
  float* rstd;
  void* h;
  int lanes;
  int per;            // places of a wave's lanes, one after another
};

// NC: turns of a row that are held in registers; 0: rows of any length, read twice.
template <class T, int NC, int Q>
__global__ void __launch_bounds__(kThreads) rms_norm_kernel(NormArgs a) {
  constexpr int V = 16 / int(sizeof(T));
  constexpr int kHeld = NC > 0 ? NC : 1;
  const int lanes = a.lanes, sub = threadIdx.x & (lanes - 1), rows = kWave / lanes;
  const int64_t wave = int64_t(blockIdx.x) * (kThreads / kWave) + threadIdx.x / kWave;
  const int64_t base = wave * rows * a.per + (threadIdx.x & (kWave - 1)) / lanes;
  const int step = lanes * V;   // entries of a turn
  const int turns = NC > 0 ? NC : (a.k + step - 1) / step;
  int g = 0, held = -1;
  int64_t end = a.ptr ? -1 : a.n;
  float gain[kHeld][V];
  auto load = [&](int64_t row, int c, float* h) {
    load_entries<T, V>(static_cast<const T*>(a.x) + row * a.ldx, c, a.k, h);
    if (a.res) {
      float r[V];
      load_entries<T, V>(static_cast<const T*>(a.res) + row * a.ldr, c, a.k, r);
#pragma unroll
      for (int j = 0; j < V; ++j) h[j] += r[j];
    }
  };
  for (int i = 0; i < a.per; ++i) {
    const int64_t place = base + int64_t(i) * rows;
    if (place >= a.n) break;   // the lanes of a row alike
    if (place >= end) {
      g = group_of(a.ptr, a.n_groups, place);
      end = g < a.n_groups ? a.ptr[g + 1] : a.n;
    }
    const int64_t row = row_at(a.order, place, a.n);
    if (row < 0) continue;
    const bool live = g < a.n_groups;
    float h[kHeld][V];
    double sum = 0.0;
#pragma unroll
    for (int t = 0; t < kHeld; ++t)
      if (NC > 0) load(row, t * step + sub * V, h[t]);
#pragma unroll
    for (int t = 0; t < turns; ++t) {
      float* v = h[NC > 0 ? t : 0];
      if (NC == 0) load(row, t * step + sub * V, v);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += double(v[j]) * double(v[j]);
    }
    const double s = live ? 1.0 / sqrt(sum_lanes(sum, lanes) / a.k + double(a.eps)) : 0.0;
    if (sub == 0 && a.rstd) a.rstd[row] = static_cast<float>(s);
    const T* own = static_cast<const T*>(a.gain) + int64_t(live ? g : 0) * a.k;
    if (NC > 0 && held != g) {
#pragma unroll
      for (int t = 0; t < kHeld; ++t) load_entries<T, V>(own, t * step + sub * V, a.k, gain[t]);
      held = g;
    }
#pragma unroll
    for (int t = 0; t < turns; ++t) {
      const int c = t * step + sub * V, at = NC > 0 ? t : 0;
      float* v = h[at];
      if (NC == 0) {
        load(row, c, v);
        load_entries<T, V>(own, c, a.k, gain[0]);
      }
      if (a.h) store_entries<T, V>(static_cast<T*>(a.h) + row * int64_t(a.k), c, a.k, v);
      float y[V];
#pragma unroll
      for (int j = 0; j < V; ++j) y[j] = live ? static_cast<float>(double(v[j]) * s * double(gain[at][j])) : 0.0f;
      if constexpr (Q == kPlain) {
        store_entries<T, V>(static_cast<T*>(a.y) + row * int64_t(a.k), c, a.k, y);
      } else {
        constexpr int L = kScaleBlock / V;
        unsigned q[V / 4];
        const unsigned scale = quantize_block<Q, V>(y, lanes < L ? lanes : L, q);
        if (c < pitch8(a.k)) __builtin_memcpy(static_cast<uint8_t*>(a.y) + row * a.ldy + c, q, V);
        if ((sub & (L - 1)) == 0 && c < a.k) a.scales[row * a.lds + c / kScaleBlock] = static_cast<uint8_t>(scale);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Gradients
// ---------------------------------------------------------------------------

struct BackArgs {
  const void *dy, *h, *dh;   // dh: or null
  int64_t lddy, ldh, lddh;
  const void* gain;
  const float* rstd;
  const int64_t* ptr;
  const int32_t* order;
  int n_groups;
  int64_t n;
  int k;
  void* dx;      // null: not formed
  void* dgain;   // null: not formed
  double* parts; // [2 blocks][k]: of each block what its first group has beside other blocks, and its last
  int rows;      // places of a block
  int lanes;
};

// The stretch of one group that a block of places works on.
struct Stretch {
  int64_t begin, end;
  int group;      // n_groups: rows of no group
  int slot;       // where its sums go: -1 dgain itself, else 0 or 1 of the block
};
__device__ inline Stretch stretch_at(const BackArgs& a, int64_t at, int64_t first, int64_t last, int g) {
  while (g < a.n_groups && a.ptr && clamp_place(a.ptr[g + 1], a.n) <= at) ++g;
  Stretch s{at, last, g, -1};
  int64_t begin = 0, end = a.n;
  if (a.ptr && g < a.n_groups) {
    begin = clamp_place(a.ptr[g], a.n);
    end = clamp_place(a.ptr[g + 1], a.n);
  }
  if (g < a.n_groups) {
    s.end = end < last ? end : last;
    s.slot = begin < first ? 0 : end > last ? 1 : -1;
  }
  return s;
}
template <class T>
__device__ inline void put_gain(const BackArgs& a, const Stretch& s, int c, double v) {
  if (s.slot < 0)
    static_cast<T*>(a.dgain)[int64_t(s.group) * a.k + c] = from_f32<T>(static_cast<float>(v));
  else
    a.parts[(2 * int64_t(blockIdx.x) + s.slot) * a.k + c] = v;
}

// Rows held in registers, with the sums over a block's rows of each group beside them.
template <class T, int NC>
__global__ void __launch_bounds__(kThreads) rms_norm_back_kernel(BackArgs a) {
  constexpr int V = 16 / int(sizeof(T)), kWaves = kThreads / kWave;
  extern __shared__ double sums[];   // [waves][lanes V NC]
  const int lanes = a.lanes, sub = threadIdx.x & (lanes - 1), wave = threadIdx.x / kWave;
  const int unit = threadIdx.x / lanes, units = kThreads / lanes, step = lanes * V, width = step * NC;
  const int64_t first = int64_t(blockIdx.x) * a.rows;
  const int64_t last = first + a.rows < a.n ? first + a.rows : a.n;
  int g = a.ptr ? group_of(a.ptr, a.n_groups, first) : 0;
  for (int64_t at = first; at < last;) {   // alike for the whole workgroup
    const Stretch s = stretch_at(a, at, first, last, g);
    g = s.group;
    at = s.end;
    const bool live = g < a.n_groups;
    const T* own = static_cast<const T*>(a.gain) + int64_t(live ? g : 0) * a.k;
    float gain[NC][V];
    double acc[NC][V];
#pragma unroll
    for (int t = 0; t < NC; ++t) {
      load_entries<T, V>(own, t * step + sub * V, a.k, gain[t]);
#pragma unroll
      for (int j = 0; j < V; ++j) acc[t][j] = 0.0;
    }
    for (int64_t place = s.begin + unit; place < s.end; place += units) {
      const int64_t row = row_at(a.order, place, a.n);
      if (row < 0) continue;
      float dy[NC][V], h[NC][V], dh[NC][V];
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        const int c = t * step + sub * V;
        load_entries<T, V>(static_cast<const T*>(a.dy) + row * a.lddy, c, a.k, dy[t]);
        load_entries<T, V>(static_cast<const T*>(a.h) + row * a.ldh, c, a.k, h[t]);
        if (a.dh && a.dx) load_entries<T, V>(static_cast<const T*>(a.dh) + row * a.lddh, c, a.k, dh[t]);
      }
      const double r = live ? double(a.rstd[row]) : 0.0;
      double sum = 0.0;
#pragma unroll
      for (int t = 0; t < NC; ++t)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const double p = double(dy[t][j]) * double(h[t][j]);
          sum += p * double(gain[t][j]);
          acc[t][j] += p * r;
        }
      if (!a.dx) continue;
      const double pull = r * r * r * (sum_lanes(sum, lanes) / a.k);
#pragma unroll
      for (int t = 0; t < NC; ++t) {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          double d = live ? double(dy[t][j]) * double(gain[t][j]) * r - double(h[t][j]) * pull : 0.0;
          if (a.dh) d += double(dh[t][j]);
          v[j] = static_cast<float>(d);
        }
        store_entries<T, V>(static_cast<T*>(a.dx) + row * int64_t(a.k), t * step + sub * V, a.k, v);
      }
    }
    if (!a.dgain || !live) continue;
#pragma unroll
    for (int t = 0; t < NC; ++t)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        double v = acc[t][j];
        for (int d = kWave / 2; d >= lanes; d /= 2) v += __shfl_xor(v, d);
        if ((threadIdx.x & (kWave - 1)) < unsigned(lanes)) sums[wave * width + t * step + sub * V + j] = v;
      }
    __syncthreads();
    for (int c = threadIdx.x; c < a.k; c += kThreads) {
      double v = 0.0;
      for (int w = 0; w < kWaves; ++w) v += sums[w * width + c];
      put_gain<T>(a, s, c, v);
    }
    __syncthreads();
  }
}

// Rows too long for that: a workgroup a row at a time, read twice ..
template <class T>
__global__ void __launch_bounds__(kThreads) rms_norm_back_rows_kernel(BackArgs a) {
  constexpr int V = 16 / int(sizeof(T));
  __shared__ double part[2][kThreads / kWave];
  int turn = 0;
  for (int64_t place = blockIdx.x; place < a.n; place += gridDim.x) {
    const int64_t row = row_at(a.order, place, a.n);
    if (row < 0) continue;   // alike for the whole workgroup
    const int g = a.ptr ? group_of(a.ptr, a.n_groups, place) : 0;
    const bool live = g < a.n_groups;
    const T* own = static_cast<const T*>(a.gain) + int64_t(live ? g : 0) * a.k;
    const T* py = static_cast<const T*>(a.dy) + row * a.lddy;
    const T* ph = static_cast<const T*>(a.h) + row * a.ldh;
    float dy[V], h[V], gain[V];
    double sum = 0.0;
    for (int c = threadIdx.x * V; c < a.k; c += kThreads * V) {
      load_entries<T, V>(py, c, a.k, dy);
      load_entries<T, V>(ph, c, a.k, h);
      load_entries<T, V>(own, c, a.k, gain);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += double(dy[j]) * double(h[j]) * double(gain[j]);
    }
    sum = sum_lanes(sum, kWave);
    turn ^= 1;   // the other half of ``part`` may still be read
    if ((threadIdx.x & (kWave - 1)) == 0) part[turn][threadIdx.x / kWave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kThreads / kWave; ++w) sum += part[turn][w];
    const double r = live ? double(a.rstd[row]) : 0.0, pull = r * r * r * (sum / a.k);
    for (int c = threadIdx.x * V; c < a.k; c += kThreads * V) {
      load_entries<T, V>(py, c, a.k, dy);
      load_entries<T, V>(ph, c, a.k, h);
      load_entries<T, V>(own, c, a.k, gain);
      float dh[V], v[V];
      if (a.dh) load_entries<T, V>(static_cast<const T*>(a.dh) + row * a.lddh, c, a.k, dh);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        double d = live ? double(dy[j]) * double(gain[j]) * r - double(h[j]) * pull : 0.0;
        if (a.dh) d += double(dh[j]);
        v[j] = static_cast<float>(d);
      }
      store_entries<T, V>(static_cast<T*>(a.dx) + row * int64_t(a.k), c, a.k, v);
    }
  }
}

// .. and the gains' gradients by strips of columns, a lane V of them.
template <class T>
__global__ void __launch_bounds__(kThreads) rms_norm_gain_kernel(BackArgs a) {
  constexpr int V = 16 / int(sizeof(T));
  const int c = (blockIdx.y * kThreads + threadIdx.x) * V;
  if (c >= a.k) return;
  const int64_t first = int64_t(blockIdx.x) * a.rows;
  const int64_t last = first + a.rows < a.n ? first + a.rows : a.n;
  int g = a.ptr ? group_of(a.ptr, a.n_groups, first) : 0;
  for (int64_t at = first; at < last;) {
    const Stretch s = stretch_at(a, at, first, last, g);
    g = s.group;
    at = s.end;
    if (g >= a.n_groups) return;
    double acc[V] = {};
    for (int64_t place = s.begin; place < s.end; ++place) {
      const int64_t row = row_at(a.order, place, a.n);
      if (row < 0) continue;
      float dy[V], h[V];
      load_entries<T, V>(static_cast<const T*>(a.dy) + row * a.lddy, c, a.k, dy);
      load_entries<T, V>(static_cast<const T*>(a.h) + row * a.ldh, c, a.k, h);
      const double r = a.rstd[row];
#pragma unroll
      for (int j = 0; j < V; ++j) acc[j] += double(dy[j]) * double(h[j]) * r;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (c + j < a.k) put_gain<T>(a, s, c + j, acc[j]);
  }
}

// The sums of the groups that lie in several blocks, added in the blocks' order, and zeros
// for the groups without rows: 64 columns of a group a workgroup, sixteen blocks at a time.
constexpr int kJoinRows = 16;
template <class T>
__global__ void __launch_bounds__(64 * kJoinRows) rms_norm_join_kernel(const int64_t* __restrict__ ptr, int64_t n,
                                                                       int k, int rows,
                                                                       const double* __restrict__ parts,
                                                                       T* __restrict__ dgain) {
  __shared__ double part[kJoinRows][64];
  const int g = blockIdx.y, col = threadIdx.x % 64, lane = threadIdx.x / 64, c = blockIdx.x * 64 + col;
  const int64_t begin = ptr ? clamp_place(ptr[g], n) : 0, end = ptr ? clamp_place(ptr[g + 1], n) : n;
  T* out = dgain + int64_t(g) * k;
  if (begin >= end) {
    if (lane == 0 && c < k) out[c] = from_f32<T>(0.0f);
    return;
  }
  const int64_t b0 = begin / rows, b1 = (end - 1) / rows;
  if (b0 == b1) return;   // written already
  double v = 0.0;
  if (c < k)
#pragma unroll 4
    for (int64_t b = b0 + lane; b <= b1; b += kJoinRows) v += parts[(2 * b + (b == b0 ? 1 : 0)) * k + c];
  part[lane][col] = v;
  __syncthreads();
  if (lane > 0 || c >= k) return;
  for (int i = 1; i < kJoinRows; ++i) v += part[i][col];
  out[c] = from_f32<T>(static_cast<float>(v));
}

// Turns of a row in registers, at most four; 0: too long for that.
template <class T>
int turns_of(int width) {
  const int64_t turns = (int64_t(width) + kWave * (16 / int(sizeof(T))) - 1) / (kWave * (16 / int(sizeof(T))));
  return turns <= 1 ? 1 : turns <= 2 ? 2 : turns <= 4 ? 4 : 0;
}
template <class Fn>
int with_turns(int turns, Fn&& fn) {
  if (turns == 1) return fn(std::integral_constant<int, 1>{});
  if (turns == 2) return fn(std::integral_constant<int, 2>{});
  if (turns == 4) return fn(std::integral_constant<int, 4>{});
  return fn(std::integral_constant<int, 0>{});
}

// places of a block of the gradients: 1,024 blocks, four to a compute unit, of 16 rows at
// the least; long rows have several strips of columns in place of as many blocks
constexpr int kBlocks = 1024;
int block_rows(int64_t n, int strips) {
  const int64_t blocks = std::max(1, kBlocks / strips);
  return static_cast<int>(std::max<int64_t>(16, (n + blocks - 1) / blocks));
}
template <class T>
int strips_of(int k) {
  if (turns_of<T>(k)) return 1;
  return (k + kThreads * (16 / int(sizeof(T))) - 1) / (kThreads * (16 / int(sizeof(T))));
}

}  // namespace

int launch_rms_norm(const dpa4c_norm& l, const NormIn& in, void* y, const dpa4c_rows8* y8, float* rstd,
                    void* h, hipStream_t st) {
  if (l.n == 0) return 0;
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    constexpr int V = 16 / int(sizeof(T));
    const int width = static_cast<int>(y8 ? pitch8(l.k) : l.k);
    NormArgs a{in.x, in.ldx, in.residual, in.ldr, l.gain, l.group_ptr, l.order, l.n_groups, l.n, l.k, in.eps,
               y8 ? y8->values : y, y8 ? y8->ld : 0, y8 ? static_cast<uint8_t*>(y8->scales) : nullptr,
               y8 ? y8->ld_scales : 0, rstd, h, lanes_for<V>(width), 1};
    // 8,192 waves, eight to a SIMD, before a wave takes several rows
    const int64_t rows = kWave / a.lanes;
    const int64_t per = std::min<int64_t>(64, (l.n + rows * 8192 - 1) / (rows * 8192));
    a.per = static_cast<int>(per);
    const int64_t each = rows * per * (kThreads / kWave), grid = (l.n + each - 1) / each;
    return with_turns(turns_of<T>(width), [&](auto turns) {
      constexpr int NC = decltype(turns)::value;
      if (!y8)
        rms_norm_kernel<T, NC, kPlain><<<grid, kThreads, 0, st>>>(a);
      else if (y8->format == DPA4C_E4M3)
        rms_norm_kernel<T, NC, DPA4C_E4M3><<<grid, kThreads, 0, st>>>(a);
      else
        rms_norm_kernel<T, NC, DPA4C_E5M2><<<grid, kThreads, 0, st>>>(a);
      DPA4C_HIP_TRY(hipGetLastError());
      return 0;
    });
  });
}

int64_t rms_norm_backward_work(const dpa4c_norm& l, bool dgain) {
  if (!dgain || l.n == 0) return 0;
  const int strips = l.dtype == DPA4C_F32 ? strips_of<float>(l.k) : strips_of<_Float16>(l.k);
  const int64_t rows = block_rows(l.n, strips), blocks = (l.n + rows - 1) / rows;
  return align_up(2 * blocks * l.k * int64_t(sizeof(double)), 256);
}

int launch_rms_norm_backward(const dpa4c_norm& l, const NormBack& in, void* dx, void* dgain, void* work,
                             hipStream_t st) {
  return with_dtype(l.dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    constexpr int V = 16 / int(sizeof(T));
    const int strips = strips_of<T>(l.k), rows = block_rows(l.n, strips);
    BackArgs a{in.dy, in.h, in.dh, in.lddy, in.ldh, in.lddh, l.gain, in.rstd, l.group_ptr, l.order, l.n_groups,
               l.n, l.k, dx, dgain, static_cast<double*>(work), rows, lanes_for<V>(l.k)};
    if (l.n > 0 && (dx || dgain)) {
      const int64_t blocks = (l.n + rows - 1) / rows;
      DPA4C_TRY(with_turns(turns_of<T>(l.k), [&](auto turns) {
        constexpr int NC = decltype(turns)::value;
        if constexpr (NC > 0) {
          const int bytes = kThreads / kWave * a.lanes * V * NC * int(sizeof(double));
          rms_norm_back_kernel<T, NC><<<blocks, kThreads, bytes, st>>>(a);
        } else {
          if (dx) rms_norm_back_rows_kernel<T><<<std::min<int64_t>(l.n, 1 << 20), kThreads, 0, st>>>(a);
          if (dgain) rms_norm_gain_kernel<T><<<dim3(blocks, strips), kThreads, 0, st>>>(a);
        }
        DPA4C_HIP_TRY(hipGetLastError());
        return 0;
      }));
    }
    if (dgain) {
      rms_norm_join_kernel<T><<<dim3((l.k + 63) / 64, l.n_groups), 64 * kJoinRows, 0, st>>>(
          l.group_ptr, l.n, l.k, rows, a.parts, static_cast<T*>(dgain));
      DPA4C_HIP_TRY(hipGetLastError());
    }
    return 0;
  });
}

}  // namespace dpa4c
