// Newton-Schulz orthogonalisation of stacks of matrices, and the Muon update.
#include <hip/hip_runtime.h>

#include "train.h"

namespace dpa4c {

namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64, kStep = 16;

// One stack with the iterate X [batch][lo][hi] (float32, the shorter side
// first), its next value, and A and B [batch][lo][lo].
struct Stack {
  const void* grad;
  void* out;
  float* momentum;
  float *x, *next, *a, *b;
  double* norm;
  int64_t batch;
  int rows, cols;
  int lo, hi;
  bool turned;   // X holds the transpose
};
struct Stacks {
  Stack s[kMaxStacks];
  int count;
};

// U into X, with the sum of its squares
template <class T, bool Muon>
__global__ void __launch_bounds__(kThreads) newton_start_kernel(Stacks all, float beta, int nesterov) {
  const Stack& s = all.s[blockIdx.y];
  __shared__ double part[kThreads];
  for (int64_t m = blockIdx.x; m < s.batch; m += gridDim.x) {
    const int64_t base = m * s.rows * s.cols;
    const T* grad = static_cast<const T*>(s.grad) + base;
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < int64_t(s.rows) * s.cols; i += kThreads) {
      float u = to_f32(grad[i]);
      if (Muon) {
        const float v = beta * s.momentum[base + i] + u;
        s.momentum[base + i] = v;
        u = nesterov ? u + beta * v : v;
      }
      const int r = static_cast<int>(i / s.cols), c = static_cast<int>(i % s.cols);
      s.x[base + (s.turned ? int64_t(c) * s.hi + r : i)] = u;
      sum += double(u) * double(u);
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    for (int d = kThreads / 2; d > 0; d /= 2) {
      if (threadIdx.x < d) part[threadIdx.x] += part[threadIdx.x + d];
      __syncthreads();
    }
    if (threadIdx.x == 0) s.norm[m] = part[0];
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kThreads) newton_scale_kernel(Stacks all, float eps) {
  const Stack& s = all.s[blockIdx.y];
  for (int64_t m = blockIdx.x; m < s.batch; m += gridDim.x) {
    const double inv = 1.0 / (sqrt(s.norm[m]) + double(eps));
    float* x = s.x + m * s.lo * s.hi;
    for (int64_t i = threadIdx.x; i < int64_t(s.lo) * s.hi; i += kThreads)
      x[i] = static_cast<float>(x[i] * inv);
  }
}

// phase 0: A = X X^T; 1: B = b A + c A A; 2: next = a X + B X
__global__ void __launch_bounds__(kThreads) newton_product_kernel(Stacks all, int phase, float ca,
                                                                  float cb, float cc) {
  const Stack& s = all.s[blockIdx.z];
  __shared__ float a[kStep][kTile + 4], b[kStep][kTile + 4];
  const int lo = s.lo, hi = s.hi;
  const int width = phase == 2 ? hi : lo, depth = phase == 0 ? hi : lo;
  const int tw = (width + kTile - 1) / kTile, th = (lo + kTile - 1) / kTile;
  for (int64_t t = blockIdx.x; t < int64_t(tw) * th * s.batch; t += gridDim.x) {
    const int64_t m = t / (tw * th);
    const int r0 = static_cast<int>(t / tw % th) * kTile, c0 = static_cast<int>(t % tw) * kTile;
    const float* x = s.x + m * lo * hi;
    const float* A = s.a + m * lo * lo;
    const float* left = phase == 0 ? x : phase == 1 ? A : s.b + m * lo * lo;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < depth; k0 += kStep) {
      for (int i = threadIdx.x; i < kTile * kStep; i += kThreads) {
        const int r = i / kStep, k = i % kStep;
        a[k][r] = r0 + r < lo && k0 + k < depth ? left[int64_t(r0 + r) * depth + k0 + k] : 0.0f;
        const int kb = phase == 0 ? k : i / kTile, c = phase == 0 ? r : i % kTile;
        const bool in = k0 + kb < depth && c0 + c < width;
        b[kb][c] = !in ? 0.0f
                   : phase == 0 ? x[int64_t(c0 + c) * hi + k0 + kb]
                   : phase == 1 ? A[int64_t(k0 + kb) * lo + c0 + c]
                                : x[int64_t(k0 + kb) * hi + c0 + c];
      }
      __syncthreads();
      const int tr = threadIdx.x / 16 * 4, tc = threadIdx.x % 16 * 4;
#pragma unroll
      for (int k = 0; k < kStep; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] += a[k][tr + i] * b[k][tc + j];
      __syncthreads();
    }
    const int tr = r0 + threadIdx.x / 16 * 4, tc = c0 + threadIdx.x % 16 * 4;
    for (int i = 0; i < 4; ++i)
      for (int j = 0; j < 4; ++j)
        if (tr + i < lo && tc + j < width) {
          const int64_t at = int64_t(tr + i) * width + tc + j;
          if (phase == 0) s.a[m * lo * lo + at] = acc[i][j];
          if (phase == 1) s.b[m * lo * lo + at] = cb * A[at] + cc * acc[i][j];
          if (phase == 2) s.next[m * lo * hi + at] = ca * x[at] + acc[i][j];
        }
  }
}

template <class T, bool Muon>
__global__ void __launch_bounds__(kThreads) newton_end_kernel(Stacks all, float lr, float decay) {
  const Stack& s = all.s[blockIdx.y];
  const float step = Muon ? lr * sqrtf(fmaxf(1.0f, float(s.cols) / float(s.rows))) : 0.0f;
  T* out = static_cast<T*>(s.out);
  for (int64_t m = blockIdx.x; m < s.batch; m += gridDim.x) {
    const int64_t base = m * s.rows * s.cols;
    for (int64_t i = threadIdx.x; i < int64_t(s.rows) * s.cols; i += kThreads) {
      const int r = static_cast<int>(i / s.cols), c = static_cast<int>(i % s.cols);
      const float o = s.x[base + (s.turned ? int64_t(c) * s.hi + r : i)];
      out[base + i] = from_f32<T>(Muon ? (1.0f - lr * decay) * to_f32(out[base + i]) - step * o : o);
    }
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
    s.x = ar.take<float>(s.batch * s.lo * s.hi);
    s.next = ar.take<float>(s.batch * s.lo * s.hi);
    s.a = ar.take<float>(s.batch * s.lo * s.lo);
    s.b = ar.take<float>(s.batch * s.lo * s.lo);
    s.norm = ar.take<double>(s.batch);
  }
  *bytes = ar.used;
  return all;
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
  Stacks all = lay_out(count, in, work, &bytes);
  if (all.count == 0) return 0;
  const dim3 each(256, all.count);
  return with_dtype(dtype, [&](auto d) {
    using T = typename Elem<decltype(d)::value>::T;
    if (muon)
      newton_start_kernel<T, true><<<each, kThreads, 0, st>>>(all, muon->momentum, muon->nesterov);
    else
      newton_start_kernel<T, false><<<each, kThreads, 0, st>>>(all, 0.0f, 0);
    DPA4C_HIP_TRY(hipGetLastError());
    newton_scale_kernel<<<each, kThreads, 0, st>>>(all, how.eps);
    DPA4C_HIP_TRY(hipGetLastError());
    for (int step = 0; step < how.steps; ++step) {
      for (int phase = 0; phase < 3; ++phase) {
        newton_product_kernel<<<dim3(1024, 1, all.count), kThreads, 0, st>>>(all, phase, how.a, how.b,
                                                                            how.c);
        DPA4C_HIP_TRY(hipGetLastError());
      }
      for (int i = 0; i < all.count; ++i) std::swap(all.s[i].x, all.s[i].next);
    }
    if (muon)
      newton_end_kernel<T, true><<<each, kThreads, 0, st>>>(all, muon->lr, muon->decay);
    else
      newton_end_kernel<T, false><<<each, kThreads, 0, st>>>(all, 0.0f, 0.0f);
    DPA4C_HIP_TRY(hipGetLastError());
    return 0;
  });
}

}  // namespace dpa4c
