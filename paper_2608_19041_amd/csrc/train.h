// Internal definitions of the operators that fit the energy MLP by element
// type: grouped layers and the Newton-Schulz update (grouped.hip, newton.hip).
#pragma once

#include "../../include/dpa4c.h"
#include "common.h"

namespace dpa4c {

constexpr int kMaxSortGroups = 512;       // of dpa4c_group_rows: its counters live in LDS
constexpr int kMaxGroups = 4096;          // of a layer: the starts of their tiles live in LDS
constexpr int kMaxWidth = 65536;
constexpr int kMaxStacks = 32;            // of one call; their descriptors are kernel arguments

constexpr int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// scratch of a call, handed out in 256-byte steps; sizes with base = nullptr
struct Arena {
  char* base;
  int64_t used = 0;
  template <class T>
  T* take(int64_t count) {
    T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
    used += align_up(count * int64_t(sizeof(T)), 256);
    return p;
  }
};

// a launch of so many workgroups can be made: HIP takes fewer than 2^32 threads
constexpr bool grid_fits(int64_t blocks, int threads) { return blocks * threads < (int64_t(1) << 32); }

int64_t group_rows_work(int64_t n, int n_groups);
int launch_group_rows(const int32_t* group, int64_t n, int n_groups, int64_t* group_ptr,
                      int32_t* order, void* work, hipStream_t st);

bool grouped_fits(const dpa4c_grouped& l);   // every launch of either direction
int64_t grouped_forward_work(const dpa4c_grouped& l);
int launch_grouped_forward(const dpa4c_grouped& l, const void* bias, bool silu, bool residual,
                           void* y, void* z, void* work, hipStream_t st);
struct Wanted {   // of a backward call: whether z is given and what is formed
  bool z, dx, dw, db;
};
int64_t grouped_backward_work(const dpa4c_grouped& l, const Wanted& want);
int launch_grouped_backward(const dpa4c_grouped& l, const void* dy, int64_t ldy, const void* z,
                            int64_t ldz, bool residual, void* dx, void* dw, void* db, void* work,
                            hipStream_t st);

// One stack of matrices of an orthogonalisation: U comes from ``grad`` alone,
// or (momentum != nullptr) from the momentum update of it; the result goes to
// ``out``, or into the weights ``param``.
struct NewtonStack {
  const void* grad;
  void* out;
  float* momentum;
  int64_t batch;
  int rows, cols;
};
struct MuonStep {
  float lr, momentum, decay;
  bool nesterov;
};
bool newton_fits(int count, const NewtonStack* s);
int64_t newton_work(int count, const NewtonStack* s);
int launch_newton(int dtype, int count, const NewtonStack* s, const dpa4c_newton& how,
                  const MuonStep* muon, void* work, hipStream_t st);

#ifdef __HIPCC__
// element types of the public arrays
template <int D>
struct Elem;
template <>
struct Elem<DPA4C_F32> {
  using T = float;
};
template <>
struct Elem<DPA4C_F16> {
  using T = _Float16;
};
template <>
struct Elem<DPA4C_BF16> {
  using T = __bf16;
};
template <class T>
__device__ inline float to_f32(T x) {
  return static_cast<float>(x);
}
template <class T>
__device__ inline T from_f32(float x) {
  return static_cast<T>(x);
}

// Calls fn(std::integral_constant<int, D>{}) for the type code.
template <class Fn>
int with_dtype(int dtype, Fn&& fn) {
  if (dtype == DPA4C_F32) return fn(std::integral_constant<int, DPA4C_F32>{});
  if (dtype == DPA4C_F16) return fn(std::integral_constant<int, DPA4C_F16>{});
  return fn(std::integral_constant<int, DPA4C_BF16>{});
}
#endif

}  // namespace dpa4c
