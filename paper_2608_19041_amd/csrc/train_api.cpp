// C-ABI entry points of the operators that fit the energy MLP by element type.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>
#include <vector>

#include "checks.h"
#include "train.h"

namespace dpa4c {

namespace {

// the sizes of a layer; its pointers too with ``all``
int check_layer(const char* who, const dpa4c_grouped* l, bool all) {
  if (!l) return invalid(std::string(who) + ": null layer");
  if (l->dtype < DPA4C_F32 || l->dtype > DPA4C_BF16) return invalid(std::string(who) + ": unknown dtype");
  DPA4C_TRY(check_rows(who, l->n, l->n_groups, kMaxGroups));
  if (l->k < 1 || l->n_out < 1 || l->k > kMaxWidth || l->n_out > kMaxWidth)
    return invalid(std::string(who) + ": widths must be 1 .. 65536");
  if (!grouped_fits(*l)) {
    set_error(std::string(who) + ": more tiles than one launch takes");
    return DPA4C_ERR_UNSUPPORTED;
  }
  if (!all) return 0;
  if (!l->group_ptr || !l->weight || (l->n > 0 && !l->x))
    return invalid(std::string(who) + ": null pointer");
  if (l->ldx != 0 && l->ldx < l->k) return invalid(std::string(who) + ": ldx below k");
  return 0;
}

int check_newton(const char* who, int dtype, const dpa4c_newton* how) {
  if (dtype < DPA4C_F32 || dtype > DPA4C_BF16) return invalid(std::string(who) + ": unknown dtype");
  if (!how || how->steps < 0 || how->steps > 100 || !(how->eps > 0) || !std::isfinite(how->eps) ||
      !std::isfinite(how->a) || !std::isfinite(how->b) || !std::isfinite(how->c))
    return invalid(std::string(who) + ": needs 0 <= steps <= 100, eps > 0, finite coefficients");
  return 0;
}

std::vector<NewtonStack> stacks_of(int count, const dpa4c_stack* s) {
  std::vector<NewtonStack> v;
  for (int i = 0; i < count; ++i)
    v.push_back({s[i].in, s[i].out, nullptr, s[i].batch, s[i].rows, s[i].cols});
  return v;
}
std::vector<NewtonStack> stacks_of(int count, const dpa4c_update* s) {
  std::vector<NewtonStack> v;
  for (int i = 0; i < count; ++i)
    v.push_back({s[i].grad, s[i].param, s[i].momentum_buf, s[i].batch, s[i].rows, s[i].cols});
  return v;
}

template <class S>
int check_stacks(const char* who, int count, const S* s) {
  if (count < 0 || count > kMaxStacks || (count > 0 && !s))
    return invalid(std::string(who) + ": 0 to " + std::to_string(kMaxStacks) + " stacks a call");
  for (int i = 0; i < count; ++i)
    if (s[i].rows < 1 || s[i].cols < 1 || s[i].rows > kMaxWidth || s[i].cols > kMaxWidth ||
        s[i].batch < 0 || s[i].batch > INT32_MAX / (int64_t(s[i].rows) + s[i].cols))
      return invalid(std::string(who) + ": stack " + std::to_string(i) + " has an unusable shape");
  if (!newton_fits(count, stacks_of(count, s).data())) {
    set_error(std::string(who) + ": more tiles than one launch takes");
    return DPA4C_ERR_UNSUPPORTED;
  }
  return 0;
}

}  // namespace

}  // namespace dpa4c

using namespace dpa4c;

extern "C" {

int dpa4c_group_rows_work(int64_t n, int n_groups, int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_rows("dpa4c_group_rows_work", n, n_groups, kMaxSortGroups));
    if (!bytes) return invalid("dpa4c_group_rows_work: null pointer");
    *bytes = group_rows_work(n, n_groups);
    return 0;
  });
}

int dpa4c_group_rows(const int32_t* group, int64_t n, int n_groups, int64_t* group_ptr,
                     int32_t* order, void* work, int64_t work_bytes, void* stream) {
  return guarded([&] {
    const char* who = "dpa4c_group_rows";
    DPA4C_TRY(check_rows(who, n, n_groups, kMaxSortGroups));
    if (!group_ptr || (n > 0 && (!group || !order))) return invalid("dpa4c_group_rows: null pointer");
    DPA4C_TRY(check_work(who, work, work_bytes, group_rows_work(n, n_groups)));
    return launch_group_rows(group, n, n_groups, group_ptr, order, work,
                             static_cast<hipStream_t>(stream));
  });
}

int dpa4c_grouped_linear_work(const dpa4c_grouped* layer, int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_layer("dpa4c_grouped_linear_work", layer, false));
    if (!bytes) return invalid("dpa4c_grouped_linear_work: null pointer");
    *bytes = grouped_forward_work(*layer);
    return 0;
  });
}

int dpa4c_grouped_linear(const dpa4c_grouped* layer, const void* bias, int activation, int residual,
                         void* y, void* z, void* work, int64_t work_bytes, void* stream) {
  return guarded([&] {
    const char* who = "dpa4c_grouped_linear";
    DPA4C_TRY(check_layer(who, layer, true));
    if (activation != DPA4C_ACT_NONE && activation != DPA4C_ACT_SILU)
      return invalid("dpa4c_grouped_linear: unknown activation");
    if (residual && layer->k != layer->n_out)
      return invalid("dpa4c_grouped_linear: a residual needs k = n_out");
    if (layer->n > 0 && !y) return invalid("dpa4c_grouped_linear: null pointer");
    DPA4C_TRY(check_work(who, work, work_bytes, grouped_forward_work(*layer)));
    return launch_grouped_forward(*layer, bias, activation == DPA4C_ACT_SILU, residual != 0, y, z,
                                  work, static_cast<hipStream_t>(stream));
  });
}

int dpa4c_grouped_linear_backward_work(const dpa4c_grouped* layer, int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_layer("dpa4c_grouped_linear_backward_work", layer, false));
    if (!bytes) return invalid("dpa4c_grouped_linear_backward_work: null pointer");
    *bytes = grouped_backward_work(*layer, {true, true, true, true});
    return 0;
  });
}

int dpa4c_grouped_linear_backward_work_of(const dpa4c_grouped* layer, int z, int dx, int dw, int db,
                                          int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_layer("dpa4c_grouped_linear_backward_work_of", layer, false));
    if (!bytes) return invalid("dpa4c_grouped_linear_backward_work_of: null pointer");
    *bytes = grouped_backward_work(*layer, {z != 0, dx != 0, dw != 0, db != 0});
    return 0;
  });
}

int dpa4c_grouped_linear_backward(const dpa4c_grouped* layer, const void* dy, int64_t ldy,
                                  const void* z, int64_t ldz, int residual, void* dx, void* dw,
                                  void* db, void* work, int64_t work_bytes, void* stream) {
  return guarded([&] {
    const char* who = "dpa4c_grouped_linear_backward";
    DPA4C_TRY(check_layer(who, layer, true));
    if (residual && layer->k != layer->n_out)
      return invalid("dpa4c_grouped_linear_backward: a residual needs k = n_out");
    if (layer->n > 0 && !dy) return invalid("dpa4c_grouped_linear_backward: null pointer");
    if ((ldy != 0 && ldy < layer->n_out) || (z && ldz != 0 && ldz < layer->n_out))
      return invalid("dpa4c_grouped_linear_backward: ldy or ldz below n_out");
    const Wanted want{z != nullptr, dx != nullptr, dw != nullptr, db != nullptr};
    DPA4C_TRY(check_work(who, work, work_bytes, grouped_backward_work(*layer, want)));
    return launch_grouped_backward(*layer, dy, ldy, z, ldz, residual != 0, dx, dw, db, work,
                                   static_cast<hipStream_t>(stream));
  });
}

int dpa4c_orthogonalize_work(int count, const dpa4c_stack* stacks, int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_stacks("dpa4c_orthogonalize_work", count, stacks));
    if (!bytes) return invalid("dpa4c_orthogonalize_work: null pointer");
    *bytes = newton_work(count, stacks_of(count, stacks).data());
    return 0;
  });
}

int dpa4c_orthogonalize(int dtype, int count, const dpa4c_stack* stacks, const dpa4c_newton* how,
                        void* work, int64_t work_bytes, void* stream) {
  return guarded([&] {
    const char* who = "dpa4c_orthogonalize";
    DPA4C_TRY(check_newton(who, dtype, how));
    DPA4C_TRY(check_stacks(who, count, stacks));
    const std::vector<NewtonStack> s = stacks_of(count, stacks);
    for (const NewtonStack& x : s)
      if (x.batch > 0 && (!x.grad || !x.out)) return invalid("dpa4c_orthogonalize: null pointer");
    DPA4C_TRY(check_work(who, work, work_bytes, newton_work(count, s.data())));
    return launch_newton(dtype, count, s.data(), *how, nullptr, work,
                         static_cast<hipStream_t>(stream));
  });
}

int dpa4c_muon_step_work(int count, const dpa4c_update* updates, int64_t* bytes) {
  return guarded([&] {
    DPA4C_TRY(check_stacks("dpa4c_muon_step_work", count, updates));
    if (!bytes) return invalid("dpa4c_muon_step_work: null pointer");
    *bytes = newton_work(count, stacks_of(count, updates).data());
    return 0;
  });
}

int dpa4c_muon_step(int dtype, int count, const dpa4c_update* updates, const dpa4c_newton* how,
                    float lr, float momentum, int nesterov, float weight_decay, void* work,
                    int64_t work_bytes, void* stream) {
  return guarded([&] {
    const char* who = "dpa4c_muon_step";
    DPA4C_TRY(check_newton(who, dtype, how));
    DPA4C_TRY(check_stacks(who, count, updates));
    if (!std::isfinite(lr) || !std::isfinite(momentum) || !std::isfinite(weight_decay))
      return invalid("dpa4c_muon_step: lr, momentum and weight_decay must be finite");
    const std::vector<NewtonStack> s = stacks_of(count, updates);
    for (const NewtonStack& x : s)
      if (x.batch > 0 && (!x.grad || !x.out || !x.momentum))
        return invalid("dpa4c_muon_step: null pointer");
    DPA4C_TRY(check_work(who, work, work_bytes, newton_work(count, s.data())));
    const MuonStep muon{lr, momentum, weight_decay, nesterov != 0};
    return launch_newton(dtype, count, s.data(), *how, &muon, work,
                         static_cast<hipStream_t>(stream));
  });
}

}  // extern "C"
