// The products of 8-bit rows that fit into registers, with results in bfloat16.
#include <hip/hip_runtime.h>

#include "layer8.h"

namespace dpa4c {

int run_held8_bf16(const HeldArgs& a, int format, bool wide, int64_t grid, hipStream_t st) {
  switch (blocks_of(a.r.kin)) {
    case 1: return run_held<__bf16, 1>(a, format, wide, grid, st);
    case 2: return run_held<__bf16, 2>(a, format, wide, grid, st);
    case 3: return run_held<__bf16, 3>(a, format, wide, grid, st);
    case 4: return run_held<__bf16, 4>(a, format, wide, grid, st);
    case 5: return run_held<__bf16, 5>(a, format, wide, grid, st);
    case 6: return run_held<__bf16, 6>(a, format, wide, grid, st);
    case 7: return run_held<__bf16, 7>(a, format, wide, grid, st);
    default: return run_held<__bf16, kHeldBlocks>(a, format, wide, grid, st);
  }
}

}  // namespace dpa4c
