// The products of 8-bit rows that fit into registers, with results in bfloat16.
#include <hip/hip_runtime.h>

#include "layer8.h"

namespace dpa4c {

int run_held8_bf16(const HeldArgs& a, int format, bool back, bool wide, int64_t grid, hipStream_t st) {
  // three blocks take rows of three, five those of four and five, eight the longer ones
  const int64_t blocks = blocks_of(a.r.kin);
  if (blocks <= 1) return run_held<__bf16, 1>(a, format, back, wide, grid, st);
  if (blocks <= 2) return run_held<__bf16, 2>(a, format, back, wide, grid, st);
  if (blocks <= 3) return run_held<__bf16, 3>(a, format, back, wide, grid, st);
  if (blocks <= 5) return run_held<__bf16, 5>(a, format, back, wide, grid, st);
  return run_held<__bf16, kHeldBlocks>(a, format, back, wide, grid, st);
}

}  // namespace dpa4c
