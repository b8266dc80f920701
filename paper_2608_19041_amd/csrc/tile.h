// The 128 x 128 product tile that the fitting operators share.
//
// A workgroup of four waves multiplies two operands that lie in LDS as rows of
// 64 reduction entries, [row][64] of 16-bit numbers; a wave forms 64 x 64 of the
// outputs from v_mfma_f32_32x32x16, the instruction with the fewest LDS bytes
// for its work.  float32 operands are pairs of float16 planes, x 2^e = hi + lo
// with both rounded to nearest (2^-24 of x 2^e or 2^-25 absolute), and a product
// is hi hi + hi lo + lo hi; a half-type factor may come as such a pair too (two
// products).  Three float16 products take 3 x 32 cycles for what
// v_mfma_f32_32x32x2_f32 takes 512 cycles for.
//
// The 16-byte slots of a row are exchanged by the row's low three bits, so that
// the eight lanes of one LDS cycle, eight rows at one slot, meet all banks.
#pragma once

#include "train.h"

namespace dpa4c {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr int kTileThreads = 256;
constexpr int kTileRows = 128, kTileCols = 128;   // outputs of a workgroup
constexpr int kDepth = 64;                        // reduction entries of a step
constexpr int kPlane = kTileRows * kDepth * 2;    // bytes of one operand's plane

// byte offset of slot (8 reduction entries) ``slot`` of row ``row`` in a plane
__device__ inline int slot_at(int row, int slot) { return row * 128 + ((slot ^ (row & 7)) << 4); }

template <bool Bf16>
__device__ inline v16f mfma(u4 a, u4 b, v16f c) {
  if constexpr (Bf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8b, a),
                                                   __builtin_bit_cast(v8b, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h, a),
                                                  __builtin_bit_cast(v8h, b), c, 0, 0, 0);
}

// two floats as float16 hi and lo pairs
__device__ inline void split2(float x, float y, unsigned* hi, unsigned* lo) {
  const v2f f = {x, y};
  const v2h h = __builtin_convertvector(f, v2h);
  const v2f r = {x - static_cast<float>(h.x), y - static_cast<float>(h.y)};
  *hi = __builtin_bit_cast(unsigned, h);
  *lo = __builtin_bit_cast(unsigned, __builtin_convertvector(r, v2h));
}

// Running power-of-two scales of float32 operands.  A row (or column) is
// multiplied by 2^e so that the largest entry seen when e was set lies in
// [2^kSet, 2^(kSet + 1)); entries up to kLimit fit, so e has to fall only when
// a later entry is 2^8 times larger, and then the sums so far are scaled
// down by the same power, which is exact.  Entries are held to 2^-24 of
// themselves or, at the least, 2^-32 of that largest one.
constexpr int kSet = 7;
constexpr float kLimit = 32768.0f;
constexpr int kFirstExp = 127;   // before any entry: the first one sets e
__device__ inline float exp2_of(int e) {   // -126 <= e <= 127
  return __builtin_bit_cast(float, static_cast<unsigned>(e + 127) << 23);
}
// the e for a largest magnitude m > 0 (an infinity or NaN: as the largest float)
__device__ inline int exp_for(float m) {
  const int e = kSet - (static_cast<int>(__builtin_bit_cast(unsigned, m) >> 23) - 127);
  return e > kFirstExp ? kFirstExp : e;
}

// sums of a wave: acc[i][j] holds the 32 x 32 outputs at (32 i, 32 j) of its
// 64 x 64; lane l has column l % 32 and rows 8 (r / 4) + 4 (l / 32) + r % 4
struct Sums {
  v16f v[2][2];
};
__device__ inline int sum_row(int lane, int r) { return 8 * (r / 4) + 4 * (lane / 32) + r % 4; }

// acc += A B^T over one step; a, b: the operands' planes in LDS at the wave's
// first row
template <bool Bf16, int PA, int PB>
__device__ inline void tile_step(Sums& acc, const char* a, const char* b, int lane) {
  const int row = lane & 31, half = lane >> 5;
#pragma unroll
  for (int ks = 0; ks < kDepth / 16; ++ks) {
    u4 fa[2][PA], fb[2][PB];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int p = 0; p < PA; ++p)
        fa[i][p] = *reinterpret_cast<const u4*>(a + p * kPlane + slot_at(32 * i + row, 2 * ks + half));
#pragma unroll
      for (int p = 0; p < PB; ++p)
        fb[i][p] = *reinterpret_cast<const u4*>(b + p * kPlane + slot_at(32 * i + row, 2 * ks + half));
    }
#pragma unroll
    for (int p = PA + PB - 2; p >= 0; --p)   // the small products first; lo lo is left out
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (PA == 2 && PB == 2) {
            if (p == 2) acc.v[i][j] = mfma<Bf16>(fa[i][PA - 1], fb[j][0], acc.v[i][j]);
            if (p == 1) acc.v[i][j] = mfma<Bf16>(fa[i][0], fb[j][PB - 1], acc.v[i][j]);
            if (p == 0) acc.v[i][j] = mfma<Bf16>(fa[i][0], fb[j][0], acc.v[i][j]);
          } else {
            acc.v[i][j] = mfma<Bf16>(fa[i][PA == 2 ? p : 0], fb[j][PB == 2 ? p : 0], acc.v[i][j]);
          }
        }
  }
}

// The tile's outputs pass through LDS once, 128 x 128 float32 in the operands'
// place; the 16-byte chunks of a row are exchanged by the row's low three bits,
// so that reads along rows and along columns both meet all banks.
constexpr int kStageBytes = kTileRows * kTileCols * 4;
__device__ inline int stage_at(int row, int col) { return row * kTileCols + (col ^ ((row & 7) << 2)); }

// this wave's sums, scaled, into the stage; a barrier has to come before and after
__device__ inline void stage_sums(float* stage, const Sums& acc, int wm, int wn, int lane, float scale) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        stage[stage_at(64 * wm + 32 * i + sum_row(lane, r), 64 * wn + 32 * j + (lane & 31))] =
            acc.v[i][j][r] * scale;
}

// vector loads and stores at the alignment of the elements (rows of odd width)
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[N];
};

}  // namespace dpa4c
