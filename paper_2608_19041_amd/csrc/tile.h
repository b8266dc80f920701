// The product tile that the fitting operators share.
//
// A workgroup of four waves multiplies two operands that lie in LDS as rows of
// 32 reduction entries, [row][32] of 16-bit numbers, into 64 NB x 64 NB outputs; a
// wave forms 32 NB x 32 NB of them from v_mfma_f32_32x32x16, the instruction with
// the fewest LDS bytes for its work.  float32 operands are pairs of float16
// planes, x 2^e = hi + lo with both rounded to nearest (2^-24 of x 2^e or 2^-25
// absolute), and a product is hi hi + hi lo + lo hi; a half-type factor may
// come as such a pair too (two products).  Three float16 products take 3 x 32
// cycles for what v_mfma_f32_32x32x2_f32 takes 512 cycles for.
//
// A step of 32 entries is 768 matrix-core cycles of a wave for float32 at NB =
// 2.  Its loads are issued two steps (from HBM four) before their use, into
// registers; they go to the other half of LDS while this step's half is read, so a
// step has one barrier.  NB = 2 halves the traffic; NB = 1 gives four times as many
// workgroups with a quarter of the latency of a step, for work that does not
// fill the chip.
//
// The 16-byte slots of a row are exchanged by bits of the row, so that the
// eight lanes of one LDS cycle, eight rows at one slot, meet all banks.
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
constexpr int kDepth = 32;                        // reduction entries of a step
constexpr int kRowBytes = kDepth * 2;
constexpr int kPad = 128;                         // rows of a laid-out operand are padded to this

template <int NB>
constexpr int kSide = 64 * NB;                    // rows and columns of a tile
template <int NB>
constexpr int kPlane = kSide<NB> * kRowBytes;     // bytes of one operand's plane of a step

// byte offset of slot (8 reduction entries) ``slot`` of row ``row`` in a plane
__device__ inline int slot_at(int row, int slot) {
  return row * kRowBytes + ((slot ^ (row >> 1 & 3)) << 4);
}

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

// sums of a wave: v[i][j] holds the 32 x 32 outputs at (32 i, 32 j) of its part;
// lane l has column l % 32 and rows 8 (r / 4) + 4 (l / 32) + r % 4
template <int NB>
struct Sums {
  v16f v[NB][NB];
  __device__ inline void clear() {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) v[i][j] = v16f{};
  }
};
__device__ inline int sum_row(int lane, int r) { return 8 * (r / 4) + 4 * (lane / 32) + r % 4; }

// a wave's part of one operand for 16 entries of a step
template <int NB, int P>
struct Part {
  u4 v[NB][P];
};
// from planes ``plane`` bytes apart in LDS, at the wave's first row
template <int NB, int P>
__device__ inline void load_part(Part<NB, P>& f, const char* a, int plane, int lane, int ks) {
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int p = 0; p < P; ++p)
      f.v[i][p] = *reinterpret_cast<const u4*>(a + p * plane + slot_at(32 * i + (lane & 31), 2 * ks + (lane >> 5)));
}
// The same of an operand whose rows are the reduction entries: blocks of 32
// columns, [block][entry 32][32 columns], slots exchanged as above.  One
// transposing read gives a lane four entries of its column: the lanes 4 j + q of
// sixteen point at columns 4 q .. 4 q + 3 of entry j.
template <int NB, int P>
__device__ inline void load_part_turned(Part<NB, P>& f, const char* a, int plane, int lane, int ks) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) v4s* Lds;
  const int group = lane >> 4, entry = 16 * ks + 8 * (group >> 1) + (lane >> 2 & 3);
  const int col = 16 * (group & 1) + 4 * (lane & 3);
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int p = 0; p < P; ++p) {
      v4s h[2];
#pragma unroll
      for (int k = 0; k < 2; ++k)
        h[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (Lds)(a + p * plane + i * 32 * kRowBytes + slot_at(entry + 4 * k, col >> 3) + (col & 7) * 2));
      __builtin_memcpy(&f.v[i][p], h, 16);
    }
}

// acc += A B^T over 16 entries
template <bool Bf16, int NB, int PA, int PB>
__device__ inline void multiply_parts(Sums<NB>& acc, const Part<NB, PA>& a, const Part<NB, PB>& b) {
#pragma unroll
  for (int p = PA + PB - 2; p >= 0; --p)   // the small products first; lo lo is left out
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        if (PA == 2 && PB == 2) {
          if (p == 2) acc.v[i][j] = mfma<Bf16>(a.v[i][PA - 1], b.v[j][0], acc.v[i][j]);
          if (p == 1) acc.v[i][j] = mfma<Bf16>(a.v[i][0], b.v[j][PB - 1], acc.v[i][j]);
          if (p == 0) acc.v[i][j] = mfma<Bf16>(a.v[i][0], b.v[j][0], acc.v[i][j]);
        } else {
          acc.v[i][j] = mfma<Bf16>(a.v[i][PA == 2 ? p : 0], b.v[j][PB == 2 ? p : 0], acc.v[i][j]);
        }
      }
}

// The steps of a tile.  near(turn, s) and far(turn, s) issue the loads of step s
// into register set ``turn`` (a constant) of Near and of Far sets: operands from L2
// and operands from HBM, Near and Far steps ahead (s may be past the end, where they
// load anything that is cheap: loads under a condition would make the compiler
// wait for all of them at every put).  Loads arrive in the order of their issue, so
// the near ones go first.  put(n, f, s) writes sets n and f to half s % 2 of LDS,
// read(ks, s) takes 16 entries of a step from there to fragment set ks, before(s)
// runs when step s - 1's sums are complete and multiply(ks) adds fragment set ks.
// The barrier of a step stands between its two products: the second one runs
// from registers while the next step's first fragments arrive.
template <int K>
using Const = std::integral_constant<int, K>;
template <int Near, int Far, class NearFn, class FarFn, class Put, class Read, class Before, class Multiply>
__device__ inline void run_steps(int steps, NearFn&& near, FarFn&& far, Put&& put, Read&& read,
                                 Before&& before, Multiply&& multiply) {
  static_assert((Near == 1 || Near == 2 || Near == Far) && (Far == 2 || Far == 4),
                "the steps are unrolled by Far");
  near(Const<0>{}, 0);
  far(Const<0>{}, 0);
  if constexpr (Near >= 2) near(Const<1>{}, 1);
  far(Const<1>{}, 1);
  if constexpr (Far == 4) {
    if constexpr (Near == 4) near(Const<2>{}, 2);
    far(Const<2>{}, 2);
    if constexpr (Near == 4) near(Const<3>{}, 3);
    far(Const<3>{}, 3);
  }
  put(Const<0>{}, Const<0>{}, 0);
  near(Const<0>{}, Near);
  far(Const<0>{}, Far);
  __syncthreads();
  read(Const<0>{}, 0);
  auto step = [&](auto next, int s) {   // next = (s + 1) % Far
    constexpr int f = decltype(next)::value, n = f % Near;
    before(s);
    read(Const<1>{}, s);
    multiply(Const<0>{});
    if (s + 1 < steps) put(Const<n>{}, next, s + 1);
    near(Const<n>{}, s + 1 + Near);
    far(next, s + 1 + Far);
    __syncthreads();
    if (s + 1 < steps) read(Const<0>{}, s + 1);
    multiply(Const<1>{});
  };
  int s = 0;
  for (; s + Far <= steps; s += Far) {
    step(Const<1>{}, s);
    if constexpr (Far == 4) {
      step(Const<2>{}, s + 1);
      step(Const<3>{}, s + 2);
    }
    step(Const<0>{}, s + Far - 1);
  }
  if (s < steps) step(Const<1>{}, s);
  if constexpr (Far == 4) {
    if (s + 1 < steps) step(Const<2>{}, s + 1);
    if (s + 2 < steps) step(Const<3>{}, s + 2);
  }
}

// The tile's outputs pass through LDS as float32, in the operands' place; the
// 16-byte chunks of a row are exchanged by bits of the row, so that reads along
// rows and along columns, sixteen columns of four slots of rows too, meet all banks.
template <int NB>
__device__ inline int stage_at(int row, int col) {
  return row * kSide<NB> + (col ^ ((row & 7) << 2) ^ ((row >> 3 & 3) << 4));
}

// this wave's sums, scaled, into the stage at its row ``row0`` and column
// ``col0``; a barrier has to come before and after
template <int NB>
__device__ inline void stage_sums(float* stage, const Sums<NB>& acc, int row0, int col0, int lane, float scale) {
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        stage[stage_at<NB>(row0 + 32 * i + sum_row(lane, r), col0 + 32 * j + (lane & 31))] =
            acc.v[i][j][r] * scale;
}

// vector loads and stores at the alignment of the elements (rows of odd width)
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
  T v[N];
};

}  // namespace dpa4c
