// Layers of 8-bit rows and weights: what their kernels share, and the product of
// rows that fit into registers (layer8.hip says what the operators compute).
#pragma once

#include "block.h"
#include "rows.h"

namespace dpa4c {

constexpr int kStep = kScaleBlock;      // reduction entries of a step, a row of 128 bytes
constexpr int kSlots8 = kStep / 16;

typedef int v8i __attribute__((ext_vector_type(8)));

struct Rows8Args {
  const int32_t* order;
  int n_groups;
  int64_t n;
  const RowTile* tiles;
  const int32_t* n_tiles;
  int kin, kout;
  const char* in;            // 8-bit rows, ldin bytes apart
  int64_t ldin;
  const uint8_t* in_scales;
  int64_t ld_scales;
  int by_place;              // ``in`` is in group order
  const char* w;             // [group][kout][pitch8(kin)]
  const uint8_t* w_scales;   // of a group: block i of kin and j of kout at i at_in + j at_out
  int64_t w_blocks, at_in, at_out;
  const void* bias;
  int silu;
  const void* residual;      // rows of kout entries, ldres apart, or null
  int64_t ldres;
  void* out;
  void* zout;
};

constexpr int kHeldBlocks = 8;   // of 128 entries

struct HeldArgs {
  Rows8Args r;              // tiles = null: a workgroup looks its tile up
  const int64_t* ptr;
  int splits;              // workgroups that share the columns of a tile
  // gradients: rows are formed from dy act'(z) (z = null: dy) of kin entries, not read
  const void *dy, *z;
  int64_t ldy, ldz;
  _Float16* dz;            // [n][pitch8(kin)] by place, or null
  uint8_t* dz_scales;      // [n][blocks of kin] by place
};

// The product over rows of up to kHeldBlocks blocks, by workgroups of 128 rows (wide) or 32; ``back``: dx,
// and dz on the way.  ``format``: of the rows in 8 bits.
int run_held8_f16(const HeldArgs& a, int format, bool back, bool wide, int64_t grid, hipStream_t st);
int run_held8_bf16(const HeldArgs& a, int format, bool back, bool wide, int64_t grid, hipStream_t st);

namespace {

// byte offset of 16-byte slot ``slot`` of row ``row`` in an operand's step: exchanged by
// bits of the row, so that eight rows at one slot meet all banks
__device__ inline int slot8_at(int row, int slot) { return row * kStep + ((slot ^ (row & 7)) << 4); }

// the first ``keep`` of sixteen bytes, zeros past them
__device__ inline u4 keep_bytes(u4 v, int keep) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int left = keep - 4 * j;
    const unsigned mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
    v[j] &= mask;
  }
  return v;
}

// dz as float16: dz 2^(kHalfUp - e), e the exponent of its block's scale, so that the largest
// entry of a block lies in (2^13.8, 2^14.8]; as 8-bit numbers: dz 2^-e
template <int F>
constexpr int kHalfUp = 14 - kTopExp<F>;

// tile ``index`` of at most ``rows`` places; false past the last.  By every wave.
__device__ inline bool find_tile(const int64_t* ptr, int n_groups, int64_t n, int rows, int64_t index, RowTile* t) {
  const int lane = threadIdx.x & (kWave - 1);
  int64_t run = 0;
  for (int g0 = 0; g0 <= n_groups; g0 += kWave) {
    const int g = g0 + lane;
    Span s{0, 0};
    if (g <= n_groups) s = span_of(ptr, g, n_groups, n);
    const int mine = static_cast<int>((s.end - s.begin + rows - 1) / rows);
    int sum = mine;
    for (int d = 1; d < kWave; d *= 2) {
      const int v = __shfl_up(sum, d);
      sum += lane >= d ? v : 0;
    }
    const int64_t at = index - run - (sum - mine);   // of this lane's group
    const uint64_t who = __ballot(at >= 0 && at < mine);
    if (who != 0) {
      const int l = __ffsll(static_cast<unsigned long long>(who)) - 1;
      t->group = g0 + l;
      t->part = __shfl(static_cast<int>(at), l);
      t->parts = __shfl(mine, l);
      const int64_t begin = __shfl(s.begin, l), end = __shfl(s.end, l);
      t->first = begin + int64_t(t->part) * rows;
      t->count = static_cast<int>(end - t->first < rows ? end - t->first : rows);
      return true;
    }
    run += __shfl(sum, kWave - 1);
  }
  return false;
}

// At most KB blocks of 128 entries a row.  A wave has 32 rows, a lane (its row lane % 32, and of each 64
// entries the half lane / 32) 64 KB bytes of them in registers, and forms 32 columns at a time:
// the weights are the first operand of the product, in an order in which a lane's sixteen sums are
// neighbouring columns of its row, so that outputs leave from the registers.  Wide: the four waves have
// 128 rows, and the columns' weights pass through LDS, the next ones on their way; else
// they have the same 32 rows and 32 columns each, whose weights they read on their own.
template <class T, int F, int KB, bool Back, bool Wide>
__global__ void __launch_bounds__(kTileThreads, Wide ? (KB < 4 ? 3 : 2) : KB < 3 ? 3 : KB < 4 ? 2 : 1) layer8_held_kernel(HeldArgs h) {
  const Rows8Args& a = h.r;
  constexpr int kRows = Wide ? 128 : 32, kCols = 32;
  constexpr int kBuffer = Wide ? kCols * KB * kStep : 16;
  __shared__ __attribute__((aligned(16))) char lds[2][kBuffer];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col_tiles = (a.kout + kCols - 1) / kCols;
  int64_t work = blockIdx.x;
  RowTile t;
  if (a.tiles) {
    const int64_t total = int64_t(*a.n_tiles) * h.splits;
    if (work >= total) return;
    // the parts of a row tile follow each other on one XCD
    work = xcd_block(work, total);
    t = a.tiles[work / h.splits];
  } else if (!find_tile(h.ptr, a.n_groups, a.n, kRows, work / h.splits, &t)) {
    return;
  }
  const int split = static_cast<int>(work % h.splits);
  // this workgroup's column tiles, and of them this wave's
  const int first = static_cast<int>(int64_t(col_tiles) * split / h.splits);
  const int last = static_cast<int>(int64_t(col_tiles) * (split + 1) / h.splits);
  T* out = static_cast<T*>(a.out);
  T* zout = static_cast<T*>(a.zout);

  if (t.group == a.n_groups) {   // rows of no group
    const int c0 = first * kCols, width = (last * kCols < a.kout ? last * kCols : a.kout) - c0;
    for (int i = tid; i < t.count * width; i += kTileThreads) {
      const int64_t row = row_at(a.order, t.first + i / width, a.n);
      if (row < 0) continue;
      out[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
      if (zout) zout[row * a.kout + c0 + i % width] = from_f32<T>(0.0f);
    }
    return;
  }

  const int mine = (Wide ? 32 * wave : 0) + (lane & 31);
  const int64_t place = t.first + (mine < t.count ? mine : t.count - 1);
  const int64_t to = row_at(a.order, place, a.n), row = to < 0 ? 0 : to;
  const bool stored = mine < t.count && to >= 0;
  const bool live = !Wide || 32 * wave < t.count;
  const int64_t pitch = pitch8(a.kin);
  const int chunks = static_cast<int>(pitch / 16), blocks = static_cast<int>(blocks_of(a.kin));   // blocks <= KB

  // weights: slot tid % 8 of row tid / 8 of the operand, which is column ``column(tid / 8)``
  auto column = [](int m) { return 16 * (m >> 2 & 1) + 4 * (m >> 3) + (m & 3); };
  const char* weights = a.w + int64_t(t.group) * a.kout * pitch;
  const uint8_t* wscales = a.w_scales + t.group * a.w_blocks;
  const int slot = tid % kSlots8, own = tid / kSlots8;
  u4 wreg[KB];
  auto fetch = [&](int tile) {   // past the end: the last column
    const int c = tile * kCols + column(own);
    const char* from = weights + int64_t(c < a.kout ? c : a.kout - 1) * pitch;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const int chunk = b * kSlots8 + slot;
      wreg[b] = *reinterpret_cast<const u4*>(from + (chunk < chunks ? chunk : chunks - 1) * 16);
    }
  };
  auto put = [&](int buffer) {
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      if (b >= blocks - 1) wreg[b] = keep_bytes(wreg[b], a.kin - b * kStep - slot * 16);
      *reinterpret_cast<u4*>(lds[buffer] + b * kCols * kStep + slot8_at(own, slot)) = wreg[b];
    }
  };
  if (Wide && first < last) fetch(first);

  // the rows
  v8i x[KB][2];
  unsigned xs[KB];
  if constexpr (!Back) {
    const char* from = a.in + row * a.ldin;
    const uint8_t* scales = a.in_scales + row * a.ld_scales;
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      xs[b] = scales[b < blocks ? b : blocks - 1];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        u4 v[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int chunk = b * kSlots8 + 4 * s + 2 * half + j;
          v[j] = *reinterpret_cast<const u4*>(from + (chunk < chunks ? chunk : chunks - 1) * 16);
          if (b >= blocks - 1) v[j] = keep_bytes(v[j], a.kin - chunk * 16);
        }
        __builtin_memcpy(&x[b][s], v, 32);
      }
    }
  } else {
    const T* dy = static_cast<const T*>(h.dy) + row * h.ldy;
    const T* z = h.z ? static_cast<const T*>(h.z) + row * h.ldz : nullptr;
    const bool keeps = split == 0 && h.dz && mine < t.count && (Wide || wave == 0);
#pragma unroll
    for (int b = 0; b < KB; ++b) {
      const bool ends = b >= blocks - 1;
      float v[2][32];
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = b * kStep + 64 * s + 32 * half + 8 * j;
          Raw<T, 8> d = load_raw_entries<T, 8>(dy, c, a.kin, ends), e;
          if (z) e = load_raw_entries<T, 8>(z, c, a.kin, ends);
          if (ends) {
            settle<T, 8>(d, c, a.kin);
            if (z) settle<T, 8>(e, c, a.kin);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float f = to < 0 ? 0.0f : d.at(i);
            if (z) f = to < 0 ? 0.0f : f * silu_slope(e.at(i));
            v[s][8 * j + i] = f;
          }
        }
      bool bad = false;
      float most = fmaxf(finite_most<32>(v[0], &bad), finite_most<32>(v[1], &bad));
      most = fmaxf(most, __shfl_xor(most, 32));
      bad |= __shfl_xor(int(bad), 32) != 0;
      const int e = scale_exp<F>(most);
      const float up = power_of_two(-e);
      xs[b] = static_cast<unsigned>(e + 127);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[s][j] *= up;
#pragma unroll
        for (int j = 0; j < 8; ++j)
          x[b][s][j] = bad ? kNaN8 : pack8<F>(v[s][4 * j], v[s][4 * j + 1], v[s][4 * j + 2], v[s][4 * j + 3]);
        if (keeps)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int c = b * kStep + 64 * s + 32 * half + 8 * j;
            if (ends && c >= pitch) continue;
            v8h f;
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = static_cast<_Float16>(v[s][8 * j + i] * power_of_two(kHalfUp<F>));
            *reinterpret_cast<v8h*>(h.dz + place * pitch + c) = f;
          }
      }
      if (keeps && half == 0 && b < blocks) h.dz_scales[place * blocks + b] = static_cast<uint8_t>(xs[b]);
    }
  }

  if (Wide && first < last) {
    put(0);
    fetch(first + 1);
    __syncthreads();
  }
  const T* bias = a.bias ? static_cast<const T*>(a.bias) + int64_t(t.group) * a.kout : nullptr;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ldres : nullptr;
  for (int tile = first + (Wide ? 0 : wave); tile < last; tile += Wide ? 1 : 4) {
    const uint8_t* ws = wscales + tile * kCols / kScaleBlock * a.at_out;
    v16f acc = {};
    const int buffer = (tile - first) & 1;
    if (live) {
      const char* direct = nullptr;
      if (!Wide) {
        const int c = tile * kCols + column(lane & 31);
        direct = weights + int64_t(c < a.kout ? c : a.kout - 1) * pitch;
      }
#pragma unroll
      for (int b = 0; b < KB; ++b) {
        const unsigned scale = ws[(b < blocks ? b : blocks - 1) * a.at_in];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          u4 v[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int in = 4 * s + 2 * half + j, chunk = b * kSlots8 + in;
            if constexpr (Wide) {
              v[j] = *reinterpret_cast<const u4*>(lds[buffer] + b * kCols * kStep + slot8_at(lane & 31, in));
            } else {
              v[j] = *reinterpret_cast<const u4*>(direct + (chunk < chunks ? chunk : chunks - 1) * 16);
              if (b >= blocks - 1) v[j] = keep_bytes(v[j], a.kin - chunk * 16);
            }
          }
          v8i f;
          __builtin_memcpy(&f, v, 32);
          acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(f, x[b][s], acc, 0, F == DPA4C_E4M3 ? 0 : 1, 0, scale,
                                                                0, xs[b]);
        }
      }
      // here, with all lanes: a product reads the registers of every lane, but the loads before it, were
      // they moved to where its sums are used, only those of the lanes whose rows are stored
      asm volatile("" : "+v"(acc));
    }
    if constexpr (Wide) {
      put(buffer ^ 1);   // last read before the barrier of the tile before
      fetch(tile + 2);
    }
    // sixteen neighbouring columns of a row a lane
    if (live && stored) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = tile * kCols + 16 * half + 8 * q;
        if (c >= a.kout) continue;
        float y[8], zv[8], v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) zv[j] = acc[8 * q + j];
        if (bias) {
          load_entries<T, 8>(bias, c, a.kout, v);
#pragma unroll
          for (int j = 0; j < 8; ++j) zv[j] += v[j];
        }
        if (res) load_entries<T, 8>(res, c, a.kout, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[j] = a.silu ? zv[j] * logistic(zv[j]) : zv[j];
          if (res) y[j] += v[j];
        }
        store_entries<T, 8>(out + row * a.kout, c, a.kout, y);
        if (zout) store_entries<T, 8>(zout + row * a.kout, c, a.kout, zv);
      }
    }
    if (Wide) __syncthreads();
  }
}

template <class T, int KB>
int run_held(const HeldArgs& a, int format, bool back, bool wide, int64_t grid, hipStream_t st) {
  auto launch = [&](auto f, auto b, auto w) {
    layer8_held_kernel<T, decltype(f)::value, KB, decltype(b)::value, decltype(w)::value>
        <<<grid, kTileThreads, 0, st>>>(a);
    DPA4C_HIP_TRY(hipGetLastError());
    return 0;
  };
  auto of_format = [&](auto b, auto w) {
    if (format == DPA4C_E4M3) return launch(std::integral_constant<int, DPA4C_E4M3>{}, b, w);
    return launch(std::integral_constant<int, DPA4C_E5M2>{}, b, w);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  if (back) return wide ? of_format(Yes{}, Yes{}) : of_format(Yes{}, No{});
  return wide ? of_format(No{}, Yes{}) : of_format(No{}, No{});
}

}  // namespace

}  // namespace dpa4c
