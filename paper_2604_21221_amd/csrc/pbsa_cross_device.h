// Device code that the kernels of the cross attention share: matrix instructions by element type, the LDS layout of a tile and
// the loads that fill it, which states of a tile are attended.
#pragma once

#include "pbsa_layer_internal.h"

namespace pbsa {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(8))) short s16x8;   // eight elements of 16 bits, whatever they are
typedef __attribute__((ext_vector_type(4))) short s16x4;

template <typename E>
struct Vec {
  typedef __attribute__((ext_vector_type(8))) E x8;
  typedef __attribute__((ext_vector_type(2))) E x2;
};

// c += a b, 32 x 32 x 16.  Lane L holds row (a) or column (b) L % 32, contraction indices 8 (L / 32) ..+7; of c column L % 32,
// rows 8 (v / 4) + 4 (L / 32) + v % 4.
template <typename E>
__device__ __forceinline__ f32x16 mfma(const s16x8& a, const s16x8& b, const f32x16& c) {
  typedef typename Vec<E>::x8 x8;
  if constexpr (__is_same(E, __bf16))
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ constexpr int row_of(int v) { return 8 * (v / 4) + v % 4; }   // of c, less 4 (L / 32)

template <typename E>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  typename Vec<E>::x2 p;
  p[0] = (E)x;
  p[1] = (E)y;
  return __builtin_bit_cast(uint32_t, p);
}
// Sixteen numbers a lane holds of one column, as operands of the two products of 16 rows each that take them as they lie: the
// contraction index 8 (L / 32) + j of product s stands for row 16 s + 8 (j / 4) + 4 (L / 32) + j % 4.
template <typename E>
__device__ __forceinline__ s16x8 pack8(const f32x16& p, int s) {
  const u32x4 v = {pack2<E>(p[8 * s], p[8 * s + 1]), pack2<E>(p[8 * s + 2], p[8 * s + 3]), pack2<E>(p[8 * s + 4], p[8 * s + 5]),
                   pack2<E>(p[8 * s + 6], p[8 * s + 7])};
  return __builtin_bit_cast(s16x8, v);
}

__device__ __forceinline__ float swap_max(float v) {   // with the other half wave's lane of the same column
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float swap_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int CTRL>
__device__ __forceinline__ float mov_dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) { return v + mov_dpp<CTRL>(v); }
__device__ __forceinline__ float swap_max16(float v) {  // with the lane 16 on or back
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The sum over the lanes of a wave that are the same in their groups of LPK (8 or 16)
template <int LPK>
__device__ __forceinline__ float over_groups(float v) {
  if constexpr (LPK == 8) v = add_dpp<0x128>(v);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return swap_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A tile in LDS: rows of D elements, unpadded, whose 16-byte chunks are permuted within the row (chunk c of row r at c ^ swz(r)),
// so that neither way of reading meets a bank twice:
//   by rows (operand a of a product over d): one chunk of 16 consecutive rows at a time;
//   by columns (operand a of a product over rows): the transposing read, four rows by 64 bytes for a half wave.
// The loads permute by what each lane fetches.  swz(r + 16) = swz(r) and swz(r + 8) = swz(r) ^ 2.
template <int D>
struct Tile {
  static constexpr int CH = D / 8, RPI = 64 / CH;      // chunks of a row, rows of a wave's 1 KiB load
  static constexpr int KS = D / 16, DT = D / 32;       // products over d, 32-wide pieces of d
  static constexpr int ROW = 2 * D, SUB = 32 * ROW;    // bytes of a row, of 32 rows
  static __device__ __forceinline__ int swz(int r) {
    if constexpr (D == 128) return (r & 3) << 2 | (r >> 2 & 3);
    else return (r >> 1 & 1) << 2 | (r >> 2 & 3);
  }
};

typedef __attribute__((address_space(3))) const s16x8* lds_row_t;
typedef __attribute__((address_space(3))) s16x4* lds_col_t;

// Where a lane reads its operands in a tile at an LDS address that is a multiple of 1 KiB: by rows of 32, k-step ks at
// row_at ^ (ks << 5); by columns, the 16 rows from 16 s on of d piece dt at (col_at ^ (dt << 6)) + 16 s ROW (read_col).
template <int D>
__device__ __forceinline__ uint32_t row_at(int lane) {
  const int r = lane & 31, half = lane >> 5;
  return (uint32_t)(r * Tile<D>::ROW + ((half ^ Tile<D>::swz(r)) << 4));
}
template <int D>
__device__ __forceinline__ uint32_t col_at(int lane) {
  const int s = lane & 15, q = (lane >> 4) & 1, half = lane >> 5;
  const int r = 4 * half + (s >> 2);
  return (uint32_t)(r * Tile<D>::ROW + (((2 * q + ((s & 3) >> 1)) ^ Tile<D>::swz(r)) << 4) + (s & 1) * 8);
}
__device__ __forceinline__ s16x8 read_row(uint32_t at) { return *(lds_row_t)(uintptr_t)at; }
template <int D>
__device__ __forceinline__ s16x8 read_col(uint32_t at) {
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)at);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)((at ^ 32) + 8 * Tile<D>::ROW));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"        // M0 is the compiler's too: it sets it anew where it needs it
// One wave's load of 16 bytes per lane to 1 KiB of LDS at `lds`, from `base` + the lane's offset; vmcnt counts it.
__device__ __forceinline__ void load_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
// The same from an address of each lane's own
__device__ __forceinline__ void load_lds(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds), "v"(from) : "memory", "m0");
}
// N such loads to consecutive KiB: the instruction's offset moves both addresses, so off[j] is less by 1024 j (and `base` is that
// much lower for all of them).
template <int N>
__device__ __forceinline__ void load_lds_n(const void* base, const uint32_t (&off)[N], uint32_t lds) {
  static_assert(N == 2 || N == 4, "");
  if constexpr (N == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                 "global_load_lds_dwordx4 %3, %5 offset:2048\n\tglobal_load_lds_dwordx4 %4, %5 offset:3072"
                 : : "s"(lds), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024"
                 : : "s"(lds), "v"(off[0]), "v"(off[1]), "s"(base) : "memory", "m0");
}
// Four bytes a lane, to 256 bytes of LDS
__device__ __forceinline__ void load_lds4(const void* from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop
// What a wave waits for before the barrier behind which the others read what it brought
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_barrier" : : : "memory"); }

// The loads of N KiB of a tile, from row r0 on, by one wave.  Rows that are not attended, or do not exist, are never fetched:
// a row that is stands in for them (their probability is zero, and zero times what it holds is zero).
template <int D, int N>
struct Loads {
  uint32_t at[N];            // of this lane: byte offset of what each load fetches
  __device__ __forceinline__ void set(int lane, int r0, uint32_t stride, uint64_t attended) {
    using T = Tile<D>;
    const int first = __builtin_ctzll(attended);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int r = r0 + j * T::RPI + lane / T::CH;
      const int c = (lane % T::CH) ^ T::swz(r);
      at[j] = (uint32_t)((attended >> r) & 1 ? r : first) * stride + (uint32_t)(c << 4);
    }
  }
  __device__ __forceinline__ void issue(const void* base, uint32_t lds) const {   // lds: where row r0 goes
#pragma unroll
    for (int j = 0; j < N; ++j) load_lds(base, at[j], lds + j * 1024);
  }
  // the offsets stay as they are up to here: until the loads are back
  __device__ __forceinline__ void keep() const {
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : : "v"(at[j]));
  }
};

// The loads of N KiB of a tile of 64 states, from row r0 on (a multiple of 16), by one wave: states 64 i .. of the first `count`,
// or of the list, whose next places lie in LDS (Picked).  States past the last one are not fetched: the last one stands in for
// them.  Offsets are 32 bits wide, from the tile's first row, or with a list from the first state (a call whose states lie further
// apart takes cross_keys_kernel: cross_shape).
constexpr int64_t kGatherSpan = 4096;      // more than a load's last byte lies behind its state's first: 256 of the row, 3 KiB (at)
struct Picked {
  int32_t at[4][64];         // of tiles i mod 4
};
typedef __attribute__((address_space(3))) const int32_t* lds_i32_t;
template <int D, int N>
struct Gather {
  const char* base;
  uint32_t picked;           // LDS address of the list's places, 0: no list
  uint32_t stride;
  int count, r;              // r, of this lane: its row of the first load
  uint32_t at[N];            // byte offsets of the loads: of a full tile, or of those on their way
  __device__ __forceinline__ uint32_t chunk(int j) const {
    // RPI rows on, the permutation differs by j (RPI = 4) or 2 j (RPI = 8)
    const uint32_t lane = threadIdx.x & 63, c = (lane % Tile<D>::CH) ^ Tile<D>::swz(r);
    return (c << 4) ^ (uint32_t)(j << (D == 128 ? 4 : 5));
  }
  __device__ __forceinline__ void init(int lane, int r0, const char* b, int64_t s, int n, uint32_t p) {
    base = b - 1024 * (N - 1);       // load_lds_n
    stride = (uint32_t)s;
    count = n;
    picked = p;
    r = r0 + lane / Tile<D>::CH;
#pragma unroll
    for (int j = 0; j < N; ++j) at[j] = (uint32_t)(r + j * Tile<D>::RPI) * stride + chunk(j) + 1024 * (N - 1 - j);
  }
  __device__ __forceinline__ void issue(int i, uint32_t lds) {     // lds: where row r0 goes
    const char* from = base;
    if (picked) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        at[j] = (uint32_t)*(lds_i32_t)(uintptr_t)(picked + 4 * (64 * (i & 3) + r + j * Tile<D>::RPI)) * stride + chunk(j) + 1024 * (N - 1 - j);
    } else {
      from += 64 * (int64_t)i * stride;
      if (64 * i + 64 > count) {     // the last tile
#pragma unroll
        for (int j = 0; j < N; ++j)
          at[j] = (uint32_t)min(r + j * Tile<D>::RPI, count - 1 - 64 * i) * stride + chunk(j) + 1024 * (N - 1 - j);
      }
    }
    load_lds_n<N>(from, at, lds);
  }
  __device__ __forceinline__ void keep() const {   // the offsets stay as they are up to here: until the loads are back
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : : "v"(at[j]));
  }
};

// Which states of a sequence are attended
struct Attended {
  const uint8_t* mask;       // of the sequence, or nullptr
  int len;
  // the N states from k0 on, as bits; the mask's bytes are read here
  template <int N>
  __device__ __forceinline__ uint64_t bits(int k0, int lane) const {
    const int n = len - k0;
    if (n <= 0) return 0;
    uint64_t b = n >= 64 ? ~0ull : (1ull << n) - 1;
    if (N < 64) b &= (1ull << (N & 63)) - 1;
    if (mask) b &= __ballot(lane < n && lane < N && mask[lane < n && lane < N ? k0 + lane : 0] != 0);
    return b;
  }
};
__device__ __forceinline__ int length_of(const int32_t* k_len, int64_t b, int Nk) {
  return k_len ? __builtin_amdgcn_readfirstlane(min(max(k_len[b], 0), Nk)) : Nk;
}
__device__ __forceinline__ Attended attended_of(const int32_t* k_len, const uint8_t* k_mask, int64_t mask_stride_b, int64_t b, int Nk) {
  Attended t;
  t.len = length_of(k_len, b, Nk);
  t.mask = k_mask ? k_mask + b * mask_stride_b : nullptr;
  return t;
}

}  // namespace
}  // namespace pbsa
