// Backward of the cross attention, for gfx950.  With P = exp(S - lse), delta = rowsum(dO O), dS = P (dO V^T - delta):
//   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
//
// dQ sums over states and dK, dV over rows; each is summed where it stays in registers, in a launch of its own, so that S and
// dO V^T are formed twice (7 products instead of 5) and nothing is added up through memory by atomics:
//   cross_dq_kernel        a wave owns 32 rows, the tiles of K and V pass by.  It also leaves, for the second launch, each row's
//                          lse in powers of two and delta.  Where rows are few the states are shared out, and
//                          cross_dq_join_kernel adds the parts in order.  Under a mask the states are those of a list.
//   cross_dkv_kernel       a wave owns 32 states, K^T and V^T of them in registers, and the tiles of Q and dO pass by; where that
//                          makes too few workgroups the rows are shared out and cross_dkv_join_kernel adds the parts.
//   cross_grad_small_kernel  both in one launch, where rows are few and one round of workgroups takes it
//   cross_grad_few_kernel  up to four rows: everything in one pass over the states
// Rows are those of all query heads that share a head of K and V (m = t G + g), which sums their gradients as it goes.
//
// P and dS are rounded to the tensors' type as operands: with the outputs' own rounding, sqrt 2 times the error of that alone; delta
// from a rounded O adds to it (sum_delta).
// In fp16 the gradients of the scores can lie far below what it holds normally (they are dO over the number of states), so dS is
// formed times 2^-k, k by the largest |dO|, of the row for dQ and of the workgroup's rows for dK; 2^-k goes into the exponent of P.
//
// Measured, 4680 x 512 x 12 x 128 in bf16: dQ 37.5 us (22 GFLOP; 8.6 us until the rows are there, 43 MB; 18 us of steps, 1.2
// PFLOP/s, a large library product's rate), dK and dV 37.8 (29 GFLOP; 25 us of steps), their join 6.6 (31 MB).  With all
// workgroups in one round, first loads and last stores have nothing beside them.
#include <algorithm>

#include "pbsa_cross_device.h"

namespace pbsa {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

struct CrossGradArgs {
  int T, Nk, Hk, G, M;
  int row_tiles, row_units;          // of 128 rows
  int key_tiles, key_units;          // of 128 states
  int parts, part_rows;              // workgroups that share out the rows of a state tile; rows of each, a multiple of 64
  int key_parts;                     // workgroups that share out the states of a row tile
  float c2, scale;
  int64_t qs[3], ks[3], vs[3], os[3], gs[3], dqs[3], dks[3], dvs[3], mask_stride_b;
  const void* Q;
  const void* K;
  const void* V;
  const void* O;
  const void* dO;
  const int32_t* k_len;
  const uint8_t* k_mask;
  const int32_t* list;               // [n][Nk] attended states and [n] their number, or nullptr: no mask, or up to four rows
  const int32_t* counts;
  const float* lse;
  void* dQ;
  void* dK;
  void* dV;
  // [n Hk][row_tiles 128], rows past the last one among them: lse in powers of two less lift_p (infinite: the row attends
  // nothing), delta
  float* stat_lse;
  float* stat_delta;
  float* top;                        // [n Hk][row_tiles]: the largest |dO| (fp16)
  float* part_q;                     // [state part][row unit][wave][D / 8][64 lanes][4]
  float* part;                       // [part][key unit][dK, dV][wave][D / 8][64 lanes][4]
};

__device__ __forceinline__ int place(int bx, int n) {
  const int per = (n + 7) / 8, at = bx % 8 * per + bx / 8;
  return bx / 8 < per && at < n ? at : -1;
}

// k of 2^-k for gradients of at most `top`, which are below 1 by it: |dS| = P |dP - sum P dP| is at most P (1 - P) times how far
// two of dO V^T lie apart, half the sum of |V| over d, and fp16 holds it as long as that sum is below 2^17.  Where it does not, the
// wave forms its sums again in binary32 (dq_plain, dk_plain): without matrix instructions, a matter of being right (4680 x 512 x 12 of
// 128 with nearly every wave doing so: 5.7 ms).
__device__ __forceinline__ float lift(float top) {
  if (!(top > 0.0f) || !(top < INFINITY)) return 0.0f;
  return fminf(fmaxf((float)__builtin_amdgcn_frexp_expf(top), -60.0f), 60.0f);
}
// P in fp16 is held times 2^14 for dV: a state that draws little from every row keeps its digits (P is at most 1)
template <typename E>
__device__ __forceinline__ constexpr float lift_p() { return __is_same(E, _Float16) ? 14.0f : 0.0f; }

// The parts of a sum in order, `step` apart, eight of them on their way at a time
__device__ __forceinline__ f32x4 sum_parts(const f32x4* from, int64_t step, int parts) {
  constexpr int kBatch = 8;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p0 = 0; p0 < parts; p0 += kBatch) {
    f32x4 u[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      u[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (p0 + k < parts) u[k] = from[(p0 + k) * step];
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) v += u[k];
  }
  return v;
}

// The sum over the lanes of a row, 8 or 16: within quads, then by mirroring eights and sixteens
template <int LPK>
__device__ __forceinline__ float over_row(float v) {
  v = add_dpp<0xB1>(v);
  v = add_dpp<0x4E>(v);
  v = add_dpp<0x141>(v);
  if constexpr (LPK == 16) v = add_dpp<0x140>(v);
  return v;
}

// Whether a row's gradients are infinite or NaN anyhow, of which nothing can be made by summing up again: it counts as one of infinite dO.
__device__ __forceinline__ bool lost(float lse, float delta) { return !(fabsf(delta) < INFINITY) || lse != lse; }
// Whether dS of a wave's has been infinite in a column that counts: then all of the column's sums are infinite or NaN, and one tells.
__device__ __forceinline__ bool beyond(float sum, bool counts) { return __any(counts && !(fabsf(sum) < INFINITY)); }
template <typename E>
__device__ __forceinline__ void store4(E* to, float x, float y, float z, float w) {
  const u32x2 v = {pack2<E>(x, y), pack2<E>(z, w)};
  *reinterpret_cast<u32x2*>(to) = v;
}

// c += a b in place, as an instruction of its own, c in the accumulator half of the register file: the compiler does not see a
// matrix instruction (settle).
template <typename E>
__device__ __forceinline__ void mfma_acc(f32x16& c, const s16x8& a, const s16x8& b) {
  if constexpr (__is_same(E, __bf16)) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
// What has to pass before vector instructions read c
__device__ __forceinline__ void settle(f32x16& c) { asm volatile("s_nop 15\n\ts_nop 15" : "+a"(c)); }
__device__ __forceinline__ s16x8 operand_of(const uint32_t* p) {
  const u32x4 v = {p[0], p[1], p[2], p[3]};
  return __builtin_bit_cast(s16x8, v);
}

// delta = sum P dP is rowsum(dO O), but O has been rounded.  Where a row has many states O is small beside V and that is lost in
// the rounding of dS; where it has a few, dP - delta can be a small difference of larger numbers.  So where a sequence attends up to
// kFewStates, however many it has room for, the sum itself is formed, in binary32.  Error of dQ and dK in bf16, of their norm, with two states 0.0050 by the outputs, 0.0023
// by the sum; eight 0.0033 and 0.0024; sixteen 0.0030 and 0.0024.  Time with three, 5 x 8676 rows of 15 heads of 64: 167 us and
// 187; with ten, 5 x 316 of 14 of 128: 26 and 37.
// With one state P = 1 and dP = delta: dS is zero, and is made so.
constexpr int kFewStates = 8;
// Those of a mask, in order, by a wave: their number if there are up to kFewStates, else more than that.  Whole waves of a workgroup
// may do so with the same `few` in LDS: they write the same.  Mostly the first 64 states tell; else 1024 to a turn, bound by latency.
__device__ __forceinline__ int few_attended(const Attended& keys, int lane, int* few) {
  constexpr int kLook = 16;
  int count = __popcll(keys.bits<64>(0, lane));
  if (__builtin_expect(count <= kFewStates, 0)) {
    count = 0;
    for (int k0 = 0; k0 < keys.len && count <= kFewStates; k0 += 64 * kLook) {
      uint64_t bits[kLook];
      int more = 0;
#pragma unroll
      for (int u = 0; u < kLook; ++u) {
        bits[u] = keys.bits<64>(k0 + 64 * u, lane);
        more += __popcll(bits[u]);
      }
      if (count + more > kFewStates) return count + more;
#pragma unroll
      for (int u = 0; u < kLook; ++u)
        for (uint64_t m = bits[u]; m != 0; m &= m - 1) few[count++] = k0 + 64 * u + __builtin_ctzll(m);
    }
  }
  return count;
}
// Of R rows, each over D / 8 lanes, 8 elements a lane; lse in powers of two; the n attended states are the first ones, or those of a
// list
template <typename E, int D, int R>
__device__ __forceinline__ void sum_delta(const CrossGradArgs& a, const int32_t* list, int n, int64_t b, int hk, int d0, const float (&q)[R][8],
                                          const float (&g)[R][8], const float (&lse)[R], float (&delta)[R]) {
  typedef typename Vec<E>::x8 x8;
#pragma unroll
  for (int r = 0; r < R; ++r) delta[r] = 0.0f;
  for (int i = 0; i < n; ++i) {
    const int j = list ? list[i] : i;
    const x8 k = *reinterpret_cast<const x8*>(reinterpret_cast<const E*>(a.K) + b * a.ks[0] + hk * a.ks[1] + j * a.ks[2] + d0);
    const x8 v = *reinterpret_cast<const x8*>(reinterpret_cast<const E*>(a.V) + b * a.vs[0] + hk * a.vs[1] + j * a.vs[2] + d0);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float s = 0.0f, dp = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s = __builtin_fmaf((float)k[e], q[r][e], s);
        dp = __builtin_fmaf((float)v[e], g[r][e], dp);
      }
      delta[r] += __builtin_amdgcn_exp2f(__builtin_fmaf(over_row<D / 8>(s), a.c2, -lse[r])) * over_row<D / 8>(dp);
    }
  }
}

// ---- dQ: a software pipeline over half tiles of 32 states ----------------------------------------------------------------
// A step forms S^T and V dO^T of the half tile after the current one, dS of the current one and what the one before it adds to
// dQ^T: a row of slots, each one matrix instruction (the three products in turn), an LDS read for a slot kAhead later and a
// slice of dS.  Nothing moves between slots.  A tile of 64 states is in LDS from its first product to its last, three half
// tiles on for K and two for V: there are three places for K and two for V, half of LDS, and registers stay below 256, so that
// two workgroups share a compute unit: one's rows come in while the other multiplies.
template <int D>
struct RowPipe {
  using T = Tile<D>;
  static constexpr int N = 3 * T::KS, kAhead = 4;                  // slots of a step: each of the three products has KS
  static constexpr int TURN = N - 3;
  static constexpr int kTile = 64 * T::ROW;                        // bytes of a tile of K or V
  uint32_t k, v, c;                                                // LDS addresses: K and V by rows, K by columns
  int32_t k_move, v_move, c_move;                                  // from a tile's place to the next one's
  s16x8 f[kAhead];                                                 // operands on their way, slot r's in r mod kAhead
  static_assert(N % kAhead == 0 && TURN >= N - kAhead, "a step's own reads are on their way at its turn");
  static constexpr int score(int r) { return 16 * r / N; }         // slot r takes scores score(r) .. score(r + 1) - 1
};
template <int D, int R, int OFF>
__device__ __forceinline__ s16x8 operand(const RowPipe<D>& z) {
  using T = Tile<D>;
  constexpr int i = R / 3;
  if constexpr (R % 3 == 0) return read_row((z.k ^ (i << 5)) + OFF);
  else if constexpr (R % 3 == 1) return read_row((z.v ^ (i << 5)) + OFF);
  else return read_col<D>((z.c ^ (i % T::DT << 6)) + OFF + 16 * (i / T::DT) * T::ROW);
}
template <int D, int OFF, int FROM, int TO>
__device__ __forceinline__ void preload(RowPipe<D>& z) {
  if constexpr (FROM < TO) {
    z.f[FROM] = operand<D, FROM, OFF>(z);
    preload<D, OFF, FROM + 1, TO>(z);
  }
}

template <int D>
struct RowGrad {
  s16x8 q[D / 16], g[D / 16];        // the wave's 32 rows of Q and dO: columns of the products over d
  f32x16 dq[D / 32];
  f32x16 s[2], dp[2];                // scores and V dO^T of the even and of the odd half tile
  uint32_t ds[2][8];
  float e[16];
  float lse, delta;                  // of the lane's row; lse in powers of two, and less what dS is scaled by
};
template <typename E, int D, int CUR, int Y, int TO>
__device__ __forceinline__ void put(RowGrad<D>& w) {               // dS of scores Y .. TO - 1, whose exponentials are there
  if constexpr (Y < TO) {
    w.e[Y] *= w.dp[CUR][Y] - w.delta;
    asm volatile("" : "+v"(w.e[Y])); // here, in its slot
    if constexpr (Y % 2 == 1) {
      w.ds[CUR][Y / 2] = pack2<E>(w.e[Y - 1], w.e[Y]);
      asm volatile("" : "+v"(w.ds[CUR][Y / 2]));
    }
    put<E, D, CUR, Y + 1, TO>(w);
  }
}

// Step A walks a tile's second half by rows and by columns the second half before it, and ends with the turn to the next places;
// step B walks first halves and issues the tile loads (extra).
template <typename E, int D, bool A, int R, typename Extra>
__device__ __forceinline__ void slots(RowGrad<D>& w, RowPipe<D>& z, float c2, Extra& extra) {
  using T = Tile<D>;
  using Z = RowPipe<D>;
  constexpr int N = Z::N, kAhead = Z::kAhead, i = R / 3, cur = A ? 0 : 1, other = 1 - cur, OFF = A ? T::SUB : 0;
  if constexpr (R < N) {
    const s16x8 u = z.f[R % kAhead];
    const f32x16 zero = {};
    if constexpr (R % 3 == 0) {
      if constexpr (i == 0) w.s[other] = mfma<E>(u, w.q[i], zero);
      else w.s[other] = mfma<E>(u, w.q[i], w.s[other]);
    } else if constexpr (R % 3 == 1) {
      if constexpr (i == 0) w.dp[other] = mfma<E>(u, w.g[i], zero);
      else w.dp[other] = mfma<E>(u, w.g[i], w.dp[other]);
    } else {
      mfma_acc<E>(w.dq[i % T::DT], u, operand_of(&w.ds[other][4 * (i / T::DT)]));
    }
    if constexpr (R + kAhead < N) z.f[R % kAhead] = operand<D, R + kAhead, OFF>(z);
    else if constexpr (!A) z.f[R % kAhead] = operand<D, R + kAhead - N, T::SUB>(z);
    if constexpr (A && R == Z::TURN) {
      wait_loads();
      barrier();
      z.k += z.k_move;
      z.v += z.v_move;
      z.c += z.c_move;
      preload<D, 0, 0, R % kAhead + 1>(z);                         // into the places of operands that have been used
    }
    if constexpr (A && R > Z::TURN) preload<D, 0, R % kAhead, R % kAhead + 1>(z);
    if constexpr (!A) extra(R);
    if constexpr (R > 0) put<E, D, cur, Z::score(R - 1), Z::score(R)>(w);
#pragma unroll
    for (int y = Z::score(R); y < Z::score(R + 1); ++y) w.e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(w.s[cur][y], c2, -w.lse));
    __builtin_amdgcn_sched_barrier(0);
    slots<E, D, A, R + 1>(w, z, c2, extra);
  } else {
    put<E, D, cur, Z::score(N - 1), 16>(w);
  }
}

// A wave's share of a tile of 64 states, N KiB of K and of V: states 64 i .. of the first `count`, or of the list.  States past
// the last one are not fetched: the last one stands in for them.
template <int D, int N>
struct StateLoads {
  const char* kb;
  const char* vb;
  const int32_t* list;
  int64_t ks, vs;
  int count, r;                      // r, of this lane: its row of the first load
  int at[N];                         // of this lane: the states that the next loads fetch
  __device__ __forceinline__ void choose(int i) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      at[j] = min(64 * i + r + j * Tile<D>::RPI, count - 1);
      if (list) at[j] = list[at[j]];
    }
  }
  __device__ __forceinline__ void issue(int lane, uint32_t to_k, uint32_t to_v) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = ((lane % Tile<D>::CH) ^ Tile<D>::swz(r + j * Tile<D>::RPI)) << 4;
      load_lds(kb + at[j] * ks + c, to_k + j * 1024);
      load_lds(vb + at[j] * vs + c, to_v + j * 1024);
    }
  }
};

// Where this lane's part of a wave's 32 rows lies in memory (whole rows to a load or store), row r of them row m0 + r of the head
template <int D>
__device__ __forceinline__ char* row_piece(const CrossGradArgs& a, const void* base, const int64_t (&st)[3], int64_t b, int hk, int m, int c) {
  const int mm = min(m, a.M - 1), t = a.G == 1 ? mm : mm / a.G, h = hk * a.G + (mm - t * a.G);
  return reinterpret_cast<char*>(const_cast<void*>(base)) + 2 * (b * st[0] + h * st[1] + t * st[2]) + c;
}

// dQ of a wave's 32 rows again where fp16 has not held their dS: in binary32, a row after the other, the states over groups of D / 8
// lanes.  Written over what has been written.
template <typename E, int D>
__device__ __forceinline__ void dq_plain(const CrossGradArgs& a, const char* kb, const char* vb, const int32_t* list, int begin, int end, int64_t b,
                                         int hk, int m0, float lse_of, float delta_of, f32x4* part) {
  typedef typename Vec<E>::x8 x8;
  constexpr int LPK = D / 8, KPI = 64 / LPK;
  const int lane = threadIdx.x & 63, grp = lane / LPK, c = lane % LPK;
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll 1
  for (int r = 0; r < 32 && m0 + r < a.M; ++r) {
    const float lse = __shfl(lse_of, r), delta = __shfl(delta_of, r);
    const x8 q = *reinterpret_cast<const x8*>(row_piece<D>(a, a.Q, a.qs, b, hk, m0 + r, 16 * c));
    const x8 g = *reinterpret_cast<const x8*>(row_piece<D>(a, a.dO, a.gs, b, hk, m0 + r, 16 * c));
    float dq[8] = {};
#pragma unroll 1
    for (int i0 = begin; i0 < end; i0 += KPI) {
      const int i = min(i0 + grp, end - 1);
      const int64_t j = list ? list[i] : i;
      const x8 k = *reinterpret_cast<const x8*>(kb + j * 2 * a.ks[2] + 16 * c), v = *reinterpret_cast<const x8*>(vb + j * 2 * a.vs[2] + 16 * c);
      float s = 0.0f, dp = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s = __builtin_fmaf((float)k[e], (float)q[e], s);
        dp = __builtin_fmaf((float)v[e], (float)g[e], dp);
      }
      s = over_row<LPK>(s);
      dp = over_row<LPK>(dp);
      const float ds = i0 + grp < end ? __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.c2, -lse)) * (dp - delta) : 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) dq[e] = __builtin_fmaf(ds, (float)k[e], dq[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dq[e] = over_groups<LPK>(dq[e]) * a.scale;
    if (grp != 0) continue;
    if (part) {
      part[c * 64 + r] = f32x4{dq[0], dq[1], dq[2], dq[3]};
      part[c * 64 + 32 + r] = f32x4{dq[4], dq[5], dq[6], dq[7]};
    } else {
      E* const to = reinterpret_cast<E*>(row_piece<D>(a, a.dQ, a.dqs, b, hk, m0 + r, 16 * c));
      store4<E>(to, dq[0], dq[1], dq[2], dq[3]);
      store4<E>(to + 4, dq[4], dq[5], dq[6], dq[7]);
    }
  }
}

// A workgroup's part of dQ; ring: kRowBytes of its LDS.  STATS: it leaves what the launch of dK and dV needs.
template <typename E, int D, bool STATS>
__device__ __forceinline__ void dq_part(const CrossGradArgs& a, unsigned char* ring, int unit_part) {
  using T = Tile<D>;
  using Z = RowPipe<D>;
  constexpr bool kLift = __is_same(E, _Float16);
  constexpr int kKeys = 64, N = kKeys / kWaves / T::RPI, kSlots = D / 8;
  const int unit = unit_part / a.key_parts, part = unit_part - unit * a.key_parts;
  const int bh = unit / a.row_tiles, hk = bh % a.Hk;
  const int64_t b = bh / a.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = (unit - bh * a.row_tiles) * 128 + wave * 32, m = m0 + (lane & 31);
  const bool on = m < a.M;
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring;

  // the attended states, in order: all of the first `count`, or those on the list; this workgroup has `n_tiles` tiles from `first` on
  StateLoads<D, N> states;
  states.list = a.list ? a.list + b * a.Nk : nullptr;
  states.count = a.list ? __builtin_amdgcn_readfirstlane(a.counts[b]) : length_of(a.k_len, b, a.Nk);
  const int all = (states.count + kKeys - 1) / kKeys, per = (all + a.key_parts - 1) / a.key_parts, first = part * per;
  const int n_tiles = max(0, min(per, all - first));
  states.kb = reinterpret_cast<const char*>(a.K) + 2 * (b * a.ks[0] + hk * a.ks[1]);
  states.vb = reinterpret_cast<const char*>(a.V) + 2 * (b * a.vs[0] + hk * a.vs[1]);
  states.ks = 2 * a.ks[2];
  states.vs = 2 * a.vs[2];
  states.r = wave * N * T::RPI + lane / T::CH;
  const auto fetch = [&](int i) {
    const uint32_t to = lds + wave * N * 1024;
    states.issue(lane, __builtin_amdgcn_readfirstlane(to + i % 3 * Z::kTile), __builtin_amdgcn_readfirstlane(to + (3 + i % 2) * Z::kTile));
  };
  if (n_tiles > 0) {
    states.choose(first);
    fetch(0);
    if (n_tiles > 1) {
      states.choose(first + 1);
      fetch(1);
    }
    if (n_tiles > 2) states.choose(first + 2);
  }

  // ---- the wave's rows of Q, dO and O --------------------------------------------------------------------------------------
  RowGrad<D> w;
  float top = 0.0f;
  w.delta = 0.0f;
  {
    typedef typename Vec<E>::x8 x8;
    const char* const qp = row_piece<D>(a, a.Q, a.qs, b, hk, m, 16 * half);
    const char* const gp = row_piece<D>(a, a.dO, a.gs, b, hk, m, 16 * half);
    const char* const op = row_piece<D>(a, a.O, a.os, b, hk, m, 16 * half);
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      w.q[ks] = *reinterpret_cast<const s16x8*>(qp + 32 * ks);
      w.g[ks] = *reinterpret_cast<const s16x8*>(gp + 32 * ks);
      const x8 o = *reinterpret_cast<const x8*>(op + 32 * ks), x = __builtin_bit_cast(x8, w.g[ks]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        w.delta += (float)o[e] * (float)x[e];
        if (kLift) top = fmaxf(top, fabsf((float)x[e]));
      }
    }
  }
  w.delta = swap_sum(w.delta);
  top = swap_max(top);
  const int mm = min(m, a.M - 1), t = a.G == 1 ? mm : mm / a.G, h = hk * a.G + (mm - t * a.G);
  const float lse = a.lse[(b * a.Hk * a.G + h) * a.T + t];
  w.lse = lse == -INFINITY ? INFINITY : lse * kLog2e;
  if (states.count <= kFewStates) {  // (sum_delta; here a lane has half of its row)
    typedef typename Vec<E>::x8 x8;
    w.delta = 0.0f;
    for (int i = 0; i < states.count; ++i) {
      const int j = states.list ? states.list[i] : i;
      const char* const kp = states.kb + j * states.ks + 16 * half;
      const char* const vp = states.vb + j * states.vs + 16 * half;
      float s = 0.0f, dp = 0.0f;
#pragma unroll
      for (int ks = 0; ks < T::KS; ++ks) {
        const x8 kx = *reinterpret_cast<const x8*>(kp + 32 * ks), vx = *reinterpret_cast<const x8*>(vp + 32 * ks);
        const x8 qx = __builtin_bit_cast(x8, w.q[ks]), gx = __builtin_bit_cast(x8, w.g[ks]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          s = __builtin_fmaf((float)kx[e], (float)qx[e], s);
          dp = __builtin_fmaf((float)vx[e], (float)gx[e], dp);
        }
      }
      w.delta += __builtin_amdgcn_exp2f(__builtin_fmaf(swap_sum(s), a.c2, -w.lse)) * swap_sum(dp);
    }
  }
  if (STATS && half == 0 && part == 0) {
    a.stat_lse[(int64_t)bh * a.row_tiles * 128 + m] = on ? w.lse - lift_p<E>() : INFINITY;
    a.stat_delta[(int64_t)bh * a.row_tiles * 128 + m] = on ? w.delta : 0.0f;
  }
  const float k = kLift ? lift(top) : 0.0f;
  if (kLift && lost(w.lse, w.delta)) top = INFINITY;
  if (states.count == 1) w.lse = INFINITY;
  w.lse += k;
  float* const tops = reinterpret_cast<float*>(ring + 2 * Z::kTile);         // (no tile is there yet)
  if constexpr (kLift && STATS) {
    float u = top;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) u = fmaxf(u, __shfl_xor(u, s));
    if (lane == 0) tops[wave] = u;
  }
  // the first step has a half tile before it like all others, of dS and states that are zero
  typedef __attribute__((address_space(3))) u32x4* lds_w_t;
  for (int c = threadIdx.x; c < T::SUB / 16; c += kThreads) *(lds_w_t)(uintptr_t)(lds + 2 * Z::kTile + T::SUB + 16 * c) = u32x4{0, 0, 0, 0};
  wait_loads();
  barrier();                         // the first tiles are there
  if (kLift && STATS && threadIdx.x == 0 && part == 0) a.top[unit] = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) w.dq[dt][v] = 0.0f;

  if (n_tiles > 0) {
    // what only matrix instructions touch, in the accumulator half
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) asm volatile("" : "+a"(w.dq[dt]));
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) asm volatile("" : "+a"(w.q[ks]), "+a"(w.g[ks]));
#pragma unroll
    for (int v = 0; v < 8; ++v) w.ds[1][v] = 0;
    const auto move = [](int tile) { return tile % 3 == 2 ? -2 * Z::kTile : Z::kTile; };        // to the next one's place
    const auto mask = [&](f32x16& s, int k0) {                     // scores of states from `count` on
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = k0 + row_of(v) + 4 * half < states.count ? s[v] : -INFINITY;
    };
    Z z;
    z.k = lds + row_at<D>(lane);
    z.v = z.k + 3 * Z::kTile;
    z.c = lds + 2 * Z::kTile + col_at<D>(lane);
#pragma unroll
    for (int v = 0; v < 16; ++v) w.s[0][v] = w.dp[0][v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      w.s[0] = mfma<E>(read_row(z.k ^ (ks << 5)), w.q[ks], w.s[0]);
      w.dp[0] = mfma<E>(read_row(z.v ^ (ks << 5)), w.g[ks], w.dp[0]);
    }
    preload<D, T::SUB, 0, Z::kAhead>(z);
    const auto none = [](int) {};
    for (int i = 0; i < n_tiles; ++i) {
      const int k0 = (first + i) * kKeys;
      z.k_move = move(i);
      z.v_move = i % 2 ? -Z::kTile : Z::kTile;
      z.c_move = move(i + 2);
      if (k0 + kKeys > states.count) mask(w.s[0], k0);
      // behind step A's turn tile i - 1, and of tile i its V, have been read and tile i + 1 is there
      slots<E, D, true, 0>(w, z, a.c2, none);
      if (k0 + kKeys > states.count) mask(w.s[1], k0 + 32);
      const auto loads = [&](int r) {
        if (r == 1 && i + 2 < n_tiles) fetch(i + 2);
        if (r == 3 && i + 3 < n_tiles) states.choose(first + i + 3);
      };
      slots<E, D, false, 0>(w, z, a.c2, loads);
    }
    // the last half tile's share
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) mfma_acc<E>(w.dq[dt], read_col<D>((z.c ^ (dt << 6)) + T::SUB + 16 * x * T::ROW), operand_of(&w.ds[1][4 * x]));
    // here, in front of any copy that the compiler makes of them where the paths meet
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) settle(w.dq[dt]);
  }
  const bool again = kLift && beyond(w.dq[0][0], on && top < INFINITY);
  const auto plain = [&](f32x4* to) {
    if constexpr (kLift)
      if (__builtin_expect(again, 0))
        dq_plain<E, D>(a, states.kb, states.vb, states.list, first * kKeys, min(states.count, (first + n_tiles) * kKeys), b, hk, m0, w.lse - k, w.delta, to);
  };
  const float f = kLift ? a.scale * __builtin_amdgcn_exp2f(k) : a.scale;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) w.dq[dt][v] *= f;
  if (a.key_parts > 1) {
    f32x4* const to = reinterpret_cast<f32x4*>(a.part_q) + (((int64_t)part * a.row_units + unit) * kWaves + wave) * kSlots * 64;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const f32x16& x = w.dq[s / 4];
      to[s * 64 + lane] = f32x4{x[4 * (s % 4)], x[4 * (s % 4) + 1], x[4 * (s % 4) + 2], x[4 * (s % 4) + 3]};
    }
    plain(to);
    return;
  }
  // through LDS: whole rows to memory
  barrier();                         // (all have read the last tile)
  typedef __attribute__((address_space(3))) u32x2* lds_8_t;
  typedef __attribute__((address_space(3))) const u32x4* lds_16_t;
  const uint32_t out = __builtin_amdgcn_readfirstlane(lds + wave * T::SUB);
  const int r = lane & 31;
#pragma unroll
  for (int s = 0; s < kSlots; ++s) {
    const f32x16& x = w.dq[s / 4];
    const u32x2 v = {pack2<E>(x[4 * (s % 4)], x[4 * (s % 4) + 1]), pack2<E>(x[4 * (s % 4) + 2], x[4 * (s % 4) + 3])};
    *(lds_8_t)(uintptr_t)(out + r * T::ROW + ((s ^ T::swz(r)) << 4) + 8 * half) = v;
  }
#pragma unroll
  for (int j = 0; j < T::SUB / 1024; ++j) {
    const int rr = j * T::RPI + lane / T::CH, c = ((lane % T::CH) ^ T::swz(rr)) << 4;
    const u32x4 v = *(lds_16_t)(uintptr_t)(out + j * 1024 + lane * 16);
    if (m0 + rr < a.M) *reinterpret_cast<u32x4*>(row_piece<D>(a, a.dQ, a.dqs, b, hk, m0 + rr, c)) = v;
  }
  plain(nullptr);
}
template <int D>
constexpr int kRowBytes = 5 * RowPipe<D>::kTile;                   // of LDS: three places of K, two of V

template <typename E, int D>
__global__ void __launch_bounds__(kThreads, 2) cross_dq_kernel(CrossGradArgs a) {
  __shared__ __align__(1024) unsigned char ring[kRowBytes<D>];
  const int unit_part = place(blockIdx.x, a.row_units * a.key_parts);
  if (unit_part >= 0) dq_part<E, D, true>(a, ring, unit_part);
}

// The parts of dQ added in order: a wave to 64 lanes' worth of eight values of d
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) cross_dq_join_kernel(CrossGradArgs a) {
  constexpr int kSlots = D / 8, kPer = kWaves * kSlots;            // pieces of a row unit
  const int64_t piece = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int unit = (int)(piece / kPer), of = (int)(piece - (int64_t)unit * kPer), wave = of / kSlots, s = of % kSlots;
  const int bh = unit / a.row_tiles, m = (unit - bh * a.row_tiles) * 128 + wave * 32 + (lane & 31);
  if (m >= a.M) return;
  const f32x4* const from = reinterpret_cast<const f32x4*>(a.part_q) + piece * 64 + lane;
  const int64_t step = (int64_t)a.row_units * kPer * 64;
  const f32x4 v = sum_parts(from, step, a.key_parts);
  store4<E>(reinterpret_cast<E*>(row_piece<D>(a, a.dQ, a.dqs, bh / a.Hk, bh % a.Hk, m, 2 * (8 * s + 4 * (lane >> 5)))), v[0], v[1], v[2], v[3]);
}

// ---- dK and dV: a software pipeline over half tiles of 32 rows -----------------------------------------------------------
// A step forms S and dO V^T of the half tile after the current one, P and dS of the current one, and what the one before it
// adds to dV and dK: a row of slots, each one matrix instruction (the four products in turn), an LDS read for a slot kAhead
// later and a slice of the probabilities.  Nothing moves between slots.  A tile of 64 rows is in LDS from its first product to
// its last, three half tiles on: there are three places.

template <int D>
struct KeyPipe {
  using T = Tile<D>;
  static constexpr int N = 4 * T::KS, kAhead = D == 128 ? 8 : 4;   // slots of a step: each of the four products has KS
  static constexpr int EACH = N / 16;                              // slots of a score: 2, or 1
  static constexpr int TURN = N - 4;
  static constexpr int kTile = 64 * T::ROW, kPlace = 2 * kTile;    // bytes of a tile of Q or dO, of both
  uint32_t k[T::KS], v[T::DT], v2[T::DT];                          // LDS addresses, by rows and by columns; v2: eight rows on
  uint32_t st;                                                     // of the rows' scalars
  int32_t k_move, v_move, st_move;                                 // from a tile's place to the next one's
  s16x8 f[kAhead];                                                 // operands on their way, slot r's in r mod kAhead
  f32x4 lse[2], delta[2];                                          // of four scores, and of the next four
  static_assert(N % kAhead == 0 && TURN >= N - kAhead, "a step's own reads are on their way at its turn");
};
constexpr int kStatPlace = 2 * 64 * 4;                             // bytes of a place's scalars: 64 lse, 64 delta

template <int D, int R, int OFF, bool MOVE>
__device__ __forceinline__ s16x8 operand(KeyPipe<D>& z) {
  using T = Tile<D>;
  constexpr int i = R / 4, kTile = KeyPipe<D>::kTile;
  if constexpr (R % 2 == 0) {        // Q, then dO by rows
    const s16x8 f = read_row(z.k[i] + OFF + (R % 4 == 2 ? kTile : 0));
    if constexpr (MOVE && R % 4 == 2) z.k[i] += z.k_move;
    return f;
  } else {                           // dO, then Q by columns
    constexpr int x = i / T::DT, dt = i % T::DT, off = OFF + 16 * x * T::ROW + (R % 4 == 1 ? kTile : 0);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)(z.v[dt] + off));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)(z.v2[dt] + off));
    if constexpr (MOVE && R % 4 == 3 && x == 1) {
      z.v[dt] += z.v_move;
      z.v2[dt] += z.v_move;
    }
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
template <int D, int OFF, bool MOVE, int FROM, int TO>
__device__ __forceinline__ void preload(KeyPipe<D>& z) {
  if constexpr (FROM < TO) {
    z.f[FROM % KeyPipe<D>::kAhead] = operand<D, FROM, OFF, MOVE>(z);
    preload<D, OFF, MOVE, FROM + 1, TO>(z);
  }
}
typedef __attribute__((address_space(3))) const f32x4* lds_f4_t;
template <int D>
__device__ __forceinline__ void scalars(KeyPipe<D>& z, int g, int off) {      // of scores 4 g ..
  z.lse[g & 1] = *(lds_f4_t)(uintptr_t)(z.st + off + 32 * g);
  z.delta[g & 1] = *(lds_f4_t)(uintptr_t)(z.st + off + 256 + 32 * g);
}

template <int D>
struct Keys {
  s16x8 kf[D / 16], vf[D / 16];      // the wave's 32 states: columns of the products over d
  f32x16 dk[D / 32], dv[D / 32];
  f32x16 s[2], dp[2];                // scores and dO V^T of the even and of the odd half tile
  uint32_t p[2][8], ds[2][8];
};

// Score Y, whose exponential is in e0 or e1: dS, and the pair as operands
template <typename E, int D, int CUR, int Y>
__device__ __forceinline__ void put(Keys<D>& w, const KeyPipe<D>& z, float f, float e0, float e1, float& d0, float& d1) {
  constexpr bool kLift = __is_same(E, _Float16);
  const float e = Y % 2 ? e1 : e0;
  float& ds = Y % 2 ? d1 : d0;
  ds = (kLift ? e * f : e) * (w.dp[CUR][Y] - z.delta[(Y / 4) & 1][Y % 4]);
  asm volatile("" : "+v"(ds));       // here, in its slot
  if constexpr (Y % 2 == 1) {
    w.p[CUR][Y / 2] = pack2<E>(e0, e1);
    w.ds[CUR][Y / 2] = pack2<E>(d0, d1);
    asm volatile("" : "+v"(w.p[CUR][Y / 2]), "+v"(w.ds[CUR][Y / 2]));
  }
}

// Step A walks rows of a tile's second half and columns of the second half before it, and ends with the turn to the next
// places; step B walks first halves and issues the tile loads (extra).
template <typename E, int D, bool A, int R, typename Extra>
__device__ __forceinline__ void slots(Keys<D>& w, KeyPipe<D>& z, float c2, float f, float& e0, float& e1, float& d0, float& d1, Extra& extra) {
  using T = Tile<D>;
  using Z = KeyPipe<D>;
  constexpr int N = Z::N, kAhead = Z::kAhead, i = R / 4, x = i / T::DT, dt = i % T::DT;
  constexpr int cur = A ? 0 : 1, other = 1 - cur, OFF = A ? T::SUB : 0;
  if constexpr (R < N) {
    const s16x8 u = z.f[R % kAhead];
    if constexpr (R % 4 == 0) {
      const f32x16 zero = {};
      if constexpr (i == 0) w.s[other] = mfma<E>(u, w.kf[i], zero);
      else w.s[other] = mfma<E>(u, w.kf[i], w.s[other]);
    } else if constexpr (R % 4 == 1) {
      mfma_acc<E>(w.dv[dt], u, operand_of(&w.p[other][4 * x]));
    } else if constexpr (R % 4 == 2) {
      const f32x16 zero = {};
      if constexpr (i == 0) w.dp[other] = mfma<E>(u, w.vf[i], zero);
      else w.dp[other] = mfma<E>(u, w.vf[i], w.dp[other]);
    } else {
      mfma_acc<E>(w.dk[dt], u, operand_of(&w.ds[other][4 * x]));
    }
    if constexpr (R + kAhead < N) z.f[R % kAhead] = operand<D, R + kAhead, OFF, A>(z);
    else if constexpr (!A) z.f[R % kAhead] = operand<D, R + kAhead - N, T::SUB, true>(z);
    if constexpr (A && R == Z::TURN) {
      wait_loads();
      barrier();
      preload<D, 0, false, 0, R % kAhead + 1>(z);                  // into the places of operands that have been used
    }
    if constexpr (A && R > Z::TURN) preload<D, 0, false, R % kAhead, R % kAhead + 1>(z);
    if constexpr (!A) extra(R);
    // a slice of the probabilities: score v takes EACH slots
    constexpr int v = R / Z::EACH;
    if constexpr (Z::EACH == 1 && v > 0) put<E, D, cur, v - 1>(w, z, f, e0, e1, d0, d1);
    if constexpr (R % Z::EACH == 0) {
      if constexpr (v % 4 == 0) {    // the next four's scalars; behind the last of a half tile, the next half tile's first
        if constexpr (v == 12) {
          if constexpr (!A) z.st += z.st_move;
          scalars<D>(z, 0, A ? 128 : 0);
        } else {
          scalars<D>(z, v / 4 + 1, A ? 0 : 128);
        }
      }
      (v % 2 ? e1 : e0) = __builtin_amdgcn_exp2f(__builtin_fmaf(w.s[cur][v], c2, -z.lse[(v / 4) & 1][v % 4]));
    } else {
      put<E, D, cur, v>(w, z, f, e0, e1, d0, d1);
    }
    __builtin_amdgcn_sched_barrier(0);
    slots<E, D, A, R + 1>(w, z, c2, f, e0, e1, d0, d1, extra);
  } else if constexpr (Z::EACH == 1) {
    put<E, D, cur, 15>(w, z, f, e0, e1, d0, d1);
  }
}
template <typename E, int D, bool A, typename Extra>
__device__ __forceinline__ void step(Keys<D>& w, KeyPipe<D>& z, float c2, float f, Extra extra) {
  float e0 = 0.0f, e1 = 0.0f, d0 = 0.0f, d1 = 0.0f;
  slots<E, D, A, 0>(w, z, c2, f, e0, e1, d0, d1, extra);
}

// A wave's share of a tile of 64 rows, N KiB of Q and of dO from row r0 on.  Rows past the last one are not fetched: the last
// one stands in for them.
template <int D, int N>
struct RowLoads {
  const char* q[N];
  const char* g[N];
  bool set;
  __device__ __forceinline__ void issue(const CrossGradArgs& a, int64_t b, int hk, int m, int r0, int lane, uint32_t lds) {
    using T = Tile<D>;
    // where 64 rows are a whole number of tokens, a tile's addresses are the last one's and a step
    if (!set || m + 64 > a.M || 64 % a.G != 0) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int r = r0 + j * T::RPI + lane / T::CH, mm = min(m + r, a.M - 1);
        const int64_t t = mm / a.G, h = (int64_t)hk * a.G + mm % a.G;
        const int c = ((lane % T::CH) ^ T::swz(r)) << 4;
        q[j] = reinterpret_cast<const char*>(a.Q) + 2 * (b * a.qs[0] + h * a.qs[1] + t * a.qs[2]) + c;
        g[j] = reinterpret_cast<const char*>(a.dO) + 2 * (b * a.gs[0] + h * a.gs[1] + t * a.gs[2]) + c;
      }
      set = true;
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        q[j] += 2 * (64 / a.G) * a.qs[2];
        g[j] += 2 * (64 / a.G) * a.gs[2];
      }
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      load_lds(q[j], lds + j * 1024);
      load_lds(g[j], lds + 64 * T::ROW + j * 1024);
    }
  }
};

// dK of a wave's states again where fp16 has not held their dS: in binary32, a state after the other, the rows over groups of D / 8
// lanes.  lse and delta: of the rows, tiles of 64 `step` apart.  Written over what has been written.
template <typename E, int D>
__device__ __forceinline__ void dk_plain(const CrossGradArgs& a, const float* lse, const float* delta, int step, int m_first, int m_end, int64_t b,
                                         int hk, int key0, uint32_t on, f32x4* part) {
  typedef typename Vec<E>::x8 x8;
  constexpr int LPK = D / 8, KPI = 64 / LPK;
  const int lane = threadIdx.x & 63, grp = lane / LPK, c = lane % LPK;
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
#pragma unroll 1
  for (; on != 0; on &= on - 1) {
    const int x = __builtin_ctz(on);
    const int64_t key = key0 + x;
    const x8 k = *reinterpret_cast<const x8*>(reinterpret_cast<const E*>(a.K) + b * a.ks[0] + hk * a.ks[1] + key * a.ks[2] + 8 * c);
    const x8 v = *reinterpret_cast<const x8*>(reinterpret_cast<const E*>(a.V) + b * a.vs[0] + hk * a.vs[1] + key * a.vs[2] + 8 * c);
    float dk[8] = {};
#pragma unroll 1
    for (int i0 = 0; i0 < m_end - m_first; i0 += KPI) {
      const int i = min(i0 + grp, m_end - m_first - 1), at = i / 64 * step + i % 64;
      const x8 q = *reinterpret_cast<const x8*>(row_piece<D>(a, a.Q, a.qs, b, hk, m_first + i, 16 * c));
      const x8 g = *reinterpret_cast<const x8*>(row_piece<D>(a, a.dO, a.gs, b, hk, m_first + i, 16 * c));
      float s = 0.0f, dp = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s = __builtin_fmaf((float)k[e], (float)q[e], s);
        dp = __builtin_fmaf((float)v[e], (float)g[e], dp);
      }
      s = over_row<LPK>(s);
      dp = over_row<LPK>(dp);
      const float ds = i0 + grp < m_end - m_first ? __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.c2, -lse[at] - lift_p<E>())) * (dp - delta[at]) : 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) dk[e] = __builtin_fmaf(ds, (float)q[e], dk[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) dk[e] = over_groups<LPK>(dk[e]) * a.scale;
    if (grp != 0) continue;
    if (part) {
      part[c * 64 + x] = f32x4{dk[0], dk[1], dk[2], dk[3]};
      part[c * 64 + 32 + x] = f32x4{dk[4], dk[5], dk[6], dk[7]};
    } else {
      E* const to = reinterpret_cast<E*>(a.dK) + b * a.dks[0] + hk * a.dks[1] + key * a.dks[2] + 8 * c;
      store4<E>(to, dk[0], dk[1], dk[2], dk[3]);
      store4<E>(to + 4, dk[4], dk[5], dk[6], dk[7]);
    }
  }
}

// A workgroup's part of dK and dV; ring: kKeyBytes of its LDS.  OWN: up to three tiles of rows, whose lse and delta it forms by
// itself; else they are those that the launch of dQ has left.
template <typename E, int D, bool OWN>
__device__ __forceinline__ void dkv_part(const CrossGradArgs& a, unsigned char* ring, int unit_part) {
  using T = Tile<D>;
  using Z = KeyPipe<D>;
  constexpr bool kLift = __is_same(E, _Float16);
  constexpr int kRows = 64, N = kRows / kWaves / T::RPI, kSlots = D / 8;
  const int unit = unit_part / a.parts, part = unit_part - unit * a.parts;
  const int bh = unit / a.key_tiles, hk = bh % a.Hk;
  const int64_t b = bh / a.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key0 = (unit - bh * a.key_tiles) * 128 + wave * 32, key = key0 + (lane & 31);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)ring, st = lds + 3 * Z::kPlace;

  const Attended keys = attended_of(a.k_len, a.k_mask, a.mask_stride_b, b, a.Nk);
  const int m_end = min(a.M, (part + 1) * a.part_rows), len = keys.len;
  const int32_t* const list = a.list ? a.list + b * a.Nk : nullptr;
  const int count = a.list ? __builtin_amdgcn_readfirstlane(a.counts[b]) : len;          // of attended states
  const uint32_t on_bits = (uint32_t)keys.bits<32>(key0, lane);
  const bool on = on_bits >> (lane & 31) & 1;
  // a tile past the sequence's states has nothing to add up
  const int m_first = (unit - bh * a.key_tiles) * 128 >= len ? m_end : min(part * a.part_rows, m_end);
  const int n_tiles = (m_end - m_first + kRows - 1) / kRows;
  Keys<D> w;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) w.dk[dt][v] = w.dv[dt][v] = 0.0f;
  float unlift = a.scale, top = 0.0f;                              // top: the largest |dO| of the rows
  if (n_tiles > 0) {
    if constexpr (kLift && !OWN) {
      for (int i = m_first / 128 + lane; i * 128 < m_end; i += 64) top = fmaxf(top, a.top[(int64_t)bh * a.row_tiles + i]);
    }
    RowLoads<D, N> rows;
    rows.set = false;
    const int r0 = wave * N * T::RPI;
    const float* scalars_at = (wave == 0 ? a.stat_lse : a.stat_delta) + (int64_t)bh * a.row_tiles * 128 + m_first + lane;
    const auto fetch = [&](int i) {  // tiles in turn
      const int to = i % 3, m = m_first + i * kRows;
      rows.issue(a, b, hk, m, r0, lane, __builtin_amdgcn_readfirstlane(lds + to * Z::kPlace + r0 * T::ROW));
      if (!OWN && wave < 2) {        // the rows' scalars: a wave brings each kind
        load_lds4(scalars_at, __builtin_amdgcn_readfirstlane(st + to * kStatPlace + wave * 256));
        if (i + 1 < n_tiles) scalars_at += kRows;
      }
    };
    // The wave's states through the second and the third place.  One that is not attended, or a last one that stands in for one
    // past the end, has a column to itself: whatever it holds reaches no other.
    const uint32_t kv = __builtin_amdgcn_readfirstlane(lds + Z::kPlace + wave * T::SUB);
    const char* from[2][T::SUB / 1024];
#pragma unroll
    for (int j = 0; j < T::SUB / 1024; ++j) {
      const int r = j * T::RPI + lane / T::CH, kk = min(key0 + r, a.Nk - 1), c = ((lane % T::CH) ^ T::swz(r)) << 4;
      from[0][j] = reinterpret_cast<const char*>(a.K) + 2 * (b * a.ks[0] + hk * a.ks[1] + kk * a.ks[2]) + c;
      from[1][j] = reinterpret_cast<const char*>(a.V) + 2 * (b * a.vs[0] + hk * a.vs[1] + kk * a.vs[2]) + c;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < T::SUB / 1024; ++j) load_lds(from[i][j], kv + i * Z::kPlace + j * 1024);
    fetch(0);
    if constexpr (OWN) {             // D / 8 lanes to a row
      typedef typename Vec<E>::x8 x8;
      float* const stat = reinterpret_cast<float*>(ring + 3 * Z::kPlace);
      constexpr int kBatch = kRows / (kWaves * T::RPI);            // loads of a tile, on their way together
      for (int i = 0; i < n_tiles; ++i) {
        x8 x[kBatch], o[kBatch];
        float lse[kBatch];
        const auto row_of_load = [&](int u) { return (u * kWaves + wave) * T::RPI + lane / T::CH; };
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int r = i * kRows + row_of_load(u), mm = min(r, a.M - 1), t = a.G == 1 ? mm : mm / a.G, h = hk * a.G + (mm - t * a.G);
          x[u] = *reinterpret_cast<const x8*>(row_piece<D>(a, a.dO, a.gs, b, hk, r, lane % T::CH * 16));
          o[u] = *reinterpret_cast<const x8*>(row_piece<D>(a, a.O, a.os, b, hk, r, lane % T::CH * 16));
          lse[u] = r < a.M ? a.lse[(b * a.Hk * a.G + h) * a.T + t] : -INFINITY;
        }
        float delta[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          delta[u] = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            delta[u] = __builtin_fmaf((float)o[u][e], (float)x[u][e], delta[u]);
            if (kLift) top = fmaxf(top, fabsf((float)x[u][e]));
          }
          delta[u] = over_row<T::CH>(delta[u]);
          lse[u] = lse[u] == -INFINITY ? INFINITY : lse[u] * kLog2e;
        }
        if (count <= kFewStates) {
          float qf[kBatch][8], gf[kBatch][8];
#pragma unroll
          for (int u = 0; u < kBatch; ++u) {
            const x8 y = *reinterpret_cast<const x8*>(row_piece<D>(a, a.Q, a.qs, b, hk, i * kRows + row_of_load(u), lane % T::CH * 16));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              qf[u][e] = (float)y[e];
              gf[u][e] = (float)x[u][e];
            }
          }
          sum_delta<E, D, kBatch>(a, list, count, b, hk, lane % T::CH * 8, qf, gf, lse, delta);
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          if (kLift && lost(lse[u], delta[u])) top = INFINITY;
          if (lane % T::CH == 0) {
            float* const to = stat + 2 * kRows * i + row_of_load(u);
            to[0] = lse[u] - lift_p<E>();
            to[kRows] = i * kRows + row_of_load(u) < a.M ? delta[u] : 0.0f;
          }
        }
      }
    }
    if constexpr (kLift) {
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
      if constexpr (OWN) {
        float* const tops = reinterpret_cast<float*>(ring + 3 * Z::kPlace + 3 * kStatPlace);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
      }
    }
    const float k_lift = kLift ? lift(top) : 0.0f, f = __builtin_amdgcn_exp2f(-k_lift - lift_p<E>());
    unlift = a.scale * __builtin_amdgcn_exp2f(k_lift);
    wait_loads();
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      w.kf[ks] = read_row((kv + row_at<D>(lane)) ^ (ks << 5));
      w.vf[ks] = read_row((kv + Z::kPlace + row_at<D>(lane)) ^ (ks << 5));
    }
#pragma unroll
    for (int j = 0; j < T::SUB / 1024; ++j) asm volatile("" : : "v"(from[0][j]), "v"(from[1][j]));
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    barrier();                       // (all have read their states)
    if (n_tiles > 1) fetch(1);
    // what only matrix instructions touch, in the accumulator half
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) asm volatile("" : "+a"(w.dk[dt]), "+a"(w.dv[dt]));
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) asm volatile("" : "+a"(w.kf[ks]), "+a"(w.vf[ks]));
    // the first step has a half tile before it like all others, of probabilities and rows that are zero
    typedef __attribute__((address_space(3))) u32x4* lds_w_t;
    for (int c = threadIdx.x; c < T::SUB / 16; c += kThreads) {
      const uint32_t to = lds + 2 * Z::kPlace + T::SUB + 16 * c;
      *(lds_w_t)(uintptr_t)to = u32x4{0, 0, 0, 0};
      *(lds_w_t)(uintptr_t)(to + Z::kTile) = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int v = 0; v < 8; ++v) w.p[1][v] = w.ds[1][v] = 0;
    const auto move = [](int tile, int bytes) { return tile % 3 == 2 ? -2 * bytes : bytes; };   // to the next one's place
    Z z;
    {
      const uint32_t k = lds + row_at<D>(lane), c = col_at<D>(lane);
#pragma unroll
      for (int ks = 0; ks < T::KS; ++ks) z.k[ks] = k ^ (ks << 5);
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) {
        z.v[dt] = lds + 2 * Z::kPlace + (c ^ (dt << 6));
        z.v2[dt] = lds + 2 * Z::kPlace + (c ^ (dt << 6) ^ 32) + 8 * T::ROW;
      }
      z.st = st + 16 * half;
      z.k_move = z.st_move = 0;
      z.v_move = 0;
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) w.s[0][v] = w.dp[0][v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) {
      w.s[0] = mfma<E>(read_row(z.k[ks]), w.kf[ks], w.s[0]);
      w.dp[0] = mfma<E>(read_row(z.k[ks] + Z::kTile), w.vf[ks], w.dp[0]);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");           // (the zeros)
    barrier();
    scalars<D>(z, 0, 0);
    z.k_move = move(0, Z::kPlace);
    z.v_move = move(2, Z::kPlace);
    preload<D, T::SUB, true, 0, Z::kAhead>(z);
    const auto none = [](int) {};
    for (int i = 0; i < n_tiles; ++i) {
      // behind step A's turn tile i - 1 has been read and tile i + 1 is there
      step<E, D, true>(w, z, a.c2, f, none);
      z.k_move = move(i + 1, Z::kPlace);
      z.v_move = move(i, Z::kPlace);
      z.st_move = move(i, kStatPlace);
      step<E, D, false>(w, z, a.c2, f, [&](int r) {
        if (r == 1 && i + 2 < n_tiles) fetch(i + 2);
      });
    }
    // the last half tile's share
    const uint32_t last = lds + (n_tiles - 1) % 3 * Z::kPlace + T::SUB, c = col_at<D>(lane);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) {
        const uint32_t at = last + 16 * x * T::ROW + (c ^ (dt << 6));
        mfma_acc<E>(w.dv[dt], read_col<D>(at + Z::kTile), operand_of(&w.p[1][4 * x]));
        mfma_acc<E>(w.dk[dt], read_col<D>(at), operand_of(&w.ds[1][4 * x]));
      }
    // here, in front of any copy that the compiler makes of them where the paths meet
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) {
      settle(w.dk[dt]);
      settle(w.dv[dt]);
    }
  }
  if (count == 1) unlift = 0.0f;
  const bool again = kLift && beyond(w.dk[0][0], on && top < INFINITY && count != 1);
  const auto plain = [&](f32x4* to) {
    if constexpr (kLift) {
      if (__builtin_expect(again, 0)) {
        const int64_t row = (int64_t)bh * a.row_tiles * 128 + m_first;
        const float* const own = reinterpret_cast<const float*>(ring + 3 * Z::kPlace);
        dk_plain<E, D>(a, OWN ? own : a.stat_lse + row, OWN ? own + kRows : a.stat_delta + row, OWN ? 2 * kRows : kRows, m_first, m_end, b, hk, key0,
                       on_bits, to);
      }
    }
  };
  const float unlift_p = __builtin_amdgcn_exp2f(-lift_p<E>());
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt) {
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      w.dk[dt][v] = on ? w.dk[dt][v] * unlift : 0.0f;
      w.dv[dt][v] = on ? w.dv[dt][v] * unlift_p : 0.0f;
    }
  }
  if (a.parts > 1) {
    f32x4* const to = reinterpret_cast<f32x4*>(a.part) + (((int64_t)part * a.key_units + unit) * 2 * kWaves + wave) * kSlots * 64;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const f32x16 &k = w.dk[s / 4], &v = w.dv[s / 4];
      to[s * 64 + lane] = f32x4{k[4 * (s % 4)], k[4 * (s % 4) + 1], k[4 * (s % 4) + 2], k[4 * (s % 4) + 3]};
      to[(kWaves * kSlots + s) * 64 + lane] = f32x4{v[4 * (s % 4)], v[4 * (s % 4) + 1], v[4 * (s % 4) + 2], v[4 * (s % 4) + 3]};
    }
    plain(to);
    return;
  }
  if (key < a.Nk) {
    E* const tk = reinterpret_cast<E*>(a.dK) + b * a.dks[0] + hk * a.dks[1] + key * a.dks[2] + 4 * half;
    E* const tv = reinterpret_cast<E*>(a.dV) + b * a.dvs[0] + hk * a.dvs[1] + key * a.dvs[2] + 4 * half;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const f32x16 &k = w.dk[s / 4], &v = w.dv[s / 4];
      store4<E>(tk + 8 * s, k[4 * (s % 4)], k[4 * (s % 4) + 1], k[4 * (s % 4) + 2], k[4 * (s % 4) + 3]);
      store4<E>(tv + 8 * s, v[4 * (s % 4)], v[4 * (s % 4) + 1], v[4 * (s % 4) + 2], v[4 * (s % 4) + 3]);
    }
  }
  plain(nullptr);
}
template <int D>
constexpr int kKeyBytes = 3 * (KeyPipe<D>::kPlace + kStatPlace) + 16;        // of LDS: three places of Q and dO, of the rows' scalars

template <typename E, int D>
__global__ void __launch_bounds__(kThreads, D == 128 ? 1 : 2) cross_dkv_kernel(CrossGradArgs a) {
  __shared__ __align__(1024) unsigned char ring[kKeyBytes<D>];
  const int unit_part = place(blockIdx.x, a.key_units * a.parts);
  if (unit_part >= 0) dkv_part<E, D, false>(a, ring, unit_part);
}

// Up to three tiles of rows: dQ, and dK and dV, in one launch
template <typename E, int D>
__global__ void __launch_bounds__(kThreads, D == 128 ? 1 : 2) cross_grad_small_kernel(CrossGradArgs a) {
  __shared__ __align__(1024) unsigned char ring[kRowBytes<D> > kKeyBytes<D> ? kRowBytes<D> : kKeyBytes<D>];
  const int n = a.row_units * a.key_parts, at = place(blockIdx.x, n + a.key_units);
  if (at < 0) return;
  if (at < n) dq_part<E, D, false>(a, ring, at);
  else dkv_part<E, D, true>(a, ring, at - n);
}

// The parts added in order: a wave to 64 lanes' worth of eight values of d
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) cross_dkv_join_kernel(CrossGradArgs a) {
  constexpr int kSlots = D / 8, kPer = 2 * kWaves * kSlots;        // pieces of a key unit
  const int64_t piece = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int unit = (int)(piece / kPer), of = (int)(piece - (int64_t)unit * kPer);
  const int which = of / (kWaves * kSlots), wave = of / kSlots % kWaves, s = of % kSlots;
  const f32x4* const from = reinterpret_cast<const f32x4*>(a.part) + piece * 64 + lane;
  const int64_t step = (int64_t)a.key_units * kPer * 64;
  const f32x4 v = sum_parts(from, step, a.parts);
  const int bh = unit / a.key_tiles, hk = bh % a.Hk, key = (unit - bh * a.key_tiles) * 128 + wave * 32 + (lane & 31);
  const int64_t b = bh / a.Hk;
  if (key >= a.Nk) return;
  const int64_t* const st = which ? a.dvs : a.dks;
  E* const to = reinterpret_cast<E*>(which ? a.dV : a.dK) + b * st[0] + hk * st[1] + key * st[2] + 8 * s + 4 * (lane >> 5);
  store4<E>(to, v[0], v[1], v[2], v[3]);
}

// ---- up to four rows -----------------------------------------------------------------------------------------------------
// No matrix instruction: D / 8 lanes hold a state's row of K and of V, 8 elements each, KPI states to a wave's load, kBatch loads
// on their way.  K and V are read once, dK and dV written once, all in binary32; dQ is summed over the states of a group of
// lanes, then over groups, waves and workgroups, in order.  Bound by memory: 36 sequences of one row, up to 4462 states of 7
// heads of 64, 114 us (matrix instructions with 31 of 32 rows empty, in two launches: 335); 2 x 2 x 1749 x 5 heads of 128: 11.
constexpr int kFewWaves = 8;
template <typename E, int D, int MR>
__global__ void __launch_bounds__(64 * kFewWaves) cross_grad_few_kernel(CrossGradArgs a) {
  constexpr int LPK = D / 8, KPI = 64 / LPK, kBatch = MR == 4 ? 2 : 4;
  __shared__ float sums[kFewWaves][MR][D];
  __shared__ int few[kFewStates];    // the attended states of a mask, if they are so few
  typedef typename Vec<E>::x8 x8;
  const int unit_part = place(blockIdx.x, a.row_units * a.key_parts);
  if (unit_part < 0) return;
  const int unit = unit_part / a.key_parts, part = unit_part - unit * a.key_parts, hk = unit % a.Hk;
  const int64_t b = unit / a.Hk;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, grp = lane / LPK, d0 = lane % LPK * 8;
  float q[MR][8], g[MR][8], dq[MR][8], lse[MR], delta[MR];
#pragma unroll
  for (int r = 0; r < MR; ++r) {
    const x8 x = *reinterpret_cast<const x8*>(row_piece<D>(a, a.Q, a.qs, b, hk, r, 2 * d0));
    const x8 y = *reinterpret_cast<const x8*>(row_piece<D>(a, a.dO, a.gs, b, hk, r, 2 * d0));
    const x8 o = *reinterpret_cast<const x8*>(row_piece<D>(a, a.O, a.os, b, hk, r, 2 * d0));
    const int mm = min(r, a.M - 1), t = mm / a.G, h = hk * a.G + (mm - t * a.G);
    const float v = a.lse[(b * a.Hk * a.G + h) * a.T + t];
    lse[r] = r >= a.M || v == -INFINITY ? INFINITY : v * kLog2e;
    delta[r] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[r][e] = (float)x[e];
      g[r][e] = (float)y[e];
      dq[r][e] = 0.0f;
      delta[r] = __builtin_fmaf((float)o[e], g[r][e], delta[r]);
    }
    delta[r] = over_row<LPK>(delta[r]);
  }
  const Attended keys = attended_of(a.k_len, a.k_mask, a.mask_stride_b, b, a.Nk);
  const int len = keys.len;
  const uint8_t* const mask = keys.mask;
  const E* const kb = reinterpret_cast<const E*>(a.K) + b * a.ks[0] + hk * a.ks[1] + d0;
  const E* const vb = reinterpret_cast<const E*>(a.V) + b * a.vs[0] + hk * a.vs[1] + d0;
  E* const dkb = reinterpret_cast<E*>(a.dK) + b * a.dks[0] + hk * a.dks[1] + d0;
  E* const dvb = reinterpret_cast<E*>(a.dV) + b * a.dvs[0] + hk * a.dvs[1] + d0;
  const int count = mask ? few_attended(keys, lane, few) : len;
  if (count <= kFewStates) sum_delta<E, D, MR>(a, mask ? few : nullptr, count, b, hk, d0, q, g, lse, delta);
  for (int64_t k0 = (int64_t)(part * waves + wave) * KPI * kBatch; k0 < a.Nk; k0 += (int64_t)a.key_parts * waves * KPI * kBatch) {
    u32x4 kr[kBatch], vr[kBatch];
    bool on[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      on[u] = false;
      kr[u] = vr[u] = u32x4{0, 0, 0, 0};
    }
    if (k0 < len) {                                // (else all of them are past the end)
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int64_t k = k0 + u * KPI + grp, at = k < len ? k : len - 1;
        on[u] = k < len && (!mask || mask[at] != 0);
        kr[u] = *reinterpret_cast<const u32x4*>(kb + at * a.ks[2]);
        vr[u] = *reinterpret_cast<const u32x4*>(vb + at * a.vs[2]);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const u32x4 zero = {0, 0, 0, 0};             // a state that is not attended may hold NaN
      const x8 kx = __builtin_bit_cast(x8, on[u] ? kr[u] : zero), vx = __builtin_bit_cast(x8, on[u] ? vr[u] : zero);
      float kf[8], vf[8], dk[8], dv[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        kf[e] = (float)kx[e];
        vf[e] = (float)vx[e];
        dk[e] = dv[e] = 0.0f;
      }
#pragma unroll
      for (int r = 0; r < MR; ++r) {
        float s = kf[0] * q[r][0], dp = vf[0] * g[r][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) {
          s = __builtin_fmaf(kf[e], q[r][e], s);
          dp = __builtin_fmaf(vf[e], g[r][e], dp);
        }
        s = over_row<LPK>(s);
        dp = over_row<LPK>(dp);
        const float p = on[u] ? __builtin_amdgcn_exp2f(__builtin_fmaf(s, a.c2, -lse[r])) : 0.0f;
        const float ds = on[u] && count != 1 ? p * (dp - delta[r]) * a.scale : 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          dq[r][e] = __builtin_fmaf(ds, kf[e], dq[r][e]);
          dk[e] = __builtin_fmaf(ds, q[r][e], dk[e]);
          dv[e] = __builtin_fmaf(p, g[r][e], dv[e]);
        }
      }
      const int64_t k = k0 + u * KPI + grp;
      if (k < a.Nk) {
        const u32x4 x = {pack2<E>(dk[0], dk[1]), pack2<E>(dk[2], dk[3]), pack2<E>(dk[4], dk[5]), pack2<E>(dk[6], dk[7])};
        const u32x4 y = {pack2<E>(dv[0], dv[1]), pack2<E>(dv[2], dv[3]), pack2<E>(dv[4], dv[5]), pack2<E>(dv[6], dv[7])};
        *reinterpret_cast<u32x4*>(dkb + k * a.dks[2]) = on[u] ? x : zero;     // (0 times a row that holds NaN is none)
        *reinterpret_cast<u32x4*>(dvb + k * a.dvs[2]) = on[u] ? y : zero;
      }
    }
  }
#pragma unroll
  for (int r = 0; r < MR; ++r) {
#pragma unroll
    for (int e = 0; e < 8; ++e) dq[r][e] = over_groups<LPK>(dq[r][e]);
    if (grp == 0) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4*>(&sums[wave][r][d0 + e]) = f32x4{dq[r][e], dq[r][e + 1], dq[r][e + 2], dq[r][e + 3]};
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < a.M * D; i += blockDim.x) {
    const int r = i / D, d = i % D;
    float v = sums[0][r][d];
    for (int k = 1; k < waves; ++k) v += sums[k][r][d];
    if (a.key_parts > 1) a.part_q[((int64_t)unit_part * a.M + r) * D + d] = v;
    else *reinterpret_cast<E*>(row_piece<D>(a, a.dQ, a.dqs, b, hk, r, 2 * d)) = (E)v;
  }
}

// dQ of a row from its parts: D / 4 lanes to its values, the others share out the parts
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) cross_grad_few_join_kernel(CrossGradArgs a) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes;
  __shared__ f32x4 sums[kGroups][kLanes];
  const int unit = blockIdx.x / a.M, r = blockIdx.x - unit * a.M, c = threadIdx.x % kLanes, g = threadIdx.x / kLanes;
  const f32x4* const from = reinterpret_cast<const f32x4*>(a.part_q) + ((int64_t)unit * a.key_parts * a.M + r) * kLanes + c;
  const int64_t step = (int64_t)a.M * kLanes;
  f32x4 v = g < a.key_parts ? sum_parts(from + g * step, kGroups * step, (a.key_parts - g + kGroups - 1) / kGroups) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  sums[g][c] = v;
  __syncthreads();
  if (g != 0) return;
#pragma unroll
  for (int k = 1; k < kGroups; ++k) v += sums[k][c];
  store4<E>(reinterpret_cast<E*>(row_piece<D>(a, a.dQ, a.dqs, unit / a.Hk, unit % a.Hk, r, 8 * c)), v[0], v[1], v[2], v[3]);
}

// How a call is shared out.
struct CrossGradShape {
  int64_t M, heads, row_tiles, key_tiles, parts, part_rows, key_parts;
  int waves;                           // up to four rows: of a workgroup; else 0
  bool small;                          // one launch for all three gradients
  size_t stat_bytes, top_bytes, list_bytes, part_q_bytes, bytes;
};
constexpr int kFill = 256, kFewFill = 512;
CrossGradShape cross_grad_shape(const pbsa_cross& p) {
  CrossGradShape s{};
  const auto up = [](size_t n) { return (n + 255) & ~(size_t)255; };
  s.heads = (int64_t)p.n * p.Hk;
  s.M = p.Hk > 0 ? (int64_t)p.T * (p.Hq / p.Hk) : 0;
  s.parts = s.key_parts = 1;
  if (s.M >= 1 && s.M <= 4 && p.Nk > 0) {
    const int64_t batch = 64 / (p.d / 8) * (s.M > 2 ? 2 : 4), turns = ((int64_t)p.Nk + batch - 1) / batch;   // states of a wave at a time
    s.row_tiles = 1;
    s.waves = 2;
    while (s.waves < kFewWaves && s.waves < turns) s.waves *= 2;
    while (s.key_parts * s.waves < turns && s.heads * s.key_parts * 2 <= kFewFill) s.key_parts *= 2;
    s.bytes = s.part_q_bytes = s.key_parts > 1 ? up((size_t)(s.heads * s.key_parts * s.M) * p.d * sizeof(float)) : 0;
    return s;
  }
  s.row_tiles = (s.M + 127) / 128;
  s.key_tiles = ((int64_t)p.Nk + 127) / 128;
  // One round of workgroups: one has a compute unit to itself.  A part saves its tiles (64 rows or states: half a microsecond to
  // one) and costs its share of a launch that adds the parts up (four microseconds).
  const int64_t units = s.heads * s.key_tiles, tiles = (s.M + 63) / 64;
  if (units > 0 && tiles >= 6) s.parts = std::max<int64_t>(1, std::min(kFill / units, tiles / 2));
  const int64_t per = (tiles + s.parts - 1) / s.parts;
  if (per > 0) s.parts = (tiles + per - 1) / per;
  s.part_rows = per * 64;
  const int64_t row_units = s.heads * s.row_tiles, states = ((int64_t)p.Nk + 63) / 64;
  if (row_units > 0 && states >= 10) s.key_parts = std::max<int64_t>(1, std::min(kFill / row_units, states / 3));
  // One launch for all three gradients where it is one round of workgroups: a launch is saved, and dK's workgroups form the row
  // sums that dQ's would have left (2 x 10 x 227 x 12 heads of 128: 14.1 us, in two launches 24.4; 6 x 24 x 25 x 11 of 64: 7.0 and
  // 13.2).  In more rounds each of them reads the rows again (3 x 23 x 2306 x 33 of 128, 11 shared: 79 us, in two launches 69).
  s.small = s.M > 0 && p.Nk > 0 && tiles <= 3 && row_units * s.key_parts + units <= (p.d == 64 ? 2 : 1) * kFill;
  s.stat_bytes = up((size_t)row_units * 128 * sizeof(float));
  s.top_bytes = up((size_t)row_units * sizeof(float));
  s.list_bytes = row_units > 0 && p.Nk > 0 ? up(attended_bytes(p.n, p.Nk)) : 0;
  s.part_q_bytes = s.key_parts > 1 ? up((size_t)(s.key_parts * row_units) * 128 * p.d * sizeof(float)) : 0;
  s.bytes = 2 * s.stat_bytes + s.top_bytes + s.list_bytes + s.part_q_bytes + (s.parts > 1 ? (size_t)(s.parts * units) * 2 * 128 * p.d * sizeof(float) : 0);
  return s;
}

template <typename E, int D>
hipError_t launch_typed(const CrossGradShape& s, const CrossGradArgs& a, int n, hipStream_t stream) {
  const auto grid = [](int64_t k) { return dim3((unsigned)((k + 7) / 8 * 8)); };
  if (s.waves > 0) {
    const dim3 at = grid((int64_t)a.row_units * a.key_parts), block(64 * s.waves);
    if (a.M == 1) hipLaunchKernelGGL((cross_grad_few_kernel<E, D, 1>), at, block, 0, stream, a);
    else if (a.M == 2) hipLaunchKernelGGL((cross_grad_few_kernel<E, D, 2>), at, block, 0, stream, a);
    else hipLaunchKernelGGL((cross_grad_few_kernel<E, D, 4>), at, block, 0, stream, a);
    if (a.key_parts > 1)
      hipLaunchKernelGGL((cross_grad_few_join_kernel<E, D>), dim3((unsigned)(a.row_units * a.M)), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  if (a.list) {
    // without its list the next launch has nothing to go by
    const hipError_t e = launch_attended(a.k_len, a.k_mask, a.mask_stride_b, n, a.Nk, const_cast<int32_t*>(a.list), const_cast<int32_t*>(a.counts), stream);
    if (e != hipSuccess) return e;
  }
  if (s.small) {
    hipLaunchKernelGGL((cross_grad_small_kernel<E, D>), grid((int64_t)a.row_units * a.key_parts + a.key_units), dim3(kThreads), 0, stream, a);
    if (a.key_parts > 1)
      hipLaunchKernelGGL((cross_dq_join_kernel<E, D>), dim3((unsigned)(a.row_units * (D / 8))), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  if (a.row_units > 0) {
    hipLaunchKernelGGL((cross_dq_kernel<E, D>), grid((int64_t)a.row_units * a.key_parts), dim3(kThreads), 0, stream, a);
    if (a.key_parts > 1)
      hipLaunchKernelGGL((cross_dq_join_kernel<E, D>), dim3((unsigned)(a.row_units * (D / 8))), dim3(kThreads), 0, stream, a);
  }
  if (a.key_units > 0) {
    hipLaunchKernelGGL((cross_dkv_kernel<E, D>), grid((int64_t)a.key_units * a.parts), dim3(kThreads), 0, stream, a);
    if (a.parts > 1)
      hipLaunchKernelGGL((cross_dkv_join_kernel<E, D>), dim3((unsigned)(a.key_units * 2 * (D / 8))), dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace

size_t cross_bwd_workspace_bytes(const pbsa_cross& p) { return cross_grad_shape(p).bytes; }

hipError_t launch_cross_bwd(const pbsa_cross& p, const void* Q, const void* K, const void* V, const int32_t* k_len, const uint8_t* k_mask,
                            const void* O, const void* dO, const float* lse, void* dQ, void* dK, void* dV, void* ws,
                            hipStream_t stream) {
  const CrossGradShape s = cross_grad_shape(p);
  if (s.heads * (s.row_tiles + s.key_tiles) == 0) return hipSuccess;
  CrossGradArgs a{};
  a.T = p.T;
  a.Nk = p.Nk;
  a.Hk = p.Hk;
  a.G = p.Hk > 0 ? p.Hq / p.Hk : 1;
  a.M = (int)s.M;
  a.row_tiles = (int)s.row_tiles;
  a.row_units = (int)(s.heads * s.row_tiles);
  a.key_tiles = (int)s.key_tiles;
  a.key_units = (int)(s.heads * s.key_tiles);
  a.parts = (int)s.parts;
  a.part_rows = (int)s.part_rows;
  a.key_parts = (int)s.key_parts;
  a.c2 = p.scale * kLog2e;
  a.scale = p.scale;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p.q[i];
    a.ks[i] = p.k[i];
    a.vs[i] = p.v[i];
    a.os[i] = p.o[i];
    a.gs[i] = p.dO[i];
    a.dqs[i] = p.dq[i];
    a.dks[i] = p.dk[i];
    a.dvs[i] = p.dv[i];
  }
  a.mask_stride_b = p.mask_stride_b;
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.O = O;
  a.dO = dO;
  a.k_len = k_len;
  a.k_mask = k_mask;
  a.lse = lse;
  a.dQ = dQ;
  a.dK = dK;
  a.dV = dV;
  char* at = static_cast<char*>(ws);
  const auto take = [&](size_t bytes) {
    char* const from = at;
    at += bytes;
    return from;
  };
  a.stat_lse = reinterpret_cast<float*>(take(s.stat_bytes));
  a.stat_delta = reinterpret_cast<float*>(take(s.stat_bytes));
  a.top = reinterpret_cast<float*>(take(s.top_bytes));
  const int32_t* const counts = reinterpret_cast<const int32_t*>(take(s.list_bytes));
  if (k_mask && s.list_bytes > 0) {
    a.counts = counts;
    a.list = counts + attended_first(p.n);
  }
  a.part_q = reinterpret_cast<float*>(take(s.part_q_bytes));
  a.part = reinterpret_cast<float*>(at);
  if (p.dtype == PBSA_BF16) return p.d == 64 ? launch_typed<__bf16, 64>(s, a, p.n, stream) : launch_typed<__bf16, 128>(s, a, p.n, stream);
  return p.d == 64 ? launch_typed<_Float16, 64>(s, a, p.n, stream) : launch_typed<_Float16, 128>(s, a, p.n, stream);
}

}  // namespace pbsa
