// Cross attention to an encoder's states, forward, for gfx950: O = softmax(scale Q K^T) V over the attended states.
//
// The query rows of all heads that share a head of K and V are taken together, row m = t (Hq / Hk) + g, so that a state is
// fetched once for all of them.  A wave owns 32 rows and walks the states with one pass of the softmax: S^T = K Q^T leaves a
// lane with scores of one row only, whose exponentials are, as they lie, the operand of O^T += V^T P^T; the reference of a
// row's exponentials (its running maximum, or one that is reset where it has to be) and the running sum are per lane, and O^T is
// rescaled where the reference has risen.  Scores and sums are binary32; the probabilities, relative to the reference, are rounded
// to the tensors' type for the second product (they meet V, which has no more digits).
//   cross_rows_kernel   four waves with 32 rows each share a tile of 64 states in LDS: many rows, bound by the matrix pipe
//   cross_keys_kernel   four waves with the same 32 rows share out the states: few rows, bound by reading K and V
//   cross_few_kernel    up to four rows and no matrix instruction: K and V from memory to registers, where a row's products cost
//                       less than a tile's way through LDS
// The last two share out the states of a head over several workgroups where heads and rows leave the chip empty;
// cross_join_kernel puts their results together.
//
// Measured, heads of 128: 21504 rows x 12 heads to 1500 states, a quarter masked, 149 GFLOP: 164 us, 907 TFLOP/s (a large library
// product: 1224).  4680 x 512 x 12: 22.8 us, of which 12 are steps at 1.2 PFLOP/s; with all workgroups in one round the rows' loads
// and stores have nothing beside them.  16 sequences of one row to 130 .. 512 states of 12 heads, 32 MB: 10.6 us, 3 TB/s.
// Four rows of 16 heads, two of K and V, to 32760 states, 34 MB: 10.3 us and 4.1 for the join.
#include <algorithm>

#include "pbsa_cross_device.h"

namespace pbsa {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct CrossArgs {
  int T, Nk, Hk, G, M;               // M = T G rows of a head of K and V
  int tiles, units, parts;           // row tiles of a head; of all heads and sequences; workgroups that share out the states
  int part_rows;                     // rows that a unit keeps room for in the parts
  float c2;                          // scale in powers of two
  int64_t qs[3], ks[3], vs[3], os[3], mask_stride_b;
  const void* Q;
  const void* K;
  const void* V;
  const int32_t* k_len;
  const uint8_t* k_mask;
  const int32_t* list;               // [n][Nk] attended states and [n] their number, or nullptr: no mask (cross_rows_kernel)
  const int32_t* counts;
  void* O;
  float* lse;
  float* part_o;                     // cross_join_kernel
  float* part_ml;
};

// Workgroups go round robin to the 8 chiplets: each gets a contiguous range, so that what shares K and V shares a cache.
__device__ __forceinline__ int place(int bx, int n) {
  const int per = (n + 7) / 8, at = bx % 8 * per + bx / 8;
  return bx / 8 < per && at < n ? at : -1;
}

template <int D>
struct Softmax {
  f32x16 o[D / 32];
  float m, l, mc;                    // of the lane's row: running maximum, sum, maximum in powers of two
};
template <int D>
__device__ __forceinline__ void clear(Softmax<D>& w) {
#pragma unroll
  for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) w.o[dt][v] = 0.0f;
  w.m = -INFINITY;
  w.l = 0.0f;
  w.mc = 0.0f;
}

// 32 states in LDS, where the lane reads K by rows and V by columns, of which those in `bits` are attended; blank() is done where
// those are not all, before V is read
template <typename E, int D, typename Blank>
__device__ __forceinline__ void attend(Softmax<D>& w, const s16x8 (&q)[D / 16], uint32_t k_at, uint32_t v_at, uint32_t bits, float c2, int half,
                                       Blank blank) {
  using T = Tile<D>;
  f32x16 s;
#pragma unroll
  for (int v = 0; v < 16; ++v) s[v] = 0.0f;
#pragma unroll
  for (int ks = 0; ks < T::KS; ++ks) s = mfma<E>(read_row(k_at ^ (ks << 5)), q[ks], s);
  if (bits != 0xFFFFFFFFu) {
    blank();
    const uint32_t on = bits >> (4 * half);
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] = (on >> row_of(v)) & 1 ? s[v] : -INFINITY;
  }
  float top = s[0];
#pragma unroll
  for (int v = 1; v < 16; ++v) top = fmaxf(top, s[v]);
  top = fmaxf(swap_max(top), w.m);
  if (__any(top > w.m)) {
    const float mc = top == -INFINITY ? 0.0f : top * c2;
    const float alpha = w.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(w.mc - mc);
    w.m = top;
    w.mc = mc;
    w.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
      for (int v = 0; v < 16; ++v) w.o[dt][v] *= alpha;
  }
  float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    s[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c2, -w.mc));
    sum[v % 4] += s[v];
  }
  w.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const s16x8 p = pack8<E>(s, x);
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) w.o[dt] = mfma<E>(read_col<D>((v_at ^ (dt << 6)) + 16 * x * T::ROW), p, w.o[dt]);
  }
}

// Rows and heads of a wave: its lane's row, and where it lies
struct Row {
  int t, h;
  bool on;
};
__device__ __forceinline__ Row row_at_m(const CrossArgs& a, int hk, int m) {
  Row r;
  r.on = m < a.M;
  const int mm = r.on ? m : a.M - 1;
  r.t = a.G == 1 ? mm : mm / a.G;
  r.h = hk * a.G + (mm - r.t * a.G);
  return r;
}
// ---- many rows: a software pipeline over half tiles of 32 states ------------------------------------------------------
// A step forms S^T of the half tile after the current one, the probabilities of the current one and O^T's share of the one
// before it.  The three do not depend on each other: the step is a row of slots, each one matrix instruction (the two products
// in turn), the LDS read for a slot some way on and a slice of the probabilities, and nothing moves between slots.
// No maximum is taken in a step: the reference of a row's exponentials is the maximum of its first half tile, and only where
// a probability passes kTop is the half tile's part done again with a new one (precision in floating point is relative;
// kTop leaves fp16, whose range ends at 2^16, room to both sides).
constexpr float kTop = 4096.0f;
constexpr float kNone = -1e30f;      // the reference where the first half tile's scores are all -infinite: the next finite one resets it

// c += a b in place, as an instruction of its own: the compiler does not copy c (as it did, for the rare rescaling's sake), and
// does not see a matrix instruction (settle).
template <typename E>
__device__ __forceinline__ void mfma_acc(f32x16& c, const s16x8& a, const s16x8& b) {
  if constexpr (__is_same(E, __bf16)) asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_32x32x16_f16 %0, %1, %2, %0" : "+v"(c) : "v"(a), "v"(b));
}
// What has to pass before vector instructions read or rewrite c, and after they have
__device__ __forceinline__ void settle(f32x16& c) { asm volatile("s_nop 15\n\ts_nop 15" : "+v"(c)); }

template <int D>
struct Pipe {
  using T = Tile<D>;
  static constexpr int N = 2 * T::KS;                              // slots of a step: both products have KS
  static constexpr int PER = 16 / N;                               // scores of a slot
  uint32_t k[T::KS], v[T::DT], v2[T::DT];                          // LDS addresses; v2: eight rows on
  static constexpr int AHEAD = 4;          // slots from a read to its use
  static constexpr int TURN = N - 2;      // slot of step A behind whose product the places are passed on
  s16x8 f[AHEAD];                                                  // operands on their way, slot r's in r mod AHEAD
  static_assert(N % AHEAD == 0 && TURN >= N - AHEAD && TURN > N - 1 - AHEAD + 1, "own reads are back at the turn");
  static constexpr uint32_t kFlip = 2 * 64 * T::ROW;               // from one place of a tile to the other
};

// The read of slot R's operand: even slots K by rows, odd ones V by columns, both OFF bytes from their addresses.  FLIP: an
// address moves to the other place after its last read.
template <int D, int R, int OFF, bool FLIP>
__device__ __forceinline__ s16x8 operand(Pipe<D>& z) {
  using T = Tile<D>;
  constexpr int i = R / 2;
  if constexpr (R % 2 == 0) {
    const s16x8 f = read_row(z.k[i] + OFF);
    if constexpr (FLIP) z.k[i] ^= Pipe<D>::kFlip;
    return f;
  } else {
    constexpr int x = i / T::DT, dt = i % T::DT, off = OFF + 16 * x * T::ROW;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)(z.v[dt] + off));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_col_t)(uintptr_t)(z.v2[dt] + off));
    if constexpr (FLIP && x == 1) {
      z.v[dt] ^= Pipe<D>::kFlip;
      z.v2[dt] ^= Pipe<D>::kFlip;
    }
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
}
// the first reads of a step, of slots FROM .. TO - 1
template <int D, int OFF, bool FLIP, int FROM, int TO>
__device__ __forceinline__ void preload(Pipe<D>& z) {
  if constexpr (FROM < TO) {
    z.f[FROM] = operand<D, FROM, OFF, FLIP>(z);
    preload<D, OFF, FLIP, FROM + 1, TO>(z);
  }
}

// What a wave keeps of its 32 rows
struct Probs {
  float e[16], sum[2], top;
  uint32_t p[8];
};
template <int D>
struct Group {
  s16x8 q[D / 16];
  f32x16 o[D / 32];
  f32x16 s[2];               // scores of the even and of the odd half tile
  uint32_t p[2][8];          // their probabilities
  float l, mc;               // of the lane's row: sum and reference, in powers of two
  Probs x;
};
__device__ __forceinline__ s16x8 operand_of(const uint32_t* p) {
  const u32x4 v = {p[0], p[1], p[2], p[3]};
  return __builtin_bit_cast(s16x8, v);
}
template <typename E>
__device__ __forceinline__ void put_pair(Probs& x, int v) {
  x.sum[0] += x.e[v];
  x.sum[1] += x.e[v + 1];
  x.top = fmaxf(fmaxf(x.top, x.e[v]), x.e[v + 1]);
  x.p[v / 2] = pack2<E>(x.e[v], x.e[v + 1]);
  asm volatile("" : "+v"(x.p[v / 2]), "+v"(x.sum[0]), "+v"(x.sum[1]), "+v"(x.top));   // here, not behind the rare branch
}

// Step A (of the even half tile) walks the second half of a tile's K and of the V before it and ends with the turn to the next
// places: some slots before its end its own reads are back, what lies in LDS is passed on, and the reads of step B begin.
// extra(slot) is what a wave does to its own loads then; in step B, which walks first halves, it issues the tile loads.
template <typename E, int D, bool A, int R, typename Extra>
__device__ __forceinline__ void slots(Group<D>& w, Pipe<D>& z, float c2, Extra& extra) {
  using T = Tile<D>;
  constexpr int N = Pipe<D>::N, PER = Pipe<D>::PER, i = R / 2, kAhead = Pipe<D>::AHEAD, kTurn = Pipe<D>::TURN;
  constexpr int cur = A ? 0 : 1, other = 1 - cur;
  if constexpr (R < N) {
    if constexpr (R % 2 == 1) {
      mfma_acc<E>(w.o[i % T::DT], z.f[R % kAhead], operand_of(&w.p[other][4 * (i / T::DT)]));
    } else if constexpr (i == 0) {
      const f32x16 zero = {};
      w.s[other] = mfma<E>(z.f[R % kAhead], w.q[i], zero);
    } else {
      w.s[other] = mfma<E>(z.f[R % kAhead], w.q[i], w.s[other]);
    }
    if constexpr (R + kAhead < N) z.f[R % kAhead] = operand<D, R + kAhead, A ? T::SUB : 0, A>(z);
    else if constexpr (!A) z.f[R % kAhead] = operand<D, R + kAhead - N, T::SUB, true>(z);
    if constexpr (A && R == kTurn) {
      wait_loads();
      extra(R);
      barrier();
      preload<D, 0, false, 0, R % kAhead + 1>(z);                  // into the places of operands that have been used
    }
    if constexpr (A && R > kTurn) preload<D, 0, false, R % kAhead, R % kAhead + 1>(z);
    if constexpr (!A) extra(R);
    Probs& x = w.x;
#pragma unroll
    for (int u = 0; u < PER; ++u) x.e[R * PER + u] = __builtin_amdgcn_exp2f(__builtin_fmaf(w.s[cur][R * PER + u], c2, -w.mc));
    if constexpr (PER == 2) {
      if constexpr (R > 0) put_pair<E>(x, 2 * R - 2);
    } else if constexpr (R % 2 == 0 && R > 0) {
      put_pair<E>(x, R - 2);
    }
    __builtin_amdgcn_sched_barrier(0);
    slots<E, D, A, R + 1>(w, z, c2, extra);
  }
}
template <typename E, int D, bool A, typename Extra>
__device__ __forceinline__ void step(Group<D>& w, Pipe<D>& z, float c2, Extra extra) {
  constexpr int cur = A ? 0 : 1;
  Probs& x = w.x;
  x.sum[0] = x.sum[1] = x.top = 0.0f;
  slots<E, D, A, 0>(w, z, c2, extra);
  put_pair<E>(x, 14);
#pragma unroll
  for (int v = 0; v < 8; ++v) w.p[cur][v] = x.p[v];
  if (__builtin_expect(__any(x.top > kTop), 0)) {
    const f32x16& s = w.s[cur];
    float m = s[0];
#pragma unroll
    for (int v = 1; v < 16; ++v) m = fmaxf(m, s[v]);
    const float mc = fmaxf(swap_max(m) * c2, w.mc), alpha = __builtin_amdgcn_exp2f(w.mc - mc);
    w.mc = mc;
    w.l *= alpha;
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt) {
      settle(w.o[dt]);
#pragma unroll
      for (int v = 0; v < 16; ++v) w.o[dt][v] *= alpha;
      settle(w.o[dt]);
    }
    x.sum[0] = x.sum[1] = 0.0f;
#pragma unroll
    for (int v = 0; v < 16; ++v) x.e[v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[v], c2, -mc));
#pragma unroll
    for (int v = 0; v < 16; v += 2) {
      put_pair<E>(x, v);
      w.p[cur][v / 2] = x.p[v / 2];
    }
  }
  w.l += x.sum[0] + x.sum[1];
}

// A wave's 32 rows between memory, where a load or store takes whole rows, and LDS, 32 ROW bytes at `lds` in the order of a tile.
// Row r of the wave is row m0 + r of the head of K and V.
template <int D>
struct Rows {
  const char* at[Tile<D>::SUB / 1024];     // of this lane: what it moves in each KiB
  __device__ __forceinline__ void set(const CrossArgs& a, const void* base, const int64_t (&st)[3], int64_t b, int hk, int m0, int lane) {
    using T = Tile<D>;
#pragma unroll
    for (int j = 0; j < T::SUB / 1024; ++j) {
      const int r = j * T::RPI + lane / T::CH;
      const Row row = row_at_m(a, hk, m0 + r);
      at[j] = reinterpret_cast<const char*>(base) + 2 * (b * st[0] + row.h * st[1] + row.t * st[2]) + (((lane % T::CH) ^ T::swz(r)) << 4);
    }
  }
};

template <typename E, int D>
__global__ void __launch_bounds__(kThreads, 2) cross_rows_kernel(CrossArgs a) {
  using T = Tile<D>;
  constexpr int kKeys = 64, N = kKeys / kWaves / T::RPI;           // states of a tile, 1 KiB loads of a wave's share of K or V
  constexpr int kTileBytes = kKeys * T::ROW;
  __shared__ __align__(4 * kTileBytes) unsigned char ring[2][2][kTileBytes];   // places of K, then V; kFlip takes one for the other
  __shared__ __align__(16) Picked picked;
  const int unit = place(blockIdx.x, a.units);
  if (unit < 0) return;
  const int bh = unit / a.tiles, hk = bh % a.Hk;
  const int64_t b = bh / a.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&ring[0][0][0];
  const auto at = [](int i) -> uint32_t { return (uint32_t)(i & 1) * 2 * kTileBytes; };   // of tile i in LDS

  // the attended states, in order: all of the first `count`, or those on the list
  const int32_t* const list = a.list ? a.list + b * a.Nk : nullptr;
  const int count = a.list ? __builtin_amdgcn_readfirstlane(a.counts[b]) : length_of(a.k_len, b, a.Nk);
  const int n_tiles = (count + kKeys - 1) / kKeys;
  Gather<D, N> lk, lv;
  const uint32_t picked_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) int32_t*)&picked.at[0][0];
  lk.init(lane, wave * N * T::RPI, reinterpret_cast<const char*>(a.K) + 2 * (b * a.ks[0] + hk * a.ks[1]), 2 * a.ks[2], count, list ? picked_at : 0);
  lv.init(lane, wave * N * T::RPI, reinterpret_cast<const char*>(a.V) + 2 * (b * a.vs[0] + hk * a.vs[1]), 2 * a.vs[2], count, list ? picked_at : 0);
  const int32_t* pick_from = list;
  const auto pick = [&](int i) {                                   // the list's places of tile i, a tile before its loads
    if (list && wave == 0) {
      pick_from = list + min(64 * i + lane, count - 1);
      load_lds4(pick_from, __builtin_amdgcn_readfirstlane(picked_at + 256 * (i & 3)));
    }
  };
  const uint32_t own = lds + wave * N * 1024;
  const uint32_t rows_at = __builtin_amdgcn_readfirstlane(lds + at(1) + wave * T::SUB);   // the wave's rows, in the second place
  const int m0 = (unit - bh * a.tiles) * 128 + wave * 32;

  Group<D> w;
  w.l = w.mc = 0.0f;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int v = 0; v < 16; ++v) w.o[dt][v] = 0.0f;
  if (n_tiles > 0) {
    Rows<D> rows;
    rows.set(a, a.Q, a.qs, b, hk, m0, lane);
    if (!list) {
      lk.issue(0, own + at(0));
      lv.issue(0, own + at(0) + kTileBytes);
    }
    pick(0);
    pick(1);
    pick(2);
#pragma unroll
    for (int j = 0; j < T::SUB / 1024; ++j) load_lds(rows.at[j], rows_at + j * 1024);
    wait_loads();
    barrier();
    if (list) {
      lk.issue(0, own + at(0));
      lv.issue(0, own + at(0) + kTileBytes);
    }
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) w.q[ks] = read_row((rows_at + row_at<D>(lane)) ^ (ks << 5));
#pragma unroll
    for (int j = 0; j < T::SUB / 1024; ++j) asm volatile("" : : "v"(rows.at[j]));
    wait_loads();
    barrier();                       // (all have read their rows: the second place is the next tile's)
    if (n_tiles > 1) lk.issue(1, own + at(1));
    // the first step has a half tile before it like all others, of probabilities and values that are zero
    typedef __attribute__((address_space(3))) u32x4* lds_w_t;
    for (int c = threadIdx.x; c < T::SUB / 16; c += kThreads) *(lds_w_t)(uintptr_t)(lds + at(1) + kTileBytes + T::SUB + 16 * c) = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < 8; ++v) w.p[1][v] = 0;
    Pipe<D> z;
    {
      const uint32_t k = lds + row_at<D>(lane), v = lds + at(1) + kTileBytes + col_at<D>(lane);
#pragma unroll
      for (int ks = 0; ks < T::KS; ++ks) z.k[ks] = k ^ (ks << 5);
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) {
        z.v[dt] = v ^ (dt << 6);
        z.v2[dt] = (v ^ (dt << 6) ^ 32) + 8 * T::ROW;
      }
    }
    const auto mask = [&](f32x16& s, int k0) {                     // scores of states from `count` on
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = k0 + row_of(v) + 4 * half < count ? s[v] : -INFINITY;
    };
#pragma unroll
    for (int v = 0; v < 16; ++v) w.s[0][v] = 0.0f;
#pragma unroll
    for (int ks = 0; ks < T::KS; ++ks) w.s[0] = mfma<E>(read_row(z.k[ks]), w.q[ks], w.s[0]);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");           // (the zeros)
    barrier();
    preload<D, T::SUB, true, 0, Pipe<D>::AHEAD>(z);
    mask(w.s[0], 0);
    float m = w.s[0][0];
#pragma unroll
    for (int v = 1; v < 16; ++v) m = fmaxf(m, w.s[0][v]);
    m = swap_max(m);
    w.mc = m == -INFINITY ? kNone : m * a.c2;
    const auto none = [](int) {};
    int i = 0;
    for (; i + 1 < n_tiles; ++i) {
      // behind step A's turn K of tile i and V of tile i - 1 have been read, K of tile i + 1 and V of tile i are there
      step<E, D, true>(w, z, a.c2, none);
      lk.keep();
      lv.keep();
      asm volatile("" : : "v"(pick_from));
      step<E, D, false>(w, z, a.c2, [&](int r) {
        if (r == 0 && i + 3 < n_tiles) pick(i + 3);
        if (r == 1 && i + 2 < n_tiles) lk.issue(i + 2, own + at(i));
        if (r == 4) lv.issue(i + 1, own + at(i + 1) + kTileBytes);
      });
    }
    mask(w.s[0], i * kKeys);
    // V of what stands in for states past the last one is zero: 0 times an infinity of the last one's would be NaN
    step<E, D, true>(w, z, a.c2, [&](int) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (i * kKeys + (wave * N + j) * T::RPI + lane / T::CH >= count) *(lds_w_t)(uintptr_t)(own + at(i) + kTileBytes + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    });
    mask(w.s[1], i * kKeys + 32);
    step<E, D, false>(w, z, a.c2, none);                           // (its S^T is of no tile)
    const uint32_t last = lds + at(i) + kTileBytes + T::SUB + col_at<D>(lane);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt) mfma_acc<E>(w.o[dt], read_col<D>((last ^ (dt << 6)) + 16 * x * T::ROW), operand_of(&w.p[1][4 * x]));
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt) settle(w.o[dt]);
    barrier();                       // all have read the last tile
  }
  // ---- O through LDS: whole rows to memory ---------------------------------------------------------------------------------
  const float l = swap_sum(w.l), inv = l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;   // (a NaN stays one)
  typedef __attribute__((address_space(3))) u32x2* lds_8_t;
  const int r = lane & 31;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f32x16& x = w.o[dt];
      const u32x2 v = {pack2<E>(x[4 * e] * inv, x[4 * e + 1] * inv), pack2<E>(x[4 * e + 2] * inv, x[4 * e + 3] * inv)};
      *(lds_8_t)(uintptr_t)(rows_at + r * T::ROW + (((4 * dt + e) ^ T::swz(r)) << 4) + 8 * half) = v;
    }
  Rows<D> rows;
  rows.set(a, a.O, a.os, b, hk, m0, lane);
#pragma unroll
  for (int j = 0; j < T::SUB / 1024; ++j) {
    typedef __attribute__((address_space(3))) const u32x4* lds_16_t;
    const u32x4 v = *(lds_16_t)(uintptr_t)(rows_at + j * 1024 + lane * 16);
    if (m0 + j * T::RPI + lane / T::CH < a.M) *reinterpret_cast<u32x4*>(const_cast<char*>(rows.at[j])) = v;
  }
  const Row row = row_at_m(a, hk, m0 + r);
  if (a.lse && half == 0 && row.on) a.lse[(b * a.Hk * a.G + row.h) * a.T + row.t] = l == 0.0f ? -INFINITY : (w.mc + __builtin_log2f(l)) * kLn2;
}

// ---- few rows ------------------------------------------------------------------------------------------------------------
// Results of a part of the states: [unit][part][R rows][D], not yet divided, and [unit][part][R][2]: reference and sum.

// Which states of a wave's tiles of 32, `step` tiles apart, are attended: of 64 tiles at a time, lane t the bits of the t-th.
struct TileBits {
  uint32_t mine;
  __device__ __forceinline__ void read(const Attended& keys, int first, int step, int n, int lane) {
    const int64_t left = (int64_t)keys.len - (int64_t)(first + lane * step) * 32;
    mine = lane >= n || left <= 0 ? 0u : left >= 32 ? ~0u : (1u << left) - 1;
    if (!keys.mask || n <= 0) return;
    constexpr int kBatch = 8;        // loads of two tiles' bytes
    for (int t = 0; t < n; t += 2 * kBatch) {
      uint8_t byte[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int64_t k = (int64_t)(first + (t + 2 * j + (lane >> 5)) * step) * 32 + (lane & 31);
        byte[j] = keys.mask[k < keys.len ? k : keys.len - 1];
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const uint64_t on = __ballot(byte[j] != 0);
        if (lane == t + 2 * j) mine &= (uint32_t)on;
        if (lane == t + 2 * j + 1) mine &= (uint32_t)(on >> 32);
      }
    }
  }
  __device__ __forceinline__ uint32_t of(int t) const { return (uint32_t)__builtin_amdgcn_readlane((int)mine, t); }
};

template <typename E, int D>
__global__ void __launch_bounds__(kThreads, 1) cross_keys_kernel(CrossArgs a) {
  using T = Tile<D>;
  constexpr int kKeys = 32, N = kKeys / T::RPI, kSlots = D / 8;    // slots: quarters of the accumulators' registers
  constexpr int kTileBytes = kKeys * T::ROW;
  __shared__ __align__(1024) unsigned char ring[kWaves][2][2][kTileBytes];
  __shared__ __align__(1024) unsigned char q_rows[kTileBytes];
  __shared__ float2 ml[kWaves][32];
  static_assert(kSlots * 64 * 16 <= 4 * kTileBytes, "a wave's O^T fits where its tiles were");
  const int unit_part = place(blockIdx.x, a.units * a.parts);
  if (unit_part < 0) return;
  const int unit = unit_part / a.parts, part = unit_part - unit * a.parts;
  const int bh = unit / a.tiles, hk = bh % a.Hk;
  const int64_t b = bh / a.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = (unit - bh * a.tiles) * 32;
  const Row row = row_at_m(a, hk, m0 + (lane & 31));

  const Attended keys = attended_of(a.k_len, a.k_mask, a.mask_stride_b, b, a.Nk);
  const int n_tiles = (keys.len + kKeys - 1) / kKeys, step = a.parts * kWaves;
  const int first = part * kWaves + wave, mine = first < n_tiles ? (n_tiles - first + step - 1) / step : 0;
  const char* const kb = reinterpret_cast<const char*>(a.K) + 2 * (b * a.ks[0] + hk * a.ks[1]);
  const char* const vb = reinterpret_cast<const char*>(a.V) + 2 * (b * a.vs[0] + hk * a.vs[1]);
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&ring[wave][0][0][0];
  const uint32_t row0 = row_at<D>(lane), col0 = col_at<D>(lane), q_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)&q_rows[0];
  Softmax<D> w;
  clear(w);
  TileBits bits;
  bits.read(keys, first, step, min(mine, 64), lane);
  // Q by all four waves, in front of the tiles
  static_assert(N % kWaves == 0, "");
  const char* q_from[N / kWaves];
#pragma unroll
  for (int j = 0; j < N / kWaves; ++j) {
    const int r = (wave * (N / kWaves) + j) * T::RPI + lane / T::CH;
    const Row at = row_at_m(a, hk, m0 + r);
    q_from[j] = reinterpret_cast<const char*>(a.Q) + 2 * (b * a.qs[0] + at.h * a.qs[1] + at.t * a.qs[2]) + (((lane % T::CH) ^ T::swz(r)) << 4);
    load_lds(q_from[j], __builtin_amdgcn_readfirstlane(q_at + (wave * (N / kWaves) + j) * 1024));
  }
  s16x8 q[T::KS];
  // Tiles are the wave's own: no barrier, and the next one is on its way before the current one is waited for.  Offsets within
  // whole tiles are alike; where they change, what is on its way is waited for first.
  Loads<D, N> lk, lv;
  uint32_t set_for = 0, on = 0;
#pragma unroll 1
  for (int t = -1; t < mine; ++t) {
    const int next = t + 1;
    uint32_t on_next = 0;
    if (next < mine) {
      if (next > 0 && (next & 63) == 0) bits.read(keys, first + next * step, step, min(mine - next, 64), lane);
      on_next = bits.of(next & 63);
      const uint32_t set = on_next != 0 ? on_next : 1u;            // (a tile without a state is passed over, but not its loads)
      if (set != set_for) {
        wait_loads();
        lk.set(lane, 0, (uint32_t)(2 * a.ks[2]), set);
        lv.set(lane, 0, (uint32_t)(2 * a.vs[2]), set);
        set_for = set;
      }
      const int64_t k0 = (int64_t)(first + next * step) * kKeys;
      const uint32_t to = lds + (next & 1) * 2 * kTileBytes;
      lk.issue(kb + 2 * k0 * a.ks[2], to);
      lv.issue(vb + 2 * k0 * a.vs[2], to + kTileBytes);
      asm volatile("s_waitcnt vmcnt(%0)" : : "n"(2 * N) : "memory");
    } else {
      wait_loads();
    }
    if (t < 0) {
      barrier();
#pragma unroll
      for (int j = 0; j < N / kWaves; ++j) asm volatile("" : : "v"(q_from[j]));
#pragma unroll
      for (int ks = 0; ks < T::KS; ++ks) q[ks] = read_row((q_at + row0) ^ (ks << 5));
    } else {
      const uint32_t here = lds + (t & 1) * 2 * kTileBytes;
      if (on != 0) {
        attend<E, D>(w, q, here + row0, here + kTileBytes + col0, on, a.c2, half, [&] {
          // V of what stands in is zero: 0 times an infinity of another state's would be NaN (LDS takes a wave's accesses in order)
          typedef __attribute__((address_space(3))) u32x4* lds_w_t;
#pragma unroll
          for (int j = 0; j < N; ++j)
            if (!(on >> (j * T::RPI + lane / T::CH) & 1)) *(lds_w_t)(uintptr_t)(here + kTileBytes + j * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
        });
      }
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");         // the tile has been read
    }
    on = on_next;
  }
  lk.keep();
  lv.keep();
  // ---- the four waves' results together, through LDS ---------------------------------------------------------------------
  const float l_mine = swap_sum(w.l);
  f32x4* const here = reinterpret_cast<f32x4*>(&ring[wave][0][0][0]);
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      here[(4 * dt + g) * 64 + lane] = f32x4{w.o[dt][4 * g], w.o[dt][4 * g + 1], w.o[dt][4 * g + 2], w.o[dt][4 * g + 3]};
  if (half == 0) ml[wave][lane] = make_float2(l_mine == 0.0f ? -INFINITY : w.mc, l_mine);
  __syncthreads();
  float mc = -INFINITY, weight[kWaves], l = 0.0f;
#pragma unroll
  for (int k = 0; k < kWaves; ++k) mc = fmaxf(mc, ml[k][lane & 31].x);
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    const float2 v = ml[k][lane & 31];
    weight[k] = v.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(v.x - mc);
    l += weight[k] * v.y;
  }
  if (!row.on) return;
  const bool whole = a.parts == 1;
  const float inv = !whole ? 1.0f : l > 0.0f ? 1.0f / l : l == 0.0f ? 0.0f : l;
  const int64_t part_row = (int64_t)unit_part * a.part_rows + (lane & 31);
#pragma unroll
  for (int s = wave; s < kSlots; s += kWaves) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const f32x4 u = reinterpret_cast<const f32x4*>(&ring[k][0][0][0])[s * 64 + lane];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += weight[k] * u[e];
    }
    if (!whole) {
      *reinterpret_cast<f32x4*>(a.part_o + part_row * D + 8 * s + 4 * half) = v;
    } else {
      E* const o = reinterpret_cast<E*>(a.O) + b * a.os[0] + row.h * a.os[1] + row.t * a.os[2] + 8 * s + 4 * half;
      const u32x2 p = {pack2<E>(v[0] * inv, v[1] * inv), pack2<E>(v[2] * inv, v[3] * inv)};
      *reinterpret_cast<u32x2*>(o) = p;
    }
  }
  if (wave == 0 && half == 0) {
    if (!whole) reinterpret_cast<float2*>(a.part_ml)[part_row] = make_float2(mc, l);
    else if (a.lse) a.lse[(b * a.Hk * a.G + row.h) * a.T + row.t] = l == 0.0f ? -INFINITY : (mc + __builtin_log2f(l)) * kLn2;
  }
}

// One to four rows: D / 8 lanes hold a state's row of K and of V, 8 elements each, KPI states to a wave's load, kBatch loads on
// their way.  Each group of lanes has a softmax of its own over its states; they are joined at the end.
constexpr int kFewWaves = 16;
template <typename E, int D, int MR>
__global__ void __launch_bounds__(64 * kFewWaves) cross_few_kernel(CrossArgs a) {
  constexpr int LPK = D / 8, KPI = 64 / LPK, kBatch = MR == 4 ? 4 : 8;
  __shared__ float sums[kFewWaves][MR][D];
  __shared__ float2 ml[kFewWaves][MR];
  typedef typename Vec<E>::x8 x8;
  const int unit_part = place(blockIdx.x, a.units * a.parts);
  if (unit_part < 0) return;
  const int unit = unit_part / a.parts, part = unit_part - unit * a.parts, hk = unit % a.Hk;
  const int64_t b = unit / a.Hk;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, grp = lane / LPK, d0 = lane % LPK * 8;
  float q[MR][8];
#pragma unroll
  for (int r = 0; r < MR; ++r) {
    const Row row = row_at_m(a, hk, r);
    const x8 v = *reinterpret_cast<const x8*>(reinterpret_cast<const E*>(a.Q) + b * a.qs[0] + row.h * a.qs[1] + row.t * a.qs[2] + d0);
#pragma unroll
    for (int e = 0; e < 8; ++e) q[r][e] = (float)v[e] * a.c2;
  }
  const int len = length_of(a.k_len, b, a.Nk);
  const uint8_t* const mask = a.k_mask ? a.k_mask + b * a.mask_stride_b : nullptr;
  const E* const kb = reinterpret_cast<const E*>(a.K) + b * a.ks[0] + hk * a.ks[1] + d0;
  const E* const vb = reinterpret_cast<const E*>(a.V) + b * a.vs[0] + hk * a.vs[1] + d0;
  float m[MR], l[MR], acc[MR][8];
#pragma unroll
  for (int r = 0; r < MR; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[r][e] = 0.0f;
  }
  for (int64_t k0 = (int64_t)(part * waves + wave) * KPI * kBatch; k0 < len; k0 += (int64_t)a.parts * waves * KPI * kBatch) {
    u32x4 kr[kBatch], vr[kBatch];
    bool on[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int64_t k = k0 + u * KPI + grp, at = k < len ? k : len - 1;
      on[u] = k < len && (!mask || mask[at] != 0);
      kr[u] = *reinterpret_cast<const u32x4*>(kb + at * a.ks[2]);
      vr[u] = *reinterpret_cast<const u32x4*>(vb + at * a.vs[2]);
    }
    float s[MR][kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const x8 k = __builtin_bit_cast(x8, kr[u]);
#pragma unroll
      for (int r = 0; r < MR; ++r) {
        float v = (float)k[0] * q[r][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) v = __builtin_fmaf((float)k[e], q[r][e], v);
        v = add_dpp<0xB1>(v);        // over the lanes of the row: within quads, then by mirroring eights and sixteens
        v = add_dpp<0x4E>(v);
        v = add_dpp<0x141>(v);
        if constexpr (LPK == 16) v = add_dpp<0x140>(v);
        s[r][u] = on[u] ? v : -INFINITY;
      }
    }
    float alpha[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
      float top = m[r];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) top = fmaxf(top, s[r][u]);
      const float mc = top == -INFINITY ? 0.0f : top;
      alpha[r] = __builtin_amdgcn_exp2f(m[r] - mc);
      m[r] = top;
      float sum = 0.0f;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        s[r][u] = __builtin_amdgcn_exp2f(s[r][u] - mc);
        sum += s[r][u];
      }
      l[r] = l[r] * alpha[r] + sum;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[r][e] *= alpha[r];
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const u32x4 zero = {0, 0, 0, 0};
      const x8 v = __builtin_bit_cast(x8, on[u] ? vr[u] : zero);   // a state that is not attended may hold NaN
#pragma unroll
      for (int r = 0; r < MR; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = __builtin_fmaf(s[r][u], (float)v[e], acc[r][e]);
    }
  }
  // ---- the groups of a wave, then the waves --------------------------------------------------------------------------------
#pragma unroll
  for (int r = 0; r < MR; ++r) {
    float top = m[r];
    if constexpr (LPK == 8) top = fmaxf(top, mov_dpp<0x128>(top));
    top = swap_max16(top);
    top = swap_max(top);
    const float weight = m[r] == -INFINITY && l[r] == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(m[r] - (top == -INFINITY ? 0.0f : top));
    l[r] = over_groups<LPK>(l[r] * weight);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[r][e] = over_groups<LPK>(acc[r][e] * weight);
    if (grp == 0) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) *reinterpret_cast<f32x4*>(&sums[wave][r][d0 + e]) = f32x4{acc[r][e], acc[r][e + 1], acc[r][e + 2], acc[r][e + 3]};
      if (lane == 0) ml[wave][r] = make_float2(top, l[r]);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < MR * D; i += blockDim.x) {
    const int r = i / D, d = i % D;
    if (r >= a.M) break;
    float top = -INFINITY, total = 0.0f, v = 0.0f;
    for (int k = 0; k < waves; ++k) top = fmaxf(top, ml[k][r].x);
    for (int k = 0; k < waves; ++k) {
      const float2 x = ml[k][r];
      const float weight = x.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(x.x - (top == -INFINITY ? 0.0f : top));
      total += weight * x.y;
      v += weight * sums[k][r][d];
    }
    const int64_t part_row = (int64_t)unit_part * a.part_rows + r;
    if (a.parts > 1) {
      a.part_o[part_row * D + d] = v;
      if (d == 0) reinterpret_cast<float2*>(a.part_ml)[part_row] = make_float2(total == 0.0f ? -INFINITY : top, total);
    } else {
      const Row row = row_at_m(a, hk, r);
      reinterpret_cast<E*>(a.O)[b * a.os[0] + row.h * a.os[1] + row.t * a.os[2] + d] = (E)(total > 0.0f ? v / total : total == 0.0f ? 0.0f : total);
      if (d == 0 && a.lse) a.lse[(b * a.Hk * a.G + row.h) * a.T + row.t] = total == 0.0f ? -INFINITY : (top + __builtin_log2f(total)) * kLn2;
    }
  }
}

// The parts of a row together: a workgroup to a row, D / 4 lanes to its values, the others share out the parts.
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) cross_join_kernel(CrossArgs a) {
  constexpr int kLanes = D / 4, kGroups = kThreads / kLanes, kBatch = 8;
  __shared__ f32x4 sums[kGroups][kLanes];
  __shared__ float2 ml[kGroups];
  const int unit = blockIdx.x / a.part_rows, r = blockIdx.x - unit * a.part_rows;
  const int bh = unit / a.tiles, hk = bh % a.Hk;
  const int64_t b = bh / a.Hk;
  const Row row = row_at_m(a, hk, (unit - bh * a.tiles) * a.part_rows + r);
  if (!row.on) return;
  const int c = threadIdx.x % kLanes, g = threadIdx.x / kLanes;
  const int64_t first = (int64_t)unit * a.parts * a.part_rows + r;
  float mc = -INFINITY, l = 0.0f;
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p0 = g; p0 < a.parts; p0 += kGroups * kBatch) {
    float2 x[kBatch];
    f32x4 u[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int p = p0 + k * kGroups;
      x[k] = make_float2(-INFINITY, 0.0f);
      u[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (p < a.parts) {
        x[k] = reinterpret_cast<const float2*>(a.part_ml)[first + (int64_t)p * a.part_rows];
        u[k] = *reinterpret_cast<const f32x4*>(a.part_o + (first + (int64_t)p * a.part_rows) * D + 4 * c);
      }
    }
    float top = mc;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, x[k].x);
    const float ref = top == -INFINITY ? 0.0f : top, alpha = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(mc - ref);
    mc = top;
    l *= alpha;
    v *= alpha;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float weight = x[k].y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(x[k].x - ref);
      l += weight * x[k].y;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += weight * u[k][e];
    }
  }
  sums[g][c] = v;
  if (c == 0) ml[g] = make_float2(mc, l);
  __syncthreads();
  if (g != 0) return;
  float top = -INFINITY, total = 0.0f;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < kGroups; ++k) top = fmaxf(top, ml[k].x);
#pragma unroll
  for (int k = 0; k < kGroups; ++k) {
    const float2 p = ml[k];
    const float weight = p.y == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(p.x - top);
    total += weight * p.y;
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += weight * sums[k][c][e];
  }
  const float inv = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
  const u32x2 p = {pack2<E>(o[0] * inv, o[1] * inv), pack2<E>(o[2] * inv, o[3] * inv)};
  *reinterpret_cast<u32x2*>(reinterpret_cast<E*>(a.O) + b * a.os[0] + row.h * a.os[1] + row.t * a.os[2] + 4 * c) = p;
  if (c == 0 && a.lse) a.lse[(b * a.Hk * a.G + row.h) * a.T + row.t] = total == 0.0f ? -INFINITY : (top + __builtin_log2f(total)) * kLn2;
}

// How a call is shared out.
enum class By { rows, keys, few };   // few: 16 rows of one to 512 states of 12 heads of 128 10.6 us, by states 20.5
struct CrossShape {
  By by;
  int64_t tiles, units;
  int parts, part_rows;
  int waves;                         // few: of a workgroup
};
constexpr int kFill = 256;           // workgroups that fill the chip
CrossShape cross_shape(const pbsa_cross& p, bool masked) {
  CrossShape s;
  const int64_t M = p.Hk > 0 ? (int64_t)p.T * (p.Hq / p.Hk) : 0, heads = (int64_t)p.n * p.Hk;
  s.parts = 1;
  s.waves = kWaves;
  s.tiles = (M + 127) / 128;
  s.units = s.tiles * heads;
  s.part_rows = 32;
  s.by = By::rows;
  if (M <= 4) {
    s.by = By::few;
    s.tiles = M > 0;
    s.units = s.tiles * heads;
    s.part_rows = (int)M;
    const int64_t batch = 64 / (p.d / 8) * (M > 2 ? 4 : 8), turns = ((int64_t)p.Nk + batch - 1) / batch;   // states of a wave at a time
    while (s.waves < kFewWaves && s.waves < turns) s.waves *= 2;
    while ((int64_t)s.parts * s.waves < turns && s.units * s.parts * 2 <= kFill) s.parts *= 2;
  } else {
    CrossShape k = s;
    k.by = By::keys;
    k.tiles = (M + 31) / 32;
    k.units = k.tiles * heads;
    const int64_t turns = ((int64_t)p.Nk + 32 * kWaves - 1) / (32 * kWaves);   // of four waves over the states
    while (k.parts * 2 <= turns && k.units * k.parts * 2 <= kFill) k.parts *= 2;
    // Microseconds of either, below a round of workgroups by rows: one of them takes 1 to a tile of 64 states, one by states 1.6
    // to a turn, and the join goes with its parts.  12 heads of 128, by rows and by states: 32 rows to 512 states 12.7 and 10.1
    // (by the model 14, 11), 128 12.6 and 12.5, 300 12.9 and 17.5, 1000 13.5 and 23.4, 2600 15.7 and 44.9; 2600 to 77 9.1 and
    // 21.7, to 2000 41 and 123.  Two heads of 32 rows to 32760 states: 15.9 by states (16; by rows, on two compute units, 518).
    const double by_rows = 6.0 + (double)(((int64_t)p.Nk + 63) / 64) + (masked ? 4.0 : 0.0), groups = (double)(k.units * k.parts);
    const double by_keys = std::max(1.0, groups / kFill) * (5.0 + 1.6 * (double)turns / k.parts) + (k.parts > 1 ? 4.0 + groups / 60.0 : 0.0);
    // Gather counts the bytes from the first state to a load of a listed one in 32 bits
    const bool far = masked && ((int64_t)p.Nk - 1) * 2 * std::max(p.k[2], p.v[2]) + kGatherSpan > ((int64_t)1 << 32);
    if (far || (s.units < kFill && by_keys < by_rows)) s = k;
  }
  return s;
}

template <typename E, int D>
hipError_t launch_typed(const CrossShape& s, const CrossArgs& a, int n, hipStream_t stream) {
  const dim3 grid((unsigned)((s.units * s.parts + 7) / 8 * 8));
  if (s.by == By::rows) {
    if (a.list) {
      // without its list the next launch has nothing to go by
      const hipError_t e = launch_attended(a.k_len, a.k_mask, a.mask_stride_b, n, a.Nk, const_cast<int32_t*>(a.list), const_cast<int32_t*>(a.counts), stream);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((cross_rows_kernel<E, D>), grid, dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const dim3 block(64 * s.waves);
  if (s.by == By::keys) hipLaunchKernelGGL((cross_keys_kernel<E, D>), grid, block, 0, stream, a);
  else if (a.M == 1) hipLaunchKernelGGL((cross_few_kernel<E, D, 1>), grid, block, 0, stream, a);
  else if (a.M == 2) hipLaunchKernelGGL((cross_few_kernel<E, D, 2>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((cross_few_kernel<E, D, 4>), grid, block, 0, stream, a);
  if (s.parts > 1) hipLaunchKernelGGL((cross_join_kernel<E, D>), dim3((unsigned)(s.units * s.part_rows)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// A launch holds fewer than 2^32 threads.  Rows in units of 128 always fit (the checks count 2^30 of them), and so do up to four rows to
// a head; units of 32, which few rows take and masked states far apart, may not.
bool cross_fits(const pbsa_cross& p, bool masked) {
  const CrossShape s = cross_shape(p, masked);
  return (s.units * s.parts + 7) / 8 * 8 * 64 * s.waves < (int64_t)1 << 32;
}

size_t cross_workspace_bytes(const pbsa_cross& p, bool masked) {
  const CrossShape s = cross_shape(p, masked);
  if (s.by == By::rows) return masked ? attended_bytes(p.n, p.Nk) : 0;
  return s.parts == 1 ? 0 : (size_t)(s.units * s.parts) * s.part_rows * (p.d + 2) * sizeof(float);
}

hipError_t launch_cross(const pbsa_cross& p, const void* Q, const void* K, const void* V, const int32_t* k_len, const uint8_t* k_mask,
                        void* O, float* lse, void* ws, hipStream_t stream) {
  const CrossShape s = cross_shape(p, k_mask != nullptr);
  if (s.units == 0) return hipSuccess;
  CrossArgs a{};
  a.T = p.T;
  a.Nk = p.Nk;
  a.Hk = p.Hk;
  a.G = p.Hq / p.Hk;
  a.M = p.T * a.G;
  a.tiles = (int)s.tiles;
  a.units = (int)s.units;
  a.parts = s.parts;
  a.c2 = p.scale * kLog2e;
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p.q[i];
    a.ks[i] = p.k[i];
    a.vs[i] = p.v[i];
    a.os[i] = p.o[i];
  }
  a.mask_stride_b = p.mask_stride_b;
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.k_len = k_len;
  a.k_mask = k_mask;
  a.O = O;
  a.lse = lse;
  if (s.by == By::rows && k_mask) {
    a.counts = static_cast<int32_t*>(ws);
    a.list = a.counts + attended_first(p.n);
  }
  a.part_o = static_cast<float*>(ws);
  a.part_rows = s.part_rows;
  a.part_ml = a.part_o + (size_t)(s.units * s.parts) * s.part_rows * p.d;
  if (p.dtype == PBSA_BF16) return p.d == 64 ? launch_typed<__bf16, 64>(s, a, p.n, stream) : launch_typed<__bf16, 128>(s, a, p.n, stream);
  return p.d == 64 ? launch_typed<_Float16, 64>(s, a, p.n, stream) : launch_typed<_Float16, 128>(s, a, p.n, stream);
}

}  // namespace pbsa
