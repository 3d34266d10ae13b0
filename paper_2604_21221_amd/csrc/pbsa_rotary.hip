// Rotary positions, and the norm of each head's row with the rotation in the same pass, forward and backward, for gfx950.
//
// y = R x,  y = R n with n = x r w, r = (mean(x^2) + eps)^-1/2;  backward, with g = R^T dy:
//   dx = r (g w - x r^2 mean(g w x)),   dw = sum over rows of g x r.
// Bound by memory: every element is read once and written once and takes about ten operations (backward: two reads, twenty).
//
// A lane owns the same 16 elements, 8 and 8, of every row it handles, chosen so that both elements of each of its pairs are
// its own whichever way pairs are formed: nothing is exchanged but the row's sum of squares.  d / 16 lanes (rounded up to a
// power of two) make a row; the rows of a workgroup are `tok` tokens of one tensor by some of its heads, and a lane keeps its
// token while it goes through the heads: the 8 pairs of cosines and sines that it needs stay in registers.  They are formed
// once per workgroup, in binary64 up to the reduced angle, while the first rows are on their way (reading them from a table
// would move more bytes than the positions, and the table would have to reach to the farthest of them).
//
// Measured, at 21504 x 12 x 128 of two tensors, 265 MB: 53 us, 5.0 TB/s (a copy of 1 GiB: 5.15).  At 4680 x 12 x 128 with the norm,
// 58 MB: 12.6 us; its backward, 86 MB: 19 us and 3.2 for the sum of the workgroups' shares of the weights' gradients: there
// a third of the time is launch and first loads, and the backward's 360 instructions for a row of a lane are another.
#include <algorithm>

#include "pbsa_layer_internal.h"

namespace pbsa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTok = 16;          // tokens of a workgroup
constexpr int kMaxGroups = 1024;     // workgroups of a backward launch for a tensor, each of which leaves one partial sum per weight
constexpr int kMostGroups = 1 << 23; // of a forward launch, which holds fewer than 2^32 threads in a dimension

struct RotaryArgs {
  int T, H[2], d, rot, n_axes, pairs0, pairs01;
  int lanes_log, tok_log;            // lanes of a row, tokens of a workgroup, as powers of two
  int groups_t;                      // groups of so many tokens per sequence
  uint32_t by_pairs;                 // 2^32 / (rot / 2), rounded up
  int64_t groups;                    // over all sequences
  float mscale, eps, sign;
  int64_t pos_stride_b;
  int64_t xs[2][3], dys[2][3], ys[2][3];
  const void* x[2];
  const void* dy[2];
  void* y[2];
  const float* w[2];
  const int64_t* pos;
  const double* freq;
  float* part;                       // backward: [tensor][workgroup][d]
};

typedef float f8[8];

// 8 consecutive elements as they lie in memory, 16 bytes at a time
template <typename E>
struct Raw {
  uint4 v[sizeof(E) / 2];
};
template <typename E>
__device__ __forceinline__ void get(Raw<E>& r, const E* p) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(E) / 2; ++i) r.v[i] = reinterpret_cast<const uint4*>(p)[i];
}
template <typename E>
__device__ __forceinline__ void unpack(const Raw<E>& r, f8& v) {
  typedef __attribute__((ext_vector_type(8))) E e8;
  const e8 a = __builtin_bit_cast(e8, r);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
}
template <typename E>
__device__ __forceinline__ void put(E* p, const f8& v) {
  typedef __attribute__((ext_vector_type(8))) E e8;
  e8 a;
#pragma unroll
  for (int i = 0; i < 8; ++i) a[i] = (E)v[i];      // nearest, ties to even
  const Raw<E> r = __builtin_bit_cast(Raw<E>, a);
#pragma unroll
  for (int i = 0; i < (int)sizeof(E) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = r.v[i];
}

// The pairs of a lane turned in place.  HALF: pair j is (a[j], b[j]); else the neighbours within a and within b.
template <bool HALF>
__device__ __forceinline__ void turn(f8& a, f8& b, const f8& c, const f8& s, bool on_a, bool on_b) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& u = HALF ? a[j] : j < 4 ? a[2 * j] : b[2 * j - 8];
    float& v = HALF ? b[j] : j < 4 ? a[2 * j + 1] : b[2 * j - 7];
    const bool on = HALF || j < 4 ? on_a : on_b;
    const float u0 = u, v0 = v;
    u = on ? u0 * c[j] - v0 * s[j] : u0;           // elements that are not rotated pass as they are, infinities too
    v = on ? u0 * s[j] + v0 * c[j] : v0;
  }
}

// The sum over the lanes of a row (up to 16, a power of two, rows aligned to it), in lane order within quads, then quads of
// eight and eights of sixteen by mirroring: the lanes of a group hold the same sum by then.
__device__ __forceinline__ float row_sum(float v, int lanes_log) {
#define PBSA_ADD_DPP(CTRL) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true))
  if (lanes_log > 0) PBSA_ADD_DPP(0xB1);           // quad_perm 1 0 3 2
  if (lanes_log > 1) PBSA_ADD_DPP(0x4E);           // quad_perm 2 3 0 1
  if (lanes_log > 2) PBSA_ADD_DPP(0x141);          // row_half_mirror
  if (lanes_log > 3) PBSA_ADD_DPP(0x140);          // row_mirror
#undef PBSA_ADD_DPP
  return v;
}
// The sum over the lanes of a wave that have the same place in their rows: by turning the 16 lanes of a DPP row, then by
// exchanging rows
__device__ __forceinline__ float column_sum(float v, int lanes_log) {
#define PBSA_ADD_DPP(CTRL) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true))
  if (lanes_log < 1) PBSA_ADD_DPP(0x121);          // row_ror 1
  if (lanes_log < 2) PBSA_ADD_DPP(0x122);
  if (lanes_log < 3) PBSA_ADD_DPP(0x124);
  if (lanes_log < 4) PBSA_ADD_DPP(0x128);
#undef PBSA_ADD_DPP
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}
__device__ __forceinline__ float inv_sqrt(float v) {    // the instruction takes no subnormal numbers
  return v < 0x1p-100f ? __builtin_amdgcn_rsqf(v * 0x1p64f) * 0x1p32f : __builtin_amdgcn_rsqf(v);
}

template <typename E, bool HALF, RotaryOp OP>
__global__ void __launch_bounds__(kThreads) rotary_kernel(RotaryArgs a) {
  constexpr bool kGrad = OP == RotaryOp::norm_grad, kNorm = OP != RotaryOp::rotate;
  constexpr int kRows = kGrad ? 1 : 2;           // rows on their way while as many are worked on (what registers leave room for)
  __shared__ __align__(16) float2 turns[kMaxTok * PBSA_ROTARY_MAX_D / 2];      // [token][pair] cosine and sine
  __shared__ __align__(16) float weights[kGrad ? PBSA_ROTARY_MAX_D : 4];
  __shared__ float sums[kGrad ? kThreads / 64 : 1][kGrad ? 16 * 16 : 1];
  const int i = blockIdx.y;                                        // the tensor
  const int tid = threadIdx.x, lanes = 1 << a.lanes_log, tok = 1 << a.tok_log;
  const int c = tid & (lanes - 1), slot = tid >> a.lanes_log;      // lanes <= 16: slots >= 16 >= tok
  const int tk = slot & (tok - 1), h0 = slot >> a.tok_log, h_step = (kThreads >> a.lanes_log) >> a.tok_log;
  // this lane's elements, oa .. oa + 7 and ob .. ob + 7, and the pairs among them that turn
  const bool own_c = c < a.d / 16;
  const int cc = own_c ? c : 0;
  int oa, ob, pa, pb;
  bool on_a, on_b;
  if constexpr (HALF) {
    const int nr = a.rot / 16;
    on_a = on_b = cc < nr;
    oa = on_a ? 8 * cc : a.rot + 8 * (cc - nr);
    ob = on_a ? oa + a.rot / 2 : oa + (a.d - a.rot) / 2;
    pa = 8 * cc;
    pb = pa + 4;
  } else {
    oa = 8 * cc;
    ob = oa + a.d / 2;
    on_a = oa < a.rot;
    on_b = ob < a.rot;
    pa = oa / 2;
    pb = ob / 2;
  }
  const int n_pairs = a.rot / 2, H = a.H[i];
  const float inv_d = 1.0f / (float)a.d;
  const E* const x0 = reinterpret_cast<const E*>(a.x[i]);
  const E* const dy0 = reinterpret_cast<const E*>(a.dy[i]);
  E* const y0 = reinterpret_cast<E*>(a.y[i]);
  const int64_t x_step = h_step * a.xs[i][1], dy_step = h_step * a.dys[i][1], y_step = h_step * a.ys[i][1];
  const float* const w = kNorm ? a.w[i] : nullptr;

  f8 wa, wb, dwa, dwb;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    dwa[j] = dwb[j] = 0.0f;
    wa[j] = wb[j] = 1.0f;
  }
  if constexpr (kGrad) {
    if (tid < a.d) weights[tid] = w ? w[tid] : 1.0f;
  } else if (w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      wa[j] = w[oa + j];
      wb[j] = w[ob + j];
    }
  }

  // The pair whose cosines and sines this thread forms, for tokens my_tok, my_tok + tok_step, ..  Revolutions: what is left of
  // whole turns is known to binary32 and better for every position that binary64 holds (the step in two pieces, 1 / 2 pi too,
  // and the product less the whole turns with one rounding).
  const int tok_step = n_pairs > 0 ? kThreads / n_pairs : 1;
  int my_tok = n_pairs > 0 ? (int)__umulhi((uint32_t)tid, a.by_pairs) : tok;       // tid / n_pairs
  const int pair = tid - my_tok * n_pairs, axis = (pair >= a.pairs0) + (pair >= a.pairs01);
  if (my_tok >= tok_step) my_tok = tok;
  constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurn2 = -0x1.6b01ec5417056p-57;
  const double f0 = my_tok < tok ? a.freq[pair] : 0.0, f = f0 * kTurn, f2 = fma(f0, kTurn, -f) + f0 * kTurn2;

  for (int64_t g = blockIdx.x; g < a.groups; g += gridDim.x) {
    const int64_t b = g / a.groups_t;
    const int t0 = (int)(g - b * a.groups_t) << a.tok_log, last = a.T - 1 - t0;   // the group's last token, from its first
    const bool on_t = own_c && tk <= last;
    const int64_t tt = t0 + min(tk, last);
    const E* x = x0 + b * a.xs[i][0] + tt * a.xs[i][2] + h0 * a.xs[i][1];
    const E* dy = kGrad ? dy0 + b * a.dys[i][0] + tt * a.dys[i][2] + h0 * a.dys[i][1] : nullptr;
    E* y = y0 + b * a.ys[i][0] + tt * a.ys[i][2] + h0 * a.ys[i][1];
    Raw<E> xa[kRows], xb[kRows], ga[kGrad ? kRows : 1], gb[kGrad ? kRows : 1];
    if constexpr (kGrad) {                         // a token past the end adds nothing to the weights' gradients
#pragma unroll
      for (int u = 0; u < kRows; ++u) ga[u] = gb[u] = Raw<E>{};
    }
    auto fetch = [&](int h) {                      // rows of heads h, h + h_step, ..; x and dy move behind them
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (h + u * h_step < H) {
          get(xa[u], x + oa);
          get(xb[u], x + ob);
          if constexpr (kGrad) {
            if (on_t) {
              get(ga[u], dy + oa);
              get(gb[u], dy + ob);
            }
          }
        }
        x += x_step;
        if constexpr (kGrad) dy += dy_step;
      }
    };
    fetch(h0);
    // ---- cosines and sines of the workgroup's tokens ------------------------------------------------------------------
    if (kGrad || g != blockIdx.x) __syncthreads(); // the previous group's are read
    if (my_tok < tok) {
      const int64_t* const pos = a.pos + b * a.pos_stride_b + axis;
      for (int k = my_tok; k < tok; k += tok_step) {
        const double at = (double)pos[(int64_t)(t0 + min(k, last)) * a.n_axes];
        const double turn = fma(at, f, -rint(at * f)) + at * f2;
        float s, co;
        sincospif((float)(2.0 * turn), &s, &co);
        turns[k * n_pairs + pair] = make_float2(a.mscale * co, a.sign * a.mscale * s);
      }
    }
    __syncthreads();
    f8 cs, sn;
    const float2* const ta = on_a ? turns + tk * n_pairs + pa : turns;
    const float2* const tb = on_b ? turns + tk * n_pairs + pb : turns;
    auto my_turns = [&] {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 v = j < 4 ? ta[j] : tb[j - 4];
        cs[j] = v.x;
        sn[j] = v.y;
      }
    };
    if constexpr (!kGrad) my_turns();
#pragma unroll 1
    for (int h = h0; h < H; h += kRows * h_step) {
      Raw<E> ua[kRows], ub[kRows], va[kGrad ? kRows : 1], vb[kGrad ? kRows : 1];
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        ua[u] = xa[u];
        ub[u] = xb[u];
        if constexpr (kGrad) {
          va[u] = ga[u];
          vb[u] = gb[u];
        }
      }
      fetch(h + kRows * h_step);
#pragma unroll
      for (int u = 0; u < kRows; ++u) {
        if (h + u * h_step >= H) break;            // (the lanes of a row go together)
        f8 p, q, gp, gq;
        unpack(ua[u], p);
        unpack(ub[u], q);
        if constexpr (kNorm) {
          float sq = 0.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) sq += p[j] * p[j] + q[j] * q[j];
          const float r = inv_sqrt(row_sum(own_c ? sq : 0.0f, a.lanes_log) * inv_d + a.eps);
          if constexpr (kGrad) {
            unpack(va[u], gp);
            unpack(vb[u], gq);
            // read again for every row: kept in registers, they and the weights would leave room for fewer waves
            asm volatile("" : : : "memory");
            my_turns();
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              wa[j] = weights[oa + j];
              wb[j] = weights[ob + j];
            }
            turn<HALF>(gp, gq, cs, sn, on_a, on_b);
            float dot = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              gp[j] *= r;
              gq[j] *= r;
              dwa[j] += gp[j] * p[j];
              dwb[j] += gq[j] * q[j];
              gp[j] *= wa[j];
              gq[j] *= wb[j];
              dot += gp[j] * p[j] + gq[j] * q[j];
            }
            const float m = row_sum(own_c ? dot : 0.0f, a.lanes_log) * inv_d * r * r;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              p[j] = gp[j] - p[j] * m;
              q[j] = gq[j] - q[j] * m;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              p[j] *= r * wa[j];
              q[j] *= r * wb[j];
            }
          }
        }
        if constexpr (!kGrad) turn<HALF>(p, q, cs, sn, on_a, on_b);
        if (on_t) {
          put(y + oa, p);
          put(y + ob, q);
        }
        y += y_step;
      }
    }
  }

  if constexpr (kGrad) {
    // the weights' gradients of this workgroup: lanes of a wave that own the same elements, then the four waves
    const int wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = column_sum(dwa[j], a.lanes_log), v = column_sum(dwb[j], a.lanes_log);
      if (lane < lanes) {
        sums[wave][lane * 16 + j] = u;
        sums[wave][lane * 16 + 8 + j] = v;
      }
    }
    __syncthreads();
    if (tid < lanes && own_c) {
      float* const to = a.part + ((int64_t)i * gridDim.x + blockIdx.x) * a.d;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float u = 0.0f, v = 0.0f;
#pragma unroll
        for (int k = 0; k < kThreads / 64; ++k) {
          u += sums[k][tid * 16 + j];
          v += sums[k][tid * 16 + 8 + j];
        }
        to[oa + j] = u;
        to[ob + j] = v;
      }
    }
  }
}

// dw = the sum of the workgroups' partial sums: 16 columns of a tensor to a workgroup, 64 rows at a time, four of them in flight
__global__ void __launch_bounds__(256) rotary_weights_kernel(const float* part, int parts_q, int parts_k, int d, float* dwq, float* dwk) {
  __shared__ float4 s[4][4];
  const int i = blockIdx.y, col = blockIdx.x * 16 + 4 * (threadIdx.x & 3), row = threadIdx.x >> 2;
  float* const dw = i ? dwk : dwq;
  if (!dw) return;
  const int n_parts = i ? parts_k : parts_q;
  const float* const from = part + (int64_t)i * parts_q * d + col;
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int g = row; g < n_parts; g += 256) {
    float4 u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      u[k] = g + 64 * k < n_parts ? *reinterpret_cast<const float4*>(from + (int64_t)(g + 64 * k) * d) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v.x += u[k].x;
      v.y += u[k].y;
      v.z += u[k].z;
      v.w += u[k].w;
    }
  }
  // threads with the same columns: every fourth lane of a wave, then the four waves
  v.x = column_sum(v.x, 2);
  v.y = column_sum(v.y, 2);
  v.z = column_sum(v.z, 2);
  v.w = column_sum(v.w, 2);
  if ((threadIdx.x & 63) < 4) s[threadIdx.x >> 6][threadIdx.x & 3] = v;
  __syncthreads();
  if (threadIdx.x < 16) {
    float u = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) u += reinterpret_cast<const float*>(&s[k][0])[threadIdx.x];
    dw[blockIdx.x * 16 + threadIdx.x] = u;
  }
}

struct RotaryShape {
  int lanes_log, tok_log, groups_t;
  int64_t groups;
};
RotaryShape rotary_shape(const pbsa_rotary& p) {
  RotaryShape s;
  s.lanes_log = 0;
  while ((1 << s.lanes_log) < p.d / 16) ++s.lanes_log;
  s.tok_log = 4;
  static_assert(kMaxTok == 16, "");
  // As many tokens as leave a workgroup to each compute unit for each tensor: what a workgroup does once costs more than the
  // uneven end of a launch (4680 tokens x 12 x 128 of two tensors: 16 tokens 13.0 us, 8 13.8, 4 16.8, 32 16.7; backward 20.6,
  // 22.8, 28, 25.7; 1000 x 5 x 64 in binary32: 4 tokens 5.7, 1 7.5).
  const auto groups_t = [&] { return ((int64_t)p.T + (1 << s.tok_log) - 1) >> s.tok_log; };
  while (s.tok_log > 0 && p.n * groups_t() < 256) --s.tok_log;
  s.groups_t = (int)groups_t();
  s.groups = (int64_t)p.n * s.groups_t;
  return s;
}
int grad_groups(const RotaryShape& s) { return (int)(s.groups < kMaxGroups ? s.groups : kMaxGroups); }

template <typename E, RotaryOp OP>
void launch_typed(const pbsa_rotary& p, const RotaryArgs& a, unsigned grid, hipStream_t stream) {
  if (p.half) hipLaunchKernelGGL((rotary_kernel<E, true, OP>), dim3(grid, p.Hk > 0 ? 2 : 1), dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL((rotary_kernel<E, false, OP>), dim3(grid, p.Hk > 0 ? 2 : 1), dim3(kThreads), 0, stream, a);
}
template <typename E>
void launch_op(const pbsa_rotary& p, RotaryOp op, const RotaryArgs& a, unsigned grid, hipStream_t stream) {
  if (op == RotaryOp::rotate) launch_typed<E, RotaryOp::rotate>(p, a, grid, stream);
  else if (op == RotaryOp::norm) launch_typed<E, RotaryOp::norm>(p, a, grid, stream);
  else launch_typed<E, RotaryOp::norm_grad>(p, a, grid, stream);
}

}  // namespace

size_t rotary_workspace_bytes(const pbsa_rotary& p) {
  const size_t n = (size_t)grad_groups(rotary_shape(p)) * 2 * p.d * sizeof(float);
  return (n + 255) & ~(size_t)255;
}

hipError_t launch_rotary(const pbsa_rotary& p, RotaryOp op, const RotaryTensors& t, void* ws, hipStream_t stream) {
  const RotaryShape s = rotary_shape(p);
  RotaryArgs a{};
  a.T = p.T;
  a.H[0] = p.Hq;
  a.H[1] = p.Hk;
  a.d = p.d;
  a.rot = p.rot;
  a.n_axes = p.n_axes;
  a.pairs0 = p.n_axes > 1 ? p.pairs[0] : p.rot / 2;
  a.pairs01 = p.n_axes > 2 ? p.pairs[0] + p.pairs[1] : p.rot / 2;
  a.lanes_log = s.lanes_log;
  a.tok_log = s.tok_log;
  a.by_pairs = p.rot > 0 ? (uint32_t)((((uint64_t)1 << 32) + p.rot / 2 - 1) / (p.rot / 2)) : 0;
  a.groups_t = s.groups_t;
  a.groups = s.groups;
  a.mscale = p.mscale;
  a.eps = p.eps;
  a.sign = op == RotaryOp::norm_grad ? -1.0f : t.sign;
  a.pos_stride_b = p.pos_stride_b;
  for (int i = 0; i < 2; ++i) {
    a.x[i] = t.x[i];
    a.dy[i] = t.dy[i];
    a.y[i] = t.y[i];
    a.w[i] = a.H[i] > 0 ? t.w[i] : nullptr;
    for (int k = 0; k < 3; ++k) {
      a.xs[i][k] = (i ? p.k : p.q)[k];
      a.dys[i][k] = (i ? p.ko : p.qo)[k];
      a.ys[i][k] = op == RotaryOp::norm_grad ? (i ? p.dk : p.dq)[k] : (i ? p.ko : p.qo)[k];
    }
  }
  a.pos = t.pos;
  a.freq = t.freq;
  a.part = static_cast<float*>(ws);
  const bool grad = op == RotaryOp::norm_grad;
  const unsigned grid = p.Hq + p.Hk == 0 ? 0 : grad ? (unsigned)grad_groups(s) : (unsigned)std::min<int64_t>(s.groups, kMostGroups);
  if (grid > 0) {
    if (p.dtype == PBSA_BF16) launch_op<__bf16>(p, op, a, grid, stream);
    else if (p.dtype == PBSA_FP16) launch_op<_Float16>(p, op, a, grid, stream);
    else launch_op<float>(p, op, a, grid, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (grad && (t.dw[0] || t.dw[1])) {
    hipLaunchKernelGGL(rotary_weights_kernel, dim3((unsigned)p.d / 16, 2), dim3(256), 0, stream, a.part, (int)grid, p.Hk > 0 ? (int)grid : 0, p.d,
                       t.dw[0], t.dw[1]);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace pbsa
