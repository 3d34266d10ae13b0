// C-ABI shim of pbsa_layer.h: host-side argument validation, then kernel launches.  Validation makes no HIP call.
#include "pbsa_internal.h"
#include "pbsa_layer_internal.h"

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// One tensor of a call: [n][H][T][d] at `s`.
struct View {
  const void* at;
  const int64_t* s;
  int64_t n, H, T;
  bool written;
};

// The pointer and the strides of a tensor; one without elements is not looked at.
int check_view(const View& v, int64_t d) {
  if (v.n == 0 || v.H == 0 || v.T == 0) return PBSA_OK;
  if (!v.at) return PBSA_EINVAL;
  int64_t ext[3] = {v.n, v.H, v.T}, st[3] = {v.s[0], v.s[1], v.s[2]};
  for (int i = 0; i < 3; ++i) {
    if (st[i] < 0) return PBSA_EINVAL;
    if (ext[i] > 1 && st[i] > ((int64_t)1 << 46) / ext[i]) return PBSA_ESHAPE;   // bytes stay within 64 bits
  }
  if (v.written) {
    // every element has a place of its own: along each dimension, by rising strides, what lies below fits into a step
    for (int i = 0; i < 3; ++i)
      for (int k = i + 1; k < 3; ++k)
        if (st[k] < st[i]) {
          int64_t t = st[i]; st[i] = st[k]; st[k] = t;
          t = ext[i]; ext[i] = ext[k]; ext[k] = t;
        }
    int64_t span = d;
    for (int i = 0; i < 3; ++i) {
      if (ext[i] == 1) continue;
      if (st[i] < span) return PBSA_EINVAL;
      span += st[i] * (ext[i] - 1);
    }
  }
  if (!aligned(v.at, 16)) return PBSA_EALIGN;
  for (int i = 0; i < 3; ++i)
    if (ext[i] > 1 && st[i] % 8 != 0) return PBSA_EALIGN;
  return PBSA_OK;
}

bool same_strides(const int64_t* a, const int64_t* b) { return a[0] == b[0] && a[1] == b[1] && a[2] == b[2]; }

int check_scratch(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return PBSA_OK;
  if (!ws || ws_bytes < need) return PBSA_EWS;
  return aligned(ws, 256) ? PBSA_OK : PBSA_EALIGN;
}

// ---- norm and rotation --------------------------------------------------------------------------------------------------
int check_rotary(const pbsa_rotary* p) {
  if (!p || p->size != sizeof(pbsa_rotary)) return PBSA_EINVAL;
  if (p->n < 0 || p->T < 0 || p->Hq < 0 || p->Hk < 0 || p->d < 1 || p->rot < 0 || p->rot > p->d) return PBSA_EINVAL;
  if (p->half != 0 && p->half != 1) return PBSA_EINVAL;
  if (p->n_axes < 1 || p->n_axes > PBSA_ROTARY_MAX_AXES) return PBSA_EINVAL;
  int64_t pairs = 0;
  for (int i = 0; i < p->n_axes; ++i) {
    if (p->pairs[i] < 0) return PBSA_EINVAL;
    pairs += p->pairs[i];
  }
  if (2 * pairs != p->rot) return PBSA_EINVAL;
  if (!(p->eps >= 0.0f) || !(p->eps < 1e30f) || !(p->mscale > -1e30f) || !(p->mscale < 1e30f)) return PBSA_EINVAL;
  if (p->dtype < PBSA_BF16 || p->dtype > PBSA_FP32) return PBSA_ESHAPE;
  if (p->d % 16 != 0 || p->d > PBSA_ROTARY_MAX_D || p->rot % 16 != 0) return PBSA_ESHAPE;
  if (p->Hq > PBSA_LAYER_MAX_HEADS || p->Hk > PBSA_LAYER_MAX_HEADS || (int64_t)p->n * p->T > INT32_MAX) return PBSA_ESHAPE;
  return PBSA_OK;
}

int check_positions(const pbsa_rotary* p, const int64_t* pos, const double* freq) {
  if (p->n == 0 || p->T == 0 || p->Hq + p->Hk == 0) return PBSA_OK;
  if (!pos || (p->rot > 0 && !freq)) return PBSA_EINVAL;
  if (!aligned(pos, 8) || !aligned(freq, 8)) return PBSA_EALIGN;
  if (p->pos_stride_b != 0 && p->pos_stride_b < (int64_t)p->T * p->n_axes) return PBSA_EINVAL;
  return p->pos_stride_b > ((int64_t)1 << 46) / (p->n > 0 ? p->n : 1) ? PBSA_ESHAPE : PBSA_OK;
}

int check_forward(const pbsa_rotary* p, const void* Q, const void* K, const int64_t* pos, const double* freq, void* Qo, void* Ko) {
  int rc = check_rotary(p);
  if (rc || (rc = check_positions(p, pos, freq))) return rc;
  const View views[4] = {{Q, p->q, p->n, p->Hq, p->T, false}, {K, p->k, p->n, p->Hk, p->T, false},
                         {Qo, p->qo, p->n, p->Hq, p->T, true}, {Ko, p->ko, p->n, p->Hk, p->T, true}};
  for (const View& v : views)
    if ((rc = check_view(v, p->d))) return rc;
  if ((p->Hq > 0 && Q && Q == Qo && !same_strides(p->q, p->qo)) || (p->Hk > 0 && K && K == Ko && !same_strides(p->k, p->ko)))
    return PBSA_EINVAL;
  return PBSA_OK;
}

// ---- cross attention ----------------------------------------------------------------------------------------------------
int check_cross(const pbsa_cross* p) {
  if (!p || p->size != sizeof(pbsa_cross)) return PBSA_EINVAL;
  if (p->n < 0 || p->T < 0 || p->Nk < 0 || p->Hq < 0 || p->Hk < 0) return PBSA_EINVAL;
  if (p->Hk == 0 ? p->Hq != 0 : p->Hq % p->Hk != 0) return PBSA_EINVAL;
  if (!(p->scale > 1e-30f) || !(p->scale < 1e30f)) return PBSA_EINVAL;
  if (p->dtype != PBSA_BF16 && p->dtype != PBSA_FP16) return PBSA_ESHAPE;
  if (p->d != 64 && p->d != 128) return PBSA_ESHAPE;
  if (p->Hq > PBSA_LAYER_MAX_HEADS || p->Nk > PBSA_CROSS_MAX_NK) return PBSA_ESHAPE;
  // rows and states of all heads are counted in 32 bits
  const int64_t most = (int64_t)1 << 30;
  if ((int64_t)p->n * p->T > most / (p->Hq > 0 ? p->Hq : 1) || (int64_t)p->n * p->Hk > most / (p->Nk + 128)) return PBSA_ESHAPE;
  return PBSA_OK;
}

// What both directions read: a tile's offsets from its first row are 32 bits wide, so the steps between tokens are bounded.
int check_cross_inputs(const pbsa_cross* p, const void* Q, const void* K, const void* V, const int32_t* k_len, const uint8_t* k_mask) {
  const View views[3] = {{Q, p->q, p->n, p->Hq, p->T, false}, {K, p->k, p->n, p->Hk, p->Nk, false}, {V, p->v, p->n, p->Hk, p->Nk, false}};
  for (const View& v : views)
    if (const int rc = check_view(v, p->d)) return rc;
  if (p->Nk > 1 && (p->k[2] > (1 << 24) || p->v[2] > (1 << 24))) return PBSA_ESHAPE;
  if (!aligned(k_len, 4)) return PBSA_EALIGN;
  if (k_mask && p->mask_stride_b != 0 && p->mask_stride_b < p->Nk) return PBSA_EINVAL;
  return k_mask && p->mask_stride_b > ((int64_t)1 << 46) / (p->n > 0 ? p->n : 1) ? PBSA_ESHAPE : PBSA_OK;
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

int pbsa_rotate(const pbsa_rotary* p, const void* Q, const void* K, const int64_t* pos, const double* freq, void* Qo, void* Ko,
                int32_t inverse, void* hip_stream) {
  const int rc = check_forward(p, Q, K, pos, freq, Qo, Ko);
  if (rc) return rc;
  if (inverse != 0 && inverse != 1) return PBSA_EINVAL;
  const pbsa::RotaryTensors t{{Q, K}, {}, {Qo, Ko}, {}, {}, pos, freq, inverse ? -1.0f : 1.0f};
  return pbsa::report(pbsa::launch_rotary(*p, pbsa::RotaryOp::rotate, t, nullptr, static_cast<hipStream_t>(hip_stream)));
}

int pbsa_norm_rotate_fwd(const pbsa_rotary* p, const void* Q, const void* K, const float* wq, const float* wk, const int64_t* pos,
                         const double* freq, void* Qo, void* Ko, void* hip_stream) {
  const int rc = check_forward(p, Q, K, pos, freq, Qo, Ko);
  if (rc) return rc;
  if (!aligned(wq, 4) || !aligned(wk, 4)) return PBSA_EALIGN;
  const pbsa::RotaryTensors t{{Q, K}, {}, {Qo, Ko}, {wq, wk}, {}, pos, freq, 1.0f};
  return pbsa::report(pbsa::launch_rotary(*p, pbsa::RotaryOp::norm, t, nullptr, static_cast<hipStream_t>(hip_stream)));
}

int pbsa_norm_rotate_workspace_bytes(const pbsa_rotary* p, size_t* out) {
  if (!out) return PBSA_EINVAL;
  const int rc = check_rotary(p);
  if (rc) return rc;
  *out = pbsa::rotary_workspace_bytes(*p);
  return PBSA_OK;
}

int pbsa_norm_rotate_bwd(const pbsa_rotary* p, const void* Q, const void* K, const float* wq, const float* wk, const int64_t* pos,
                         const double* freq, const void* dQo, const void* dKo, void* dQ, void* dK, float* dwq, float* dwk, void* ws,
                         size_t ws_bytes, void* hip_stream) {
  int rc = check_rotary(p);
  if (rc || (rc = check_positions(p, pos, freq))) return rc;
  const View views[6] = {{Q, p->q, p->n, p->Hq, p->T, false},   {K, p->k, p->n, p->Hk, p->T, false},
                         {dQo, p->qo, p->n, p->Hq, p->T, false}, {dKo, p->ko, p->n, p->Hk, p->T, false},
                         {dQ, p->dq, p->n, p->Hq, p->T, true},  {dK, p->dk, p->n, p->Hk, p->T, true}};
  for (const View& v : views)
    if ((rc = check_view(v, p->d))) return rc;
  if ((p->Hq > 0 && dQ && dQ == dQo && !same_strides(p->dq, p->qo)) || (p->Hk > 0 && dK && dK == dKo && !same_strides(p->dk, p->ko)))
    return PBSA_EINVAL;
  if (!aligned(wq, 4) || !aligned(wk, 4) || !aligned(dwq, 4) || !aligned(dwk, 4)) return PBSA_EALIGN;
  if ((rc = check_scratch(ws, ws_bytes, pbsa::rotary_workspace_bytes(*p)))) return rc;
  const pbsa::RotaryTensors t{{Q, K}, {dQo, dKo}, {dQ, dK}, {wq, wk}, {dwq, dwk}, pos, freq, -1.0f};
  return pbsa::report(pbsa::launch_rotary(*p, pbsa::RotaryOp::norm_grad, t, ws, static_cast<hipStream_t>(hip_stream)));
}

int pbsa_cross_workspace_bytes(const pbsa_cross* p, size_t* out) {
  if (!out) return PBSA_EINVAL;
  const int rc = check_cross(p);
  if (rc) return rc;
  const size_t plain = pbsa::cross_workspace_bytes(*p, false), masked = pbsa::cross_workspace_bytes(*p, true);
  *out = plain > masked ? plain : masked;
  return PBSA_OK;
}

int pbsa_cross_attention_fwd(const pbsa_cross* p, const void* Q, const void* K, const void* V, const int32_t* k_len,
                             const uint8_t* k_mask, void* O, float* lse, void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check_cross(p);
  if (rc || (rc = check_cross_inputs(p, Q, K, V, k_len, k_mask))) return rc;
  if ((rc = check_view({O, p->o, p->n, p->Hq, p->T, true}, p->d))) return rc;
  if (!aligned(lse, 4)) return PBSA_EALIGN;
  if (!pbsa::cross_fits(*p, k_mask != nullptr)) return PBSA_ESHAPE;
  if ((rc = check_scratch(ws, ws_bytes, pbsa::cross_workspace_bytes(*p, k_mask != nullptr)))) return rc;
  return pbsa::report(pbsa::launch_cross(*p, Q, K, V, k_len, k_mask, O, lse, ws, static_cast<hipStream_t>(hip_stream)));
}

int pbsa_cross_bwd_workspace_bytes(const pbsa_cross* p, size_t* out) {
  if (!out) return PBSA_EINVAL;
  const int rc = check_cross(p);
  if (rc) return rc;
  *out = pbsa::cross_bwd_workspace_bytes(*p);
  return PBSA_OK;
}

int pbsa_cross_attention_bwd(const pbsa_cross* p, const void* Q, const void* K, const void* V, const int32_t* k_len,
                             const uint8_t* k_mask, const void* O, const void* dO, const float* lse, void* dQ, void* dK, void* dV,
                             void* ws, size_t ws_bytes, void* hip_stream) {
  int rc = check_cross(p);
  if (rc || (rc = check_cross_inputs(p, Q, K, V, k_len, k_mask))) return rc;
  const View views[5] = {{O, p->o, p->n, p->Hq, p->T, false}, {dO, p->dO, p->n, p->Hq, p->T, false}, {dQ, p->dq, p->n, p->Hq, p->T, true},
                         {dK, p->dk, p->n, p->Hk, p->Nk, true}, {dV, p->dv, p->n, p->Hk, p->Nk, true}};
  for (const View& v : views)
    if ((rc = check_view(v, p->d))) return rc;
  if ((int64_t)p->n * p->Hq * p->T > 0 && !lse) return PBSA_EINVAL;
  if (!aligned(lse, 4)) return PBSA_EALIGN;
  if ((rc = check_scratch(ws, ws_bytes, pbsa::cross_bwd_workspace_bytes(*p)))) return rc;
  return pbsa::report(pbsa::launch_cross_bwd(*p, Q, K, V, k_len, k_mask, O, dO, lse, dQ, dK, dV, ws, static_cast<hipStream_t>(hip_stream)));
}

#pragma GCC visibility pop
}
