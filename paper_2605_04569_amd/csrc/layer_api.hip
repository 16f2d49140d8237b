// Host side of the operators that stand beside the sparse attention in a transformer's layer (include/isa.h): argument checks,
// workspace sizes and launches.
#include <math.h>

#include "cross.h"
#include "rms_norm.h"

namespace isa {

static bool type_ok(int t) { return t == ISA_BF16 || t == ISA_F32; }

static int check_norm(const isa_norm_problem* p) {
  if (!p) return ISA_ERR_NULL;
  if (!type_ok(p->dtype) || !type_ok(p->weight_dtype)) return ISA_ERR_DTYPE;
  if (p->rows < 0 || p->rows > 0x7fffffffLL || p->channels < 1 || p->channels > 32768) return ISA_ERR_SHAPE;
  if (p->group != 0 && (p->group != 128 || p->channels % 128)) return ISA_ERR_SHAPE;
  if (!(p->eps >= 0.0) || !isfinite(p->eps)) return ISA_ERR_UNSUPPORTED;
  return ISA_OK;
}
static bool read_stride(int64_t s) { return s >= 0 && s < (1ll << 40); }
static bool write_stride(const isa_norm_problem* p, int64_t s) { return s >= p->channels && s < (1ll << 40); }
// a pointer to whole elements
static bool whole(const void* q, int dtype) { return ((uintptr_t)q & (dtype == ISA_BF16 ? 1u : 3u)) == 0; }

static NormArgs norm_args(const isa_norm_problem* p) {
  NormArgs a = {};
  a.rows = p->rows;
  a.C = p->channels;
  a.group = p->group;
  a.w_f32 = p->weight_dtype == ISA_F32;
  a.eps = (float)p->eps;
  const int half_bits = (int)lround(0.5 * log2((double)p->channels));
  a.square_scale = (float)ldexp(1.0, -half_bits);
  a.sum_scale = (float)(ldexp(1.0, 2 * half_bits) / p->channels);
  return a;
}

static int run_norm(const isa_norm_problem* p, const void* x, const void* residual, const void* weight, void* h, void* y, float* rstd,
                    float* scales, bool eight, void* hip_stream) {
  int rc = check_norm(p);
  if (rc != ISA_OK) return rc;
  if (p->rows == 0) return ISA_OK;
  if (!x || !y || (residual && !h) || (!residual && h) || (eight && !scales)) return ISA_ERR_NULL;
  if (!read_stride(p->stride_x) || !write_stride(p, p->stride_y)) return ISA_ERR_SHAPE;
  if (residual && (!read_stride(p->stride_residual) || !write_stride(p, p->stride_h))) return ISA_ERR_SHAPE;
  if (!whole(x, p->dtype) || !whole(residual, p->dtype) || !whole(h, p->dtype) || !whole(weight, p->weight_dtype)) return ISA_ERR_SHAPE;
  if ((!eight && !whole(y, p->dtype)) || !whole(rstd, ISA_F32) || !whole(scales, ISA_F32) || (h && h == y)) return ISA_ERR_SHAPE;
  // in place only row by row
  if (eight && (y == x || y == residual)) return ISA_ERR_SHAPE;
  if ((y == x && p->stride_y != p->stride_x) || (residual && y == residual && p->stride_y != p->stride_residual)) return ISA_ERR_SHAPE;
  if (h && ((h == x && p->stride_h != p->stride_x) || (h == residual && p->stride_h != p->stride_residual))) return ISA_ERR_SHAPE;
  NormArgs a = norm_args(p);
  a.x = x; a.residual = residual; a.weight = weight; a.h = h; a.y = y; a.rstd = rstd; a.scales = scales;
  a.sx = p->stride_x; a.sr = p->stride_residual; a.sh = p->stride_h; a.sy = p->stride_y;
  hipStream_t st = (hipStream_t)hip_stream;
  ISA_STAGE(launch_rms_norm(a, p->dtype, eight, st));
  return ISA_OK;
}

static bool read_strides(const isa_strides& s) {
  const int64_t all[3] = {s.b, s.h, s.t};
  for (int64_t v : all)
    if (v < 0 || v >= (1ll << 40) || v % 8) return false;
  return s.t < (1ll << 22);
}
static bool write_strides(const isa_cross_problem* p, const isa_strides& s, int heads) {
  return read_strides(s) && s.t >= p->D && (heads == 1 || s.h >= p->D) && (p->B <= 1 || s.b >= p->D);
}

static int check_cross(const isa_cross_problem* p) {
  if (!p) return ISA_ERR_NULL;
  if (!type_ok(p->dtype)) return ISA_ERR_DTYPE;
  if (p->D != 64 && p->D != 128) return ISA_ERR_SHAPE;
  if (p->B < 0 || p->H < 1 || p->H_kv < 1 || p->H % p->H_kv) return ISA_ERR_SHAPE;
  if (p->S_q < 0 || p->S_k < 0 || p->S_q > (1 << 28) || p->S_k > (1 << 28)) return ISA_ERR_SHAPE;
  const long long bh = (long long)p->B * p->H;             // (no count of rows or workgroups passes 31 bits)
  if (bh > (1 << 20) || bh * p->S_q > (1 << 30) || bh / (p->H / p->H_kv) * p->S_k > (1 << 30)) return ISA_ERR_SHAPE;
  if (!(p->scale > 0.0) || !isfinite(p->scale) || !isfinite((float)(p->scale * 1.4426950408889634)) || !((float)p->scale > 0.0f))
    return ISA_ERR_UNSUPPORTED;
  if (!read_strides(p->q) || !read_strides(p->k) || !read_strides(p->v) || !write_strides(p, p->out, p->H)) return ISA_ERR_SHAPE;
  return ISA_OK;
}

static CrossArgs cross_args(const isa_cross_problem* p, const void* q, const void* k, const void* v, const int32_t* kv_len,
                            const uint8_t* key_mask, int64_t key_mask_stride) {
  CrossArgs a = {};
  a.q = q; a.k = k; a.v = v;
  a.kv_len = kv_len; a.mask = key_mask; a.mask_stride = key_mask_stride;
  a.B = p->B; a.H = p->H; a.Hkv = p->H_kv; a.group = p->H / p->H_kv; a.Sq = p->S_q; a.Sk = p->S_k;
  a.sq = p->q; a.sk = p->k; a.sv = p->v; a.so = p->out;
  a.scale = (float)p->scale;
  a.cscale = (float)(p->scale * 1.4426950408889634);     // log2(e)
  a.rows = a.group * p->S_q;
  return a;
}

static int check_masks(const isa_cross_problem* p, const int32_t* kv_len, const uint8_t* key_mask, int64_t key_mask_stride) {
  if (!whole(kv_len, ISA_F32)) return ISA_ERR_SHAPE;
  if (key_mask && (key_mask_stride < 0 || key_mask_stride >= (1ll << 40))) return ISA_ERR_SHAPE;
  return ISA_OK;
}

}  // namespace isa

using namespace isa;

extern "C" {

size_t isa_cross_workspace_bytes(const isa_cross_problem* p, int backward) {
  if (check_cross(p) != ISA_OK || p->B == 0) return 0;
  if (backward) {
    const CrossBackwardPlan c = cross_backward_plan(*p);
    return c.side_bytes + c.part_bytes + c.ml_bytes;
  }
  const CrossPlan c = cross_forward_plan(*p);
  return align256(c.part_rows * p->D * 4) + align256(c.part_rows * sizeof(float4));
}

int isa_cross_attention(const isa_cross_problem* p, const void* q, const void* k, const void* v, const int32_t* kv_len,
                        const uint8_t* key_mask, int64_t key_mask_stride, void* out, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
  int rc = check_cross(p);
  if (rc != ISA_OK) return rc;
  if (p->B == 0 || p->S_q == 0) return ISA_OK;
  if (!q || !out || (p->S_k > 0 && (!k || !v))) return ISA_ERR_NULL;
  if (!all_aligned16(q, k, v, out) || !whole(lse, ISA_F32)) return ISA_ERR_SHAPE;
  if (out == q || out == k || out == v) return ISA_ERR_SHAPE;
  if ((rc = check_masks(p, kv_len, key_mask, key_mask_stride)) != ISA_OK) return rc;
  const size_t need = isa_cross_workspace_bytes(p, 0);
  if (need && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return ISA_ERR_WORKSPACE;
  CrossArgs a = cross_args(p, q, k, v, kv_len, key_mask, key_mask_stride);
  a.out = out; a.lse = lse;
  a.part_o = (float*)workspace;
  a.part_ml = (float4*)((uintptr_t)workspace + align256(cross_forward_plan(*p).part_rows * p->D * 4));
  hipStream_t st = (hipStream_t)hip_stream;
  ISA_STAGE(launch_cross_forward(a, *p, st));
  return ISA_OK;
}

int isa_cross_attention_backward(const isa_cross_problem* p, const void* q, const void* k, const void* v, const int32_t* kv_len,
                                 const uint8_t* key_mask, int64_t key_mask_stride, const void* out, const float* lse,
                                 const void* d_out, void* dq, void* dk, void* dv, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
  int rc = check_cross(p);
  if (rc != ISA_OK) return rc;
  const bool states = dk || dv;                          // neither: dq alone is worked out
  if (!read_strides(p->d_out) || !write_strides(p, p->dq, p->H)) return ISA_ERR_SHAPE;
  if (states && (!write_strides(p, p->dk, p->H_kv) || !write_strides(p, p->dv, p->H_kv))) return ISA_ERR_SHAPE;
  if (p->B == 0 || (p->S_q == 0 && p->S_k == 0)) return ISA_OK;
  if (p->S_q > 0 && (!q || !out || !lse || !d_out || !dq)) return ISA_ERR_NULL;
  if (p->S_k > 0 && (!k || !v || (states && (!dk || !dv)))) return ISA_ERR_NULL;
  if (!all_aligned16(q, k, v, out, d_out, dq, dk, dv) || !whole(lse, ISA_F32)) return ISA_ERR_SHAPE;
  const void* ins[] = {q, k, v, out, d_out};
  const void* outs[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    for (const void* in : ins)
      if (outs[i] && outs[i] == in) return ISA_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return ISA_ERR_SHAPE;
  }
  if ((rc = check_masks(p, kv_len, key_mask, key_mask_stride)) != ISA_OK) return rc;
  const size_t need = isa_cross_workspace_bytes(p, 1);
  if (need && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return ISA_ERR_WORKSPACE;
  CrossArgs a = cross_args(p, q, k, v, kv_len, key_mask, key_mask_stride);
  a.sdo = p->d_out; a.sdq = p->dq; a.sdk = p->dk; a.sdv = p->dv;
  a.d_out = d_out; a.fwd_out = out; a.fwd_lse = lse;
  a.dq = dq; a.dk = dk; a.dv = dv;
  a.side = (float*)workspace;
  const CrossBackwardPlan c = cross_backward_plan(*p);
  a.part_o = (float*)((uintptr_t)workspace + c.side_bytes);
  a.part_ml = (float4*)((uintptr_t)workspace + c.side_bytes + c.part_bytes);
  hipStream_t st = (hipStream_t)hip_stream;
  ISA_STAGE(launch_cross_backward(a, *p, st));
  return ISA_OK;
}

int isa_rms_norm(const isa_norm_problem* p, const void* x, const void* residual, const void* weight, void* h, void* y, float* rstd,
                 void* hip_stream) {
  return run_norm(p, x, residual, weight, h, y, rstd, nullptr, false, hip_stream);
}

int isa_rms_norm_8bit(const isa_norm_problem* p, const void* x, const void* residual, const void* weight, void* h, void* y8,
                      float* scales, void* hip_stream) {
  return run_norm(p, x, residual, weight, h, y8, nullptr, scales, true, hip_stream);
}

size_t isa_rms_norm_workspace_bytes(const isa_norm_problem* p) {
  if (check_norm(p) != ISA_OK) return 0;
  const int wgs = norm_backward_workgroups(p);
  return align256((size_t)(wgs > 0 ? wgs : 1) * (size_t)p->channels * 4);
}

int isa_rms_norm_backward(const isa_norm_problem* p, const void* x, const void* residual, const void* weight, const float* rstd,
                          const void* dy, const void* dh, void* dx, void* d_weight, void* workspace, size_t workspace_bytes,
                          void* hip_stream) {
  int rc = check_norm(p);
  if (rc != ISA_OK) return rc;
  if (p->rows > 0) {
    if (!x || !rstd || !dy || !dx) return ISA_ERR_NULL;
    if (!read_stride(p->stride_x) || (residual && !read_stride(p->stride_residual)) || !read_stride(p->stride_dy) ||
        (dh && !read_stride(p->stride_dh)) || !write_stride(p, p->stride_dx))
      return ISA_ERR_SHAPE;
    if (!whole(x, p->dtype) || !whole(residual, p->dtype) || !whole(dy, p->dtype) || !whole(dh, p->dtype) || !whole(dx, p->dtype) ||
        !whole(rstd, ISA_F32) || dx == x || dx == residual)
      return ISA_ERR_SHAPE;
    if ((dx == dy && p->stride_dx != p->stride_dy) || (dh && dx == dh && p->stride_dx != p->stride_dh)) return ISA_ERR_SHAPE;
  }
  if (!whole(weight, p->weight_dtype) || !whole(d_weight, p->weight_dtype)) return ISA_ERR_SHAPE;
  const int wgs = norm_backward_workgroups(p);
  if (d_weight) {
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < isa_rms_norm_workspace_bytes(p)) return ISA_ERR_WORKSPACE;
  }
  NormArgs a = norm_args(p);
  a.x = x; a.residual = residual; a.weight = weight; a.y = dx; a.rstd = const_cast<float*>(rstd); a.dy = dy; a.dh = dh;
  a.sx = p->stride_x; a.sr = p->stride_residual; a.sy = p->stride_dx; a.sdy = p->stride_dy; a.sdh = p->stride_dh;
  a.partial = d_weight ? (float*)workspace : nullptr;
  hipStream_t st = (hipStream_t)hip_stream;
  ISA_STAGE(launch_rms_norm_backward(a, p->dtype, wgs, d_weight, st));
  return ISA_OK;
}

}  // extern "C"
