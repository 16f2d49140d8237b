// Cross attention in fp32 (the checking mode), forward and backward, gfx950: the structure of cross_fwd.hip and cross_bwd.hip with fp32
// products (v_mfma_f32_16x16x4_f32, which bound it).
//
// A workgroup of 4 waves owns 64 rows, 16 to a wave, in registers, and streams tiles of 32 rows of the other side through one LDS
// stage; the next tile waits in registers.  Rows in LDS are D + 4 floats apart, so that both kinds of reads meet all banks: 16 bytes of 16
// rows (scores), and 16 neighbouring floats of rows 4 apart (the transposed side of the second product).  5280 queries x 231 keys, 8 heads of 128: forward
// 68 us, dq 100, dk and dv 117; matrix pipe busy 67 to 76 % where a compute unit works.  Three workgroups to a compute unit: no difference.
#include "cross_tiles.h"

namespace isa {
namespace {

constexpr int FT = 32;                                   // streamed rows of a tile
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// One tile of FT rows on its way to LDS: 8 threads to a row, D / 32 pieces of 16 bytes each
template <int D> struct TileRegs {
  f32x4 r[D / 32];
  __device__ __forceinline__ void fetch(const float* base, long long stride, int tid, bool ok) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) r[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (!ok) return;
    const float* p = base + (long long)(tid >> 3) * stride + (tid & 7) * 4;
#pragma unroll
    for (int j = 0; j < D / 32; ++j) r[j] = *reinterpret_cast<const f32x4*>(p + 32 * j);
  }
  __device__ __forceinline__ void put(float* tile, int tid) const {
#pragma unroll
    for (int j = 0; j < D / 32; ++j) *reinterpret_cast<f32x4*>(tile + (tid >> 3) * (D + 4) + (tid & 7) * 4 + 32 * j) = r[j];
  }
};

// T = tile rows 16 kt .. x own rows: lane (r, q): tile rows 16 kt + 4 q + i of own row r.  Both sides take channel 16 t + 4 q + e in step (t, e).
template <int D> __device__ __forceinline__ f32x4 scores(const float* tile, const f32x4 (&own)[D / 16], int kt, int r16, int q, f32x4 c) {
  const float* p = tile + (16 * kt + r16) * (D + 4) + 4 * q;
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p + 16 * t);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = mfma4(x[e], own[t][e], c);
  }
  return c;
}
// acc[ct] (channels 16 ct + 4 q + i of own row r) += sum over the tile's rows 16 kt + 4 q' + i of w[i] times the row
template <int D> __device__ __forceinline__ void add_rows(const float* tile, const f32x4 w, int kt, int r16, int q, f32x4 (&acc)[D / 16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float* p = tile + (16 * kt + 4 * q + i) * (D + 4) + r16;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) acc[ct] = mfma4(p[16 * ct], w[i], acc[ct]);
  }
}
template <int D> __device__ __forceinline__ void load_own(const float* row, int q, bool ok, f32x4 (&own)[D / 16]) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) own[t] = ok ? *reinterpret_cast<const f32x4*>(row + 16 * t + 4 * q) : f32x4{0.f, 0.f, 0.f, 0.f};
}
template <int D> __device__ __forceinline__ void store_own(const f32x4 (&acc)[D / 16], float f, float* row, int q) {
#pragma unroll
  for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f32x4*>(row + 16 * t + 4 * q) = acc[t] * f;
}

}  // namespace

// BWD: dq (and the rows' deltas and log-sum-exps for k_cross_dkv_f32); otherwise the forward pass
template <int D, bool BWD>
__global__ __launch_bounds__(256, 2) void k_cross_rows_f32(CrossArgs a) {
  constexpr int CT = D / 16;
  __shared__ __attribute__((aligned(16))) float lds[2 * FT * (D + 4)];
  float* const kt_ = lds;
  float* const vt_ = lds + FT * (D + 4);
  uint32_t item;
  if (!cross_item(a, item)) return;
  const int part = (int)(item % (uint32_t)a.parts);
  item /= (uint32_t)a.parts;
  const long long slot = item;
  const int tile0 = (int)(item % (uint32_t)a.items) * 64;
  const int bh = (int)(item / (uint32_t)a.items), b = bh % a.B, hk = bh / a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, q = lane >> 4;
  const int n_keys = key_count(a, b), n_tiles = (n_keys + FT - 1) / FT;
  const int t_begin = (int)((long long)n_tiles * part / a.parts), t_end = (int)((long long)n_tiles * (part + 1) / a.parts);
  const uint8_t* const mask_row = a.mask ? a.mask + (long long)b * a.mask_stride : nullptr;

  const int row = tile0 + wave * 16 + r16;
  const bool ok = row < a.rows;
  const int use = ok ? row : tile0, head = hk * a.group + use / a.Sq, query = use % a.Sq;
  f32x4 own_q[CT], own_o[CT];
  load_own<D>(reinterpret_cast<const float*>(a.q) + at_row(a.sq, b, head, query), q, true, own_q);
  float neg_m = -LOWEST, l = 0.f, nd = 0.f;              // BWD: neg_m is minus the log-sum-exp
  if constexpr (BWD) {
    f32x4 o[CT];
    load_own<D>(reinterpret_cast<const float*>(a.d_out) + at_row(a.sdo, b, head, query), q, true, own_o);
    load_own<D>(reinterpret_cast<const float*>(a.fwd_out) + at_row(a.so, b, head, query), q, true, o);
    float d = 0.f;
#pragma unroll
    for (int t = 0; t < CT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) d = fmaf(own_o[t][e], o[t][e], d);
    nd = -sum_over_q(d);
    const float lse = a.fwd_lse[((long long)b * a.H + head) * a.Sq + query];
    neg_m = lse == -INFINITY ? -INFINITY : -lse * LOG2E;
    if (part == 0 && q == 0 && ok) {
      float* s = a.side + (((long long)b * a.H + head) * a.side_tiles + (query >> 6)) * 128 + (query & 63);
      s[0] = neg_m;
      s[64] = nd;
      if (query == a.Sq - 1)
        for (int i = 1; i < 64 - (query & 63); ++i) { s[i] = -INFINITY; s[64 + i] = 0.f; }
    }
  }
  f32x4 acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};

  const float* const k_head = reinterpret_cast<const float*>(a.k) + at_row(a.sk, b, hk, 0);
  const float* const v_head = reinterpret_cast<const float*>(a.v) + at_row(a.sv, b, hk, 0);
  TileRegs<D> rk, rv;
  unsigned long long valid = 0, valid_next = 0, seen = 0;
  auto fetch = [&](int t) __attribute__((always_inline)) {
    valid_next = valid_keys(mask_row, t * FT, min(n_keys, t * FT + FT), lane);
    const bool live = (valid_next >> (tid >> 3)) & 1ull;
    rk.fetch(k_head + (long long)t * FT * a.sk.t, a.sk.t, tid, live);
    rv.fetch(v_head + (long long)t * FT * a.sv.t, a.sv.t, tid, live);
  };
  if (t_begin < t_end) fetch(t_begin);
  for (int t = t_begin; t < t_end; ++t) {
    valid = valid_next;
    seen |= valid;
    __syncthreads();
    rk.put(kt_, tid);
    rv.put(vt_, tid);
    __syncthreads();
    if (t + 1 < t_end) fetch(t + 1);
    f32x4 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      s[kt] = scores<D>(kt_, own_q, kt, r16, q, zero4);
      const unsigned long long w = valid >> (16 * kt + 4 * q);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[kt][i] = (w >> i) & 1ull ? s[kt][i] * a.cscale : -INFINITY;
    }
    if constexpr (BWD) {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const f32x4 dp = scores<D>(vt_, own_o, kt, r16, q, f32x4{nd, nd, nd, nd});
        f32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_exp2f(s[kt][i] + neg_m) * dp[i];
        add_rows<D>(kt_, w, kt, r16, q, acc);
      }
    } else {
      float m = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, s[kt][i]);
      m = max_over_q(m);
      if (__ballot(m > -neg_m) != 0ull) {
        const float m_new = fmaxf(m, -neg_m), alpha = __builtin_amdgcn_exp2f(-neg_m - m_new);
        neg_m = -m_new;
        l *= alpha;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) acc[ct] *= alpha;
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        f32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          w[i] = __builtin_amdgcn_exp2f(s[kt][i] + neg_m);
          l += w[i];
        }
        add_rows<D>(vt_, w, kt, r16, q, acc);
      }
    }
  }
  if (!BWD) l = sum_over_q(l);
  if (BWD && neg_m == -INFINITY) {                       // no valid key: zeros (0 times an infinite gradient is no zero)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4;
  }
  if (a.parts > 1) {
    const long long at = (slot * a.parts + part) * 64 + wave * 16 + r16;
    store_own<D>(acc, 1.0f, a.part_o + at * D, q);
    if (!BWD && q == 0) a.part_ml[at] = make_float4(-neg_m, l, l, seen ? 1.f : 0.f);
    return;
  }
  if (!ok) return;
  if constexpr (BWD) {
    store_own<D>(acc, a.scale, reinterpret_cast<float*>(a.dq) + at_row(a.sdq, b, head, query), q);
  } else {
    // (a valid key whose score is minus infinity, and no other: no weights to speak of)
    const float none = seen ? __builtin_nanf("") : 0.f;
    store_own<D>(acc, l == 0.f ? none : 1.0f / l, reinterpret_cast<float*>(a.out) + at_row(a.so, b, head, query), q);
    if (a.lse && q == 0)
      a.lse[((long long)b * a.H + head) * a.Sq + query] = l > 0.f ? 0.6931471805599453f * (log2f(l) - neg_m) : l == 0.f ? (seen ? none : -INFINITY) : l;
  }
}

template <int D>
__global__ __launch_bounds__(256, 2) void k_cross_dkv_f32(CrossArgs a) {
  constexpr int CT = D / 16;
  __shared__ __attribute__((aligned(16))) float lds[2 * FT * (D + 4)];
  __shared__ __attribute__((aligned(16))) float side[2][FT];
  float* const qt_ = lds;
  float* const ot_ = lds + FT * (D + 4);
  uint32_t item;
  if (!cross_item(a, item)) return;
  const int key0 = (int)(item % (uint32_t)a.items) * 64;
  const long long slot = item / (uint32_t)a.items;
  const int part = (int)(slot % a.parts);
  const int bh = (int)(slot / a.parts), b = bh % a.B, hk = bh / a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r16 = lane & 15, q = lane >> 4;
  const int n_keys = key_count(a, b);
  const uint8_t* const mask_row = a.mask ? a.mask + (long long)b * a.mask_stride : nullptr;

  const int key = key0 + wave * 16 + r16;
  const bool live = key < n_keys && (!mask_row || mask_row[key] != 0);
  f32x4 own_k[CT], own_v[CT], ak[CT], av[CT];
  load_own<D>(reinterpret_cast<const float*>(a.k) + at_row(a.sk, b, hk, live ? key : 0), q, live, own_k);
  load_own<D>(reinterpret_cast<const float*>(a.v) + at_row(a.sv, b, hk, live ? key : 0), q, live, own_v);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) ak[ct] = av[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};

  // tiles of 32 queries: two of each of the 64 that share a place in `side`
  bool any = key0 < n_keys;                               // a block without a valid key streams nothing
  if (any && mask_row) any = __syncthreads_or(live) != 0;
  const int per_head = 2 * a.side_tiles, units = any ? a.group * per_head : 0;
  const int u_begin = (int)((long long)units * part / a.parts), u_end = (int)((long long)units * (part + 1) / a.parts);
  TileRegs<D> rq, ro;
  float rs = 0.f;
  auto fetch = [&](int u) __attribute__((always_inline)) {
    const int h = hk * a.group + u / per_head, t = u % per_head;
    const bool in = t * FT + (tid >> 3) < a.Sq;
    rq.fetch(reinterpret_cast<const float*>(a.q) + at_row(a.sq, b, h, t * FT), a.sq.t, tid, in);
    ro.fetch(reinterpret_cast<const float*>(a.d_out) + at_row(a.sdo, b, h, t * FT), a.sdo.t, tid, in);
    if (tid < 64) rs = a.side[(((long long)b * a.H + h) * a.side_tiles + (t >> 1)) * 128 + (tid >> 5) * 64 + (t & 1) * FT + (tid & 31)];
  };
  if (u_begin < u_end) fetch(u_begin);
  for (int u = u_begin; u < u_end; ++u) {
    __syncthreads();
    rq.put(qt_, tid);
    ro.put(ot_, tid);
    if (tid < 64) side[tid >> 5][tid & 31] = rs;
    __syncthreads();
    if (u + 1 < u_end) fetch(u + 1);
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const f32x4 nl = *reinterpret_cast<const f32x4*>(&side[0][16 * rt + 4 * q]), nd = *reinterpret_cast<const f32x4*>(&side[1][16 * rt + 4 * q]);
      const f32x4 s = scores<D>(qt_, own_k, rt, r16, q, zero4), dp = scores<D>(ot_, own_v, rt, r16, q, nd);
      f32x4 p, w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[i] = live ? __builtin_amdgcn_exp2f(s[i] * a.cscale + nl[i]) : 0.f;
        w[i] = p[i] * dp[i];
      }
      add_rows<D>(ot_, p, rt, r16, q, av);
      add_rows<D>(qt_, w, rt, r16, q, ak);
    }
  }
  if (!live) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) ak[ct] = av[ct] = zero4;
  }
  if (a.parts > 1) {
    const long long at = (((long long)bh * a.items + key0 / 64) * a.parts + part) * 128 + wave * 16 + r16;
    store_own<D>(ak, 1.0f, a.part_o + at * D, q);
    store_own<D>(av, 1.0f, a.part_o + (at + 64) * D, q);
    return;
  }
  if (key >= a.Sk) return;
  store_own<D>(ak, a.scale, reinterpret_cast<float*>(a.dk) + at_row(a.sdk, b, hk, key), q);
  store_own<D>(av, 1.0f, reinterpret_cast<float*>(a.dv) + at_row(a.sdv, b, hk, key), q);
}

hipError_t launch_cross_forward_f32(const CrossArgs& a, int D, hipStream_t st) {
  const dim3 grid = cross_grid(a.total), blk(256);
  if (D == 128) hipLaunchKernelGGL((k_cross_rows_f32<128, false>), grid, blk, 0, st, a);
  else hipLaunchKernelGGL((k_cross_rows_f32<64, false>), grid, blk, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_cross_dq_f32(const CrossArgs& a, int D, hipStream_t st) {
  const dim3 grid = cross_grid(a.total), blk(256);
  if (D == 128) hipLaunchKernelGGL((k_cross_rows_f32<128, true>), grid, blk, 0, st, a);
  else hipLaunchKernelGGL((k_cross_rows_f32<64, true>), grid, blk, 0, st, a);
  return hipGetLastError();
}
hipError_t launch_cross_dkv_f32(const CrossArgs& a, int D, hipStream_t st) {
  const dim3 grid = cross_grid(a.total), blk(256);
  if (D == 128) hipLaunchKernelGGL(k_cross_dkv_f32<128>, grid, blk, 0, st, a);
  else hipLaunchKernelGGL(k_cross_dkv_f32<64>, grid, blk, 0, st, a);
  return hipGetLastError();
}

}  // namespace isa
