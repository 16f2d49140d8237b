// Backward pass of cross attention, gfx950: its host side and the sums over parts.  With P the softmax weights, delta = rowsum(d_out * out),
// dP = d_out v^T:
//     dS = P (dP - delta),   dq = scale dS k,   dk = scale dS^T q,   dv = P^T d_out.
// Two launches: dq, with the rows' deltas (cross_dq.hip), then dk and dv (cross_dkv.hip), eight matrix products where five are needed: no
// atomics, and no sums in memory but those of the parts.  A workgroup of the first owns query rows and streams the keys, one of the second owns 128
// keys and streams the queries; as there are few keys and many queries the queries are cut into parts, whose sums k_cross_sum adds in a fixed order.
// In fp32 (cross_f32.hip) the same with seven products: the output is not rounded there.
#include "cross_tiles.h"

namespace isa {
// Adds the parts' sums in their order.  KV: dk and dv of every key (tiles of `tile_rows` keys: dk's, then dv's); otherwise dq.
template <typename T, int D, bool KV>
__global__ __launch_bounds__(256) void k_cross_sum(CrossArgs a, int tile_rows) {
  constexpr int TPR = D / 4;
  const long long idx = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int c = (threadIdx.x % TPR) * 4;
  const int rows = KV ? 2 * a.Sk : a.rows;
  const int bh = (int)(idx / rows);
  if (bh >= a.B * a.Hkv) return;
  const int at_rows = (int)(idx % rows), which = KV ? at_rows / a.Sk : 0, row = KV ? at_rows % a.Sk : at_rows;
  const int b = bh % a.B, hk = bh / a.B;
  const int per = KV ? 2 * tile_rows : tile_rows;        // rows of a part
  const long long base = ((long long)bh * a.items + row / tile_rows) * a.parts * per + which * tile_rows + row % tile_rows;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < a.parts; ++p) o += *reinterpret_cast<const f32x4*>(a.part_o + (base + (long long)p * per) * D + c);
  if (which == 0) o *= a.scale;
  T* to;
  if (KV) to = which ? reinterpret_cast<T*>(a.dv) + at_row(a.sdv, b, hk, row) : reinterpret_cast<T*>(a.dk) + at_row(a.sdk, b, hk, row);
  else to = reinterpret_cast<T*>(a.dq) + at_row(a.sdq, b, hk * a.group + row / a.Sq, row % a.Sq);
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to + c) = bf16x4_of(o);
  else *reinterpret_cast<f32x4*>(to + c) = o;
}

// dq of the parts of cross_dq.hip, and the deltas of the rows
template <int D>
__global__ __launch_bounds__(256) void k_cross_sum_dq(CrossArgs a) {
  constexpr int TPR = D / 4;
  const long long idx = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int c = (threadIdx.x % TPR) * 4;
  const int bh = (int)(idx / a.rows), row = (int)(idx % a.rows);
  if (bh >= a.B * a.Hkv) return;
  const int b = bh % a.B, hk = bh / a.B;
  const long long base = ((long long)bh * a.items + row / 128) * a.parts * 128 + row % 128;
  f32x4 s = {0.f, 0.f, 0.f, 0.f}, p = s;
  float e = 0.f;
  for (int i = 0; i < a.parts; ++i) {
    const long long at = base + (long long)i * 128;
    s += *reinterpret_cast<const f32x4*>(a.part_o + 2 * at * D + c);
    p += *reinterpret_cast<const f32x4*>(a.part_o + (2 * at + 1) * D + c);
    e += a.part_ml[at].x;
  }
  const int head = hk * a.group + row / a.Sq, query = row % a.Sq;
  if (c == 0) a.side[(((long long)b * a.H + head) * a.side_tiles + (query >> 6)) * 128 + 64 + (query & 63)] -= e;
  *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.dq) + at_row(a.sdq, b, head, query) + c) = bf16x4_of((s - p * e) * a.scale);
}

// Parts of `units` pieces of work for each of `wgs` workgroups on `resident` places: as many as make the rounds over the places
// shortest, each part taking `fixed` pieces' time beside its share (its start, its result and the sum over them).  With many rounds there is
// nothing to gain, and the room for partial results stays bounded.
static int parts_for(long long wgs, int units, long long resident, int fixed) {
  if (wgs < 1 || units < 2) return 1;
  int best = 1;
  long long best_cost = -1;
  for (int p = 1; p <= 64 && p <= units && (p == 1 || wgs * p <= 2048); ++p) {
    const long long cost = (wgs * p + resident - 1) / resident * ((units + p - 1) / p + (p > 1 ? fixed : 0));
    if (best_cost < 0 || cost < best_cost) {
      best = p;
      best_cost = cost;
    }
  }
  return best;
}

// Row tiles of a workgroup of cross_dq.hip with 128 channels, at most 32: the fewest within 5 % of the shortest rounds over the `resident` places, as what
// a workgroup begins and ends with takes half of a row tile (512 keys) where it has a compute unit for itself.  With 64 channels, where two fill each
// other's waits, that is next to nothing, and one row tile is never more than 5 % behind.
static int chunk_for(long long bh, int tiles, long long resident) {
  auto cost = [&](int c) { return (double)((bh * ((tiles + c - 1) / c) + resident - 1) / resident) * (c + 0.5); };
  const int most = tiles < 32 ? tiles : 32;
  double best = cost(1);
  for (int c = 2; c <= most; ++c) best = cost(c) < best ? cost(c) : best;
  int c = 1;
  while (c < most && cost(c) > 1.05 * best) ++c;
  return c;
}

CrossBackwardPlan cross_backward_plan(const isa_cross_problem& p) {
  CrossBackwardPlan c = {};
  const bool f32 = p.dtype == ISA_F32;
  const int group = p.H / p.H_kv;
  const long long rows = (long long)group * p.S_q, bh = (long long)p.B * p.H_kv, chip = (long long)N_XCD * cus_per_xcd();
  c.dq_rows = f32 ? 64 : 128;
  c.kv_rows = f32 ? 64 : 128;
  c.side_tiles = (p.S_q + 63) / 64;
  c.dq_items = (int)((rows + c.dq_rows - 1) / c.dq_rows);
  c.kv_items = (p.S_k + c.kv_rows - 1) / c.kv_rows;
  c.dq_parts = parts_for(bh * c.dq_items, (p.S_k + 63) / 64, (f32 || p.D == 64 ? 2 : 1) * chip, 4);
  c.kv_parts = parts_for(bh * c.kv_items, group * c.side_tiles, (f32 || p.D == 64 ? 2 : 1) * chip, 4);
  c.side_bytes = align256((size_t)p.B * p.H * c.side_tiles * 128 * 4);
  const size_t dq_rows = c.dq_parts > 1 ? (size_t)bh * c.dq_items * c.dq_parts * c.dq_rows : 0, dq = dq_rows * p.D * (f32 ? 4 : 8);
  const size_t kv = c.kv_parts > 1 ? (size_t)bh * c.kv_items * c.kv_parts * 2 * c.kv_rows * p.D * 4 : 0;
  c.part_bytes = align256(dq > kv ? dq : kv);
  c.ml_bytes = f32 ? 0 : align256(dq_rows * sizeof(float4));
  return c;
}

template <typename T, bool KV> static hipError_t sum_parts(const CrossArgs& a, int D, int tile_rows, hipStream_t st) {
  const long long rows = (long long)a.B * a.Hkv * (KV ? 2ll * a.Sk : a.rows);
  const int per = 256 / (D / 4);
  const dim3 grid((unsigned)((rows + per - 1) / per)), blk(256);
  if (D == 128) hipLaunchKernelGGL((k_cross_sum<T, 128, KV>), grid, blk, 0, st, a, tile_rows);
  else hipLaunchKernelGGL((k_cross_sum<T, 64, KV>), grid, blk, 0, st, a, tile_rows);
  return hipGetLastError();
}

hipError_t launch_cross_backward(CrossArgs a, const isa_cross_problem& p, hipStream_t st) {
  const CrossBackwardPlan c = cross_backward_plan(p);
  const bool f32 = p.dtype == ISA_F32;
  const long long bh = (long long)p.B * p.H_kv;
  hipError_t e = hipSuccess;
  a.side_tiles = c.side_tiles;
  if (p.S_q > 0) {
    a.items = c.dq_items;
    a.parts = c.dq_parts;
    a.chunk = 1;
    if (!f32 && p.D == 128 && c.dq_parts == 1) {
      a.chunk = chunk_for(bh, c.dq_items, (long long)N_XCD * cus_per_xcd());
      a.items = (c.dq_items + a.chunk - 1) / a.chunk;
    }
    a.total = bh * a.items * c.dq_parts;
    e = f32 ? launch_cross_dq_f32(a, p.D, st) : launch_cross_dq(a, p.D, st);
    if (e == hipSuccess && c.dq_parts > 1) {
      if (f32) {
        e = sum_parts<float, false>(a, p.D, c.dq_rows, st);
      } else {
        const int per = 256 / (p.D / 4);
        const dim3 grid((unsigned)((bh * a.rows + per - 1) / per)), blk(256);
        if (p.D == 128) hipLaunchKernelGGL(k_cross_sum_dq<128>, grid, blk, 0, st, a);
        else hipLaunchKernelGGL(k_cross_sum_dq<64>, grid, blk, 0, st, a);
        e = hipGetLastError();
      }
    }
    if (e != hipSuccess) return e;
  }
  if (p.S_k > 0 && a.dk) {
    a.items = c.kv_items;
    a.parts = c.kv_parts;
    a.total = bh * c.kv_items * c.kv_parts;
    if (f32) e = launch_cross_dkv_f32(a, p.D, st);
    else e = launch_cross_dkv(a, p.D, st);
    if (e == hipSuccess && c.kv_parts > 1) e = f32 ? sum_parts<float, true>(a, p.D, c.kv_rows, st) : sum_parts<uint16_t, true>(a, p.D, c.kv_rows, st);
  }
  return e;
}

}  // namespace isa
