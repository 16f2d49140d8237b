// dq of cross attention in bf16, and the rows' deltas for dk and dv (cross_bwd.hip has the formulas).
//
// delta = rowsum(d_out * out) wants an output that is neither rounded nor made of rounded weights.  What this kernel starts from is delta' of the
// output as stored; with dS' = P (dP - delta') the row sum e of dS' is delta - delta' (the weights of a row add up to 1), so that
//     dq = scale sum_j dS_j k_j = scale (sum_j dS'_j k_j - e sum_j P_j k_j),   delta = delta' + e.
// The second sum is one more matrix product (P k beside dS' k, on the same fragments), in place of an output in more bits that the forward pass
// would have to write and this one to read.
//
// A workgroup is 4 waves, one to a SIMD, 32 query rows to a wave; it takes several tiles of 128 rows, one after the other, through one sequence of
// key tiles: keys and values come global -> LDS two tiles ahead, in four stages, across the row tiles' borders, and (128 channels) the next row
// tile's queries are fetched to registers while the present one is multiplied.  An iteration is laid out as in cross_dkv.hip.  65 520 queries x 512
// keys, 40 heads of 128: 1.62 ms, 0.85 PFLOP/s over its four products.
#include "cross_tiles.h"

namespace isa {

template <int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void k_cross_dq(CrossArgs a) {
  constexpr int TILE = KT * D * 2, CT = D / 16, KS = D / 32;               // bytes of a tile of 64 rows
  constexpr int NST = 4, STAGE = 2 * TILE;                                 // a stage: keys, values
  constexpr int T_STEPS = 4 * KS, C_STEPS = 2 * CT, N_STEPS = T_STEPS + C_STEPS;
  constexpr int LOADS = 2 * TileLoad<D, KT, 4>::N;                         // load instructions of a wave per tile
  constexpr bool AHEAD = D == 128;                                         // (64 channels: two workgroups share a compute unit and fill each other's waits)
  constexpr float LOG2E = 1.4426950408889634f;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[NST * STAGE];
  uint32_t item;
  if (!cross_item(a, item)) return;
  const int part = (int)(item % (uint32_t)a.parts);
  item /= (uint32_t)a.parts;
  const uint32_t slot = item;                                              // (several parts: one row tile to an item)
  int tile = (int)(item % (uint32_t)a.items) * a.chunk;
  const int tile_end = min(tile + a.chunk, (a.rows + 127) / 128);
  const int bh = (int)(item / (uint32_t)a.items), b = bh % a.B, hk = bh / a.B;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  KeyBits<32> bits;
  bits.init(a.mask ? a.mask + (long long)b * a.mask_stride : nullptr, key_count(a, b), lane);
  const int n_keys = min(bits.n_keys, 32 * bits.used((bits.n_keys + 31) / 32)), n_tiles = (n_keys + KT - 1) / KT;
  const int t_begin = (int)((long long)n_tiles * part / a.parts), n_real = (int)((long long)n_tiles * (part + 1) / a.parts) - t_begin;
  const int n = max(n_real, 1);                                            // (no key at all: one tile without a valid one)

  // ---- the streamed tiles, row tile after row tile; behind the last they go on, so that the number of loads in flight stays the same
  bits.init(bits.mask_row, min(n_keys, (t_begin + n_real) * KT), lane);
  const uint16_t* const k_head = reinterpret_cast<const uint16_t*>(a.k) + at_row(a.sk, b, hk, 0) + (long long)t_begin * KT * a.sk.t;
  const uint16_t* const v_head = reinterpret_cast<const uint16_t*>(a.v) + at_row(a.sv, b, hk, 0) + (long long)t_begin * KT * a.sv.t;
  const uint32_t lds0 = lds_addr_of(lds);
  TileLoad<D, KT, 4> lk, lv;
  lk.init(wave, lane, (uint32_t)a.sk.t * 2u);
  lv.init(wave, lane, (uint32_t)a.sv.t * 2u);
  int f_pos = 0, f_stage = 0;                                              // the next tile to be fetched, its stage
  unsigned long long w_now = 0, w_1 = 0, w_2 = 0;                          // valid keys of tiles i, i + 1, i + 2
  const char *k_tile = nullptr, *v_tile = nullptr;
  uint32_t dst = 0;
  auto fetch = [&](int f) __attribute__((always_inline)) {                 // in slices: 0 works the addresses out, 1 and 2 issue the loads
    if (f == 0) {
      const uint32_t lo = bits.of(2 * (t_begin + f_pos)), hi = bits.of(2 * (t_begin + f_pos) + 1);
      w_2 = ((unsigned long long)hi << 32) | lo;
      k_tile = uniform_ptr(k_head + (long long)f_pos * KT * a.sk.t);
      v_tile = uniform_ptr(v_head + (long long)f_pos * KT * a.sv.t);
      dst = lds0 + (uint32_t)f_stage * (uint32_t)STAGE;
      f_stage = (f_stage + 1) & (NST - 1);
      f_pos = f_pos + 1 == n ? 0 : f_pos + 1;
    } else if (f == 1) {
      lk.issue(k_tile, dst, wave, lane, w_2);
    } else if (f == 2) {
      lv.issue(v_tile, dst + TILE, wave, lane, w_2);
    }
  };

  // ---- the stationary rows: those at hand and, on their way, the next row tile's
  bf16x8 qf[2][KS], of[2][KS], qn[2][KS], on[2][KS], un[2][KS];
  float lse_n[2], nlse[2], nd[2], e[2];                                    // nd: minus delta'
  auto load_rows = [&](int of_tile) __attribute__((always_inline)) {
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const RowOf row(a, hk, of_tile * 128, wave * 32 + 16 * qt + r16);
      const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + at_row(a.sq, b, row.head, row.query) + 8 * q;
      const uint16_t* dp = reinterpret_cast<const uint16_t*>(a.d_out) + at_row(a.sdo, b, row.head, row.query) + 8 * q;
      const uint16_t* op = reinterpret_cast<const uint16_t*>(a.fwd_out) + at_row(a.so, b, row.head, row.query) + 8 * q;
      lse_n[qt] = a.fwd_lse[((long long)b * a.H + row.head) * a.Sq + row.query];
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qn[qt][ks] = *reinterpret_cast<const bf16x8*>(qp + 32 * ks);
        on[qt][ks] = *reinterpret_cast<const bf16x8*>(dp + 32 * ks);
        un[qt][ks] = *reinterpret_cast<const bf16x8*>(op + 32 * ks);
      }
    }
  };
  auto take_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      float d = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[qt][ks] = qn[qt][ks];
        of[qt][ks] = on[qt][ks];
#pragma unroll
        for (int i = 0; i < 8; i += 2)                                     // (what this sum rounds away is put right with the rest)
          d = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{on[qt][ks][i], on[qt][ks][i + 1]}, bf16x2{un[qt][ks][i], un[qt][ks][i + 1]}, d, false);
      }
      nd[qt] = -sum_over_q(d);
      nlse[qt] = lse_n[qt] == -INFINITY ? -INFINITY : -lse_n[qt] * LOG2E;
      e[qt] = 0.f;
    }
  };
  if (AHEAD) load_rows(tile);
#pragma unroll
  for (int f = 0; f < 3; ++f) fetch(f);
  w_now = w_2;
#pragma unroll
  for (int f = 0; f < 3; ++f) fetch(f);
  w_1 = w_2;

  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  const float cscale = a.cscale;
  // as, ap: sums of dS' k and of P k
  auto store = [&](int of_tile, f32x4 (&as)[CT][2], f32x4 (&ap)[CT][2]) __attribute__((always_inline)) {
    settle(as[0][0]);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) { settled(as[ct][qt]); settled(ap[ct][qt]); }
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const bool none = nlse[qt] == -INFINITY;                             // no valid key: zeros (0 times an infinite gradient is no zero)
      const float es = none ? 0.f : sum_over_q(e[qt]), ndq = none ? 0.f : nd[qt];
      const RowOf row(a, hk, of_tile * 128, wave * 32 + 16 * qt + r16);
      const bool whole = a.parts == 1;
      if (part == 0 && q == 0 && row.ok) {
        float* s = a.side + (((long long)b * a.H + row.head) * a.side_tiles + (row.query >> 6)) * 128 + (row.query & 63);
        s[0] = nlse[qt];
        s[64] = whole ? ndq - es : ndq;
        if (row.query == a.Sq - 1)                                         // the places behind the last query: weight 0
          for (int i = 1; i < 64 - (row.query & 63); ++i) { s[i] = -INFINITY; s[64 + i] = 0.f; }
      }
      if (!whole) {
        const long long at = ((long long)slot * a.parts + part) * 128 + wave * 32 + 16 * qt + r16;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          *reinterpret_cast<f32x4*>(a.part_o + 2 * at * D + 16 * ct + 4 * q) = none ? zero4 : as[ct][qt];
          *reinterpret_cast<f32x4*>(a.part_o + (2 * at + 1) * D + 16 * ct + 4 * q) = none ? zero4 : ap[ct][qt];
        }
        if (q == 0) a.part_ml[at] = make_float4(es, 0.f, 0.f, 0.f);
        continue;
      }
      f32x4 r[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) r[ct] = none ? zero4 : as[ct][qt] - ap[ct][qt] * es;
      store_row<D>(r, a.scale, reinterpret_cast<uint16_t*>(a.dq) + at_row(a.sdq, b, row.head, row.query), q, row.ok);
    }
  };

  FragsAt<D> at;
  at.init(r16, q, lds0);
  constexpr int PF = 3, NB = 4;                                            // fragments are requested PF steps ahead, in NB rotating sets
  static_assert(N_STEPS % NB == 0, "the sets of a tile's first steps do not depend on the tile");
  bf16x8 fa[NB], fb[NB];                                                   // T steps: key, value rows; C steps: K^T
  auto load = [&](int m) __attribute__((always_inline)) {
    if (m < T_STEPS) {
      const uint32_t add = (uint32_t)(m / KS) * 32u * D;
      fa[m % NB] = read_rows(at.row[m % KS], add);
      fb[m % NB] = read_rows(at.row[m % KS], add + TILE);
    } else {
      fa[m % NB] = read_tr<D>(at.tr[(m - T_STEPS) % CT], (uint32_t)((m - T_STEPS) / CT) * 64u * D);
    }
  };

  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
  __syncthreads();
#pragma unroll
  for (int m = 0; m < PF; ++m) load(m);
  int stage = 0;
  for (;;) {
  if (!AHEAD) load_rows(tile);
  take_rows();
  if (AHEAD && tile + 1 < tile_end) load_rows(tile + 1);                   // the next row tile's rows are on their way
  f32x4 as[CT][2], ap[CT][2];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) as[ct][qt] = ap[ct][qt] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int pos = 0; pos < n; ++pos) {
    const uint32_t step = stage == NST - 1 ? (uint32_t)(-(NST - 1) * STAGE) : (uint32_t)STAGE;      // to the next tile's stage
    stage = (stage + 1) & (NST - 1);
    f32x4 t1[2][2], t2[2][2];                                              // [sub-tile % 2][query tile]
    uint32_t wp[2][2][4], ws[2][2][4];                                     // [half][query tile]: P and dS' in pairs
    auto weight2 = [&](int s, int j) __attribute__((always_inline)) {      // weights 2 j, 2 j + 1 of sub-tile s: query tile j / 2
      const int hh = s >> 1, rt = s & 1, qt = j >> 1, i0 = 2 * (j & 1);
      const float p0 = __builtin_amdgcn_exp2f(fmaf(t1[rt][qt][i0], cscale, nlse[qt]));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(t1[rt][qt][i0 + 1], cscale, nlse[qt]));
      const float s0 = p0 * t2[rt][qt][i0], s1 = p1 * t2[rt][qt][i0 + 1];
      e[qt] += s0 + s1;
      pin(e[qt]);
      wp[hh][qt][2 * rt + (j & 1)] = pin_pair(p0, p1);
      ws[hh][qt][2 * rt + (j & 1)] = pin_pair(s0, s1);
    };
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int rt = s & 1;
      f32x4 bias = zero4;                                                  // minus infinity for keys that are not valid (their rows are zeros in LDS)
      if (__builtin_expect(w_now != ~0ull, 0)) {
        asm volatile("");
        const uint32_t w = (uint32_t)(w_now >> (16 * s)) >> (4 * q);
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = (w >> i) & 1u ? 0.f : -INFINITY;
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int m = KS * s + ks, cb = m % NB;
        ISA_CROSS_FENCE();
        load(m + PF);
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) t1[rt][qt] = mfma16(fa[cb], qf[qt][ks], ks == 0 ? bias : t1[rt][qt]);
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) t2[rt][qt] = mfma16(fb[cb], of[qt][ks], ks == 0 ? f32x4{nd[qt], nd[qt], nd[qt], nd[qt]} : t2[rt][qt]);
#pragma unroll
        for (int j = ks * 4 / KS; j < (ks + 1) * 4 / KS; ++j) {
          if (s > 0) weight2(s - 1, j);
          else fetch(j);
        }
      }
    }
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      if (hh == 1) {
        // All but the newest loads (tile i + 2's) have landed: tile i + 1 is complete, for everybody behind the barrier, and everybody is through
        // tile i - 1.  In a row tile's first iteration this waits for the next row tile's rows too, which went before tile i + 2: their number
        // is the compiler's to choose, and a wait that allowed for it would be sound only as long as it keeps to it.
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) at.row[ks] += step;
      }
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const int m = T_STEPS + CT * hh + ct, cb = m % NB;
        ISA_CROSS_FENCE();
        load((m + PF) % N_STEPS);
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) mfma16_acc(fa[cb], __builtin_bit_cast(bf16x8, make_uint4(ws[hh][qt][0], ws[hh][qt][1], ws[hh][qt][2], ws[hh][qt][3])), as[ct][qt]);
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) mfma16_acc(fa[cb], __builtin_bit_cast(bf16x8, make_uint4(wp[hh][qt][0], wp[hh][qt][1], wp[hh][qt][2], wp[hh][qt][3])), ap[ct][qt]);
        if (hh == 0 && ct % (CT / 4) == 0) weight2(3, ct / (CT / 4));
      }
    }
    ISA_CROSS_FENCE();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) at.tr[ct] += step;
    w_now = w_1;
    w_1 = w_2;
  }
  store(tile, as, ap);
  if (++tile == tile_end) break;
  }
  // the loads past the end still target this workgroup's LDS: let them land before the waves end
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

hipError_t launch_cross_dq(const CrossArgs& a, int D, hipStream_t st) {
  const dim3 grid = cross_grid(a.total), blk(256);
  if (D == 128) hipLaunchKernelGGL(k_cross_dq<128>, grid, blk, 0, st, a);
  else hipLaunchKernelGGL(k_cross_dq<64>, grid, blk, 0, st, a);
  return hipGetLastError();
}

}  // namespace isa
