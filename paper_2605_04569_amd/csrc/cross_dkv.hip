// dk and dv of cross attention in bf16 (cross_bwd.hip has the formulas): the scores and dP of 128 keys against the streamed queries
// are formed once and feed both accumulations, four matrix products per query-key pair.
//
// A workgroup is 128 keys and 4 waves, one to a SIMD: a wave keeps 32 rows of keys and values and both accumulators beside a tile's state, for which
// it needs the registers of a SIMD by itself (64 channels: two workgroups share a compute unit).  Tiles of 64 rows of Q and dO come global ->
// LDS two tiles ahead, in four stages.  What an iteration does in the shadow of its matrix instructions is laid out as in attn_bwd_kv.hip: the
// weights of a sub-tile of 16 rows are issued between the products of the next one, the set-up of a tile between those of the first sub-tile, the
// first fragments of the next tile between the last accumulations.  65 520 queries x 512 keys, 40 heads of 128: 1.33 ms, 1.04 PFLOP/s; the fragment
// reads of a wave's 32 keys take as many cycles of the LDS as its matrix instructions take of their pipe.
#include "cross_tiles.h"

namespace isa {
template <int D>
__global__ __launch_bounds__(256, D == 128 ? 1 : 2) void k_cross_dkv(CrossArgs a) {
  constexpr int TILE = KT * D * 2, CT = D / 16, KS = D / 32;               // bytes of a tile of 64 rows
  constexpr int NST = 4, STAGE = 2 * TILE + 512;                           // a stage: Q, dO, 64 minus-log-sum-exps, 64 minus-deltas
  constexpr int T_STEPS = 4 * KS, C_STEPS = 2 * CT, N_STEPS = T_STEPS + C_STEPS;
  constexpr int LD = KT * (D / 8) / 64 / 4, LOADS = 2 * LD + 1;            // load instructions of a wave per tensor, per tile
  __shared__ __attribute__((aligned(1024))) unsigned char lds[NST * STAGE];
  uint32_t item;
  if (!cross_item(a, item)) return;
  const int key0 = (int)(item % (uint32_t)a.items) * 128;
  const uint32_t slot = item / (uint32_t)a.items;                          // (batch item, key head) and part
  const int part = (int)(slot % (uint32_t)a.parts);
  const int bh = (int)(slot / (uint32_t)a.parts), b = bh % a.B, hk = bh / a.B;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int n_keys = key_count(a, b);
  const uint8_t* const mask_row = a.mask ? a.mask + (long long)b * a.mask_stride : nullptr;

  // ---- the streamed tiles: 64 queries of a head of the group, head after head; a block without a valid key streams nothing
  bool any = key0 < n_keys;
  if (any && mask_row) any = __syncthreads_or(tid < 128 && key0 + tid < n_keys && mask_row[key0 + tid] != 0) != 0;
  const int units = any ? a.group * a.side_tiles : 0;
  const int u_begin = (int)((long long)units * part / a.parts), n = (int)((long long)units * (part + 1) / a.parts) - u_begin;
  const uint32_t lds0 = lds_addr_of(lds);
  const uint32_t sq_b = (uint32_t)a.sq.t * 2u, so_b = (uint32_t)a.sdo.t * 2u;
  int row_l[LD];
  uint32_t chunk_b[LD];
#pragma unroll
  for (int i = 0; i < LD; ++i) {
    row_l[i] = (wave * LD + i) * (512 / D) + lane / (D / 8);
    chunk_b[i] = (uint32_t)(chunk_at<D>(lane % (D / 8), row_l[i]) * 16);
  }
  int u_next = u_begin, in_stage = 0;                                      // the next tile to be fetched and its stage
  int h_next = 0, t_next = 0;
  if (n > 0) { h_next = u_begin / a.side_tiles; t_next = u_begin % a.side_tiles; }
  const char *q_tile = nullptr, *o_tile = nullptr, *side_tile = nullptr;
  uint32_t dst = 0, q_off[LD], o_off[LD];
  // The loads of a tile in four slices: 0 works its addresses out, 1 to 3 issue the loads.  A sequence that has ended loads its last tile
  // again: the number of loads in flight stays the same.
  auto fetch = [&](int f) __attribute__((always_inline)) {
    if (f == 0) {
      const int head = hk * a.group + h_next, t0 = t_next * KT, nk = min(KT, a.Sq - t0);
      q_tile = uniform_ptr(reinterpret_cast<const uint16_t*>(a.q) + at_row(a.sq, b, head, t0));
      o_tile = uniform_ptr(reinterpret_cast<const uint16_t*>(a.d_out) + at_row(a.sdo, b, head, t0));
      side_tile = uniform_ptr(a.side + (((long long)b * a.H + head) * a.side_tiles + t_next) * 128);
      dst = lds0 + (uint32_t)in_stage * (uint32_t)STAGE;
      in_stage = (in_stage + 1) & (NST - 1);
#pragma unroll
      for (int i = 0; i < LD; ++i) {                                       // rows past the end repeat the last one (their weights are 0)
        const uint32_t row = (uint32_t)min(row_l[i], nk - 1);
        q_off[i] = row * sq_b + chunk_b[i];
        o_off[i] = row * so_b + chunk_b[i];
      }
      if (u_next + 1 < u_begin + n) {
        ++u_next;
        if (++t_next == a.side_tiles) { t_next = 0; ++h_next; }
      }
    } else if (f < 3) {
      constexpr int PER = (LD + 1) / 2;
#pragma unroll
      for (int i = (f - 1) * PER; i < (f == 1 ? PER : LD); ++i) {
        dma16(q_tile, q_off[i], dst + (uint32_t)(wave * LD + i) * 1024u);
        dma16(o_tile, o_off[i], dst + (uint32_t)TILE + (uint32_t)(wave * LD + i) * 1024u);
      }
    } else {
      // 512 B, lanes 32..63 repeat lanes 0..31; every wave loads them, so that all waves have the same number of loads in flight.  (The upper
      // half of what they write is the start of the next stage's Q or, in the last stage, nothing: it is kept out.)
      if (lane < 32) dma16(side_tile, (uint32_t)lane * 16u, dst + 2u * TILE);
    }
  };
  if (n > 0) {
#pragma unroll
    for (int f = 0; f < 4; ++f) fetch(f);
#pragma unroll
    for (int f = 0; f < 4; ++f) fetch(f);
  }

  // ---- the stationary rows: 32 keys and values; those that are not valid enter as zeros, with scores of minus infinity
  bf16x8 kf[2][KS], vf[2][KS];
  f32x4 kbias[2];
  int key[2];
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    key[kt] = key0 + wave * 32 + 16 * kt + r16;
    const bool live = key[kt] < n_keys && (!mask_row || mask_row[key[kt]] != 0);
    const float kb = live ? 0.f : -INFINITY;
    kbias[kt] = f32x4{kb, kb, kb, kb};
    const uint16_t* kp = reinterpret_cast<const uint16_t*>(a.k) + at_row(a.sk, b, hk, live ? key[kt] : 0) + 8 * q;
    const uint16_t* vp = reinterpret_cast<const uint16_t*>(a.v) + at_row(a.sv, b, hk, live ? key[kt] : 0) + 8 * q;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      kf[kt][ks] = vf[kt][ks] = __builtin_bit_cast(bf16x8, make_uint4(0u, 0u, 0u, 0u));
      if (live) {
        kf[kt][ks] = *reinterpret_cast<const bf16x8*>(kp + 32 * ks);
        vf[kt][ks] = *reinterpret_cast<const bf16x8*>(vp + 32 * ks);
      }
    }
  }
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(kf[kt][ks]), "+v"(vf[kt][ks]));

  f32x4 ak[CT][2], av[CT][2];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) ak[ct][kt] = av[ct][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float cscale = a.cscale;

  // Fragment places of the tile at hand; the rows' and the side array's move on to the next tile before the last accumulations of the present one
  FragsAt<D> at;
  at.init(r16, q, lds0);
  uint32_t side_at = lds0 + 2u * TILE + 16u * (uint32_t)q;
  constexpr int PF = 3, NB = 4;                                            // fragments are requested PF steps ahead, in NB rotating sets
  static_assert(N_STEPS % NB == 0, "the sets of a tile's first steps do not depend on the tile");
  bf16x8 fa[NB], fb[NB];                                                   // T steps: Q, dO rows; C steps: Q^T, dO^T
  f32x4 nd[2], nl[2];                                                      // minus-deltas / minus-log-sum-exps of the rows of a sub-tile
  // steps 0 .. T_STEPS - 1: T (sub-tile m / KS, k-slice m % KS); the others: C (half, channel tile)
  auto load = [&](int m) __attribute__((always_inline)) {
    if (m < T_STEPS) {
      const uint32_t add = (uint32_t)(m / KS) * 32u * D;
      fa[m % NB] = read_rows(at.row[m % KS], add);
      fb[m % NB] = read_rows(at.row[m % KS], add + TILE);
    } else {
      const uint32_t add = (uint32_t)((m - T_STEPS) / CT) * 64u * D;
      fa[m % NB] = read_tr<D>(at.tr[(m - T_STEPS) % CT], add);
      fb[m % NB] = read_tr<D>(at.tr[(m - T_STEPS) % CT], add + TILE);
    }
  };
  auto side4 = [&](uint32_t add) __attribute__((always_inline)) -> f32x4 {
    return *(__attribute__((address_space(3))) const f32x4*)((__attribute__((address_space(3))) const char*)(uintptr_t)side_at + add);
  };

  if (n > 0) {
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");          // (the stationary rows' loads came after: they are here too)
    __syncthreads();
#pragma unroll
    for (int m = 0; m < PF; ++m) load(m);
    nd[0] = side4(256);
    for (int i = 0, stage = 0; i < n; ++i) {
      // To the next tile's stage
      const uint32_t step = stage == NST - 1 ? (uint32_t)(-(NST - 1) * STAGE) : (uint32_t)STAGE;
      stage = (stage + 1) & (NST - 1);
      f32x4 t1[2][2], t2[2][2];                                            // [sub-tile % 2][key tile]
      uint32_t wp[2][2][4], ws[2][2][4];                                   // [half][key tile]: P and dS in pairs; element 4 rt + i = row 32 half + 16 rt + 4 q + i
      // weights 2 j, 2 j + 1 of sub-tile s: key tile j / 2
      auto weight2 = [&](int s, int j) __attribute__((always_inline)) {
        const int hh = s >> 1, rt = s & 1, kt = j >> 1, i0 = 2 * (j & 1);
        const float p0 = __builtin_amdgcn_exp2f(fmaf(t1[rt][kt][i0], cscale, nl[rt][i0]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(t1[rt][kt][i0 + 1], cscale, nl[rt][i0 + 1]));
        wp[hh][kt][2 * rt + (j & 1)] = pin_pair(p0, p1);
        ws[hh][kt][2 * rt + (j & 1)] = pin_pair(p0 * t2[rt][kt][i0], p1 * t2[rt][kt][i0 + 1]);
      };
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int rt = s & 1;
        if (s > 0) nl[rt ^ 1] = side4(64 * (s - 1));
        if (s < 3) nd[rt ^ 1] = side4(256 + 64 * (s + 1));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int m = KS * s + ks, cb = m % NB;
          ISA_CROSS_FENCE();
          load(m + PF);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) t1[rt][kt] = mfma16(fa[cb], kf[kt][ks], ks == 0 ? kbias[kt] : t1[rt][kt]);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) t2[rt][kt] = mfma16(fb[cb], vf[kt][ks], ks == 0 ? nd[rt] : t2[rt][kt]);
#pragma unroll
          for (int j = ks * 4 / KS; j < (ks + 1) * 4 / KS; ++j) {
            if (s > 0) weight2(s - 1, j);
            else fetch(j);
          }
        }
      }
      nl[1] = side4(64 * 3);
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        if (hh == 1) {
          // all but the newest tile's loads have landed: the next tile is complete, for everybody behind the barrier, and everybody is through
          // the tile before the present one
          asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
          __builtin_amdgcn_s_barrier();                                    // the fragments in flight are of this tile, whose stage nobody fills yet
          asm volatile("" ::: "memory");
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) at.row[ks] += step;
          side_at += step;
        }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const int m = T_STEPS + CT * hh + ct, cb = m % NB;
          ISA_CROSS_FENCE();
          load((m + PF) % N_STEPS);
          if (m == N_STEPS - 1) nd[0] = side4(256);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) mfma16_acc(fa[cb], __builtin_bit_cast(bf16x8, make_uint4(ws[hh][kt][0], ws[hh][kt][1], ws[hh][kt][2], ws[hh][kt][3])), ak[ct][kt]);
#pragma unroll
          for (int kt = 0; kt < 2; ++kt) mfma16_acc(fb[cb], __builtin_bit_cast(bf16x8, make_uint4(wp[hh][kt][0], wp[hh][kt][1], wp[hh][kt][2], wp[hh][kt][3])), av[ct][kt]);
          if (hh == 0 && ct % (CT / 4) == 0) weight2(3, ct / (CT / 4));
        }
      }
      ISA_CROSS_FENCE();
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) at.tr[ct] += step;
    }
    // the loads past the end still target this workgroup's LDS: let them land before the waves end
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  }
  settle(ak[0][0]);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) { settled(ak[ct][kt]); settled(av[ct][kt]); }
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) {
    f32x4 rk[CT], rv[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {                                      // (0 times an infinite gradient is no zero)
      rk[ct] = kbias[kt][0] == 0.f ? ak[ct][kt] : f32x4{0.f, 0.f, 0.f, 0.f};
      rv[ct] = kbias[kt][0] == 0.f ? av[ct][kt] : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (a.parts > 1) {
      const long long row = ((long long)bh * a.items + key0 / 128) * a.parts + part;
      float* to = a.part_o + (row * 256 + wave * 32 + 16 * kt + r16) * D;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        *reinterpret_cast<f32x4*>(to + 16 * ct + 4 * q) = rk[ct];
        *reinterpret_cast<f32x4*>(to + 128 * D + 16 * ct + 4 * q) = rv[ct];
      }
      continue;
    }
    const bool in = key[kt] < a.Sk;
    store_row<D>(rk, a.scale, reinterpret_cast<uint16_t*>(a.dk) + at_row(a.sdk, b, hk, in ? key[kt] : 0), q, in);
    store_row<D>(rv, 1.0f, reinterpret_cast<uint16_t*>(a.dv) + at_row(a.sdv, b, hk, in ? key[kt] : 0), q, in);
  }
}

hipError_t launch_cross_dkv(const CrossArgs& a, int D, hipStream_t st) {
  const dim3 grid = cross_grid(a.total), blk(256);
  if (D == 128) hipLaunchKernelGGL(k_cross_dkv<128>, grid, blk, 0, st, a);
  else hipLaunchKernelGGL(k_cross_dkv<64>, grid, blk, 0, st, a);
  return hipGetLastError();
}

}  // namespace isa
