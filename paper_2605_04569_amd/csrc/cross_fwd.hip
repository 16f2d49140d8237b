// Cross attention in bf16: out = softmax(scale q k^T) v over the valid keys, gfx950.
//
// k_cross: a workgroup of 4 waves owns 128 query rows (the heads that share a key head are one sequence of rows) and streams tiles
// of 32 keys and values through LDS, four stages, two tiles behind a barrier while the loads of the next two are in flight; two workgroups share a
// compute unit and fill each other's waits.  The scores are computed transposed, so that the weights go from the accumulators to the
// second product without leaving their lanes; the values are read transposed out of their row-major tile.  The running maximum is
// raised only when a tile exceeds it by 2^RESCALE_TAU.  Measured (40 heads of 128 channels, 65 520 queries): 212 us and 1.09 us a key, that is
// 1.26 PFLOP/s in the loop and 0.8 with 512 keys, where the rows' bytes cost time beside the products: the chip is at its power limit (2.37 GHz with 16
// keys, 1.5 to 1.9 GHz with 512 or 8192).  One step of 64 keys behind a barrier, with its weights after its scores: 880 us for 512 keys instead of 805; row
// tiles that begin in the shadow of the one before, or 256 rows to a workgroup: within 3 % of this form either way.
//
// k_cross_narrow: 16 rows or fewer (single tokens): bound by reading the keys and values once.  The 4 waves take tiles of 32 keys in
// turn, each with its own stages in LDS and no barrier, and join their results at the end.  8 rows over 4096 to 16 384 states of 8 heads
// (421 MB): 77 us, 5.5 TB/s, and 5 us for the join.
//
// Where the items do not fill the chip each runs as several workgroups over a share of the keys, and k_cross_merge joins their sums.
#include <type_traits>

#include "cross_tiles.h"

namespace isa {
namespace {

// Scores of 32 keys: two sub-tiles of 16, lane: keys 16 kt + 4 q + i.  Bits of `valid` that are not set: minus infinity.
__device__ __forceinline__ void mask_scores(f32x4 (&s)[2], uint32_t valid, int q) {
  const uint32_t w = valid >> (4 * q);
#pragma unroll
  for (int kt = 0; kt < 2; ++kt)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!((w >> (16 * kt + i)) & 1u)) s[kt][i] = -INFINITY;
}

struct RowState {
  float neg_m, thr;                 // minus the running maximum (log2 domain); the score from which it is raised
  f32x4 l;                          // the lane's share of the sum of the rounded weights (all elements alike)
  float lu;                         // of the weights before they are rounded
};
__device__ __forceinline__ RowState row_state() { return RowState{-LOWEST, LOWEST, f32x4{0.f, 0.f, 0.f, 0.f}, 0.f}; }

__device__ __forceinline__ float top_of(const f32x4 (&s)[2]) {
  float m = -INFINITY;
#pragma unroll
  for (int kt = 0; kt < 2; ++kt) m = fmaxf(fmaxf(fmaxf(fmaxf(m, s[kt][0]), s[kt][1]), s[kt][2]), s[kt][3]);      // pairs of these are one instruction
  return m;
}
// The running maximum with a tile's, `m`, where that exceeds it enough: the factor of what has been summed
__device__ __forceinline__ float raise_row(float m, RowState& st) {
  const float m_new = m > st.thr ? m : -st.neg_m, alpha = __builtin_amdgcn_exp2f(-st.neg_m - m_new);
  st.neg_m = -m_new;
  st.thr = m_new + RESCALE_TAU;
  st.l *= alpha;
  st.lu *= alpha;
  return alpha;
}

// The weights of 32 keys: B fragment, element 4 kt + i = key 16 kt + 4 q + i
template <bool LSE> __device__ __forceinline__ bf16x8 weights(const f32x4 s0, const f32x4 s1, float cscale, RowState& st) {
  uint32_t p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 x = j < 2 ? s0 : s1;
    const float w0 = __builtin_amdgcn_exp2f(fmaf(x[2 * (j & 1)], cscale, st.neg_m)), w1 = __builtin_amdgcn_exp2f(fmaf(x[2 * (j & 1) + 1], cscale, st.neg_m));
    if (LSE) st.lu += w0 + w1;
    p[j] = pin_pair(w0, w1);
  }
  // The sum that normalises the output is that of the rounded weights, so that the rounding of a dominant one cancels.  A 4x4x4 product
  // with ones adds the four bf16 values of a lane.
  const bf16x4 ones = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int j = 0; j < 2; ++j)
    st.l = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(short4v, ones), __builtin_bit_cast(short4v, make_uint2(p[2 * j], p[2 * j + 1])), st.l, 0, 0, 0);
  return __builtin_bit_cast(bf16x8, make_uint4(p[0], p[1], p[2], p[3]));
}

// The weights of a row with a valid key add up to 2^-RESCALE_TAU at least, unless its scores are so large (2^31) that their rounding takes the weights
// out of range: NaN then, so that the row is not taken for one without a key.
__device__ __forceinline__ float inverse_of(float l, bool keys) { return l != 0.f ? 1.0f / l : keys ? __builtin_nanf("") : 0.f; }
__device__ __forceinline__ float natural_lse(float m, float lu, bool keys) {      // m: log2 domain
  return lu > 0.f ? 0.6931471805599453f * (m + __log2f(lu)) : lu == 0.f ? (keys ? __builtin_nanf("") : -INFINITY) : lu;
}

}  // namespace

template <int D, bool LSE>
__global__ __launch_bounds__(256, 2) void k_cross(CrossArgs a) {
  constexpr int NK = 32, TILE = NK * D * 2, CT = D / 16, KS = D / 32;      // TILE: bytes
  constexpr int STEPS = 2 * KS, NST = 4;                   // steps of two matrix instructions each, in both products; stages of keys and of values
  static_assert(STEPS == CT, "both products have as many steps");
  __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * NST * TILE];
  uint32_t item;
  if (!cross_item(a, item)) return;
  const int part = (int)(item % (uint32_t)a.parts);
  item /= (uint32_t)a.parts;
  const uint32_t slot = item;
  const int tile0 = (int)(item % (uint32_t)a.items) * 128;
  const int bh = (int)(item / (uint32_t)a.items), b = bh % a.B, hk = bh / a.B;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int n_keys = key_count(a, b);
  KeyBits<NK> bits;
  bits.init(a.mask ? a.mask + (long long)b * a.mask_stride : nullptr, n_keys, lane);
  const int n_tiles = bits.used((n_keys + NK - 1) / NK);
  const int t_begin = (int)((long long)n_tiles * part / a.parts), n = (int)((long long)n_tiles * (part + 1) / a.parts) - t_begin;

  // ---- tiles u = 0 .. n - 1 of 32 keys, stage u % 4.  Step u forms the scores of tile u from fragments that were read a step before, and adds the
  // values of tile u - 1.  The loop takes two steps u, u + 1 (u odd) behind one barrier: they read keys u + 1, u + 2 and values u - 1, u, which have
  // landed, while keys u + 3, u + 4 and values u + 1, u + 2 are on their way into the stages that the two steps before have read.
  const uint16_t* const k_head = reinterpret_cast<const uint16_t*>(a.k) + at_row(a.sk, b, hk, 0) + (long long)t_begin * NK * a.sk.t;
  const uint16_t* const v_head = reinterpret_cast<const uint16_t*>(a.v) + at_row(a.sv, b, hk, 0) + (long long)t_begin * NK * a.sv.t;
  TileLoad<D, NK, 4> lk, lv;
  lk.init(wave, lane, (uint32_t)a.sk.t * 2u);
  lv.init(wave, lane, (uint32_t)a.sv.t * 2u);
  const uint32_t lds0 = lds_addr_of(lds);
  auto load_k = [&](int u, uint32_t stage, uint32_t w) __attribute__((always_inline)) {
    lk.issue(uniform_ptr(k_head + (long long)u * NK * a.sk.t), lds0 + stage * (uint32_t)TILE, wave, lane, w);
  };
  auto load_v = [&](int u, uint32_t stage, uint32_t w) __attribute__((always_inline)) {
    lv.issue(uniform_ptr(v_head + (long long)u * NK * a.sv.t), lds0 + (NST + stage) * (uint32_t)TILE, wave, lane, w);
  };
  uint32_t w[5] = {0, 0, 0, 0, 0}, seen = 0;               // key bits of tiles u .. u + 4; a tile behind the last has none.  seen: of all tiles
  if (n > 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < n) {
        w[i] = bits.of(t_begin + i);
        seen |= w[i];
        load_k(i, i, w[i]);
        if (i < 2) load_v(i, i, w[i]);
      }
    }
  }
  bf16x8 qf[2][KS];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const RowOf row(a, hk, tile0, wave * 32 + 16 * qt + r16);
    const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + at_row(a.sq, b, row.head, row.query) + 8 * q;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[qt][ks] = *reinterpret_cast<const bf16x8*>(qp + 32 * ks);
  }
#pragma unroll
  for (int qt = 0; qt < 2; ++qt)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[qt][ks]));      // consumed here, not by a wait inside the loop
  FragsAt<D> at;
  at.init(r16, q, lds0);

  f32x4 acc[2][CT], s_even[2][2], s_odd[2][2];             // scores of even and odd tiles: [qt][kt]
  RowState st[2];
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    st[qt] = row_state();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[qt][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  const float cscale = a.cscale;
  const bf16x4 ones = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};

  bf16x8 kf[STEPS];                                        // keys of the next scores: step f reads sub-tile f % 2, k-slice f / 2
  auto read_k = [&](int stage, int f) __attribute__((always_inline)) { kf[f] = read_rows(at.row[f >> 1], stage * TILE + (f & 1) * 32 * D); };
  // The scores that a tile's key bits leave, its maxima, and the running maxima with them; the sums so far follow.  Most tiles have all keys
  // and raise nothing.
  auto finish = [&](f32x4 (&s)[2][2], float (&m)[2], uint32_t valid) __attribute__((always_inline)) {
    if (__builtin_expect(valid != 0xffffffffu, 0)) {
      asm volatile("");
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) {
        mask_scores(s[qt], valid, q);
        m[qt] = top_of(s[qt]) * cscale;
      }
    }
    if (__builtin_expect((__ballot(m[0] > st[0].thr) | __ballot(m[1] > st[1].thr)) == 0ull, 1)) return;
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) {
      const float alpha = raise_row(max_over_q(m[qt]), st[qt]);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) acc[qt][ct] *= alpha;
    }
  };
  // A step: scores of a tile into `sn` (fragments in kf), weights of the tile before it from `sp` and its values (stage v_stage); the next tile's
  // fragments from stage k_stage.  exp2 runs at half the vector rate: the weights are spread over the first product's steps.
  auto step = [&](f32x4 (&sp)[2][2], f32x4 (&sn)[2][2], int k_stage, int v_stage, uint32_t valid) __attribute__((always_inline)) {
    bf16x8 vf[STEPS];
    uint32_t pw[2][4];                                     // weights in pairs: [qt], elements 4 kt + i of the fragment
#pragma unroll
    for (int f = 0; f < STEPS; ++f) {
      ISA_CROSS_FENCE();
      vf[f] = read_tr<D>(at.tr[f], (NST + v_stage) * TILE);
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) sn[qt][f & 1] = mfma16(kf[f], qf[qt][f >> 1], f < 2 ? zero4 : sn[qt][f & 1]);
#pragma unroll
      for (int j = f * 8 / STEPS; j < (f + 1) * 8 / STEPS; ++j) {      // pair j: query tile j / 4, elements 2 (j % 4), + 1
        const int qt = j >> 2, kt = (j >> 1) & 1, i = 2 * (j & 1);
        const float w0 = __builtin_amdgcn_exp2f(fmaf(sp[qt][kt][i], cscale, st[qt].neg_m));
        const float w1 = __builtin_amdgcn_exp2f(fmaf(sp[qt][kt][i + 1], cscale, st[qt].neg_m));
        if (LSE) { st[qt].lu += w0 + w1; pin(st[qt].lu); }
        pw[qt][j & 3] = pin_pair(w0, w1);
      }
    }
    float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int c = 0; c < STEPS; ++c) {
      ISA_CROSS_FENCE();
      read_k(k_stage, c);
#pragma unroll
      for (int qt = 0; qt < 2; ++qt)
        acc[qt][c] = mfma16(vf[c], __builtin_bit_cast(bf16x8, make_uint4(pw[qt][0], pw[qt][1], pw[qt][2], pw[qt][3])), acc[qt][c]);
      if (c < 2) {
        // The sum that normalises the output is that of the rounded weights, so that the rounding of a dominant one cancels: a 4x4x4 product
        // with ones adds the four bf16 values of a lane.
#pragma unroll
        for (int j = 0; j < 2; ++j)
          st[c].l = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(__builtin_bit_cast(short4v, ones), __builtin_bit_cast(short4v, make_uint2(pw[c][2 * j], pw[c][2 * j + 1])),
                                                           st[c].l, 0, 0, 0);
      }
      if (c < 4) {
        const int qt = c >> 1, kt = c & 1;
        m[qt] = fmaxf(fmaxf(fmaxf(fmaxf(m[qt], sn[qt][kt][0]), sn[qt][kt][1]), sn[qt][kt][2]), sn[qt][kt][3]);
        if (kt == 1) m[qt] *= cscale;
        pin(m[qt]);
      }
    }
    ISA_CROSS_FENCE();
    finish(sn, m, valid);
  };
  // Steps u and u + 1 (which may be behind the last tile: all masked), u % 4 == PAR
  auto two_steps = [&](int u, auto par) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par)::value;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // loads issued two steps ago
    __syncthreads();
    if (u + 3 < n) { w[3] = bits.of(t_begin + u + 3); load_k(u + 3, (PAR + 3) % NST, w[3]); }
    if (u + 4 < n) { w[4] = bits.of(t_begin + u + 4); load_k(u + 4, PAR, w[4]); }
    seen |= w[3] | w[4];
    if (u + 1 < n) load_v(u + 1, (PAR + 1) % NST, w[1]);
    if (u + 2 < n) load_v(u + 2, (PAR + 2) % NST, w[2]);
    step(s_even, s_odd, (PAR + 1) % NST, (PAR + 3) % NST, w[0]);
    step(s_odd, s_even, (PAR + 2) % NST, PAR, w[1]);
    w[0] = w[2];
    w[1] = w[3];
    w[2] = w[4];
    w[3] = w[4] = 0;
  };

  if (n > 0) {
    // the first tile's scores
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int f = 0; f < STEPS; ++f) read_k(0, f);
#pragma unroll
    for (int f = 0; f < STEPS; ++f)
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) s_even[qt][f & 1] = mfma16(kf[f], qf[qt][f >> 1], f < 2 ? zero4 : s_even[qt][f & 1]);
#pragma unroll
    for (int f = 0; f < STEPS; ++f) read_k(1, f);
    float m[2];
#pragma unroll
    for (int qt = 0; qt < 2; ++qt) m[qt] = top_of(s_even[qt]) * cscale;
    finish(s_even, m, w[0]);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = w[i + 1];
    w[4] = 0;
    for (int u = 1;;) {
      if (u >= n) break;
      two_steps(u, std::integral_constant<int, 1>());
      u += 2;
      if (u >= n) break;
      two_steps(u, std::integral_constant<int, 3>());
      u += 2;
    }
    if (n & 1) {                                           // the last tile's values (otherwise the step behind it has added them)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const uint32_t add = (uint32_t)(NST + ((n - 1) & 3)) * (uint32_t)TILE;
      bf16x8 p[2];
#pragma unroll
      for (int qt = 0; qt < 2; ++qt) p[qt] = weights<LSE>(s_even[qt][0], s_even[qt][1], cscale, st[qt]);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        const bf16x8 vf = read_tr<D>(at.tr[ct] + add, 0);
#pragma unroll
        for (int qt = 0; qt < 2; ++qt) acc[qt][ct] = mfma16(vf, p[qt], acc[qt][ct]);
      }
    }
  }
#pragma unroll
  for (int qt = 0; qt < 2; ++qt) {
    const float l = sum_over_q(st[qt].l[0]), lu = LSE ? sum_over_q(st[qt].lu) : 0.f;
    if (a.parts > 1) {
      const long long row = ((long long)slot * a.parts + part) * 128 + wave * 32 + 16 * qt + r16;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) *reinterpret_cast<f32x4*>(a.part_o + row * D + 16 * ct + 4 * q) = acc[qt][ct];
      if (q == 0) a.part_ml[row] = make_float4(-st[qt].neg_m, l, lu, seen ? 1.f : 0.f);
      continue;
    }
    const RowOf row(a, hk, tile0, (int)opaque((uint32_t)(wave * 32 + 16 * qt + r16)));      // (worked out again: nothing of it stays in registers)
    const long long o = at_row(a.so, b, row.head, row.query);
    store_row<D>(acc[qt], inverse_of(l, seen != 0), reinterpret_cast<uint16_t*>(a.out) + o, q, row.ok);
    if (LSE && q == 0 && row.ok) a.lse[((long long)b * a.H + row.head) * a.Sq + row.query] = natural_lse(-st[qt].neg_m, lu, seen != 0);
  }
}

// STREAM: keys and values are loaded past the caches, which is quicker where those cannot keep them from call to call (more than 256 MB, the size of the
// cache in front of the memory): 8 rows over 16 384 states of 8 heads, 537 MB 103 -> 89 us (6.0 TB/s), 1074 MB 185 -> 161 (6.7).  268 MB: 46 -> 48 us if
// they were read the call before, 56 -> 49 if not.
// States that several batch items or heads share (a stride of 0) count once, as they are read from memory once (8 requests of 5 rows a head on one document
// of 67 or 134 MB: 51 and 86 us a call, past the caches 51 and 87).
constexpr long long KEPT_BYTES = 256ll << 20;
template <int D, bool LSE, bool STREAM>
__global__ __launch_bounds__(256, 2) void k_cross_narrow(CrossArgs a) {
  constexpr int NK = 32, TILE = NK * D, CT = D / 16, KS = D / 32;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[8 * TILE];      // [wave][stage] V tiles; at the end the waves' results
  __shared__ float4 ml[4][16];
  const long long id = blockIdx.x;
  const int part = (int)(id % a.parts);
  const int bh = (int)(id / a.parts), b = bh % a.B, hk = bh / a.B;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  const int n_keys = key_count(a, b), n_tiles = (n_keys + NK - 1) / NK;
  const int t_begin = (int)((long long)n_tiles * part / a.parts), t_end = (int)((long long)n_tiles * (part + 1) / a.parts);
  const uint8_t* const mask_row = a.mask ? a.mask + (long long)b * a.mask_stride : nullptr;

  const bool ok = r16 < a.rows;
  const int use = ok ? r16 : 0, head = hk * a.group + use / a.Sq, query = use % a.Sq;
  bf16x8 qf[KS];
  {
    const uint16_t* qp = reinterpret_cast<const uint16_t*>(a.q) + at_row(a.sq, b, head, query) + 8 * q;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8*>(qp + 32 * ks);
  }
  const uint16_t* const k_head = reinterpret_cast<const uint16_t*>(a.k) + at_row(a.sk, b, hk, 0) + 8 * q;
  const char* const v_head = reinterpret_cast<const char*>(reinterpret_cast<const uint16_t*>(a.v) + at_row(a.sv, b, hk, 0));
  TileLoad<D, NK, 1> lv;
  lv.init(0, lane, (uint32_t)a.sv.t * 2u);
  FragAt<D> at;
  at.init(r16, q);
  uint16_t* const stage = lds + wave * 2 * TILE;

  bf16x8 kf[2][KS], kn[2][KS];
  auto issue = [&](int t, int buf, unsigned long long valid) __attribute__((always_inline)) {
    // keys go to registers: a row that is not valid reads the last of the item's (its scores are masked)
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint16_t* kp = k_head + (long long)min(t * NK + 16 * kt + r16, n_keys - 1) * a.sk.t;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        if constexpr (STREAM) kn[kt][ks] = __builtin_nontemporal_load(reinterpret_cast<const bf16x8*>(kp + 32 * ks));
        else kn[kt][ks] = *reinterpret_cast<const bf16x8*>(kp + 32 * ks);
      }
    }
    lv.template issue<STREAM>(uniform_ptr(v_head + (long long)t * NK * a.sv.t * 2), lds_addr_of(stage) + buf * (2u * TILE), 0, lane, valid & 0xffffffffull);
  };
  f32x4 acc[CT];
  RowState st = row_state();
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};

  unsigned long long valid = 0, valid_next = 0, seen = 0;
  int t = t_begin + wave;
  if (t < t_end) {
    valid_next = valid_keys(mask_row, t * NK, min(n_keys, t * NK + NK), lane);
    issue(t, 0, valid_next);
  }
  for (int buf = 0; t < t_end; t += 4, buf ^= 1) {
    valid = valid_next;
    seen |= valid;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // this tile is here, and the reads of the one before it are over
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kf[kt][ks] = kn[kt][ks];
    if (t + 4 < t_end) {
      valid_next = valid_keys(mask_row, (t + 4) * NK, min(n_keys, (t + 4) * NK + NK), lane);
      issue(t + 4, buf ^ 1, valid_next);
    }
    f32x4 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[kt] = mfma16(kf[kt][ks], qf[ks], ks == 0 ? zero4 : s[kt]);
    if (valid != 0xffffffffull) mask_scores(s, (uint32_t)valid, q);
    const float m = top_of(s) * a.cscale;
    if (__builtin_expect(__ballot(m > st.thr) != 0ull, 0)) {
      const float alpha = raise_row(max_over_q(m), st);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) acc[ct] *= alpha;
    }
    const bf16x8 p = weights<LSE>(s[0], s[1], a.cscale, st);
    const uint32_t v_at = opaque(lds_addr_of(stage + buf * TILE) + at.tr);
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) acc[ct] = mfma16(frag_tr<D>(v_at, ct), p, acc[ct]);
  }
  // the waves' results meet in LDS: 16 rows x D of each in its own stages
  const float l = sum_over_q(st.l[0]), lu = LSE ? sum_over_q(st.lu) : 0.f;
  __syncthreads();
  float* const mine = reinterpret_cast<float*>(stage);
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) *reinterpret_cast<f32x4*>(mine + r16 * D + 16 * ct + 4 * q) = acc[ct];
  if (q == 0) ml[wave][r16] = make_float4(-st.neg_m, l, lu, seen ? 1.f : 0.f);
  __syncthreads();
  // 16 threads to a row, D / 16 channels each
  const int row = tid >> 4, c0 = (tid & 15) * (D / 16);
  if (row >= a.rows) return;
  float m = LOWEST;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w][row].x);
  float o[D / 16], sum = 0.f, sum_u = 0.f, keys = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) o[i] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float4 e = ml[w][row];
    const float f = __builtin_amdgcn_exp2f(e.x - m);
    sum = fmaf(e.y, f, sum);
    sum_u = fmaf(e.z, f, sum_u);
    keys = fmaxf(keys, e.w);
    const float* from = reinterpret_cast<const float*>(lds + w * 2 * TILE) + row * D + c0;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = fmaf(from[i], f, o[i]);
  }
  if (a.parts > 1) {
    const long long at_part = ((long long)bh * a.parts + part) * 16 + row;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) a.part_o[at_part * D + c0 + i] = o[i];
    if (c0 == 0) a.part_ml[at_part] = make_float4(m, sum, sum_u, keys);
    return;
  }
  const int oh = hk * a.group + row / a.Sq, oq = row % a.Sq;
  const float inv = inverse_of(sum, keys != 0.f);
  const long long to = at_row(a.so, b, oh, oq) + c0;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    reinterpret_cast<__bf16*>(a.out)[to + i] = (__bf16)(o[i] * inv);
  }
  if (LSE && c0 == 0) a.lse[((long long)b * a.H + oh) * a.Sq + oq] = natural_lse(m, sum_u, keys != 0.f);
}

// out = sum_p O_p 2^(m_p - m) / sum_p l_p 2^(m_p - m), m = max_p m_p.  D / 4 threads take a row of a part; `split` such groups share a row's parts
// and meet in LDS.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_cross_merge(CrossArgs a, int tile_rows, int split) {
  constexpr int TPR = D / 4, GROUPS = 256 / TPR;
  __shared__ float4 ml[GROUPS];
  __shared__ f32x4 sums[GROUPS][TPR];
  const int group = threadIdx.x / TPR, c = (threadIdx.x % TPR) * 4, share = group % split;
  const long long idx = (long long)blockIdx.x * (GROUPS / split) + group / split;      // row of a (batch item, key head)
  const int bh = (int)(idx / a.rows), row = (int)(idx % a.rows);
  const bool in = bh < a.B * a.Hkv;
  const int b = bh % a.B, hk = bh / a.B;
  const long long base = ((long long)bh * a.items + row / tile_rows) * a.parts * tile_rows + row % tile_rows;
  float m = LOWEST, l = 0.f, lu = 0.f, keys = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (in) {
    // four parts' loads in flight
    for (int p0 = share; p0 < a.parts; p0 += 4 * split) {
      float4 e[4];
      f32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long at = base + (long long)min(p0 + i * split, a.parts - 1) * tile_rows;
        e[i] = a.part_ml[at];
        x[i] = *reinterpret_cast<const f32x4*>(a.part_o + at * D + c);
        if (p0 + i * split >= a.parts) e[i] = make_float4(LOWEST, 0.f, 0.f, 0.f);
      }
      const float m_new = fmaxf(fmaxf(fmaxf(m, e[0].x), fmaxf(e[1].x, e[2].x)), e[3].x), f0 = __builtin_amdgcn_exp2f(m - m_new);
      l *= f0;
      lu *= f0;
      o *= f0;
      m = m_new;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (p0 + i * split >= a.parts) break;
        const float f = __builtin_amdgcn_exp2f(e[i].x - m);
        l = fmaf(e[i].y, f, l);
        lu = fmaf(e[i].z, f, lu);
        keys = fmaxf(keys, e[i].w);
        o += x[i] * f;
      }
    }
  }
  if (split > 1) {
    if (c == 0) ml[group] = make_float4(m, l, lu, keys);
    sums[group][c >> 2] = o;
    __syncthreads();
    if (share) return;
    for (int g = 1; g < split; ++g) {
      const float4 e = ml[group + g];
      const float m_new = fmaxf(m, e.x), f0 = __builtin_amdgcn_exp2f(m - m_new), f1 = __builtin_amdgcn_exp2f(e.x - m_new);
      l = l * f0 + e.y * f1;
      lu = lu * f0 + e.z * f1;
      o = o * f0 + sums[group + g][c >> 2] * f1;
      keys = fmaxf(keys, e.w);
      m = m_new;
    }
  }
  if (!in) return;
  o *= inverse_of(l, keys != 0.f);
  const int head = hk * a.group + row / a.Sq, query = row % a.Sq;
  const long long to = at_row(a.so, b, head, query) + c;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + to) = bf16x4_of(o);
  else *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + to) = o;
  if (a.lse && c == 0) a.lse[((long long)b * a.H + head) * a.Sq + query] = natural_lse(m, lu, keys != 0.f);
}

CrossPlan cross_forward_plan(const isa_cross_problem& p) {
  CrossPlan c = {};
  const long long rows = (long long)(p.H / p.H_kv) * p.S_q, bh = (long long)p.B * p.H_kv;
  const bool f32 = p.dtype == ISA_F32;
  c.narrow = !f32 && rows <= 16;
  c.tile_rows = c.narrow ? 16 : f32 ? 64 : 128;
  c.items = (int)((rows + c.tile_rows - 1) / c.tile_rows);
  const long long wgs = bh * c.items, resident = 2ll * N_XCD * cus_per_xcd();
  // keys that a workgroup takes at a time, and the fewest that are worth one of its own
  const int step = c.narrow ? 128 : f32 ? 32 : 64;
  const int units = (p.S_k + step - 1) / step / 2;
  long long parts = 1;
  if (wgs > 0 && wgs < resident) parts = (c.narrow ? 2 : 1) * resident / wgs;
  if (parts > units) parts = units;
  if (parts > 64) parts = 64;
  c.parts = parts < 1 ? 1 : (int)parts;
  c.part_rows = c.parts > 1 ? (size_t)wgs * c.parts * c.tile_rows : 0;
  return c;
}

bool cross_states_streamed(const isa_cross_problem& p) {
  long long bytes = 0;
  for (const isa_strides* s : {&p.k, &p.v})
    bytes += 2ll * p.D * (s->b ? p.B : 1) * (s->h ? p.H_kv : 1) * (s->t ? p.S_k : 1);
  return bytes > KEPT_BYTES;
}

template <typename T> static hipError_t merge(const CrossArgs& a, int D, int tile_rows, hipStream_t st) {
  const long long rows = (long long)a.B * a.Hkv * a.rows;
  const int groups = 256 / (D / 4);
  int split = 1;                                           // a group takes four parts at a time
  while (split < groups && 4 * split < a.parts) split *= 2;
  const int per = groups / split;
  const dim3 grid((unsigned)((rows + per - 1) / per)), blk(256);
  if (D == 128) hipLaunchKernelGGL((k_cross_merge<T, 128>), grid, blk, 0, st, a, tile_rows, split);
  else hipLaunchKernelGGL((k_cross_merge<T, 64>), grid, blk, 0, st, a, tile_rows, split);
  return hipGetLastError();
}

hipError_t launch_cross_forward(CrossArgs a, const isa_cross_problem& p, hipStream_t st) {
  const CrossPlan c = cross_forward_plan(p);
  a.items = c.items;
  a.parts = c.parts;
  a.total = (long long)a.B * a.Hkv * c.items * c.parts;
  hipError_t e;
  if (p.dtype == ISA_F32) {
    e = launch_cross_forward_f32(a, p.D, st);
  } else {
    const bool lse = a.lse != nullptr;
    const dim3 grid = c.narrow ? dim3((unsigned)a.total) : cross_grid(a.total), blk(256);
#define ISA_CROSS(kernel, D)                                                                 \
  do {                                                                                       \
    if (lse) hipLaunchKernelGGL((kernel<D, true>), grid, blk, 0, st, a);                     \
    else hipLaunchKernelGGL((kernel<D, false>), grid, blk, 0, st, a);                        \
  } while (0)
#define ISA_NARROW(D, LSE)                                                                                \
  do {                                                                                                    \
    if (stream) hipLaunchKernelGGL((k_cross_narrow<D, LSE, true>), grid, blk, 0, st, a);                  \
    else hipLaunchKernelGGL((k_cross_narrow<D, LSE, false>), grid, blk, 0, st, a);                        \
  } while (0)
    if (c.narrow) {
      const bool stream = cross_states_streamed(p);
      if (p.D == 128) { if (lse) ISA_NARROW(128, true); else ISA_NARROW(128, false); }
      else { if (lse) ISA_NARROW(64, true); else ISA_NARROW(64, false); }
    } else {
      if (p.D == 128) ISA_CROSS(k_cross, 128); else ISA_CROSS(k_cross, 64);
    }
#undef ISA_NARROW
#undef ISA_CROSS
    e = hipGetLastError();
  }
  if (e != hipSuccess || c.parts == 1) return e;
  return p.dtype == ISA_F32 ? merge<float>(a, p.D, c.tile_rows, st) : merge<uint16_t>(a, p.D, c.tile_rows, st);
}

}  // namespace isa
