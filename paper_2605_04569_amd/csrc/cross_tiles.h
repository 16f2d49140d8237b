// Pieces of the bf16 cross attention kernels: tiles of 64 rows x D channels in LDS, loaded past the registers, and the fragments
// of v_mfma_f32_16x16x32_bf16 that are read out of them.
//
// Layouts (as in attn_sp.hip and attn_bwd.hip): with r = lane % 16, q = lane / 16, a score tile S^T = K Q^T of 16 keys x 16 queries gives lane
// (r, q) keys 4 q + i of query r; two of them, rounded, are the B operand of the next product (32 keys), whose A operand is
// read transposed out of the row-major tile with ds_read_b64_tr_b16 in the same key order.
#pragma once

#include "cross.h"

namespace isa {
namespace {

typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v* lds_s4_ptr;

#define ISA_CROSS_FENCE() __builtin_amdgcn_sched_barrier(0)

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// acc += a b with the accumulator in accumulation registers (in files built so that every other matrix instruction writes ordinary ones): with
// those for the scores as well every one of their values would be copied there and back.  Nothing but these instructions touches the
// accumulators inside a loop; `settle` (of the first one that is read) and `settled` (of the others) keep the first read behind the last write.
__device__ __forceinline__ void mfma16_acc(bf16x8 a, bf16x8 b, f32x4& acc) {
  asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void settle(f32x4& acc) { asm volatile("s_nop 15\n\ts_nop 15" : "+a"(acc)); }
__device__ __forceinline__ void settled(f32x4& acc) { asm volatile("" : "+a"(acc)); }
// 16 bytes per active lane from global memory straight into LDS: lane i -> LDS bytes lds_addr + 16 i.  Inline assembly so that the
// only wait for these loads is the explicit one.
template <bool NT = false> __device__ __forceinline__ void dma16(const void* sbase, uint32_t voff_bytes, uint32_t lds_addr) {
  lds_addr = __builtin_amdgcn_readfirstlane(lds_addr);
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt"
                 :: "s"(lds_addr), "v"(voff_bytes), "s"(sbase) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds_addr), "v"(voff_bytes), "s"(sbase) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_addr_of(const void* p) {
  return (uint32_t)(size_t)(__attribute__((address_space(3))) const void*)p;
}
__device__ __forceinline__ const char* uniform_ptr(const void* p) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
  return reinterpret_cast<const char*>((uintptr_t)(((uint64_t)hi << 32) | lo));
}

// Where the 16-byte chunk c of row `row` of a tile sits in its row: rows of 256 bytes (D = 128) meet all banks at once, rows of 128 bytes
// in pairs; with these the lanes of a fragment read hit different banks.
template <int D> __device__ __forceinline__ int chunk_at(int c, int row) { return D == 128 ? c ^ (row & 15) : c ^ ((row >> 1) & 7); }

// The same from an address of each lane's own
__device__ __forceinline__ void dma16_from(const void* src, uint32_t lds_addr) {
  lds_addr = __builtin_amdgcn_readfirstlane(lds_addr);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(lds_addr), "v"(src) : "memory", "m0");
}
__device__ const uint32x4 zero_chunk = {0u, 0u, 0u, 0u};

// The loads of a wave's share of one tile of ROWS rows (`WAVES` waves load it): row `row` of the tile from src + row * stride_b.  Bits of
// `valid` that are not set: the row is not read, its place gets zeros.  N load instructions in any case.
template <int D, int ROWS, int WAVES> struct TileLoad {
  static constexpr int CH = D / 8;                     // chunks of a row
  static constexpr int N = ROWS * CH / 64 / WAVES;     // load instructions of a wave
  static constexpr int PER = 64 / CH;                  // rows of an instruction
  static_assert(N >= 1, "a wave loads whole instructions");
  uint32_t off[N];
  __device__ __forceinline__ void init(int wave, int lane, uint32_t stride_b) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (wave * N + i) * PER + lane / CH;
      off[i] = (uint32_t)row * stride_b + (uint32_t)(chunk_at<D>(lane % CH, row) * 16);
    }
  }
  // tile: LDS address
  template <bool NT = false> __device__ __forceinline__ void issue(const char* src, uint32_t tile, int wave, int lane, unsigned long long valid) const {
    if (__builtin_expect(valid == (ROWS == 64 ? ~0ull : (1ull << (ROWS & 63)) - 1), 1)) {
#pragma unroll
      for (int i = 0; i < N; ++i) dma16<NT>(src, off[i], tile + (uint32_t)(wave * N + i) * 1024u);
    } else {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int row = (wave * N + i) * PER + lane / CH;
        const void* from = (valid >> row) & 1ull ? (const void*)(src + off[i]) : (const void*)&zero_chunk;
        dma16_from(from, tile + (uint32_t)(wave * N + i) * 1024u);
      }
    }
  }
};

// Places of a lane's fragments in a tile of rows of D channels, as LDS addresses: the chunk's bits of an address are apart from the row's, so
// that the fragments of a row follow from the first one by an exclusive or (one instruction where a register each would cost occupancy).
template <int D> struct FragAt {
  uint32_t row;                                        // rows as they are: k-slice 0 of row r of a 16-row sub-tile
  uint32_t tr;                                         // transposed: channel tile 0 of rows 4 q + ..
  __device__ __forceinline__ void init(int r16, int q) {
    row = (uint32_t)(r16 * D + chunk_at<D>(q, r16) * 8) * 2u;
    const int tr_row = 4 * q + (r16 >> 2);
    tr = (uint32_t)(tr_row * D + chunk_at<D>((r16 & 3) >> 1, tr_row) * 8 + 4 * (r16 & 1)) * 2u;
  }
};
// `at`: FragAt's place plus the LDS address of the sub-tile (a multiple of 256 bytes)
template <int D> __device__ __forceinline__ bf16x8 frag_tr(uint32_t at, int ct) {
  const uint32_t p = at ^ (32u * (uint32_t)ct);
  const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(uintptr_t)p);
  const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(uintptr_t)(p + 32 * D));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Keep a value, and what it depends on, on this side of the next fence
__device__ __forceinline__ void pin(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ uint32_t pin_pair(float a, float b) {       // two numbers rounded to bf16
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  uint32_t w = __builtin_bit_cast(uint32_t, p);
  asm volatile("" : "+v"(w));
  return w;
}
// The same as numbers of their own, for loops that know a tile's stage at compile time: what is added is part of the instruction then
template <int D> struct FragsAt {
  uint32_t row[D / 32], tr[D / 16];
  __device__ __forceinline__ void init(int r16, int q, uint32_t lds) {
    FragAt<D> at;
    at.init(r16, q);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks) row[ks] = lds + (at.row ^ (64u * (uint32_t)ks));
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct) tr[ct] = lds + (at.tr ^ (32u * (uint32_t)ct));
  }
};
__device__ __forceinline__ bf16x8 read_rows(uint32_t at, uint32_t add) {
  return *(__attribute__((address_space(3))) const bf16x8*)((__attribute__((address_space(3))) const char*)(uintptr_t)at + add);
}
template <int D> __device__ __forceinline__ bf16x8 read_tr(uint32_t at, uint32_t add) {
  const auto p = (__attribute__((address_space(3))) char*)(uintptr_t)at + add;
  const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)p);
  const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_ptr)(p + 32 * D));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Keeps a value that is the same from tile to tile from being spread over registers
__device__ __forceinline__ uint32_t opaque(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The valid keys of the 64 from key0 on that lie before `end`, one bit each
__device__ __forceinline__ unsigned long long valid_keys(const uint8_t* mask_row, int key0, int end, int lane) {
  const int key = key0 + lane;
  bool ok = key < end;
  if (mask_row && ok) ok = mask_row[key] != 0;
  return __ballot(ok);
}

// The valid keys of tiles of NK keys, one bit each: lane L holds those of tile `first` + L, worked out for 64 tiles at a time, so that no
// load of mask bytes is waited for from tile to tile.
template <int NK> struct KeyBits {
  static_assert(NK == 32, "one 32-bit word a tile");
  const uint8_t* mask_row;
  int n_keys, lane, first;
  uint32_t word;
  __device__ __forceinline__ void init(const uint8_t* mask_row_, int n_keys_, int lane_) {
    mask_row = mask_row_;
    n_keys = n_keys_;
    lane = lane_;
    first = -64;
  }
  // Tiles up to the last one with a valid key, of n_tiles (those of a long mask are not looked at)
  __device__ __forceinline__ int used(int n_tiles) {
    if (!mask_row || n_tiles > 64) return n_tiles;
    of(0);
    const unsigned long long any = __ballot(word != 0u);   // (0 for tiles behind the last)
    return any ? 64 - __builtin_clzll(any) : 0;
  }
  __device__ __forceinline__ uint32_t of(int t) {
    if (t < first || t >= first + 64) {
      first = t;
      const int key0 = (t + lane) * NK, n = n_keys - key0;
      word = n >= NK ? 0xffffffffu : n > 0 ? (1u << n) - 1u : 0u;
      if (mask_row && n > 0) {
        uint32_t w = 0;
        if (n >= NK) {
          typedef uint32_t __attribute__((ext_vector_type(4), aligned(1))) bytes16;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const bytes16 x = *reinterpret_cast<const bytes16*>(mask_row + key0 + 16 * j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t set = ((((x[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x[i]) >> 7) & 0x01010101u;      // bytes that are not 0
              w |= ((set * 0x10204080u) >> 28) << (16 * j + 4 * i);
            }
          }
        } else {
          for (int i = 0; i < n; ++i) w |= (mask_row[key0 + i] != 0 ? 1u : 0u) << i;
        }
        word &= w;
      }
      asm volatile("" : "+v"(word));                       // consumed here
    }
    return __builtin_amdgcn_readlane(word, t - first);
  }
};

// over the four lanes (r, 0..3) that share a query
__device__ __forceinline__ float max_over_q(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_q(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The 8-byte pieces that a lane holds of two neighbouring 16-channel tiles of its row (lane (r, q): channels 4 q .. 4 q + 3 of each)
// become 16 consecutive bytes: lane q has channels 8 (q / 2) .. + 7 of tile q % 2.
__device__ __forceinline__ uint4 pair_halves(uint2 a, uint2 b) {
  const auto x = __builtin_amdgcn_permlane16_swap(a.x, b.x, false, false);
  const auto y = __builtin_amdgcn_permlane16_swap(a.y, b.y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}
__device__ __forceinline__ uint2 bf16x4_of(const f32x4 r) {
  const bf16x2 lo = {(__bf16)r[0], (__bf16)r[1]}, hi = {(__bf16)r[2], (__bf16)r[3]};
  return make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi));
}
// A row's results (acc[ct]: channels 16 ct + 4 q + i) times f, rounded, to dst
template <int D> __device__ __forceinline__ void store_row(const f32x4 (&acc)[D / 16], float f, uint16_t* dst, int q, bool ok) {
#pragma unroll
  for (int ct = 0; ct < D / 16; ct += 2) {
    const uint4 o = pair_halves(bf16x4_of(acc[ct] * f), bf16x4_of(acc[ct + 1] * f));
    if (ok) *reinterpret_cast<uint4*>(dst + 16 * (ct + (q & 1)) + 8 * (q >> 1)) = o;
  }
}

__device__ __forceinline__ long long at_row(const isa_strides& s, int b, int h, int t) {
  return (long long)b * s.b + (long long)h * s.h + (long long)t * s.t;
}

// Row tile0 + i of the sequence of a key head; past its end the tile's first (which is not stored)
struct RowOf {
  int head, query;
  bool ok;
  __device__ __forceinline__ RowOf(const CrossArgs& a, int hk, int tile0, int i) {
    ok = tile0 + i < a.rows;
    const uint32_t use = ok ? tile0 + i : tile0;
    head = hk;
    query = (int)use;
    if (a.group > 1) {
      head = hk * a.group + (int)(use / (uint32_t)a.Sq);
      query = (int)(use % (uint32_t)a.Sq);
    }
  }
};

}  // namespace
}  // namespace isa
