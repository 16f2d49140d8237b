// Root-mean-square norm with the residual's addition, an output in 8 bits, and the backward pass, for gfx950.
//
//   h = x + residual,  r = 1 / sqrt(mean(h^2) + eps),  y = h r w;     8 bits: s = max |y| / 448,  y8 = e4m3(y / s)
//   g = w dy,  n = h r:  dx = r (g - n mean(g n)) + dh,  dw = sum over rows of dy n
//
// Bound by memory: every element is loaded once, a row stays in registers between the sums and the outputs (up to 8192 channels: see by_size).  LPR lanes share a
// row (8 lanes to 1024), each holds NV chunks of 16 bytes of it; a workgroup takes rows in turn, with the next row's loads in
// flight while it sums the present one, and keeps the weight in registers.  Chunks are loaded at the alignment of an element (the
// chip's vector loads need no more), so that odd row lengths and strides take the same path; the last chunk of a row whose
// length is no multiple of a chunk goes element by element (TAIL).  65 520 x 5120 bf16 with a residual: 484 us (5.5 TB/s), 8 bits 422 us (5.6), backward
// 575 us (5.8); a copy reaches 5.1.
#include <type_traits>

#include "rms_norm.h"

namespace isa {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <typename T> struct Row;
template <> struct Row<uint16_t> {
  static constexpr int E = 8;               // elements of a chunk
  typedef u32x4 __attribute__((aligned(2))) mem;
  static __device__ __forceinline__ void floats(const u32x4 r, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(r[i] << 16);
      f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 raw(const float (&f)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x2 p = {(__bf16)f[2 * i], (__bf16)f[2 * i + 1]};
      r[i] = __builtin_bit_cast(uint32_t, p);
    }
    return r;
  }
};
template <> struct Row<float> {
  static constexpr int E = 4;
  typedef u32x4 __attribute__((aligned(4))) mem;
  static __device__ __forceinline__ void floats(const u32x4 r, float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(r[i]);
  }
  static __device__ __forceinline__ u32x4 raw(const float (&f)[4]) {
    return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};

// How a row's chunks are loaded and stored.  WHOLE: all of them whole chunks, through the caches; TAIL: the last one element by element; STREAMED:
// whole chunks past the caches, where a call's tensors are STREAM_BYTES or more together, the size of the cache in front of the memory: it then keeps little
// of them for the next kernel anyway.  Chains projection -> norm -> projection of rows of 5120 bf16, us, through the caches / streamed, by the size of one
// tensor: with the residual (four tensors) 54 MB 159 / -, 66 MB 193 / 184, 130 MB 353 / 343, 512 MB 1438 / 1402; without (two) 66 MB 124 / 135, 96 MB
// 174 / 189, 130 MB 245 / 235; 8 bits with the residual 96 MB 249 / 238; backward with dh (five) 54 MB 149 / 146, 130 MB 325 / 308.
enum Mode { WHOLE, TAIL, STREAMED };
constexpr long long STREAM_BYTES = 256ll << 20;

// Chunk c of a row of C elements; zeros past its end.
template <typename T, Mode M> __device__ __forceinline__ u32x4 load_chunk(const T* row, int c, int C) {
  constexpr int E = Row<T>::E;
  u32x4 r = {0u, 0u, 0u, 0u};
  if ((c + 1) * E <= C) {
    if constexpr (M == STREAMED) r = __builtin_nontemporal_load(reinterpret_cast<const typename Row<T>::mem*>(row + c * E));
    else r = *reinterpret_cast<const typename Row<T>::mem*>(row + c * E);
  } else if (M == TAIL) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (c * E + i < C) {
        if constexpr (E == 8) r[i / 2] |= (uint32_t)row[c * E + i] << (16 * (i & 1));
        else r[i] = __float_as_uint(row[c * E + i]);
      }
  }
  return r;
}
template <typename T, Mode M> __device__ __forceinline__ void store_chunk(T* row, int c, int C, const u32x4 r) {
  constexpr int E = Row<T>::E;
  if ((c + 1) * E <= C) {
    if constexpr (M == STREAMED) __builtin_nontemporal_store(r, reinterpret_cast<typename Row<T>::mem*>(row + c * E));
    else *reinterpret_cast<typename Row<T>::mem*>(row + c * E) = r;
  } else if (M == TAIL) {
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (c * E + i < C) {
        if constexpr (E == 8) row[c * E + i] = (uint16_t)(r[i / 2] >> (16 * (i & 1)));
        else row[c * E + i] = __uint_as_float(r[i]);
      }
  }
}
template <typename T, int NV, Mode M> __device__ __forceinline__ void load_weight(const NormArgs& a, int lane, int lpr, float (&w)[NV][Row<T>::E]) {
  constexpr int E = Row<T>::E;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = lane + v * lpr;
#pragma unroll
    for (int i = 0; i < E; ++i) w[v][i] = 1.0f;
    if (!a.weight) continue;
    if (a.w_f32) {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (c * E + i < a.C) w[v][i] = reinterpret_cast<const float*>(a.weight)[c * E + i];
    } else if (E == 8) {
      Row<uint16_t>::floats(load_chunk<uint16_t, M == STREAMED ? WHOLE : M>(reinterpret_cast<const uint16_t*>(a.weight), c, a.C), reinterpret_cast<float(&)[8]>(w[v]));
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (c * E + i < a.C) w[v][i] = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(a.weight)[c * E + i] << 16);
    }
  }
}

struct Sum { static __device__ __forceinline__ float of(float a, float b) { return a + b; } };
struct Max { static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); } };
// Over the LPR lanes of a row.  More than a wave: through `lds`, one float per wave, of which the caller alternates two sets, so that one
// barrier is enough.
template <int LPR, typename Op> __device__ __forceinline__ float over_row(float x, float* lds) {
#pragma unroll
  for (int d = 1; d < (LPR < 64 ? LPR : 64); d <<= 1) x = Op::of(x, __shfl_xor(x, d));
  if constexpr (LPR > 64) {
    constexpr int W = LPR / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    float t = lds[threadIdx.x & (W - 1)];             // lane l reads wave l mod W's
#pragma unroll
    for (int d = 1; d < W; d <<= 1) t = Op::of(t, __shfl_xor(t, d));
    x = t;
  }
  return x;
}

constexpr int threads_of(int lpr) { return lpr > 256 ? lpr : 256; }

__device__ __forceinline__ float in_e4m3(float v) {   // NaN stays NaN
  return v != v ? v : fminf(fmaxf(v, -448.0f), 448.0f);
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int r = 0;
  r = __builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(a), in_e4m3(b), r, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in_e4m3(c), in_e4m3(d), r, true);
}

template <typename T, int LPR, int NV, Mode M, bool EIGHT>
__global__ __launch_bounds__(threads_of(LPR)) void k_rms_norm(NormArgs a) {
  constexpr int E = Row<T>::E, SLOTS = threads_of(LPR) / LPR;
  __shared__ float lds[4][16];
  const int lane = threadIdx.x % LPR;
  const long long step = (long long)gridDim.x * SLOTS;
  long long row = (long long)blockIdx.x * SLOTS + threadIdx.x / LPR;
  if (row >= a.rows) return;                           // (more than a wave to a row: the whole workgroup)
  float w[NV][E];
  u32x4 rx[NV], rr[NV];
  auto fetch = [&](long long at) __attribute__((always_inline)) {
    const T* px = reinterpret_cast<const T*>(a.x) + at * a.sx;
    const T* pr = reinterpret_cast<const T*>(a.residual) + at * a.sr;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rx[v] = load_chunk<T, M>(px, lane + v * LPR, a.C);
      if (a.residual) rr[v] = load_chunk<T, M>(pr, lane + v * LPR, a.C);
    }
  };
  fetch(row);
  load_weight<T, NV, M>(a, lane, LPR, w);
  for (int turn = 0; row < a.rows; row += step, turn ^= 2) {
    float f[NV][E], sum = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Row<T>::floats(rx[v], f[v]);
      if (a.residual) {
        float g[E];
        Row<T>::floats(rr[v], g);
#pragma unroll
        for (int i = 0; i < E; ++i) f[v][i] += g[i];
      }
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float t = f[v][i] * a.square_scale;
        sum = fmaf(t, t, sum);
      }
    }
    if (row + step < a.rows) fetch(row + step);        // in flight while this row is finished
    sum = over_row<LPR, Sum>(sum, lds[turn]);
    const float r = 1.0f / sqrtf(fmaf(sum, a.sum_scale, a.eps));
    if (a.rstd && lane == 0) a.rstd[row] = r;
    T* ph = reinterpret_cast<T*>(a.h) + row * a.sh;
    if (a.h) {
#pragma unroll
      for (int v = 0; v < NV; ++v) store_chunk<T, M>(ph, lane + v * LPR, a.C, Row<T>::raw(f[v]));
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < E; ++i) f[v][i] = f[v][i] * r * w[v][i];
    if constexpr (!EIGHT) {
      T* py = reinterpret_cast<T*>(a.y) + row * a.sy;
#pragma unroll
      for (int v = 0; v < NV; ++v) store_chunk<T, M>(py, lane + v * LPR, a.C, Row<T>::raw(f[v]));
    } else {
      uint8_t* py = reinterpret_cast<uint8_t*>(a.y) + row * a.sy;
      float top[NV], all = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        top[v] = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) top[v] = fmaxf(top[v], fabsf(f[v][i]));
        all = fmaxf(all, top[v]);
      }
      constexpr int GL = 128 / E;                      // lanes that hold a group's chunks
      if (a.group) {
        if constexpr (LPR >= GL) {
#pragma unroll
          for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int d = 1; d < GL; d <<= 1) top[v] = fmaxf(top[v], __shfl_xor(top[v], d));
        }
      } else {
        all = over_row<LPR, Max>(all, lds[turn + 1]);
#pragma unroll
        for (int v = 0; v < NV; ++v) top[v] = all;
      }
      const int n_scales = a.group ? a.C / 128 : 1;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = lane + v * LPR;
        // (not below the smallest normal number, whose reciprocal is finite)
        const float s = top[v] > 0.f ? fmaxf(top[v] * (1.0f / 448.0f), 0x1p-126f) : 1.0f, inv = 1.0f / s;
        if (a.group ? (c % GL == 0 && c * E < a.C) : c == 0) a.scales[row * n_scales + (a.group ? c / GL : 0)] = s;
        uint32_t q[E / 4];
#pragma unroll
        for (int j = 0; j < E / 4; ++j) q[j] = e4m3x4(f[v][4 * j] * inv, f[v][4 * j + 1] * inv, f[v][4 * j + 2] * inv, f[v][4 * j + 3] * inv);
        if ((c + 1) * E <= a.C) {
          typedef uint32_t q_mem __attribute__((ext_vector_type(E / 4), aligned(1)));
          q_mem o;
#pragma unroll
          for (int j = 0; j < E / 4; ++j) o[j] = q[j];
          if constexpr (M == STREAMED) __builtin_nontemporal_store(o, reinterpret_cast<q_mem*>(py + c * E));
          else *reinterpret_cast<q_mem*>(py + c * E) = o;
        } else if (M == TAIL) {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (c * E + i < a.C) py[c * E + i] = (uint8_t)(q[i / 4] >> (8 * (i & 3)));
        }
      }
    }
  }
}

// The sums of dw run down the rows of a workgroup in registers (a lane holds the same channels of every row), then over its row slots
// in LDS; k_norm_dw adds the workgroups' sums in a fixed order.
template <typename T, int LPR, int NV, Mode M>
__global__ __launch_bounds__(threads_of(LPR)) void k_rms_norm_bwd(NormArgs a) {
  constexpr int E = Row<T>::E, SLOTS = threads_of(LPR) / LPR;
  __shared__ float lds[2][16];
  __shared__ float slots[SLOTS > 1 ? SLOTS * LPR * NV * E : 1];
  const int lane = threadIdx.x % LPR;
  const long long step = (long long)gridDim.x * SLOTS;
  long long row = (long long)blockIdx.x * SLOTS + threadIdx.x / LPR;
  float w[NV][E], acc[NV][E];
  u32x4 rx[NV], rr[NV], rg[NV], rd[NV];
  float rs = 0.f;
  auto fetch = [&](long long at) __attribute__((always_inline)) {
    const T* px = reinterpret_cast<const T*>(a.x) + at * a.sx;
    const T* pr = reinterpret_cast<const T*>(a.residual) + at * a.sr;
    const T* pg = reinterpret_cast<const T*>(a.dy) + at * a.sdy;
    const T* pd = reinterpret_cast<const T*>(a.dh) + at * a.sdh;
    rs = a.rstd[at];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      rx[v] = load_chunk<T, M>(px, lane + v * LPR, a.C);
      if (a.residual) rr[v] = load_chunk<T, M>(pr, lane + v * LPR, a.C);
      rg[v] = load_chunk<T, M>(pg, lane + v * LPR, a.C);
      if (a.dh) rd[v] = load_chunk<T, M>(pd, lane + v * LPR, a.C);
    }
  };
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < E; ++i) acc[v][i] = 0.f;
  if (row < a.rows) fetch(row);
  load_weight<T, NV, M>(a, lane, LPR, w);
  const float inv_c = 1.0f / (float)a.C;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    float n[NV][E], g[NV][E], d[NV][E], dot = 0.f;
    const float r = rs;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      Row<T>::floats(rx[v], n[v]);
      if (a.residual) {
        Row<T>::floats(rr[v], g[v]);
#pragma unroll
        for (int i = 0; i < E; ++i) n[v][i] += g[v][i];
      }
      Row<T>::floats(rg[v], g[v]);
      if (a.dh) Row<T>::floats(rd[v], d[v]);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        n[v][i] *= r;
        acc[v][i] = fmaf(g[v][i], n[v][i], acc[v][i]);
        g[v][i] *= w[v][i];
        dot = fmaf(g[v][i], n[v][i], dot);
      }
    }
    if (row + step < a.rows) fetch(row + step);
    dot = over_row<LPR, Sum>(dot, lds[turn]) * inv_c;
    T* px = reinterpret_cast<T*>(a.y) + row * a.sy;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        g[v][i] = r * fmaf(-n[v][i], dot, g[v][i]);
        if (a.dh) g[v][i] += d[v][i];
      }
      store_chunk<T, M>(px, lane + v * LPR, a.C, Row<T>::raw(g[v]));
    }
  }
  if (!a.partial) return;
  float* const out = a.partial + (long long)blockIdx.x * a.C;
  if constexpr (SLOTS > 1) {
    constexpr int N = LPR * NV * E;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < E; ++i) slots[(threadIdx.x / LPR) * N + (lane + v * LPR) * E + i] = acc[v][i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += threads_of(LPR)) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < SLOTS; ++k) s += slots[k * N + c];
      out[c] = s;
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int c = (lane + v * LPR) * E + i;
        if (c < a.C) out[c] = acc[v][i];
      }
  }
}

// dw: 32 channels a workgroup, 4 to a thread, 128 threads to a channel, each of which adds a few of the workgroups' sums (so many loads are in
// flight at once); the additions in 64 bits and in a fixed order.  At most 512 sums, of 5120 channels 256: 5 us.
__global__ __launch_bounds__(1024) void k_norm_dw(const float* partial, int n, int C, void* dw, int w_f32) {
  __shared__ double sums[128][33];
  const int c = blockIdx.x * 32 + (threadIdx.x & 7) * 4, part = threadIdx.x >> 3;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  const bool wide = C % 4 == 0;                         // (the sums of a workgroup then start at 16-byte places)
  for (int k = part; k < n; k += 128) {
    const float* p = partial + (long long)k * C + c;
    if (wide && c < C) {
      const float4 x = *reinterpret_cast<const float4*>(p);
      s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < C) s[i] += p[i];
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[part][(threadIdx.x & 7) * 4 + i] = s[i];
  __syncthreads();
  // 32 threads to a channel, four parts each, then over the 32
  const int ch = threadIdx.x >> 5, l = threadIdx.x & 31;
  double t = (sums[l][ch] + sums[l + 32][ch]) + (sums[l + 64][ch] + sums[l + 96][ch]);
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) t += __shfl_xor(t, d);
  const int o = blockIdx.x * 32 + ch;
  if (l || o >= C) return;
  if (w_f32) reinterpret_cast<float*>(dw)[o] = (float)t;
  else reinterpret_cast<__bf16*>(dw)[o] = (__bf16)(float)t;
}

// Lanes to a row and chunks to a lane: few enough chunks that a row's working set stays in registers beside the next row's loads, up to 8192 channels.
// Beyond, 1024 threads leave 128 registers a lane, and some of what a lane holds goes through scratch memory (bytes a lane, forward / 8 bits / backward):
// bf16 to 16 384 channels 0 / 0 / 92, to 32 768 0 / 28 / 632; fp32 to 16 384 0 / 0 / 220, to 32 768 240 / 256 / 1100.
template <typename T, typename F> hipError_t by_size(int chunks, F f) {
#define ISA_NORM(LPR, NV) return f(std::integral_constant<int, LPR>(), std::integral_constant<int, NV>())
  if (chunks <= 8) ISA_NORM(8, 1);
  if (chunks <= 16) ISA_NORM(16, 1);
  if (chunks <= 32) ISA_NORM(32, 1);
  if (chunks <= 64) ISA_NORM(64, 1);
  if (chunks <= 128) ISA_NORM(64, 2);
  if (chunks <= 256) ISA_NORM(256, 1);
  if (chunks <= 512) ISA_NORM(256, 2);
  if (chunks <= 768) ISA_NORM(256, 3);
  if (chunks <= 1024) ISA_NORM(256, 4);
  if (chunks <= 2048) ISA_NORM(1024, 2);
  if constexpr (Row<T>::E == 8) {                        // (4096 chunks are 32 768 channels)
    ISA_NORM(1024, 4);
  } else {
    if (chunks <= 4096) ISA_NORM(1024, 4);
    ISA_NORM(1024, 8);
  }
#undef ISA_NORM
}
template <typename T, typename F> void by_mode(const NormArgs& a, bool eight, F f) {
  if (a.C % Row<T>::E != 0) f(std::integral_constant<Mode, TAIL>());
  else if (norm_streams(a, Row<T>::E == 8 ? ISA_BF16 : ISA_F32, eight)) f(std::integral_constant<Mode, STREAMED>());
  else f(std::integral_constant<Mode, WHOLE>());
}
int slots_of(int chunks) { return chunks <= 8 ? 32 : chunks <= 16 ? 16 : chunks <= 32 ? 8 : chunks <= 128 ? 4 : 1; }
int chunks_of(int C, int dtype) { return dtype == ISA_BF16 ? (C + 7) / 8 : (C + 3) / 4; }

}  // namespace

bool norm_streams(const NormArgs& a, int dtype, bool eight) {
  const long long size = dtype == ISA_BF16 ? 2 : 4;
  long long bytes = eight ? 1 : size;                      // of an element of every tensor: y or dx, then those that the call has
  for (const void* t : {a.x, a.residual, (const void*)a.h, a.dy, a.dh})
    if (t) bytes += size;
  return a.C % (16 / size) == 0 && a.rows * a.C * bytes >= STREAM_BYTES;
}

int norm_backward_workgroups(const isa_norm_problem* p) {
  const int chunks = chunks_of(p->channels, p->dtype);
  // One workgroup to a compute unit where a lane has two chunks of a row or more (16 loads in flight), else two; more leave more sums to add and take
  // turns at the memory.  160 million bf16 elements, 1 / 2 / 3 to a compute unit: 5120 channels 280 / 304 / 328 us, 1024 channels 289 / 303 / 304; one chunk to
  // a lane: 512 channels 318 / 276 / 296, 2048 channels 320 / 281 / 285.
  const bool one_chunk = chunks <= 64 || (chunks > 128 && chunks <= 256);
  const long long most = (one_chunk ? 2 : 1) * (long long)N_XCD * cus_per_xcd(), slots = slots_of(chunks);
  const long long n = (p->rows + slots - 1) / slots;
  return (int)(n < most ? n : most);
}

template <typename T> static hipError_t launch_t(const NormArgs& a, bool eight, hipStream_t st) {
  const int chunks = chunks_of(a.C, Row<T>::E == 8 ? ISA_BF16 : ISA_F32);
  return by_size<T>(chunks, [&](auto lpr, auto nv) -> hipError_t {
    constexpr int L = decltype(lpr)::value, N = decltype(nv)::value;
    // Many short turns where the rows are streamed (5120 channels, 8 / 16 / 32 workgroups to a compute unit: 245 / 238 / 230 us, in 8 bits 213 / 207 / 199), fewer
    // loads of the weight where they are few (4096 rows: 25 / 30 / 30)
    const long long slots = threads_of(L) / L, wide = norm_streams(a, Row<T>::E == 8 ? ISA_BF16 : ISA_F32, eight) ? 32 : 8, most = (L > 256 ? 2 : wide) * (long long)N_XCD * cus_per_xcd(), n = (a.rows + slots - 1) / slots;
    const dim3 grid((unsigned)(n < most ? n : most)), blk(threads_of(L));
    by_mode<T>(a, eight, [&](auto mode) {
      constexpr Mode M = decltype(mode)::value;
      if (eight) hipLaunchKernelGGL((k_rms_norm<T, L, N, M, true>), grid, blk, 0, st, a);
      else hipLaunchKernelGGL((k_rms_norm<T, L, N, M, false>), grid, blk, 0, st, a);
    });
    return hipGetLastError();
  });
}

hipError_t launch_rms_norm(const NormArgs& a, int dtype, bool eight, hipStream_t st) {
  return dtype == ISA_BF16 ? launch_t<uint16_t>(a, eight, st) : launch_t<float>(a, eight, st);
}

template <typename T> static hipError_t launch_bwd_t(const NormArgs& a, int wgs, hipStream_t st) {
  return by_size<T>(chunks_of(a.C, Row<T>::E == 8 ? ISA_BF16 : ISA_F32), [&](auto lpr, auto nv) -> hipError_t {
    constexpr int L = decltype(lpr)::value, N = decltype(nv)::value;
    const dim3 grid((unsigned)wgs), blk(threads_of(L));
    by_mode<T>(a, false, [&](auto mode) { hipLaunchKernelGGL((k_rms_norm_bwd<T, L, N, decltype(mode)::value>), grid, blk, 0, st, a); });
    return hipGetLastError();
  });
}

hipError_t launch_rms_norm_backward(const NormArgs& a, int dtype, int wgs, void* d_weight, hipStream_t st) {
  if (wgs > 0) {
    const hipError_t e = dtype == ISA_BF16 ? launch_bwd_t<uint16_t>(a, wgs, st) : launch_bwd_t<float>(a, wgs, st);
    if (e != hipSuccess) return e;
  }
  if (d_weight) hipLaunchKernelGGL(k_norm_dw, dim3((a.C + 31) / 32), dim3(1024), 0, st, a.partial, wgs, a.C, d_weight, a.w_f32);
  return hipGetLastError();
}

}  // namespace isa
