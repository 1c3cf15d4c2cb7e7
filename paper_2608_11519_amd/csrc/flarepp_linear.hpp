// Shared by the kernels of the linear layer: activations, operand tiles in LDS,
// the epilogue.
#pragma once

#include <algorithm>

#include "flarepp_device.hpp"
#include "flarepp_layers.hpp"

namespace flarepp {
namespace {

// ---- activations ---------------------------------------------------------------
// Phi(y) - 1/2 and exp(-y^2 / 2) of the normal distribution, by Abramowitz and
// Stegun 7.1.26: 1 - erf(x) = (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x), absolute
// error 1.5e-7 in erf (the coefficients are halved here).
__device__ __forceinline__ float normal_half(float y, float& gauss) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678f, __builtin_fabsf(y), 1.f));
  gauss = __builtin_amdgcn_exp2f(y * -0.72134752f * y);
  float q = 0.5f * 1.061405429f;
  q = __builtin_fmaf(q, t, 0.5f * -1.453152027f);
  q = __builtin_fmaf(q, t, 0.5f * 1.421413741f);
  q = __builtin_fmaf(q, t, 0.5f * -0.284496736f);
  q = __builtin_fmaf(q, t, 0.5f * 0.254829592f);
  return __builtin_copysignf(__builtin_fmaf(-q * t, gauss, 0.5f), y);
}
__device__ __forceinline__ float sigmoid(float y) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * -1.44269504f));
}
template <int ACT> __device__ __forceinline__ float activate(float y) {
  if constexpr (ACT == kActRelu) return y < 0.f ? 0.f : y;  // a NaN stays
  if constexpr (ACT == kActGelu) {
    float gauss;
    const float h = normal_half(y, gauss);
    return __builtin_fmaf(y, h, 0.5f * y);
  }
  if constexpr (ACT == kActSilu) return y * sigmoid(y);
  return y;
}
template <int ACT> __device__ __forceinline__ float slope(float y) {
  if constexpr (ACT == kActRelu) return y > 0.f ? 1.f : 0.f;
  if constexpr (ACT == kActGelu) {
    float gauss;
    const float h = normal_half(y, gauss);
    return __builtin_fmaf(y * 0.39894228f, gauss, 0.5f) + h;
  }
  if constexpr (ACT == kActSilu) {
    const float s = sigmoid(y);
    return s * __builtin_fmaf(y, 1.f - s, 1.f);
  }
  return 1.f;
}
// f with the activation as a constant (one uniform branch for a whole block)
template <int V> struct ActC { static constexpr int value = V; };
template <typename Fn> __device__ __forceinline__ void with_act(int act, Fn f) {
  if (act == kActGelu) f(ActC<kActGelu>{});
  else if (act == kActSilu) f(ActC<kActSilu>{});
  else if (act == kActRelu) f(ActC<kActRelu>{});
  else f(ActC<kActNone>{});
}

// f(0), .. f(N - 1) with the index as a constant
template <int I, int N, typename Fn> __device__ __forceinline__ void static_for(Fn f) {
  if constexpr (I < N) {
    f(ActC<I>{});
    static_for<I + 1, N>(f);
  }
}

// A value every lane agrees on, in scalar registers
__device__ __forceinline__ int64_t scalar64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
// lds_copy16 from a wave-uniform base and a byte offset per lane
__device__ __forceinline__ void lds_copy16_at(const void* base, uint32_t off, char* dst) {
  const unsigned to = __builtin_amdgcn_readfirstlane(
      (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)dst);
  unsigned m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "v"(off), "s"(scalar64((int64_t)base)), "s"(to) : "memory");
}

// ---- operand tiles in LDS ----------------------------------------------------------
// A step holds KB bytes (128 or 64) of the reduction of every row.
// k-contiguous operands lie as [ROWS][KB] with a row's 16-byte chunks permuted by
// the row, the others as [k][ROWS] with groups of four chunks permuted by k for
// the transposing reads: the 256 bytes of a read's turn (one chunk of 16 rows; 64
// bytes of four k) fall in different banks.
template <typename T, bool TR, int ROWS, int KB = 128> struct Tile {
  static constexpr int EPC = 16 / (int)sizeof(T), BK = KB / (int)sizeof(T);
  static constexpr int CPR = TR ? ROWS / EPC : KB / 16;  // chunks of a stored row
  static constexpr int BYTES = ROWS * KB, CHUNKS = BYTES / 16;
  // the source chunk that LDS slot s of stored row `row` holds (an involution)
  static __device__ __forceinline__ int swap(int row, int s) {
    if constexpr (!TR) return s ^ (row / (256 / KB) & (KB / 16 - 1));
    else if constexpr (sizeof(T) == 4) return s;
    else return s ^ (ROWS >= 128 ? 4 * (row & 3) : ROWS == 64 ? 4 * (row >> 1 & 1) : 0);
  }
  // rows 32 blk .. + 31, reduction elements 16 ks .. + 15: lane (c, g) holds
  // row c, elements 8 g .. + 7
  static __device__ __forceinline__ typename Frag<T>::type frag(const char* buf, int blk, int ks) {
    const int lane = lane_id(), g = lane >> 5, c = lane & 31;
    if constexpr (!TR && sizeof(T) == 2) {
      const int row = 32 * blk + c;
      return load_frag(reinterpret_cast<const T*>(buf + row * KB + swap(row, 2 * ks + g) * 16));
    } else if constexpr (!TR) {
      const int row = 32 * blk + c;
      return join<T>(load_half(reinterpret_cast<const T*>(buf + row * KB + swap(row, 4 * ks + 2 * g) * 16)),
                     load_half(reinterpret_cast<const T*>(buf + row * KB + swap(row, 4 * ks + 2 * g + 1) * 16)));
    } else if constexpr (sizeof(T) == 2) {
      const int i16 = lane & 15, k = 16 * ks + 8 * g + (i16 >> 2);
      const int s = 4 * blk + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1);
      return lds_tr_frag(buf + k * ROWS * 2 + swap(k, s) * 16 + 8 * (i16 & 1),
                         buf + (k + 4) * ROWS * 2 + swap(k + 4, s) * 16 + 8 * (i16 & 1));
    } else {
      const T* p = reinterpret_cast<const T*>(buf) + (16 * ks + 8 * g) * ROWS + 32 * blk + c;
      typename Frag<T>::type f;
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = p[j * ROWS];
      return f;
    }
  }
};

// One 16-byte chunk of an operand with `rows` rows and reduction length kend,
// zeros outside; `whole`: rows of the array are whole chunks.
template <typename T, bool TR>
__device__ __forceinline__ f32x4 guarded_chunk(const T* src, int64_t ld, int64_t rows, int64_t kend, int64_t row, int64_t k,
                                               bool whole) {
  constexpr int EPC = 16 / (int)sizeof(T);
  // stored row and column, and their ends
  const int64_t sr = TR ? k : row, sc = TR ? row : k, re = TR ? kend : rows, ce = TR ? rows : kend;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (sr >= re) return v;
  const T* s = src + sr * ld + sc;
  if (whole) {
    if (sc < ce) v = *reinterpret_cast<const f32x4*>(s);
    return v;
  }
  if (sc + EPC <= ce) {
    __builtin_memcpy(&v, s, 16);  // at any address
    return v;
  }
  T e[EPC];
#pragma unroll
  for (int j = 0; j < EPC; ++j) e[j] = sc + j < ce ? s[j] : from_f32<T>(0.f);
  __builtin_memcpy(&v, e, 16);
  return v;
}

// ---- epilogue ---------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void store_part(T* out, int64_t Q, int64_t row, int64_t q, const float (&v)[4], bool whole) {
  if (whole) {
    store4(out + row * Q + q, v[0], v[1], v[2], v[3]);
    return;
  }
  T w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = from_f32<T>(v[e]);
  T* at = out + row * Q + q;
  if (q + 4 <= Q) {
    __builtin_memcpy(at, w, sizeof(w));  // at any address
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (q + e < Q) at[e] = w[e];
}
// Four consecutive values from q on, zeros past the end of the row
template <typename T>
__device__ __forceinline__ void read_part(const T* src, int64_t at, int64_t q, int64_t Q, bool whole, float (&v)[4]) {
  if (whole) {
    const auto x = load_half(src + at + q);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_f32(x[e]);
  } else if (q + 4 <= Q) {
    T w[4];
    __builtin_memcpy(w, src + at + q, sizeof(w));  // at any address
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_f32(w[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = q + e < Q ? to_f32(src[at + q + e]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void finish4(float (&y)[4], float (&o)[4], const LinGemmParams& p, int64_t row, int64_t q, bool whole) {
  float b[4], r[4];
  if (p.bias) {
    read_part(static_cast<const T*>(p.bias), 0, q, p.Q, whole, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += b[e];
  }
  with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = activate<decltype(act)::value>(y[e]);
  });
  if (p.res) {
    read_part(static_cast<const T*>(p.res), row * p.Q, q, p.Q, whole, r);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += r[e];
  }
}

// A 32 x 32 block (lane (c, g): row c, columns 8 u + 4 g .. + 3 in v[4 u ..]) as the
// 16-byte vectors 2 m + g of its row, m in order
template <typename T> __device__ __forceinline__ void row_vectors(const f32x16& v, f32x4* q) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 w;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = (__bf16)v[8 * u + e];
      q[u] = __builtin_bit_cast(f32x4, runs_of_8(w));
    }
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = f32x4{v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]};
  }
}
// The 32 values of a row of the residual that go with a block, in its layout
// (element 4 u + e: column 8 u + 4 g + e), read 16 bytes per lane
template <typename T> struct ResBlock {
  f32x4 v[sizeof(T)];
  __device__ __forceinline__ void load(const T* row) {
    const int g = lane_id() >> 5;
#pragma unroll
    for (int u = 0; u < (int)sizeof(T); ++u)
      v[u] = *reinterpret_cast<const f32x4*>(row + (sizeof(T) == 2 ? 16 * u + 8 * g : 8 * u + 4 * g));
  }
  __device__ __forceinline__ void add_to(f32x16& y) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const bf16x8 w = runs_of_8(__builtin_bit_cast(bf16x8, v[u]));  // (its own inverse)
#pragma unroll
        for (int e = 0; e < 8; ++e) y[8 * u + e] += (float)w[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) y[e] += v[e / 4][e % 4];
    }
  }
};
// One 32 x 32 block of C inside the row (Q % EPC == 0): lane (c, g) holds row c,
// outputs 8 u + 4 g .. + 3 of the block in y[4 u ..].  res, out and pre point to
// the row's first output of the block (or are null); bias adds to a block.
// Stores of 16 bytes per lane.
template <typename T, int ACT, typename Bias>
__device__ __forceinline__ void epilogue_whole(f32x16 y, const T* res, T* out, T* pre, bool in, Bias bias) {
  const int g = lane_id() >> 5;
  ResBlock<T> r;
  if (res) r.load(res);
  bias(y);
  auto put = [&](T* d, const f32x16& v) __attribute__((always_inline)) {
    f32x4 q[sizeof(T)];
    row_vectors<T>(v, q);
#pragma unroll
    for (int m = 0; m < (int)sizeof(T); ++m)
      if (in) *reinterpret_cast<f32x4*>(d + (2 * m + g) * (16 / (int)sizeof(T))) = q[m];
  };
  if (pre) put(pre, y);
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = activate<ACT>(y[e]);
  if (res) r.add_to(y);
  put(out, y);
}
// the same for rows of any width and blocks that pass the row's end
template <typename T>
__device__ __forceinline__ void epilogue_parts(const f32x16& y, const LinGemmParams& p, int64_t row, int64_t qb) {
  const int g = lane_id() >> 5;
  const bool whole = p.Q % 4 == 0;
  if (row >= p.P) return;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t q = qb + 8 * u + 4 * g;
    if (q >= p.Q) continue;
    float v[4], o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = y[4 * u + e];
    finish4<T>(v, o, p, row, q, whole);
    store_part(static_cast<T*>(p.out), p.Q, row, q, o, whole);
    if (p.pre) store_part(static_cast<T*>(p.pre), p.Q, row, q, v, whole);
  }
}

}  // namespace
}  // namespace flarepp
