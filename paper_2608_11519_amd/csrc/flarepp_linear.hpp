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
  // the same where the row ends after `left` columns (a multiple of a vector, maybe none)
  __device__ __forceinline__ void load_cut(const T* row, int left) {
    const int g = lane_id() >> 5;
#pragma unroll
    for (int u = 0; u < (int)sizeof(T); ++u) {
      const int col = sizeof(T) == 2 ? 16 * u + 8 * g : 8 * u + 4 * g;
      v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (col < left) v[u] = *reinterpret_cast<const f32x4*>(row + col);
    }
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
// Stores NV * 32 bytes (the first `vectors` 16-byte ones) of each of a tile's 32 rows: lane (c, g) holds row c, 16-byte
// vectors 2 m + g in q[m].  Through 2 KiB of the wave's LDS, 16 rows at a time, so
// that an instruction stores whole 64- or 128-byte runs of its rows: straight from
// the product's layout (32 bytes of 32 rows) part of the lines are written twice
// (131,072 x 128 -> 256 with pre: 161 MB for 134; GELU 56 us, 46 so; 1,048,576 x 128 -> 128
// with residual 209, 160).
template <int NV>
__device__ __forceinline__ void store_rows(char* region, const f32x4 (&q)[NV], void* dst, uint32_t row_bytes, int rows,
                                           int vectors) {
  const int lane = lane_id(), g = lane >> 5, c = lane & 31;
  constexpr int RB = NV * 32, PER = 64 / (2 * NV);  // bytes of a row, rows of an instruction
  auto slot = [](int row, int v) __attribute__((always_inline)) { return v ^ (row / (256 / RB) & (2 * NV - 1)); };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if ((c >> 4) == h) {
#pragma unroll
      for (int m = 0; m < NV; ++m) *reinterpret_cast<f32x4*>(region + (c & 15) * RB + slot(c & 15, 2 * m + g) * 16) = q[m];
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < 16 / PER; ++j) {
      const int r = j * PER + lane / (2 * NV), v = lane % (2 * NV);
      const f32x4 x = *reinterpret_cast<const f32x4*>(region + r * RB + slot(r, v) * 16);
      const int row = 16 * h + r;
      if (row < rows && v < vectors) *reinterpret_cast<f32x4*>(static_cast<char*>(dst) + (uint32_t)row * row_bytes + v * 16) = x;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Bias, activation, residual and stores of NG 32 x 32 blocks of C side by side,
// rows row0 .., outputs q .. (Q whole 16-byte vectors; vectors past the row's end
// are not stored): lane (c, g) holds row c, outputs 8 u + 4 g .. + 3 of a block in
// v[4 u ..]; bias(u) gives the four biases of run u of all blocks.
template <typename T, int NG, typename Bias>
__device__ __forceinline__ void epilogue_group(f32x16 (&v)[NG], const LinGemmParams& p, char* region, int64_t row0, int64_t q,
                                               Bias bias) {
  constexpr int ES = sizeof(T), NV = NG * ES;  // 16-byte vectors of a row per lane
  const int c = lane_id() & 31;
  const int rows = (int)min((int64_t)32, p.P - row0), vectors = (int)min((int64_t)2 * NV, (p.Q - q) * ES / 16);
  const int64_t first = row0 * p.Q + q;
  f32x4 o[NV], y[NV];
#pragma unroll
  for (int d = 0; d < NG; ++d) {
    ResBlock<T> r;
    const bool inside = q + 32 * d + 32 <= p.Q;  // uniform; a cut block's residual is read by vectors
    if (p.res) {
      const T* at = static_cast<const T*>(p.res) + first + (int64_t)min(c, rows - 1) * p.Q + 32 * d;
      if (inside) r.load(at);
      else r.load_cut(at, (int)(p.Q - q) - 32 * d);
    }
    if (p.bias) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 b = bias(4 * d + u);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[d][4 * u + e] += b[e];
      }
    }
    if (p.pre) row_vectors<T>(v[d], &y[d * ES]);
    with_act(p.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) v[d][e] = activate<decltype(act)::value>(v[d][e]);
    });
    if (p.res) r.add_to(v[d]);
    row_vectors<T>(v[d], &o[d * ES]);
  }
  store_rows<NV>(region, o, static_cast<T*>(p.out) + first, (uint32_t)(p.Q * ES), rows, vectors);
  if (p.pre) store_rows<NV>(region, y, static_cast<T*>(p.pre) + first, (uint32_t)(p.Q * ES), rows, vectors);
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
