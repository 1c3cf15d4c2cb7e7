// AdamW step over many tensors in one launch:
//   m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
// Every element is read and written once, with no product worth counting: memory
// bounds it.  A wave takes blocks of 256 elements, whose 8-bit states share a
// scale: one reduction over the wave.  The 8-bit states are m and sqrt(v), in e4m3,
// rounded at random: a step moves sqrt(v) by far less than half a step of e4m3,
// which rounding to the nearest would never pass.  8-bit states, 49.6 M elements:
// 166 us, 5.4 TB/s (a large copy 5.2); four small tensors, fp32: 4.5 us.
#include <hip/hip_runtime.h>

#include "flarepp_device.hpp"
#include "flarepp_layers.hpp"

// every operation is rounded by itself: the stored codes depend on the last
// bits, and a program must get the same ones from the same formulas
#pragma clang fp contract(off)

namespace flarepp {
namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kScaleFloor = 1e-30f;  // a block whose largest value is below this is stored as zeros

// 16 + 16 random bits of element i of a step
__device__ __forceinline__ uint32_t noise(int64_t i, uint32_t step) {
  uint32_t h = (uint32_t)i * 0x9E3779B1u + (uint32_t)((uint64_t)i >> 32) * 0x6A09E667u + step * 0xBB67AE85u;
  h ^= h >> 16;
  h *= 0x6A09E667u;
  h ^= h >> 15;
  h *= 0xBB67AE85u;
  return h ^ (h >> 16);
}

// y (at most 448 in magnitude) on the e4m3 grid, rounded away from zero with
// the probability of the part cut off (u of 65536); with keep, a positive
// value is not rounded to zero
__device__ __forceinline__ float e4m3_random(float y, uint32_t u, bool keep) {
  float a = __builtin_fabsf(y);
  a = a > kE4m3Max ? kE4m3Max : a;
  const float normal = __uint_as_float((__float_as_uint(a) + (u << 4)) & ~0xFFFFFu);
  const float fixed = __builtin_floorf(a * 512.f + (float)u * (1.f / 65536)) * (1.f / 512);
  float q = a < 1.f / 64 ? fixed : normal;
  if (keep && y > 0.f && q < 1.f / 512) q = 1.f / 512;
  return y < 0.f ? -q : q;
}

__device__ __forceinline__ void decode4(uint32_t c, float scale, float (&v)[4]) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  v[0] = a[0] * scale; v[1] = a[1] * scale; v[2] = b[0] * scale; v[3] = b[1] * scale;
}

// Codes and scale of a block of 256 (four values per lane)
__device__ __forceinline__ uint32_t encode4(const float (&v)[4], const uint32_t (&u)[4], bool keep, float& scale) {
  float big = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float a = __builtin_fabsf(v[e]);
    big = __int_as_float(max(__float_as_int(big), __float_as_int(a)));  // as bits: a NaN is the largest
  }
  big = wave_max_nonneg(big);
  const bool zero = big < kScaleFloor;
  scale = zero ? 0.f : big * (1.f / kE4m3Max);
  const float inv = zero ? 0.f : 1.f / scale;
  float q[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) q[e] = e4m3_random(v[e] * inv, u[e], keep);
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], c, true);
}

template <typename V> __device__ __forceinline__ V load4(const void* p, int64_t i) {
  return *reinterpret_cast<const V*>(static_cast<const char*>(p) + i * (sizeof(V) / 4));
}

// One block of 256 elements per wave and turn, four elements per lane.
template <bool Q8>
__global__ __launch_bounds__(256) void k_adamw(AdamwParams p) {
  // this workgroup's tensor: one compare per lane (a search would wait for the
  // argument's memory at every step)
  const int mine = lane_id() < p.count && p.first[lane_id() < kAdamwPerLaunch ? lane_id() : 0] <= (int)blockIdx.x;
  const int k = __builtin_popcountll(__builtin_amdgcn_ballot_w64(mine)) - 1;
  const AdamwTensor& t = p.t[k];
  const AdamwSchedule now = p.schedule ? *p.schedule : p.now;
  const float keep = (float)(1.0 - now.lr * t.decay);
  const int lane = lane_id();
  const int64_t base = ((int64_t)((int)blockIdx.x - p.first[k]) * 4 + wave_id()) * (kAdamwBlock * kAdamwTurns);
  f32x4 pv[kAdamwTurns], gv[kAdamwTurns], mv[kAdamwTurns], vv[kAdamwTurns];
  uint32_t mc[kAdamwTurns], vc[kAdamwTurns];
  float ms[kAdamwTurns], vs[kAdamwTurns];
#pragma unroll
  for (int r = 0; r < kAdamwTurns; ++r) {
    const int64_t b = base + r * kAdamwBlock, i = b + 4 * lane;
    if (b >= t.n) break;
    if (Q8) { ms[r] = t.m_scale[b / kAdamwBlock]; vs[r] = t.v_scale[b / kAdamwBlock]; }
    if (b + kAdamwBlock <= t.n) {
      pv[r] = load4<f32x4>(t.p, i);
      gv[r] = load4<f32x4>(t.g, i);
      if (Q8) {
        mc[r] = load4<uint32_t>(t.m, i);
        vc[r] = load4<uint32_t>(t.v, i);
      } else {
        mv[r] = load4<f32x4>(t.m, i);
        vv[r] = load4<f32x4>(t.v, i);
      }
    } else {
      mc[r] = vc[r] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = i + e < t.n;
        pv[r][e] = in ? t.p[i + e] : 0.f;
        gv[r][e] = in ? t.g[i + e] : 0.f;
        if (Q8) {
          mc[r] |= (in ? (uint32_t)static_cast<const uint8_t*>(t.m)[i + e] : 0u) << (8 * e);
          vc[r] |= (in ? (uint32_t)static_cast<const uint8_t*>(t.v)[i + e] : 0u) << (8 * e);
        } else {
          mv[r][e] = in ? static_cast<const float*>(t.m)[i + e] : 0.f;
          vv[r][e] = in ? static_cast<const float*>(t.v)[i + e] : 0.f;
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kAdamwTurns; ++r) {
    const int64_t b = base + r * kAdamwBlock, i = b + 4 * lane;
    if (b >= t.n) return;
    float m[4], v[4], root[4], x[4];
    if (Q8) {
      decode4(mc[r], ms[r], m);
      decode4(vc[r], vs[r], v);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = v[e] * v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) { m[e] = mv[r][e]; v[e] = vv[r][e]; }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float g = gv[r][e];
      m[e] = m[e] * p.b1 + g * p.a1;
      v[e] = v[e] * p.b2 + (g * g) * p.a2;
      root[e] = sqrtf(v[e]);
      x[e] = pv[r][e] * keep - (m[e] / (root[e] * now.root + p.eps)) * now.size;
    }
    uint32_t mq = 0, vq = 0;
    if (Q8) {
      uint32_t um[4], uv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t h = noise(i + e, now.step);
        um[e] = h & 0xFFFFu;
        uv[e] = h >> 16;
        if (i + e >= t.n) m[e] = root[e] = 0.f;
      }
      float sm, sv;
      mq = encode4(m, um, false, sm);
      vq = encode4(root, uv, true, sv);
      if (lane == 0) {
        t.m_scale[b / kAdamwBlock] = sm;
        t.v_scale[b / kAdamwBlock] = sv;
      }
    }
    if (b + kAdamwBlock <= t.n) {
      store4(t.p + i, x[0], x[1], x[2], x[3]);
      if (Q8) {
        static_cast<uint32_t*>(t.m)[i / 4] = mq;
        static_cast<uint32_t*>(t.v)[i / 4] = vq;
      } else {
        store4(static_cast<float*>(t.m) + i, m[0], m[1], m[2], m[3]);
        store4(static_cast<float*>(t.v) + i, v[0], v[1], v[2], v[3]);
      }
      if (t.p_low) store4(static_cast<__bf16*>(t.p_low) + i, x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (i + e >= t.n) continue;
        t.p[i + e] = x[e];
        if (Q8) {
          static_cast<uint8_t*>(t.m)[i + e] = (uint8_t)(mq >> (8 * e));
          static_cast<uint8_t*>(t.v)[i + e] = (uint8_t)(vq >> (8 * e));
        } else {
          static_cast<float*>(t.m)[i + e] = m[e];
          static_cast<float*>(t.v)[i + e] = v[e];
        }
        if (t.p_low) static_cast<__bf16*>(t.p_low)[i + e] = (__bf16)x[e];
      }
    }
  }
}

}  // namespace

hipError_t launch_adamw(const AdamwParams& p, bool q8, hipStream_t s) {
  if (q8) k_adamw<true><<<dim3((unsigned)p.blocks), 256, 0, s>>>(p);
  else k_adamw<false><<<dim3((unsigned)p.blocks), 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace flarepp
