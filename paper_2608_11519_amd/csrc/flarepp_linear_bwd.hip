// Linear-layer backward (bf16) in one pass over the tokens.
#include <hip/hip_runtime.h>

#include "flarepp_linear.hpp"

namespace flarepp {
namespace {

using T = __bf16;
constexpr int TS = 32;  // tokens of a step

// LDS slot of 16-byte chunk s of token `row` in a dP tile [TS][NT].  Read two
// ways: one chunk of 16 rows (rows of dP, for dX), and 64 bytes of four rows (dP
// as the other operand of dW); both fall in different banks.
template <int NT> __device__ __forceinline__ int p_slot(int row, int s) {
  return NT >= 128 ? s ^ ((row & 3) << 2 | (row >> 2 & 3)) : s ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
}

// A workgroup takes a chunk of tokens, KT inputs and NT outputs: steps of 32
// tokens whose dP = dOut * act'(pre) is formed once, in fp32, and left in LDS as
// bf16 hi and lo parts; dW += X^T (hi + lo) stays in registers over the chunk, dbias
// sums dP in fp32, and with DX (K = KT, N = NT, the weights in LDS) dX = hi W^T
// of the step is stored; else hi goes to memory for dX.  Beside a step's products
// the next step's dP is formed, and the one after is loaded.
// 131,072 x 128 -> 256, GELU: 62 us (and 8 for the sums over the chunks) for 201 MB, 39 us
// at a large copy's rate; the VALU is busy for 36 us of it (some 40 instructions
// per element of dP), the matrix cores for 10.
template <int KT, int NT, bool SLOPE, bool DX> struct Bwd {
  static constexpr int KB = KT / 32, NB = NT / 32, BLOCKS = KB * NB;
  static constexpr int WB = BLOCKS >= 8 ? BLOCKS / 8 : 1;         // blocks of dW per wave, as BK x BN
  static constexpr int BK = WB == 4 ? 2 : WB == 2 && KB >= NB ? 2 : 1, BN = WB / BK;
  static constexpr int WN = NB / BN, WAVES = BLOCKS / WB;
  static constexpr int XB = TS * KT * 2, PB = TS * NT * 2, PARTS = SLOPE ? 2 : 1;
  static constexpr int XAT = DX ? KT * NT * 2 : 0, PAT = XAT + 3 * XB, LDS = PAT + 2 * PARTS * PB;
  static_assert(WB <= 4 && LDS <= 160 * 1024 && 512 * 8 * 4 <= 3 * XB + 2 * PARTS * PB, "layout");
};

template <int KT, int NT, int ACT, bool DX>
__global__ __launch_bounds__(512) void k_linear_backward(LinBwdParams p) {
  constexpr bool SLOPE = ACT != kActNone;
  using B = Bwd<KT, NT, SLOPE, DX>;
  using X = Tile<T, true, KT>;
  using W = Tile<T, false, KT>;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = lane_id(), wave = wave_id(), g = lane >> 5, c = lane & 31, i16 = lane & 15, r4 = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.y * NT, c0 = (int64_t)blockIdx.z * KT;
  const int64_t t0 = (int64_t)blockIdx.x * p.chunk, t1 = min(p.T, t0 + p.chunk);
  const int nsteps = (int)((t1 - t0 + TS - 1) / TS);
  const T* dout = static_cast<const T*>(p.dout);
  const T* pre = static_cast<const T*>(p.pre);

  // X rows of a step: a ring of three buffers filled by direct copies
  constexpr int XC = B::XB / 1024, XPW = (XC + 7) / 8;  // 1 KiB copies of a step, per wave
  auto issue_x = [&](int s) __attribute__((always_inline)) {
    if (s >= nsteps) return;
#pragma unroll
    for (int u = 0; u < XPW; ++u) {
      const int kib = wave * XPW + u;
      if (kib >= XC) break;
      const int e = kib * 64 + lane, row = e / X::CPR, ch = X::swap(row, e % X::CPR);
      const int64_t first = t0 + (int64_t)s * TS;
      const uint32_t at = (uint32_t)min((int64_t)row, p.T - 1 - first) * (uint32_t)p.K + ch * 8;
      lds_copy16_at(static_cast<const T*>(p.x) + first * p.K + c0, at * 2, smem + B::XAT + s % 3 * B::XB + kib * 1024);
    }
  };
  // this thread's chunks of dOut and pre: column chunk cc, rows r0 + j * RP
  constexpr int CH = NT / 8, RP = 512 / CH < TS ? 512 / CH : TS, NJ = TS / RP;
  const int cc = threadIdx.x % CH, r0 = threadIdx.x / CH;
  const bool mine = r0 < RP;
  struct Raw {
    bf16x8 d[NJ], y[SLOPE ? NJ : 1];
  };
  auto load_p = [&](Raw& r, int s) __attribute__((always_inline)) {
    // a uniform base per step and an offset per lane; rows past the end repeat the last one
    const int64_t first = t0 + (int64_t)min(s, nsteps - 1) * TS;
    const T* db = dout + first * p.N + n0;
    const T* yb = SLOPE ? pre + first * p.N + n0 : nullptr;
    const int last = (int)min(p.T - 1 - first, (int64_t)TS - 1);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const uint32_t at = (uint32_t)min(r0 + j * RP, last) * (uint32_t)p.N + cc * 8;
      r.d[j] = load_frag(db + at);
      if constexpr (SLOPE) r.y[j] = load_frag(yb + at);
    }
  };
  float bias[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) bias[e] = 0.f;
  auto produce = [&](const Raw& r, int s) __attribute__((always_inline)) {
    char* buf = smem + B::PAT + (s & 1) * (B::PARTS * B::PB);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int row = r0 + j * RP;
      const int64_t t = t0 + (int64_t)s * TS + row;
      bf16x8 hi, lo;
      if constexpr (SLOPE) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = (float)r.d[j][e] * slope<ACT>((float)r.y[j][e]);
          v[e] = t < t1 ? v[e] : 0.f;
          bias[e] += v[e];
          hi[e] = (__bf16)v[e];
          lo[e] = (__bf16)(v[e] - (float)hi[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          hi[e] = t < t1 ? r.d[j][e] : (__bf16)0.f;
          bias[e] += (float)hi[e];
        }
      }
      if (mine) {
        char* at = buf + row * NT * 2 + p_slot<NT>(row, cc) * 16;
        *reinterpret_cast<bf16x8*>(at) = hi;
        if constexpr (SLOPE) *reinterpret_cast<bf16x8*>(at + B::PB) = lo;
        if (!DX && SLOPE && p.hi && blockIdx.z == 0 && t < t1) *reinterpret_cast<bf16x8*>(static_cast<T*>(p.hi) + t * p.N + n0 + cc * 8) = hi;
      }
    }
  };

  issue_x(0);
  issue_x(1);
  Raw first;
  load_p(first, 0);
  if constexpr (DX) {  // the weights, k-contiguous per input
    const T* w = static_cast<const T*>(p.w);
    constexpr int N16 = KT * NT / 8;
#pragma unroll 8
    for (int e0 = 0; e0 < N16; e0 += 512) {
      const int e = e0 + threadIdx.x, b = e / W::CHUNKS, ee = e % W::CHUNKS, row = ee / W::CPR, ch = W::swap(row, ee % W::CPR);
      reinterpret_cast<f32x4*>(smem)[e] = *reinterpret_cast<const f32x4*>(w + (int64_t)row * p.N + b * W::BK + ch * 8);
    }
  }
  produce(first, 0);

  const int wk = wave / B::WN, wn = wave % B::WN;
  f32x16 acc[B::BK][B::BN];
#pragma unroll
  for (int i = 0; i < B::BK; ++i)
#pragma unroll
    for (int j = 0; j < B::BN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  auto dx_part = [&](int s, const char* pb, int left) __attribute__((always_inline)) {
    if constexpr (DX) {
      // the step's dX: 32 inputs per wave; groups of KB waves take the steps in turn
      constexpr int GROUPS = 8 / B::KB;
      if (p.dx && s % GROUPS == wave / B::KB) {
        const int kb = wave % B::KB;
        f32x16 d;
#pragma unroll
        for (int e = 0; e < 16; ++e) d[e] = 0.f;
#pragma unroll 1  // (unrolled, the loads of all its steps would be in registers at once)
        for (int b = 0; b < NT / 64; ++b) {
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4) {
            const bf16x8 l = load_frag(reinterpret_cast<const T*>(pb + c * NT * 2 + p_slot<NT>(c, 8 * b + 2 * k4 + g) * 16));
            mma(d, W::frag(smem + b * W::BYTES, kb, k4), l);
          }
        }
        if (c < left) {
          T* out = static_cast<T*>(p.dx) + (t0 + (int64_t)s * TS + c) * p.K + 32 * kb;
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            bf16x8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (__bf16)d[8 * u + e];
            *reinterpret_cast<bf16x8*>(out + 16 * u + 8 * g) = runs_of_8(v);
          }
        }
      }
    }
  };
  auto dw_part = [&](const char* xb, const char* pb) __attribute__((always_inline)) {
    if (wave < B::WAVES) {
#pragma unroll
      for (int ks = 0; ks < TS / 16; ++ks) {
        bf16x8 xf[B::BK], pf[B::PARTS][B::BN];
#pragma unroll
        for (int i = 0; i < B::BK; ++i) xf[i] = X::frag(xb, wk * B::BK + i, ks);
        const int k = 16 * ks + 8 * g + (i16 >> 2);
#pragma unroll
        for (int j = 0; j < B::BN; ++j) {
          const int sl = 4 * (wn * B::BN + j) + 2 * (r4 & 1) + ((i16 & 3) >> 1);
#pragma unroll
          for (int h = 0; h < B::PARTS; ++h)
            pf[h][j] = lds_tr_frag(pb + h * B::PB + k * NT * 2 + p_slot<NT>(k, sl) * 16 + 8 * (i16 & 1),
                                   pb + h * B::PB + (k + 4) * NT * 2 + p_slot<NT>(k + 4, sl) * 16 + 8 * (i16 & 1));
        }
#pragma unroll
        for (int h = 0; h < B::PARTS; ++h)
#pragma unroll
          for (int i = 0; i < B::BK; ++i)
#pragma unroll
            for (int j = 0; j < B::BN; ++j) mma(acc[i][j], pf[h][j], xf[i]);
      }
    }
  };

  // one step: `ahead` holds the next step's raw values, `spare` takes those of
  // the step after
  auto turn = [&](int s, Raw& ahead, Raw& spare) __attribute__((always_inline)) {
    // The step's dP is in LDS, and its X: a wave's own copies are older than
    // the 2 PARTS NJ loads of the last two turns.  Every wave has left the buffers of
    // the step before.
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(2 * B::PARTS * NJ) : "memory");
    issue_x(s + 2);
    load_p(spare, s + 2);
    char* xb = smem + B::XAT + s % 3 * B::XB;
    const char* pb = smem + B::PAT + (s & 1) * (B::PARTS * B::PB);
    const int left = (int)min((int64_t)TS, t1 - t0 - (int64_t)s * TS);
    if (left < TS) {  // rows past the end count as zero, also where X is not finite
      for (int e = threadIdx.x; e < B::XB / 16; e += 512)
        if (e / X::CPR >= left) reinterpret_cast<f32x4*>(xb)[e] = f32x4{0.f, 0.f, 0.f, 0.f};
      lds_barrier();
    }
    dx_part(s, pb, left);
    dw_part(xb, pb);
    produce(ahead, s + 1);  // (past the end: zeros into a buffer that is not read)
  };
  Raw a, b;
  load_p(a, 1);  // (a step past the end repeats the last rows)
  for (int s = 0; s < nsteps; s += 2) {
    turn(s, a, b);
    if (s + 1 < nsteps) turn(s + 1, b, a);
  }

  if (p.part && wave < B::WAVES) {
    float* out = p.part + blockIdx.x * p.part_stride;
#pragma unroll
    for (int i = 0; i < B::BK; ++i) {
      float* row = out + (c0 + 32 * (wk * B::BK + i) + c) * p.N + n0 + 32 * wn * B::BN + 4 * g;
#pragma unroll
      for (int j = 0; j < B::BN; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          store4(row + 32 * j + 8 * u, acc[i][j][4 * u], acc[i][j][4 * u + 1], acc[i][j][4 * u + 2], acc[i][j][4 * u + 3]);
    }
  }
  if (p.bias_part && blockIdx.z == 0) {
    __syncthreads();
    float* sums = reinterpret_cast<float*>(smem + B::XAT);
    if (mine) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[r0 * NT + cc * 8 + e] = bias[e];
    }
    __syncthreads();
    if (threadIdx.x < NT) {
      float v = 0.f;
      for (int r = 0; r < RP; ++r) v += sums[r * NT + threadIdx.x];
      p.bias_part[blockIdx.x * p.bias_ld + n0 + threadIdx.x] = v;
    }
  }
}

template <int KT, int NT, int ACT, bool DX>
hipError_t launch_form(const LinBwdParams& p, hipStream_t s) {
  constexpr int lds = Bwd<KT, NT, ACT != kActNone, DX>::LDS;
  auto* kernel = k_linear_backward<KT, NT, ACT, DX>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)p.nchunks, (unsigned)(p.N / NT), (unsigned)(p.K / KT)), 512, lds, s>>>(p);
  return hipGetLastError();
}
template <int KT, int NT, bool DX> hipError_t launch_act(const LinBwdParams& p, hipStream_t s) {
  if (p.act == kActGelu) return launch_form<KT, NT, kActGelu, DX>(p, s);
  if (p.act == kActSilu) return launch_form<KT, NT, kActSilu, DX>(p, s);
  if (p.act == kActRelu) return launch_form<KT, NT, kActRelu, DX>(p, s);
  if constexpr (DX) return launch_form<KT, NT, kActNone, DX>(p, s);
  return hipErrorInvalidValue;
}
template <int KT, int NT> hipError_t launch_size(const LinBwdParams& p, bool fused, hipStream_t s) {
  if constexpr (KT * NT <= 128 * 256) {
    if (fused) return launch_act<KT, NT, true>(p, s);
  }
  if constexpr (KT >= 128 && NT == 128) return launch_act<KT, NT, false>(p, s);
  return hipErrorInvalidValue;
}

}  // namespace

// The tile of inputs and outputs (kt, nt) of the one-pass backward; fused: dX
// too.  False where the products of k_linear take less time: sizes that are not
// whole tiles, tokens too few for their chunks' sums of dW, and, where dX is not
// formed in the pass, no activation (nothing is formed twice) or more than 256
// inputs (dP is formed again per tile of inputs).  One pass / products, us, GELU:
// 64 x 64, 2048 tokens 8.4 / 10.7; 128 x 256, 8192 24 / 21, 16,384 25 / 27, 131,072 67 / 121;
// 256 x 512, 24,576 50 / 58, 131,072 202 / 272; 256 x 256, 32,768 51 / 44, 49,152 60 / 68;
// 512 x 128, 131,072 135 / 139; without activation 256 x 256, 131,072 102 / 99.
bool lin_bwd_tile(int64_t T, int64_t K, int64_t N, int act, int& kt, int& nt, bool& fused) {
  auto ok = [](int64_t v) { return v == 64 || v == 128 || v == 256; };
  fused = ok(K) && ok(N) && K * N <= 128 * 256;
  kt = (int)K;
  nt = fused ? (int)N : 128;
  if (fused) return 2 * T >= K * N;
  return act != kActNone && T >= (N > K ? 3 << 13 : 3 << 14) && (K == 128 || K == 256) && N % 128 == 0;
}

hipError_t launch_lin_bwd(const LinBwdParams& p, int kt, int nt, bool fused, hipStream_t s) {
  switch (kt * 1000 + nt) {
    case 64064: return launch_size<64, 64>(p, fused, s);
    case 64128: return launch_size<64, 128>(p, fused, s);
    case 64256: return launch_size<64, 256>(p, fused, s);
    case 128064: return launch_size<128, 64>(p, fused, s);
    case 128128: return launch_size<128, 128>(p, fused, s);
    case 128256: return launch_size<128, 256>(p, fused, s);
    case 256064: return launch_size<256, 64>(p, fused, s);
    default: return launch_size<256, 128>(p, fused, s);
  }
}

}  // namespace flarepp
