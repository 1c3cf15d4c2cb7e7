// Linear-layer products over many rows with the weights resident in LDS.
#include <hip/hip_runtime.h>

#include "flarepp_linear.hpp"

namespace flarepp {
namespace {

// C[P][Q] = L[P][K] R[K][Q] for a strip of NB outputs whose weights fit the
// LDS: persistent workgroups of eight waves, each wave walking tiles of 32 rows
// on its own.  Rows come straight from memory as MFMA fragments, a segment of SEG
// 16-element steps ahead, so every element of L passes a CU once and no barrier
// follows the weights' copy.  Memory bounds it: 131,072 x 128 -> 256 with GELU and
// its pre-activation 44 us, 3.8 TB/s.
// STEPS: K is whole steps of 16 (else rows are read by single elements).
// WHOLE: Q is whole blocks of 32.
// Waves per SIMD: four for the narrowest strip (500,000 x 64 -> 4 25 -> 21 us), two
// for the others, whose loads ahead are worth more than the waves (1,048,576 x
// 64 -> 64 101 us, 115 with four; 200,000 x 512 -> 128 82, 109).
constexpr int rows_waves(int nb, int elem_bytes) { return nb == 32 && elem_bytes == 2 ? 4 : 2; }
template <typename T, bool RT, int NB, bool STEPS, bool WHOLE>
__global__ __launch_bounds__(512, rows_waves(NB, sizeof(T))) void k_linear_rows(LinGemmParams p) {
  using F = typename Frag<T>::type;
  using R = Tile<T, RT, NB>;
  constexpr int EPC = R::EPC, BK = R::BK, NQ = NB / 32, KPB = BK / 16;  // steps of a buffer of BK
  constexpr int SEG = !STEPS ? 1 : sizeof(T) == 4 || NB == 256 ? 4 : 8;
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int lane = lane_id(), wave = wave_id(), g = lane >> 5, c = lane & 31;
  const int64_t q0 = (int64_t)blockIdx.y * NB;
  const int K = (int)p.K, KS = (K + 15) / 16, nbuf = (KS + KPB - 1) / KPB;

  // the strip's weights, zeros past the end of the reduction, and its biases
  float* lbias = reinterpret_cast<float*>(smem + nbuf * R::BYTES);
  if (WHOLE && p.bias && threadIdx.x < NB)
    lbias[threadIdx.x] = q0 + threadIdx.x < p.Q ? to_f32(static_cast<const T*>(p.bias)[q0 + threadIdx.x]) : 0.f;
  {
    const T* w = static_cast<const T*>(p.r);
    const int64_t ld = RT ? p.Q : p.K;
    const bool whole = ld % EPC == 0;
    const int chunks = nbuf * R::CHUNKS;
    for (int e0 = threadIdx.x; e0 < chunks; e0 += 512 * 8) {
      f32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int e = e0 + u * 512;
        if (e >= chunks) break;
        // RT: stored rows run through all buffers; else a buffer holds BK elements of every row
        const int b = e / R::CHUNKS, ee = e % R::CHUNKS, row = ee / R::CPR, ch = R::swap(row, ee % R::CPR);
        v[u] = RT ? guarded_chunk<T, true>(w, ld, p.Q, K, q0 + ch * EPC, b * BK + row, whole)
                  : guarded_chunk<T, false>(w, ld, p.Q, K, q0 + row, b * BK + ch * EPC, whole);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int e = e0 + u * 512;
        if (e >= chunks) break;
        reinterpret_cast<f32x4*>(smem)[e] = v[u];
      }
    }
  }
  const int64_t tiles = (p.P + 31) / 32, stride = (int64_t)gridDim.x * 8;
  int64_t tile = (int64_t)blockIdx.x * 8 + wave;
  const int nseg = (KS + SEG - 1) / SEG;

  struct Rows {
    F x[SEG];
  };
  auto load = [&](Rows& r, int64_t t, int seg) __attribute__((always_inline)) {
    const int64_t at = min(t * 32 + c, p.P - 1) * K;
    const T* l = static_cast<const T*>(p.l) + at;
#pragma unroll
    for (int j = 0; j < SEG; ++j) {
      const int k = (seg * SEG + j) * 16 + 8 * g;
      if constexpr (STEPS) {
        const int kc = min(k, K - 16 + 8 * g);  // steps past the end are not used
        r.x[j] = load_frag(l + kc);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int kc = min(k + e, K - 1);
          const T v = l[kc];
          r.x[j][e] = k + e < K ? v : from_f32<T>(0.f);
        }
      }
    }
  };

  f32x16 acc[NQ];
#pragma unroll
  for (int i = 0; i < NQ; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;

  Rows now, next;
  if (tile < tiles) load(now, tile, 0);
  __syncthreads();
  int seg = 0;
  while (tile < tiles) {
    // the next segment's loads, this one's products, and a tile's end
    const bool last = seg == nseg - 1;
    const int64_t ntile = last ? tile + stride : tile;
    const int nxt = last ? 0 : seg + 1;
    if (ntile < tiles) load(next, ntile, nxt);
    auto step = [&](int j) __attribute__((always_inline)) {
      const int ks = seg * SEG + j;
#pragma unroll
      for (int i = 0; i < NQ; ++i)
        mma(acc[i], RT ? R::frag(smem, i, ks) : R::frag(smem + ks / KPB * R::BYTES, i, ks % KPB), now.x[j]);
    };
#pragma unroll
    for (int j = 0; j < SEG; ++j)
      if (seg * SEG + j < KS) step(j);  // uniform
    if (last) {
      const int64_t row = tile * 32 + c;
      if constexpr (WHOLE) {
        constexpr int NG = sizeof(T) == 2 && NB >= 64 ? 2 : 1;  // blocks stored together
        char* region = smem + nbuf * R::BYTES + NB * sizeof(float) + wave * 2048;
        static_for<0, NQ / NG>([&](auto ic) __attribute__((always_inline)) {
          constexpr int i0 = decltype(ic)::value * NG;
          if (q0 + 32 * i0 >= p.Q) return;
          f32x16 v[NG];
#pragma unroll
          for (int d = 0; d < NG; ++d) v[d] = acc[i0 + d];
          epilogue_group<T, NG>(v, p, region, scalar64(tile * 32), q0 + 32 * i0, [&](int u) __attribute__((always_inline)) {
            return *reinterpret_cast<const f32x4*>(lbias + 32 * i0 + 8 * u + 4 * g);
          });
        });
      } else {
#pragma unroll
        for (int i = 0; i < NQ; ++i)
          if (q0 + 32 * i < p.Q) epilogue_parts<T>(acc[i], p, row, q0 + 32 * i);
      }
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][e] = 0.f;
    }
    now = next;
    tile = ntile;
    seg = nxt;
  }
}

template <typename T, bool RT, int NB, bool STEPS, bool WHOLE>
hipError_t launch_strip(const LinGemmParams& p, hipStream_t s) {
  const int64_t tiles = (p.P + 31) / 32, strips = (p.Q + NB - 1) / NB;
  const size_t lds = lin_rows_lds(sizeof(T), NB, p.K);
  const int64_t per_cu = rows_waves(NB, sizeof(T)) == 4 && 2 * lds <= 160 * 1024 ? 2 : 1;
  const int64_t groups = std::min<int64_t>((tiles + 7) / 8, std::max<int64_t>(1, 256 * per_cu / strips));
  auto* kernel = k_linear_rows<T, RT, NB, STEPS, WHOLE>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)groups, (unsigned)strips), 512, lds, s>>>(p);
  return hipGetLastError();
}

template <typename T, bool RT>
hipError_t launch_form(const LinGemmParams& p, int strip, hipStream_t s) {
  const bool whole = p.Q % 32 == 0, steps = p.K % 16 == 0;
  if constexpr (RT) {
    if (!whole && strip == 32) return launch_strip<T, RT, 32, true, false>(p, s);
    if (!whole) return launch_strip<T, RT, 64, true, false>(p, s);
  }
#define FORM(NB) return steps ? launch_strip<T, RT, NB, true, true>(p, s) : launch_strip<T, RT, NB, false, true>(p, s)
  if constexpr (sizeof(T) == 2) {
    if (strip == 256) FORM(256);
    if (strip == 128) FORM(128);
  }
  if (strip == 64) FORM(64);
  FORM(32);
#undef FORM
}

}  // namespace

size_t lin_rows_lds(int elem_bytes, int strip, int64_t K) {
  const int64_t bk = lin_step(elem_bytes);
  return (size_t)((K + bk - 1) / bk) * strip * 128 + strip * sizeof(float) + 8 * 2048;  // weights, biases, stores
}

// The strip for a product, or 0 where the tiles take less time.  Weights that
// every CU copies pay over many rows only: from 49,152 for at most 16 inputs
// (rows / tiles, us: fp32 4 -> 64, 32,768 rows 7.7 / 7.2, 49,152 8.4 / 9.0; bf16 16 -> 256,
// 24,576 16.5 / 12.2, 49,152 18.0 / 20.1), from 65,536 for at most 32 inputs or outputs
// (bf16 64 -> 3, 24,576 4.5 / 4.5, 65,536 5.2 / 5.6; 32 -> 64, 49,152 7.0 / 6.6, 65,536 7.4 /
// 8.9), and in bf16 from 98,304 to outputs
// that are many and no fewer than the inputs, so that the stores are most of the
// work (128 -> 256, 65,536 22 / 21, 100,000 35 / 37, 200,000 65 / 74; 256 -> 512, 65,536
// 43 / 43, 200,000 133 / 150; not 256 -> 128, 200,000 48 / 47, nor fp32 256 -> 256, 257 / 257).
// The kernel itself needs rows of L that are whole steps, or short; outputs that
// are whole blocks, or (forward) few; weights that fit, and L read at most twice.
int lin_rows_strip(int prod, int elem_bytes, int64_t P, int64_t Q, int64_t K) {
  const bool whole = Q % 32 == 0, steps = K % 16 == 0, few = K <= 32 || Q <= 32;
  if (few ? P < (K <= 16 ? 3 << 14 : 1 << 16) : elem_bytes != 2 || P < (3 << 15) || Q < 256 || Q < K) return 0;
  if (prod == kLinWeight || K > 512 || (!steps && (K > 32 || !whole)) || (!whole && (prod != kLinForward || Q > 64))) return 0;
  const int widest = elem_bytes == 2 ? 256 : 64;
  int strip = 32;
  while (strip < widest && strip < Q) strip *= 2;
  while (strip > 32 && lin_rows_lds(elem_bytes, strip, K) > kLinRowsLds) strip /= 2;
  return lin_rows_lds(elem_bytes, strip, K) <= kLinRowsLds && (Q + strip - 1) / strip <= 2 ? strip : 0;
}

template <typename T>
hipError_t launch_lin_rows(const LinGemmParams& p, int prod, int strip, hipStream_t s) {
  return prod == kLinForward ? launch_form<T, true>(p, strip, s) : launch_form<T, false>(p, strip, s);
}
template hipError_t launch_lin_rows<float>(const LinGemmParams&, int, int, hipStream_t);
template hipError_t launch_lin_rows<__bf16>(const LinGemmParams&, int, int, hipStream_t);

}  // namespace flarepp
