// Linear layer out = res + act(X W + b) and its gradients
// dP = dOut act'(pre), dX = dP W^T, dW = X^T dP, dbias = the sums of dP's columns.
// Tiles of L and R go to LDS by direct copies, two steps' buffers in turn, and
// from there to MFMA; the epilogue works on the fp32 accumulators.  Large products
// are bound by the matrix cores (8192 x 2048 -> 2048, SiLU: 65 us, 1.06 PFLOP/s), long
// ones by memory (100,000 x 512 -> 256 with residual: 61 us, 3.3 TB/s), small ones by
// the launches (one token: 5 us).
#include <hip/hip_runtime.h>

#include "flarepp_linear.hpp"

namespace flarepp {
namespace {

// ---- the product -------------------------------------------------------------------
template <typename T, int PROD, bool LO, int BP, int BQ, int NBUF, int KB> constexpr int lin_lds() {
  return (Tile<T, lin_l_t(PROD), BP, KB>::BYTES + Tile<T, lin_r_t(PROD), BQ, KB>::BYTES * (LO ? 2 : 1)) * NBUF;
}
template <typename T, int PROD, bool LO, int BP, int BQ, int WP, int WQ, bool DIRECT, int NBUF, int KB>
__device__ __forceinline__ void linear_tile(const LinGemmParams& p, int block, char* smem) {
  constexpr bool LT = lin_l_t(PROD), RT = lin_r_t(PROD);
  using L = Tile<T, LT, BP, KB>;
  using R = Tile<T, RT, BQ, KB>;
  constexpr int EPC = L::EPC, BK = L::BK, NP = BP / WP / 32, NQ = BQ / WQ / 32, NW = WP * WQ, NT = 64 * NW;
  constexpr int BUF = L::BYTES + R::BYTES * (LO ? 2 : 1);
  const int lane = lane_id(), wave = wave_id(), g = lane >> 5, c = lane & 31;
  const int wp = wave / WQ, wq = wave % WQ;

  // tiles in the order q, p, split; the workgroups of one XCD (dealt out in
  // turn) take a run of them, so they share the rows of L and R in its L2
  const int64_t ntp = (p.P + BP - 1) / BP, ntq = (p.Q + BQ - 1) / BQ, total = ntp * ntq * p.splits;
  const int64_t per = (total + 7) / 8, tile = (block & 7) * per + (block >> 3);
  if ((block >> 3) >= per || tile >= total) return;  // whole workgroup, before any barrier
  const int64_t q0 = tile % ntq * BQ, p0 = tile / ntq % ntp * BP;
  const int z = (int)(tile / (ntq * ntp));
  const int64_t k0 = z * p.kchunk, k1 = min(p.K, k0 + p.kchunk);
  const int nsteps = (int)((k1 - k0 + BK - 1) / BK);
  const int64_t lld = LT ? p.P : p.K, rld = RT ? p.Q : p.K;
  const T* lsrc = static_cast<const T*>(p.l);
  const T* rsrc = static_cast<const T*>(p.r);
  const T* rlo = static_cast<const T*>(p.r_lo);

  f32x16 acc[NQ][NP];
#pragma unroll
  for (int i = 0; i < NQ; ++i)
#pragma unroll
    for (int j = 0; j < NP; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  auto compute = [&](const char* buf) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < BK / 16; ++ks) {
      typename Frag<T>::type lf[NP], rf[NQ];
#pragma unroll
      for (int j = 0; j < NP; ++j) lf[j] = L::frag(buf, wp * NP + j, ks);
#pragma unroll
      for (int i = 0; i < NQ; ++i) rf[i] = R::frag(buf + L::BYTES, wq * NQ + i, ks);
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int j = 0; j < NP; ++j) mma(acc[i][j], rf[i], lf[j]);
      if constexpr (LO) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) rf[i] = R::frag(buf + L::BYTES + R::BYTES, wq * NQ + i, ks);
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
          for (int j = 0; j < NP; ++j) mma(acc[i][j], rf[i], lf[j]);
      }
    }
  };

  if constexpr (DIRECT) {
    // 1 KiB copies of a step per wave: L, then R (and its low part)
    constexpr int LC = L::BYTES / 1024 / NW, RC = R::BYTES / 1024 / NW, IPW = LC + RC * (LO ? 2 : 1);
    static_assert(L::BYTES % (1024 * NW) == 0 && R::BYTES % (1024 * NW) == 0, "whole copies per wave");
    // A copy's source: a base per step (uniform) and an offset per lane, the
    // same in every step.  Rows and columns past the end repeat the last ones:
    // their products are not stored; reduction rows past the end (of the last
    // step) repeat too, and are cleared below.
    uint32_t loff[LC], roff[RC];
    auto offsets = [&](int64_t kleft) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < LC; ++u) {
        const int e = (wave * LC + u) * 64 + lane, row = e / L::CPR, ch = L::swap(row, e % L::CPR);
        const int64_t n = p.P - p0, r = min((int64_t)row, (LT ? kleft : n) - 1);
        loff[u] = (uint32_t)((r * lld + min((int64_t)ch * EPC, (LT ? n : kleft) - EPC)) * sizeof(T));
      }
#pragma unroll
      for (int u = 0; u < RC; ++u) {
        const int e = (wave * RC + u) * 64 + lane, row = e / R::CPR, ch = R::swap(row, e % R::CPR);
        const int64_t n = p.Q - q0, r = min((int64_t)row, (RT ? kleft : n) - 1);
        roff[u] = (uint32_t)((r * rld + min((int64_t)ch * EPC, (RT ? n : kleft) - EPC)) * sizeof(T));
      }
    };
    offsets(BK);
    const int64_t rfirst = (RT ? k0 * rld + q0 : q0 * rld + k0);
    int64_t lat = scalar64((int64_t)(lsrc + (LT ? k0 * lld + p0 : p0 * lld + k0)));  // bytes
    int64_t rat = scalar64((int64_t)(rsrc + rfirst));
    int64_t rlo_at = LO ? scalar64((int64_t)(rlo + rfirst)) : 0;
    const int64_t ladd = (LT ? BK * lld : BK) * (int64_t)sizeof(T), radd = (RT ? BK * rld : BK) * (int64_t)sizeof(T);
    auto issue = [&](int s) __attribute__((always_inline)) {
      if (s >= nsteps) return;
      char* dst = smem + s % NBUF * BUF;
      const int64_t kleft = p.K - k0 - (int64_t)s * BK;
      if (kleft < BK) offsets(kleft);  // (the last step, or none)
#pragma unroll
      for (int u = 0; u < LC; ++u) lds_copy16_at(reinterpret_cast<const void*>(lat), loff[u], dst + (wave * LC + u) * 1024);
#pragma unroll
      for (int u = 0; u < RC; ++u)
        lds_copy16_at(reinterpret_cast<const void*>(rat), roff[u], dst + L::BYTES + (wave * RC + u) * 1024);
      if constexpr (LO) {
#pragma unroll
        for (int u = 0; u < RC; ++u)
          lds_copy16_at(reinterpret_cast<const void*>(rlo_at), roff[u], dst + L::BYTES + R::BYTES + (wave * RC + u) * 1024);
        rlo_at += radd;
      }
      lat += ladd;
      rat += radd;
    };
    for (int s = 0; s < NBUF - 1; ++s) issue(s);
    for (int s = 0; s < nsteps; ++s) {
      // step s has landed: at most the NBUF - 2 steps after it are in flight
      if (s + NBUF - 2 < nsteps) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(IPW * (NBUF - 2)) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      lds_barrier();
      issue(s + NBUF - 1);  // into the buffer of step s - 1, which every wave has left
      char* buf = smem + s % NBUF * BUF;
      const int left = (int)min((int64_t)BK, k1 - k0 - (int64_t)s * BK);
      if (left < BK) {  // reduction elements past the end count as zero, on both sides
        for (int e = threadIdx.x; e < BUF / 16; e += NT) {
          const bool isl = e < L::CHUNKS;
          const int ee = isl ? e : (e - L::CHUNKS) % R::CHUNKS;
          const int row = ee / (isl ? L::CPR : R::CPR), slot = ee % (isl ? L::CPR : R::CPR);
          const int k = (isl ? LT : RT) ? row : (isl ? L::swap(row, slot) : R::swap(row, slot)) * EPC;
          if (k >= left) reinterpret_cast<f32x4*>(buf)[e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        __syncthreads();
      }
      compute(buf);
    }
  } else {
    static_assert(NBUF == 2, "one step ahead in registers");
    constexpr int NL = (L::CHUNKS + NT - 1) / NT, NR = (BUF / 16 - L::CHUNKS + NT - 1) / NT;
    const bool lwhole = lld % EPC == 0, rwhole = rld % EPC == 0;
    f32x4 lv[NL], rv[NR];
    // Steps with rows of the arrays left after them are read without a guard,
    // vectors at any address from a uniform base: rows past the end repeat the last
    // one, and a vector that passes a stored row's end takes what follows there
    // (their products are not stored).
    uint32_t loff[NL], roff[NR];
#pragma unroll
    for (int u = 0; u < NL; ++u) {
      const int e = min(u * NT + (int)threadIdx.x, L::CHUNKS - 1), row = e / L::CPR, ch = L::swap(row, e % L::CPR);
      const int64_t n = p.P - p0;
      loff[u] = (uint32_t)((LT ? row * lld + min((int64_t)ch * EPC, n - 1) : min((int64_t)row, n - 1) * lld + ch * EPC) * sizeof(T));
    }
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int e = (u * NT + (int)threadIdx.x) % R::CHUNKS, row = e / R::CPR, ch = R::swap(row, e % R::CPR);
      const int64_t n = p.Q - q0;
      roff[u] = (uint32_t)((RT ? row * rld + min((int64_t)ch * EPC, n - 1) : min((int64_t)row, n - 1) * rld + ch * EPC) * sizeof(T));
    }
    const int64_t lfirst = LT ? k0 * lld + p0 : p0 * lld + k0, rfirst = RT ? k0 * rld + q0 : q0 * rld + k0;
    const int64_t ladd = LT ? BK * lld : BK, radd = RT ? BK * rld : BK;
    auto load = [&](int s) __attribute__((always_inline)) {
      const int64_t k = k0 + (int64_t)s * BK;
      if (s < nsteps - 1 && lld >= EPC && rld >= EPC) {
        const char* lb = reinterpret_cast<const char*>(lsrc + lfirst + s * ladd);
        const char* rb = reinterpret_cast<const char*>(rsrc + rfirst + s * radd);
        const char* rl = LO ? reinterpret_cast<const char*>(rlo + rfirst + s * radd) : nullptr;
#pragma unroll
        for (int u = 0; u < NL; ++u) __builtin_memcpy(&lv[u], lb + loff[u], 16);
#pragma unroll
        for (int u = 0; u < NR; ++u)
          __builtin_memcpy(&rv[u], (LO && u * NT + (int)threadIdx.x >= R::CHUNKS ? rl : rb) + roff[u], 16);
        return;
      }
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const int e = u * NT + threadIdx.x, row = e / L::CPR, ch = L::swap(row, e % L::CPR);
        if (e >= L::CHUNKS) continue;
        lv[u] = LT ? guarded_chunk<T, true>(lsrc, lld, p.P, k1, p0 + ch * EPC, k + row, lwhole)
                   : guarded_chunk<T, false>(lsrc, lld, p.P, k1, p0 + row, k + ch * EPC, lwhole);
      }
#pragma unroll
      for (int u = 0; u < NR; ++u) {
        const int e0 = u * NT + threadIdx.x;
        const bool lo = LO && e0 >= R::CHUNKS;
        const int e = lo ? e0 - R::CHUNKS : e0, row = e / R::CPR, ch = R::swap(row, e % R::CPR);
        if (e >= R::CHUNKS) continue;
        const T* base = lo ? rlo : rsrc;
        rv[u] = RT ? guarded_chunk<T, true>(base, rld, p.Q, k1, q0 + ch * EPC, k + row, rwhole)
                   : guarded_chunk<T, false>(base, rld, p.Q, k1, q0 + row, k + ch * EPC, rwhole);
      }
    };
    load(0);
    for (int s = 0; s < nsteps; ++s) {
      char* buf = smem + (s & 1) * BUF;
#pragma unroll
      for (int u = 0; u < NL; ++u) {
        const int e = u * NT + threadIdx.x;
        if (e < L::CHUNKS) reinterpret_cast<f32x4*>(buf)[e] = lv[u];
      }
#pragma unroll
      for (int u = 0; u < NR; ++u) {
        const int e = u * NT + threadIdx.x;
        if (e < BUF / 16 - L::CHUNKS) reinterpret_cast<f32x4*>(buf + L::BYTES)[e] = rv[u];
      }
      lds_barrier();  // the buffer two steps on is written after the next barrier, when every wave has left this one
      if (s + 1 < nsteps) load(s + 1);
      compute(buf);
    }
  }

  if (!p.part && p.Q % EPC == 0) {
    // whole vectors: rows go out through LDS, which every wave has left
    __syncthreads();
    char* region = smem + wave * 2048;
    constexpr int NG = sizeof(T) == 2 && NQ % 2 == 0 ? 2 : 1;
    static_for<0, NP>([&](auto jc) __attribute__((always_inline)) {
      constexpr int j = decltype(jc)::value;
      const int64_t row0 = scalar64(p0 + 32 * (wp * NP + j));
      if (row0 >= p.P) return;
      static_for<0, NQ / NG>([&](auto ic) __attribute__((always_inline)) {
        constexpr int i0 = decltype(ic)::value * NG;
        const int64_t qb = scalar64(q0 + 32 * (wq * NQ + i0));
        if (qb >= p.Q) return;
        f32x16 v[NG];
#pragma unroll
        for (int d = 0; d < NG; ++d) v[d] = acc[i0 + d][j];
        epilogue_group<T, NG>(v, p, region, row0, qb, [&](int u) __attribute__((always_inline)) {
          const auto b = load_half(static_cast<const T*>(p.bias) + min(qb + 8 * u + 4 * g, p.Q - 4));
          return f32x4{to_f32(b[0]), to_f32(b[1]), to_f32(b[2]), to_f32(b[3])};
        });
      });
    });
    return;
  }
  static_for<0, NP>([&](auto jc) __attribute__((always_inline)) {
    constexpr int j = decltype(jc)::value;
    const int64_t row = p0 + 32 * (wp * NP + j) + c;
    static_for<0, NQ>([&](auto ic) __attribute__((always_inline)) {
      constexpr int i = decltype(ic)::value;
      const int64_t qb = q0 + 32 * (wq * NQ + i);
      if (qb >= p.Q) return;
      if (!p.part) {
        epilogue_parts<T>(acc[i][j], p, row, qb);
        return;
      }
      const bool whole = p.Q % 4 == 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t q = qb + 8 * u + 4 * g;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * u + e];
        if (row < p.P && q < p.Q) store_part(p.part + z * p.part_stride, p.Q, row, q, v, whole);
      }
    });
  });
}

template <typename T, int PROD, bool LO, int BP, int BQ, int WP, int WQ, bool DIRECT, int NBUF, int KB>
__global__ __launch_bounds__(64 * WP * WQ) void k_linear(LinGemmParams p) {
  __shared__ __attribute__((aligned(16))) char smem[lin_lds<T, PROD, LO, BP, BQ, NBUF, KB>()];
  linear_tile<T, PROD, LO, BP, BQ, WP, WQ, DIRECT, NBUF, KB>(p, blockIdx.x, smem);
}

// Both products of a small backward in one launch (64 x 64 tiles): the input
// gradient's workgroups, then the weight gradient's.
template <typename T, bool LO, bool DIRECT>
__global__ __launch_bounds__(256) void k_linear_pair(LinGemmParams dx, LinGemmParams dw, int first) {
  constexpr int NBUF = DIRECT ? 3 : 2;
  constexpr int A = lin_lds<T, kLinInput, false, 64, 64, NBUF, 128>(), B = lin_lds<T, kLinWeight, LO, 64, 64, NBUF, 128>();
  __shared__ __attribute__((aligned(16))) char smem[A > B ? A : B];
  if ((int)blockIdx.x < first) linear_tile<T, kLinInput, false, 64, 64, 2, 2, DIRECT, NBUF, 128>(dx, blockIdx.x, smem);
  else linear_tile<T, kLinWeight, LO, 64, 64, 2, 2, DIRECT, NBUF, 128>(dw, blockIdx.x - first, smem);
}

// ---- epilogue of a product whose reduction was split ----------------------------------
template <typename T>
__global__ __launch_bounds__(256) void k_linear_finish(LinGemmParams p) {
  const int64_t nq = (p.Q + 3) / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= p.P * nq) return;
  const int64_t row = i / nq, q = i % nq * 4;
  const bool whole = p.Q % 4 == 0;
  float y[4] = {0.f, 0.f, 0.f, 0.f}, o[4];
  for (int z = 0; z < p.splits; ++z) {
    const float* s = p.part + z * p.part_stride + row * p.Q + q;
    if (whole) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(s);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (q + e < p.Q) y[e] += s[e];
    }
  }
  finish4<T>(y, o, p, row, q, whole);
  store_part(static_cast<T*>(p.out), p.Q, row, q, o, whole);
  if (p.pre) store_part(static_cast<T*>(p.pre), p.Q, row, q, y, whole);
}

// ---- dP = dOut * act'(pre) and its column sums --------------------------------------------
// A workgroup takes a chunk of rows and a strip of columns: VEC columns per
// lane, 2^cl lanes across, 256 / 2^cl rows at a time.  WHOLE: rows are whole
// vectors; else the vectors lie at any address and a row's last one is cut.
template <typename T, int VEC, int ACT, bool WHOLE>
__global__ __launch_bounds__(256) void k_linear_slope(LinSlopeParams p, int cl_log2) {
  __shared__ float sums[256 * VEC];
  const int cl = 1 << cl_log2, lc = threadIdx.x & (cl - 1), lr = threadIdx.x >> cl_log2, rl = 256 >> cl_log2;
  const int64_t col = ((int64_t)blockIdx.y * cl + lc) * VEC;
  const int64_t r0 = (int64_t)blockIdx.x * p.chunk, r1 = min(p.T, r0 + p.chunk);
  const T* d = static_cast<const T*>(p.dout);
  const T* a = static_cast<const T*>(p.pre);
  const bool full = WHOLE || col + VEC <= p.N;
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  auto get = [&](const T* src, T (&v)[VEC]) __attribute__((always_inline)) {
    if (WHOLE) __builtin_memcpy(v, __builtin_assume_aligned(src, VEC * sizeof(T)), VEC * sizeof(T));
    else if (full) __builtin_memcpy(v, src, VEC * sizeof(T));
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[e] = col + e < p.N ? src[e] : from_f32<T>(0.f);
  };
  auto put = [&](T* dst, const T (&v)[VEC]) __attribute__((always_inline)) {
    if (WHOLE) __builtin_memcpy(__builtin_assume_aligned(dst, VEC * sizeof(T)), v, VEC * sizeof(T));
    else if (full) __builtin_memcpy(dst, v, VEC * sizeof(T));
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (col + e < p.N) dst[e] = v[e];
  };
  if (col < p.N) {
    for (int64_t r = r0 + lr; r < r1; r += rl) {
      const int64_t at = r * p.N + col;
      T dv[VEC], av[VEC], hi[VEC], lo[VEC];
      get(d + at, dv);
      if (ACT != kActNone) get(a + at, av);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float v = to_f32(dv[e]);
        if (ACT != kActNone) v *= slope<ACT>(to_f32(av[e]));
        s[e] += v;
        hi[e] = from_f32<T>(v);
        lo[e] = from_f32<T>(v - to_f32(hi[e]));
      }
      if (p.dp) put(static_cast<T*>(p.dp) + at, hi);
      if (p.dp_lo) put(static_cast<T*>(p.dp_lo) + at, lo);
    }
  }
  if (!p.part) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[(lr * cl + lc) * VEC + e] = s[e];
  for (int h = rl / 2; h > 0; h /= 2) {
    __syncthreads();
    if (lr < h)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[(lr * cl + lc) * VEC + e] += sums[((lr + h) * cl + lc) * VEC + e];
  }
  if (lr == 0)
#pragma unroll
    for (int e = 0; e < VEC; ++e)
      if (col + e < p.N) p.part[blockIdx.x * p.part_ld + col + e] = sums[lc * VEC + e];
}

// ---- sums of partials in a fixed order ---------------------------------------------------
// 64 outputs per workgroup: 16 lanes of four outputs, 16 groups of lanes that
// each sum every 16th split with eight loads in flight, then the groups in order.
__global__ __launch_bounds__(256) void k_linear_sum(LinSumParams p, int64_t first1) {
  __shared__ f32x4 sums[16][16];
  const int jb = p.njobs > 1 && (int64_t)blockIdx.x >= first1 ? 1 : 0;
  const LinSumJob& j = p.job[jb];
  const int l = threadIdx.x & 15, gr = threadIdx.x >> 4;
  const int64_t i = (((int64_t)blockIdx.x - (jb ? first1 : 0)) * 16 + l) * 4;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (i < j.n) {  // (strides are multiples of four: the last vector may read padding)
    const float* x = j.part + i;
    for (int z = gr; z < j.splits; z += 128) {
      f32x4 v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const f32x4*>(x + min(z + 16 * e, j.splits - 1) * j.stride);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (z + 16 * e < j.splits) s += v[e];
    }
  }
  sums[gr][l] = s;
  __syncthreads();
  if (gr == 0 && i < j.n) {
    s = sums[0][l];
#pragma unroll
    for (int e = 1; e < 16; ++e) s += sums[e][l];
    if (i + 4 <= j.n) *reinterpret_cast<f32x4*>(j.out + i) = s;
    else
      for (int e = 0; i + e < j.n; ++e) j.out[i + e] = s[e];
  }
}

template <typename T, int PROD, bool LO, int BP, int BQ, int WP, int WQ, bool DIRECT, int NBUF, int KB = 128>
hipError_t launch_tile(const LinGemmParams& p, hipStream_t s) {
  const int64_t total = (p.P + BP - 1) / BP * ((p.Q + BQ - 1) / BQ) * p.splits;
  const int64_t grid = (total + 7) / 8 * 8;
  k_linear<T, PROD, LO, BP, BQ, WP, WQ, DIRECT, NBUF, KB><<<dim3((unsigned)grid), 64 * WP * WQ, 0, s>>>(p);
  return hipGetLastError();
}

template <typename T, int PROD, bool LO>
hipError_t launch_prod(const LinGemmParams& p, int tile, bool direct, hipStream_t s) {
  if constexpr (sizeof(T) == 2 && PROD != kLinWeight) {
    if (tile == kTile256) return launch_tile<T, PROD, LO, 256, 256, 2, 4, true, 2>(p, s);
  }
  switch (tile) {
    case kTile128:
      return direct ? launch_tile<T, PROD, LO, 128, 128, 2, 2, true, 2>(p, s) : launch_tile<T, PROD, LO, 128, 128, 2, 2, false, 2>(p, s);
    case kTile64:
      return direct ? launch_tile<T, PROD, LO, 64, 64, 2, 2, true, 3>(p, s) : launch_tile<T, PROD, LO, 64, 64, 2, 2, false, 2>(p, s);
    case kTile128x32: return launch_tile<T, PROD, LO, 128, 32, 4, 1, false, 2>(p, s);
    default: return launch_tile<T, PROD, LO, 32, 128, 1, 4, false, 2>(p, s);
  }
}

int64_t tile64_blocks(const LinGemmParams& p) {
  return ((p.P + 63) / 64 * ((p.Q + 63) / 64) * p.splits + 7) / 8 * 8;
}

}  // namespace

bool lin_direct(int prod, int elem_bytes, int64_t P, int64_t Q, int64_t K) {
  const int64_t epc = 16 / elem_bytes;
  return (lin_l_t(prod) ? P : K) % epc == 0 && (lin_r_t(prod) ? Q : K) % epc == 0;
}

template <typename T>
hipError_t launch_lin_gemm(const LinGemmParams& p, int prod, int tile, bool direct, hipStream_t s) {
  if (prod == kLinForward) return launch_prod<T, kLinForward, false>(p, tile, direct, s);
  if (prod == kLinInput) return launch_prod<T, kLinInput, false>(p, tile, direct, s);
  if constexpr (sizeof(T) == 2) {
    if (p.r_lo) return launch_prod<T, kLinWeight, true>(p, tile, direct, s);
  }
  return launch_prod<T, kLinWeight, false>(p, tile, direct, s);
}
template hipError_t launch_lin_gemm<float>(const LinGemmParams&, int, int, bool, hipStream_t);
template hipError_t launch_lin_gemm<__bf16>(const LinGemmParams&, int, int, bool, hipStream_t);

template <typename T>
hipError_t launch_lin_pair(const LinGemmParams& dx, const LinGemmParams& dw, bool direct, hipStream_t s) {
  const int64_t first = tile64_blocks(dx), grid = first + tile64_blocks(dw);
  auto go = [&](auto lo, auto dir) {
    k_linear_pair<T, decltype(lo)::value != 0, decltype(dir)::value != 0><<<dim3((unsigned)grid), 256, 0, s>>>(dx, dw, (int)first);
    return hipGetLastError();
  };
  if constexpr (sizeof(T) == 2) {
    if (dw.r_lo) return direct ? go(ActC<1>{}, ActC<1>{}) : go(ActC<1>{}, ActC<0>{});
  }
  return direct ? go(ActC<0>{}, ActC<1>{}) : go(ActC<0>{}, ActC<0>{});
}
template hipError_t launch_lin_pair<float>(const LinGemmParams&, const LinGemmParams&, bool, hipStream_t);
template hipError_t launch_lin_pair<__bf16>(const LinGemmParams&, const LinGemmParams&, bool, hipStream_t);

template <typename T>
hipError_t launch_lin_finish(const LinGemmParams& p, hipStream_t s) {
  const int64_t n = p.P * ((p.Q + 3) / 4);
  k_linear_finish<T><<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>(p);
  return hipGetLastError();
}
template hipError_t launch_lin_finish<float>(const LinGemmParams&, hipStream_t);
template hipError_t launch_lin_finish<__bf16>(const LinGemmParams&, hipStream_t);

template <typename T>
hipError_t launch_lin_slope(const LinSlopeParams& p, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  const int vec = p.N >= V ? V : 1;
  int cl = 0;
  while ((1 << cl) < (vec == 1 ? 256 : 32) && (int64_t)vec << cl < p.N) ++cl;
  const dim3 grid((unsigned)p.nchunks, (unsigned)((p.N + ((int64_t)vec << cl) - 1) / ((int64_t)vec << cl)));
  auto go = [&](auto act) {
    constexpr int A = decltype(act)::value;
    if (vec == 1) k_linear_slope<T, 1, A, true><<<grid, 256, 0, s>>>(p, cl);
    else if (p.N % V == 0) k_linear_slope<T, V, A, true><<<grid, 256, 0, s>>>(p, cl);
    else k_linear_slope<T, V, A, false><<<grid, 256, 0, s>>>(p, cl);
  };
  if (p.act == kActGelu) go(ActC<kActGelu>{});
  else if (p.act == kActSilu) go(ActC<kActSilu>{});
  else if (p.act == kActRelu) go(ActC<kActRelu>{});
  else go(ActC<kActNone>{});
  return hipGetLastError();
}
template hipError_t launch_lin_slope<float>(const LinSlopeParams&, hipStream_t);
template hipError_t launch_lin_slope<__bf16>(const LinSlopeParams&, hipStream_t);

hipError_t launch_lin_sum(const LinSumParams& p, hipStream_t s) {
  const int64_t first1 = (p.job[0].n + 63) / 64, second = p.njobs > 1 ? (p.job[1].n + 63) / 64 : 0;
  k_linear_sum<<<dim3((unsigned)(first1 + second)), 256, 0, s>>>(p, first1);
  return hipGetLastError();
}

}  // namespace flarepp
