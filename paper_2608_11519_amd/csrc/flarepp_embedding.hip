// Embedding lookup with scaling and its gradient.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "flarepp_device.hpp"
#include "flarepp_layers.hpp"

namespace flarepp {
namespace {

int pow2_log2(int64_t n, int most) {  // of the smallest power of two >= n, at most `most`
  int l = 0;
  while (l < most && (int64_t(1) << l) < n) ++l;
  return l;
}

// N values of T from column col of a row of C as floats, and back.  WHOLE: rows
// are whole vectors of 16 bytes; else the vectors lie at any address and the
// row's last one is cut.
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void load_n(const T* row, int64_t col, int64_t C, float (&v)[N]) {
  T e[N];
  if constexpr (WHOLE) {
    __builtin_memcpy(e, __builtin_assume_aligned(row + col, N * sizeof(T) < 16 ? N * sizeof(T) : 16), N * sizeof(T));
  } else if (col + N <= C) {
    __builtin_memcpy(e, row + col, N * sizeof(T));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = col + i < C ? row[col + i] : from_f32<T>(0.f);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_f32(e[i]);
}
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void store_n(T* row, int64_t col, int64_t C, const float (&v)[N]) {
  T e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = from_f32<T>(v[i]);
  if constexpr (WHOLE) {
    __builtin_memcpy(__builtin_assume_aligned(row + col, N * sizeof(T) < 16 ? N * sizeof(T) : 16), e, N * sizeof(T));
  } else if (col + N <= C) {
    __builtin_memcpy(row + col, e, N * sizeof(T));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (col + i < C) row[col + i] = e[i];
  }
}

// out[t] = scale * table[ids[t]]: VEC channels per lane, 2^cl lanes across a
// row, four rows per lane so that their loads are in flight together.  The rows
// written bound it: 131,072 x 128 bf16 9.8 us, 3.5 TB/s.
template <typename T, int VEC, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed(EmbedParams p, int cl) {
  constexpr int ROWS = 4;
  const int rl = 256 >> cl, lr = threadIdx.x >> cl;
  const int64_t col = (((int64_t)blockIdx.y << cl) + (threadIdx.x & ((1 << cl) - 1))) * VEC;
  const int64_t t0 = (int64_t)blockIdx.x * rl * ROWS + lr;
  if (col >= p.C) return;
  int64_t id[ROWS];
  float v[ROWS][VEC];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) id[r] = t0 + r * rl < p.T ? p.ids[t0 + r * rl] : -1;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (id[r] >= 0 && id[r] < p.V) load_n<T, VEC, WHOLE>(static_cast<const T*>(p.table) + id[r] * p.C, col, p.C, v[r]);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) v[r][e] = id[r] < 0 ? 0.f : __builtin_nanf("");
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (t0 + r * rl >= p.T) continue;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[r][e] *= p.scale;
    store_n<T, VEC, WHOLE>(static_cast<T*>(p.out) + (t0 + r * rl) * p.C, col, p.C, v[r]);
  }
}

// ---- gradient -------------------------------------------------------------------
// A stable radix sort of the positions by symbol (ids outside [0, V) sort
// last, as V), then sums over the runs of equal symbols in ascending position: an
// order that no atomic sets, so the results are the same bits every time.  The
// sums read dOut once and the table is written once; beyond this the launches of
// the sort cost most.  131,072 x 128 fp32, 256 symbols: count 4.7, scan 4.2, scatter 7.2,
// runs 14.0 (68 MB, 4.8 TB/s), join 8.0 us; 65,536 x 256 bf16, 32,000 symbols: two passes of
// 8.0 / 3.0 / 6.0 (median), runs 16.1, join 12.7 us.

__device__ __forceinline__ uint32_t embed_key(const EmbedGradParams& p, int pass, int64_t i) {
  if (pass > 0) return p.key[pass & 1][i];
  const int64_t id = p.ids[i];
  return id < 0 || id >= p.V ? (uint32_t)p.V : (uint32_t)id;
}

__device__ __forceinline__ void clear_slice(float* p, int64_t n) {
  const int64_t stride = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n / 4; i += stride)
    reinterpret_cast<f32x4*>(p)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int64_t tail = n / 4 * 4 + threadIdx.x;
  if (blockIdx.x == 0 && tail < n) p[tail] = 0.f;
}
int clear_groups(int64_t n) { return (int)std::min<int64_t>(2048, (n + 1023) / 1024); }
__global__ __launch_bounds__(256) void k_embed_clear(float* p, int64_t n) { clear_slice(p, n); }

// counts[digit][workgroup] of tiles of TILE positions; the first pass also
// clears the table's gradient, by workgroups past the nb of the positions where
// these are few
template <int TILE>
__global__ __launch_bounds__(256) void k_embed_count(EmbedGradParams p, int pass, int nb) {
  __shared__ int hist[1024];
  const int bins = 1 << p.bits, shift = pass * p.bits;
  for (int b = threadIdx.x; b < bins; b += 256) hist[b] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * TILE;
#pragma unroll
  for (int u = 0; u < TILE / 256; ++u) {
    const int64_t i = i0 + u * 256 + threadIdx.x;
    if (i < p.T) atomicAdd(&hist[embed_key(p, pass, i) >> shift & (bins - 1)], 1);
  }
  if (pass == 0) clear_slice(p.dtable, p.V * p.C);
  if ((int)blockIdx.x >= nb) return;  // whole workgroup
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 256) p.counts[(int64_t)b * nb + blockIdx.x] = hist[b];
}

// exclusive sums over the workgroups of a digit, one wave per digit
__global__ __launch_bounds__(64) void k_embed_scan(EmbedGradParams p, int nb) {
  int* row = p.counts + (int64_t)blockIdx.x * nb;
  const int lane = lane_id();
  int run = 0;
  for (int b = 0; b < nb; b += 64) {
    const int v = b + lane < nb ? row[b + lane] : 0;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(s, d);
      if (lane >= d) s += o;
    }
    if (b + lane < nb) row[b + lane] = run + s - v;
    run += __shfl(s, 63);
  }
  if (lane == 0) p.totals[blockIdx.x] = run;
}

// keys and positions to their places: each wave ranks a run of its
// workgroup's tile, 64 positions at a time
template <int TILE>
__global__ __launch_bounds__(256) void k_embed_scatter(EmbedGradParams p, int pass, int nb) {
  __shared__ int place[4][1024];
  __shared__ int sums[256];
  const int bins = 1 << p.bits, shift = pass * p.bits, lane = lane_id(), wave = wave_id();
  constexpr int PER = TILE / 4;  // positions of a wave
  const int64_t i0 = (int64_t)blockIdx.x * TILE + wave * PER;
  uint32_t key[PER / 64];
#pragma unroll
  for (int u = 0; u < PER / 64; ++u) {
    const int64_t i = i0 + u * 64 + lane;
    key[u] = i < p.T ? embed_key(p, pass, i) : 0;
  }
  for (int b = threadIdx.x; b < bins; b += 256)
#pragma unroll
    for (int w = 0; w < 4; ++w) place[w][b] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < PER / 64; ++u)
    if (i0 + u * 64 + lane < p.T) atomicAdd(&place[wave][key[u] >> shift & (bins - 1)], 1);
  // first place of every digit: sums over the digits (a run of them per thread)
  const int run = (bins + 255) / 256, b0 = threadIdx.x * run;
  int total = 0;
  for (int j = 0; j < run; ++j) total += b0 + j < bins ? p.totals[b0 + j] : 0;
  sums[threadIdx.x] = total;
  __syncthreads();
  for (int d = 1; d < 256; d *= 2) {
    const int o = threadIdx.x >= (unsigned)d ? sums[threadIdx.x - d] : 0;
    __syncthreads();
    sums[threadIdx.x] += o;
    __syncthreads();
  }
  int at = sums[threadIdx.x] - total;
  for (int j = 0; j < run; ++j) {
    const int b = b0 + j;
    if (b >= bins) break;
    int to = at + p.counts[(int64_t)b * nb + blockIdx.x];
    at += p.totals[b];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const int n = place[w][b];
      place[w][b] = to;
      to += n;
    }
  }
  __syncthreads();
  volatile int* mine = place[wave];  // only this wave reads and writes it from here on
#pragma unroll
  for (int u = 0; u < PER / 64; ++u) {
    const int64_t i = i0 + u * 64 + lane;
    const bool in = i < p.T;
    const int digit = (int)(key[u] >> shift & (bins - 1));
    uint64_t same = __builtin_amdgcn_ballot_w64(in);
    for (int b = 0; b < p.bits; ++b) {
      const uint64_t set = __builtin_amdgcn_ballot_w64(digit >> b & 1);
      same &= digit >> b & 1 ? set : ~set;
    }
    if (in) {
      const int before = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
      const int first = mine[digit];
      __builtin_amdgcn_wave_barrier();  // every lane has read the place before its group's last lane moves it
      const int to = first + before;
      if ((same >> lane) == 1) mine[digit] = to + 1;
      p.key[(pass + 1) & 1][to] = key[u];
      p.pos[(pass + 1) & 1][to] = pass > 0 ? p.pos[pass & 1][i] : (int32_t)i;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Sums over the runs of equal symbols inside chunks of p.chunk sorted
// positions, 2^cl lanes per chunk and strip of columns.  A run inside one
// chunk is a row of the result; parts of longer runs go to part[chunk][0]
// (began before the chunk) or [1] (goes on after it).
template <typename T, int VEC, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_runs(EmbedGradParams p, int cl) {
  const int64_t col = (((int64_t)blockIdx.y << cl) + (threadIdx.x & ((1 << cl) - 1))) * VEC;
  const int64_t chunk = ((int64_t)blockIdx.x << (8 - cl)) + (threadIdx.x >> cl);
  const int64_t i0 = chunk * p.chunk, i1 = min(p.T, i0 + p.chunk);
  if (i0 >= p.T || col >= p.C) return;
  const uint32_t* key = p.key[p.passes & 1];
  const int32_t* pos = p.pos[p.passes & 1];
  uint32_t cur = key[i0];
  bool head = i0 > 0 && key[i0 - 1] == cur;
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  auto flush = [&](bool tail) __attribute__((always_inline)) {
    if (cur >= (uint32_t)p.V) return;  // padding
    if (head || tail) {
      store_n<float, VEC, WHOLE>(p.part + (2 * chunk + (head ? 0 : 1)) * p.C, col, p.C, s);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[e] *= p.scale;
      store_n<float, VEC, WHOLE>(p.dtable + (int64_t)cur * p.C, col, p.C, s);
    }
  };
  constexpr int AHEAD = 8;
  for (int64_t i = i0; i < i1; i += AHEAD) {
    uint32_t k[AHEAD];
    float v[AHEAD][VEC];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t at = min(i + u, i1 - 1);
      k[u] = key[at];
      load_n<T, VEC, WHOLE>(static_cast<const T*>(p.dout) + (int64_t)pos[at] * p.C, col, p.C, v[u]);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (i + u >= i1) break;
      if (k[u] != cur) {
        flush(false);
        cur = k[u];
        head = false;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[e] += v[u][e];
    }
  }
  flush(i1 < p.T && key[i1] == cur);
}

constexpr int kJoin = 512, kJoinLanes = 4;
// Rows whose runs cross chunks: the workgroup of the chunk in which a run
// begins sums its parts, kJoin / 2^cl groups of lanes taking every so many
// chunks, and then the groups' sums in order.
template <int VEC, bool WHOLE>
__global__ __launch_bounds__(kJoin) void k_embed_join(EmbedGradParams p, int cl) {
  __shared__ float sums[kJoin * VEC];
  const int64_t chunk = blockIdx.x, i0 = chunk * p.chunk, i1 = i0 + p.chunk;
  if (i1 >= p.T) return;
  const uint32_t* key = p.key[p.passes & 1];
  const uint32_t cur = key[i1 - 1];
  if (cur >= (uint32_t)p.V || key[i1] != cur || (i0 > 0 && key[i0 - 1] == cur)) return;  // whole workgroup
  const int lc = threadIdx.x & ((1 << cl) - 1), lr = threadIdx.x >> cl, rl = kJoin >> cl;
  const int64_t col = (((int64_t)blockIdx.y << cl) + lc) * VEC;
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  if (col < p.C) {
    if (lr == 0) load_n<float, VEC, WHOLE>(p.part + (2 * chunk + 1) * p.C, col, p.C, s);
    constexpr int AHEAD = 4;
    for (int64_t q = chunk + 1 + lr; q * p.chunk < p.T && key[q * p.chunk] == cur; q += AHEAD * rl) {
      float v[AHEAD][VEC];
      bool in[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int64_t at = q + u * rl;
        in[u] = at * p.chunk < p.T && key[at * p.chunk] == cur;
        if (in[u]) load_n<float, VEC, WHOLE>(p.part + 2 * at * p.C, col, p.C, v[u]);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (in[u])
#pragma unroll
          for (int e = 0; e < VEC; ++e) s[e] += v[u][e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] = s[e];
  for (int h = rl / 2; h > 0; h /= 2) {
    __syncthreads();
    if (lr < h)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] += sums[(threadIdx.x + (h << cl)) * VEC + e];
  }
  if (lr == 0 && col < p.C) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = sums[threadIdx.x * VEC + e] * p.scale;
    store_n<float, VEC, WHOLE>(p.dtable + (int64_t)cur * p.C, col, p.C, s);
  }
}

// Few positions: the workgroup of a symbol's first position lists all of its
// positions in order and sums their rows, groups of 2^cl lanes taking every so
// many of them, and then the groups' sums in order.
template <typename T, int VEC, bool WHOLE>
__global__ __launch_bounds__(256) void k_embed_few(EmbedGradParams p, int cl) {
  constexpr int PER = kEmbedFew / 256;  // positions of a thread, consecutive
  __shared__ int list[kEmbedFew];
  __shared__ int counts[5];
  __shared__ float sums[256 * VEC];
  const int t = blockIdx.x, n = (int)p.T, lane = lane_id(), wave = wave_id();
  const int64_t id = p.ids[t];
  if (id < 0 || id >= p.V) return;  // whole workgroup
  bool same[PER], earlier = false;
  int mine = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = threadIdx.x * PER + j;
    same[j] = i < n && p.ids[i] == id;
    earlier |= same[j] && i < t;
    mine += same[j];
  }
  if (__syncthreads_or(earlier)) return;
  // places: positions before this thread's, over the wave and the waves before
  int before = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(before, d);
    if (lane >= d) before += o;
  }
  if (lane == 63) counts[wave] = before;
  __syncthreads();
  int total = 0, base = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) base += counts[w];
    total += counts[w];
  }
  base += before - mine;
#pragma unroll
  for (int j = 0; j < PER; ++j)
    if (same[j]) list[base++] = threadIdx.x * PER + j;
  __syncthreads();
  const int lc = threadIdx.x & ((1 << cl) - 1), lr = threadIdx.x >> cl, rl = 256 >> cl;
  const int64_t col = (((int64_t)blockIdx.y << cl) + lc) * VEC;
  float s[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s[e] = 0.f;
  if (col < p.C) {
    constexpr int AHEAD = 8;
    for (int q = lr; q < total; q += AHEAD * rl) {
      float v[AHEAD][VEC];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        load_n<T, VEC, WHOLE>(static_cast<const T*>(p.dout) + (int64_t)list[min(q + u * rl, total - 1)] * p.C, col, p.C, v[u]);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (q + u * rl < total)
#pragma unroll
          for (int e = 0; e < VEC; ++e) s[e] += v[u][e];
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] = s[e];
  for (int h = rl / 2; h > 0; h /= 2) {
    __syncthreads();
    if (lr < h)
#pragma unroll
      for (int e = 0; e < VEC; ++e) sums[threadIdx.x * VEC + e] += sums[(threadIdx.x + (h << cl)) * VEC + e];
  }
  if (lr == 0 && col < p.C) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) s[e] = sums[threadIdx.x * VEC + e] * p.scale;
    store_n<float, VEC, WHOLE>(p.dtable + id * p.C, col, p.C, s);
  }
}

template <typename T, int VEC, bool WHOLE>
void embed_sums(const EmbedGradParams& p, hipStream_t s) {
  const int64_t lanes = (p.C + VEC - 1) / VEC, chunks = (p.T + p.chunk - 1) / p.chunk;
  const int cl = pow2_log2(lanes, 6);
  const unsigned strips = (unsigned)((lanes + (1 << cl) - 1) >> cl), per = 256u >> cl;
  k_embed_runs<T, VEC, WHOLE><<<dim3((unsigned)((chunks + per - 1) / per), strips), 256, 0, s>>>(p, cl);
  if (chunks > 1) {
    // narrow strips: one symbol may have every chunk, and its parts are then
    // joined by a single workgroup per strip
    const int jl = std::min(cl, kJoinLanes);
    k_embed_join<VEC, WHOLE><<<dim3((unsigned)(chunks - 1), (unsigned)((lanes + (1 << jl) - 1) >> jl)), kJoin, 0, s>>>(p, jl);
  }
}

}  // namespace

template <typename T>
hipError_t launch_embed(const EmbedParams& p, hipStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  const int64_t lanes = p.C >= V ? (p.C + V - 1) / V : p.C;
  const int cl = pow2_log2(lanes, 8), rows = 4 * (256 >> cl);
  const dim3 grid((unsigned)((p.T + rows - 1) / rows), (unsigned)((lanes + (1 << cl) - 1) >> cl));
  if (p.C % V == 0) k_embed<T, V, true><<<grid, 256, 0, s>>>(p, cl);
  else if (p.C > V) k_embed<T, V, false><<<grid, 256, 0, s>>>(p, cl);
  else k_embed<T, 1, true><<<grid, 256, 0, s>>>(p, cl);
  return hipGetLastError();
}
template hipError_t launch_embed<float>(const EmbedParams&, hipStream_t);
template hipError_t launch_embed<__bf16>(const EmbedParams&, hipStream_t);

template <typename T, int VEC, bool WHOLE>
void embed_unsorted(const EmbedGradParams& p, hipStream_t s) {
  const int64_t lanes = (p.C + VEC - 1) / VEC;
  const int cl = pow2_log2(lanes, 5);  // eight groups at least: one symbol may have every position
  k_embed_few<T, VEC, WHOLE><<<dim3((unsigned)p.T, (unsigned)((lanes + (1 << cl) - 1) >> cl)), 256, 0, s>>>(p, cl);
}
template <int TILE> void embed_sort(const EmbedGradParams& p, hipStream_t s) {
  const int nb = (int)((p.T + TILE - 1) / TILE);
  for (int pass = 0; pass < p.passes; ++pass) {
    k_embed_count<TILE><<<dim3(pass ? nb : std::max(nb, clear_groups(p.V * p.C))), 256, 0, s>>>(p, pass, nb);
    k_embed_scan<<<dim3(1u << p.bits), 64, 0, s>>>(p, nb);
    k_embed_scatter<TILE><<<dim3(nb), 256, 0, s>>>(p, pass, nb);
  }
}

template <typename T>
hipError_t launch_embed_grad(const EmbedGradParams& p, hipStream_t s) {
  // 16 bytes of a row of dOut per lane; the sums are stored as whole vectors too
  constexpr int V = 16 / (int)sizeof(T);
  const bool whole = p.C % V == 0, cut = p.C > V;
  if (embed_few(p.T, p.C)) {
    const int64_t n = p.V * p.C;
    k_embed_clear<<<dim3(clear_groups(n)), 256, 0, s>>>(p.dtable, n);
    if (whole) embed_unsorted<T, V, true>(p, s);
    else if (cut) embed_unsorted<T, V, false>(p, s);
    else embed_unsorted<T, 1, true>(p, s);
    return hipGetLastError();
  }
  if (embed_tile(p.T) == kEmbedTileSmall) embed_sort<kEmbedTileSmall>(p, s);
  else embed_sort<kEmbedTile>(p, s);
  if (whole) embed_sums<T, V, true>(p, s);
  else if (cut) embed_sums<T, V, false>(p, s);
  else embed_sums<T, 1, true>(p, s);
  return hipGetLastError();
}
template hipError_t launch_embed_grad<float>(const EmbedGradParams&, hipStream_t);
template hipError_t launch_embed_grad<__bf16>(const EmbedGradParams&, hipStream_t);

}  // namespace flarepp
