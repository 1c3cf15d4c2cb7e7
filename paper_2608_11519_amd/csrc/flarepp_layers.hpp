// Parameter blocks and launchers of the operators around the mixer: linear
// layer, embedding, optimiser step.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace flarepp {

// ---- linear layer ------------------------------------------------------------
enum Activation { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// The three products of a linear layer, C[P][Q] = sum_k L(p, k) R(k, q), row-major C:
//   kLinForward  P = tokens, Q = outputs, k = inputs:  L = X rows, R = W
//   kLinInput    P = tokens, Q = inputs,  k = outputs: L = dP rows, R = W^T
//   kLinWeight   P = inputs, Q = outputs, k = tokens:  L = X^T, R = dP
// A k-contiguous operand is stored [rows][K], the others [K][rows] ("T").
enum LinProduct { kLinForward = 0, kLinInput = 1, kLinWeight = 2 };
constexpr bool lin_l_t(int prod) { return prod == kLinWeight; }
constexpr bool lin_r_t(int prod) { return prod != kLinInput; }

// Output tiles (P x Q) of a workgroup
enum LinTile { kTile128 = 0, kTile64 = 1, kTile128x32 = 2, kTile32x128 = 3, kTile256 = 4 };

struct LinGemmParams {
  const void* l; const void* r;
  const void* r_lo;        // kLinWeight, bf16: R = r + r_lo, or null
  int64_t P, Q, K;
  int splits; int64_t kchunk;  // split z sums k in [z * kchunk, (z + 1) * kchunk); a multiple of lin_step
  float* part; int64_t part_stride;  // fp32 sums per split, or null: the epilogue
  const void* bias; const void* res; void* out; void* pre;
  int act;
};
// reduction elements of one step
constexpr int lin_step(int elem_bytes) { return 128 / elem_bytes; }
// Whether the operands can be copied straight to LDS: whole 16-byte chunks,
// and whole steps where the reduction is contiguous.
bool lin_direct(int prod, int elem_bytes, int64_t P, int64_t Q, int64_t K);
template <typename T> hipError_t launch_lin_gemm(const LinGemmParams&, int prod, int tile, bool direct, hipStream_t);

// The input and the weight gradient in one launch, both in 64 x 64 tiles
template <typename T> hipError_t launch_lin_pair(const LinGemmParams& dx, const LinGemmParams& dw, bool direct, hipStream_t);

// The same product for many rows and a strip of outputs (32, 64, 128 or 256
// wide) whose weights fit the LDS.
constexpr size_t kLinRowsLds = 160 * 1024;
size_t lin_rows_lds(int elem_bytes, int strip, int64_t K);
int lin_rows_strip(int prod, int elem_bytes, int64_t P, int64_t Q, int64_t K);
template <typename T>
hipError_t launch_lin_rows(const LinGemmParams&, int prod, int strip, hipStream_t);

// out = epilogue of the sum over the splits of part
template <typename T> hipError_t launch_lin_finish(const LinGemmParams&, hipStream_t);

// dP = dOut * act'(pre): fp32 type one array, bf16 type hi (+ lo when given);
// and the column sums of dP per chunk of rows.  act none: sums only.
struct LinSlopeParams {
  const void* dout; const void* pre; int act;
  int64_t T; int64_t N;
  void* dp; void* dp_lo;   // or null
  float* part; int64_t part_ld;  // [nchunks][part_ld] column sums, or null
  int nchunks; int64_t chunk;
};
template <typename T> hipError_t launch_lin_slope(const LinSlopeParams&, hipStream_t);

// bf16: dP, dbias, dW and (fused) dX in one pass over the tokens
struct LinBwdParams {
  const void *x, *w, *pre, *dout;
  void* dx;                 // fused: or null
  void* hi;                 // not fused, act: dP rounded to bf16, or null
  float* part; int64_t part_stride;      // [nchunks] dW of each chunk, or null
  float* bias_part; int64_t bias_ld;     // [nchunks][bias_ld], or null
  int64_t T, K, N, chunk;
  int nchunks, act;
};
bool lin_bwd_tile(int64_t T, int64_t K, int64_t N, int act, int& kt, int& nt, bool& fused);
hipError_t launch_lin_bwd(const LinBwdParams&, int kt, int nt, bool fused, hipStream_t);

// out[i] = sum_s part[s * stride + i], i < n: two independent jobs in a launch
struct LinSumJob { const float* part; int64_t stride, n; int splits; float* out; };
struct LinSumParams { LinSumJob job[2]; int njobs; };
hipError_t launch_lin_sum(const LinSumParams&, hipStream_t);

// ---- embedding -----------------------------------------------------------------
struct EmbedParams {
  const int64_t* ids; const void* table; void* out;
  int64_t T, V, C;
  float scale;
};
template <typename T> hipError_t launch_embed(const EmbedParams&, hipStream_t);

struct EmbedGradParams {
  const int64_t* ids; const void* dout;
  int64_t T, V, C;
  float scale;
  float* dtable;
  // sort workspace: keys and positions of a pass and of the next, counts per
  // (digit, workgroup) and per digit
  uint32_t* key[2]; int32_t* pos[2];
  int32_t* counts; int32_t* totals;
  float* part;  // [chunks][2][C]: the sums of runs that cross a chunk's start, end
  int passes, bits;
  int chunk;  // sorted positions summed by one group of lanes
};
// Positions up to which no sort is needed: every position looks through all of
// them, once per strip of columns, so up to 2048 and by T * T * C.  Unsorted /
// sorted, us: 300 x 256 (30,000 symbols) 12 / 30; 2048 x 256 21 / 36, x 512 35 / 41, x 1024
// 61 / 48; 1536 x 1024 47 / 47; 4096 x 128 (256 symbols) 35 / 20.
constexpr int kEmbedFew = 2048;
inline bool embed_few(int64_t T, int64_t C) { return T <= kEmbedFew && T * T * C <= int64_t(5) << 29; }
// positions of a workgroup of the sort: small ones until they would make more
// workgroups than the card takes at once
constexpr int kEmbedTileSmall = 512, kEmbedTile = 2048;
constexpr int embed_tile(int64_t T) { return T <= (1 << 18) ? kEmbedTileSmall : kEmbedTile; }
// Sorted positions summed by one group of lanes: few, so that there are waves
// enough, while joining the parts of long runs costs little.  Chunks of 16 / 32 /
// 64 / 128: 16,384 positions x 512 25 / 26 / 30 us; 65,536 x 256 (words) 54 / 53 / 59;
// 131,072 x 128 (256 symbols) 41 / 38 / 36 / 41; 1,048,576 x 128 188 / 145 / 123 / 112.
constexpr int embed_chunk(int64_t T) { return T < (1 << 15) ? 16 : T < (1 << 17) ? 32 : T <= (1 << 19) ? 64 : 128; }
template <typename T> hipError_t launch_embed_grad(const EmbedGradParams&, hipStream_t);

// ---- optimiser ------------------------------------------------------------------
constexpr int kAdamwBlock = 256;      // elements that share a scale
constexpr int kAdamwTurns = 2;        // of them per wave
constexpr int64_t kAdamwUnit = 4 * kAdamwBlock * kAdamwTurns;  // elements of a workgroup
constexpr int kAdamwPerLaunch = 40;   // tensors of a launch: their table travels as a kernel argument
struct AdamwSchedule {
  double lr;
  float size;     // lr / (1 - b1^t)
  float root;     // 1 / sqrt(1 - b2^t)
  uint32_t step;  // t
  uint32_t pad;
};
struct AdamwTensor {
  float* p; const float* g; void* m; void* v; float* m_scale; float* v_scale; void* p_low;
  int64_t n;
  double decay;
};
struct AdamwParams {
  int first[kAdamwPerLaunch];  // workgroups of the tensors before each one
  AdamwTensor t[kAdamwPerLaunch];
  int count, blocks;
  float b1, a1, b2, a2, eps;
  AdamwSchedule now;              // what changes from step to step,
  const AdamwSchedule* schedule;  // or null: in device memory
};
hipError_t launch_adamw(const AdamwParams&, bool q8, hipStream_t);

}  // namespace flarepp
