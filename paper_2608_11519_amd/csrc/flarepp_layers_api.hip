// C ABI of the operators around the mixer (linear layer, embedding, optimiser
// step): argument checks, workspace layout and launch sequencing.
// Declarations and the contract of every entry point are in include/flarepp.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <initializer_list>
#include <new>
#include <vector>

#include "../../include/flarepp.h"
#include "flarepp_layers.hpp"

namespace flarepp {
int api_error(int code, const char* text);
int api_ok();
}  // namespace flarepp

namespace {

using namespace flarepp;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return api_error(code, buf);
}

#define TRY(x) do { int _rc = (x); if (_rc != FLAREPP_OK) return _rc; } while (0)
#define HIPTRY(x) do { hipError_t _e = (x); if (_e != hipSuccess) \
    return fail(FLAREPP_ERR_HIP, "%s: %s", #x, hipGetErrorString(_e)); } while (0)

constexpr int64_t kMaxRows = int64_t(1) << 30;
constexpr int64_t kMaxWidth = 1 << 16;
constexpr int64_t kMaxElems = int64_t(1) << 40;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

int check_dtype(int dtype) {
  if (dtype != FLAREPP_F32 && dtype != FLAREPP_BF16)
    return fail(FLAREPP_ERR_UNSUPPORTED, "unknown dtype %d (expected FLAREPP_F32=0 or FLAREPP_BF16=1)", dtype);
  return FLAREPP_OK;
}
int check_size(int64_t v, const char* name, int64_t most) {
  if (v < 1) return fail(FLAREPP_ERR_INVALID_ARG, "%s=%lld must be >= 1", name, (long long)v);
  if (v > most) return fail(FLAREPP_ERR_UNSUPPORTED, "%s=%lld exceeds %lld", name, (long long)v, (long long)most);
  return FLAREPP_OK;
}
int check_ptr(const void* p, const char* name, bool may_be_null = false) {
  if (!p) return may_be_null ? FLAREPP_OK : fail(FLAREPP_ERR_INVALID_ARG, "%s is NULL", name);
  if (reinterpret_cast<uintptr_t>(p) & 15) return fail(FLAREPP_ERR_INVALID_ARG, "%s is not 16-byte aligned", name);
  return FLAREPP_OK;
}
int check_ws(const void* ws, size_t have, size_t need) {
  if (!need) return FLAREPP_OK;
  if (!ws) return fail(FLAREPP_ERR_WORKSPACE, "workspace is NULL (%zu bytes required)", need);
  if (reinterpret_cast<uintptr_t>(ws) & 15) return fail(FLAREPP_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  if (have < need)
    return fail(FLAREPP_ERR_WORKSPACE, "workspace of %zu bytes is smaller than the %zu required", have, need);
  return FLAREPP_OK;
}

// A buffer that a call reads or writes; no written one may overlap another.
struct Range {
  uintptr_t from, to;
  bool written;
};
Range range(const void* p, int64_t bytes, bool written) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return {a, p ? a + (uintptr_t)bytes : a, written};
}
int check_disjoint(std::initializer_list<Range> rs) {
  for (const Range* x = rs.begin(); x != rs.end(); ++x)
    for (const Range* y = x + 1; y != rs.end(); ++y)
      if ((x->written || y->written) && x->from < y->to && y->from < x->to)
        return fail(FLAREPP_ERR_INVALID_ARG, "an output overlaps another buffer of the call");
  return FLAREPP_OK;
}

struct Carver {
  char* base;
  size_t off = 0;
  void* take(size_t bytes) {
    void* p = base ? base + off : nullptr;
    off += (bytes + 255) & ~size_t(255);
    return p;
  }
};

// ---- linear layer ----------------------------------------------------------------
int check_linear_shape(int dtype, int act, int64_t T, int64_t K, int64_t N) {
  TRY(check_dtype(dtype));
  if (act < FLAREPP_ACT_NONE || act > FLAREPP_ACT_SILU)
    return fail(FLAREPP_ERR_UNSUPPORTED, "unknown activation %d (FLAREPP_ACT_NONE .. FLAREPP_ACT_SILU)", act);
  TRY(check_size(T, "T", kMaxRows));
  TRY(check_size(K, "K", kMaxWidth));
  TRY(check_size(N, "N", kMaxWidth));
  if (T * std::max(K, N) > kMaxElems) return fail(FLAREPP_ERR_UNSUPPORTED, "T * max(K, N) too large");
  return FLAREPP_OK;
}

struct LinPlan {
  int strip;  // not 0: k_linear_rows with strips of this width
  int tile, splits;
  bool direct;
  int64_t kchunk, part_stride;
  size_t part_bytes;  // fp32 sums per split (0: the product runs its epilogue)
};

// Tile by the product's shape: narrow ones (at most 32 outputs or rows) take a
// narrow tile, others 128 x 128 where these give every CU a workgroup, else
// 64 x 64.  The weight gradient, whose tokens can be split, takes 128 x 128 where
// its tiles times tokens times bytes of an element pass 2^19, else 64 x 64, which split
// finer and let both products of a backward go in one launch.  Both products, 128 x 128 /
// 64 x 64, us: bf16 2000 x 1000 x 1000 44 / 30, 16,384 x 512 x 512 44 / 42, 4096 x 1024 x
// 1024 48 / 46, 8000 x 1000 x 1000 67 / 76, 4096 x 2048 x 2048 93 / 126; fp32 2000 x 1000 x
// 1000 96 / 82, 60,969 x 128 x 256 104 / 100, 8000 x 512 x 640 118 / 121, 8000 x 1000 x 1000
// 278 / 324; off at fp32 21,668 x 274 x 459 (212 / 190).  A reduction is
// split when the tiles alone would leave CUs idle: the weight gradient's, or that
// of a forward or input-gradient product of eight steps or more (fewer cost less
// than the second launch).
LinPlan lin_plan(int prod, int bs, int64_t P, int64_t Q, int64_t K) {
  LinPlan pl{};
  const int64_t bk = lin_step(bs), steps = cdiv(K, bk);
  const bool weight = prod == kLinWeight;
  pl.splits = 1;
  pl.strip = lin_rows_strip(prod, bs, P, Q, K);
  if (pl.strip) return pl;
  int64_t bp, bq;
  if (Q <= 32 && P > 64) { pl.tile = kTile128x32; bp = 128; bq = 32; }
  else if (P <= 32 && Q > 64) { pl.tile = kTile32x128; bp = 32; bq = 128; }
  else if (P > 64 && Q > 64 && (weight ? cdiv(P, 128) * cdiv(Q, 128) * K * bs > (1 << 19)
                                        : cdiv(P, 128) * cdiv(Q, 128) >= 256)) { pl.tile = kTile128; bp = bq = 128; }
  else { pl.tile = kTile64; bp = bq = 64; }
  if (pl.tile == kTile128 && !weight && bs == 2 && lin_direct(prod, bs, P, Q, K)) {
    // 256 x 256 where they fill the CUs' rounds to three quarters and pass the
    // outputs' end by little: with GELU 8192 x 2048 -> 2048 74 / 82 us (128 x 128), 65,536 x
    // 1024 -> 512 91 / 106; but 60,969 x 1248 -> 200 99 / 72, 4096 x 2048 -> 2048 73 / 40
    const int64_t t = cdiv(P, 256) * cdiv(Q, 256);
    if (4 * t >= 3 * 256 * cdiv(t, 256) && 8 * cdiv(Q, 256) * 256 <= 9 * Q) { pl.tile = kTile256; bp = bq = 256; }
  }
  pl.direct = (pl.tile == kTile256 || pl.tile == kTile128 || pl.tile == kTile64) && lin_direct(prod, bs, P, Q, K);
  const int64_t tiles = cdiv(P, bp) * cdiv(Q, bq);
  int64_t splits = 1;
  if (tiles < 256 && steps >= 8) splits = std::min(cdiv(512, tiles), steps / 4);
  const int64_t per = cdiv(steps, splits);
  pl.splits = (int)cdiv(steps, per);
  pl.kchunk = per * bk;
  pl.part_stride = cdiv(P * Q, 4) * 4;
  pl.part_bytes = pl.splits > 1 ? sizeof(float) * pl.splits * pl.part_stride : 0;
  return pl;
}

LinGemmParams lin_params(const LinPlan& pl, int64_t P, int64_t Q, int64_t K, const void* l, const void* r, void* part) {
  LinGemmParams p{};
  p.l = l; p.r = r; p.P = P; p.Q = Q; p.K = K;
  p.splits = pl.splits; p.kchunk = pl.kchunk; p.part_stride = pl.part_stride;
  p.part = pl.part_bytes ? static_cast<float*>(part) : nullptr;
  return p;
}

template <typename T>
int run_linear(int act, int64_t rows, int64_t K, int64_t N, const void* X, const void* W, const void* bias, const void* res,
               void* out, void* pre, void* ws, hipStream_t s) {
  const LinPlan pl = lin_plan(kLinForward, sizeof(T), rows, N, K);
  LinGemmParams p = lin_params(pl, rows, N, K, X, W, ws);
  p.bias = bias; p.res = res; p.out = out; p.pre = pre; p.act = act;
  if (pl.strip) HIPTRY(launch_lin_rows<T>(p, kLinForward, pl.strip, s));
  else HIPTRY(launch_lin_gemm<T>(p, kLinForward, pl.tile, pl.direct, s));
  if (p.part) HIPTRY(launch_lin_finish<T>(p, s));
  return api_ok();
}

struct LinBwdWs {
  LinPlan dx, dw;
  bool pass, fused;  // one pass over the tokens; dX in it
  int kt, nt;
  void *dp, *dp_lo, *part;
  float* bias_part;
  int64_t bias_ld, chunk;
  int nchunks;
  size_t bytes;
};

LinBwdWs lin_bwd_ws(void* base, int dtype, int act, int64_t rows, int64_t K, int64_t N) {
  const size_t bs = dtype == FLAREPP_F32 ? 4 : 2;
  LinBwdWs w{};
  w.dx = lin_plan(kLinInput, (int)bs, rows, K, N);
  w.dw = lin_plan(kLinWeight, (int)bs, K, N, rows);
  Carver cv{static_cast<char*>(base)};
  if (act != FLAREPP_ACT_NONE) {
    w.dp = cv.take(bs * rows * N);
    if (dtype == FLAREPP_BF16) w.dp_lo = cv.take(bs * rows * N);
  }
  // (few rows: one chunk, and no sum of partials)
  w.chunk = rows <= 128 ? rows : std::max<int64_t>(32, cdiv(rows, 512));
  w.pass = dtype == FLAREPP_BF16 && lin_bwd_tile(rows, K, N, act, w.kt, w.nt, w.fused);
  if (w.pass) {  // a workgroup per CU, of two steps at least
    const int64_t tiles = (K / w.kt) * (N / w.nt);
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(256 / tiles, rows / 64));
    w.chunk = cdiv(cdiv(rows, groups), 32) * 32;
  }
  w.nchunks = (int)cdiv(rows, w.chunk);
  if (w.pass) w.dw.part_bytes = std::max(w.dw.part_bytes, sizeof(float) * w.nchunks * w.dw.part_stride);
  w.bias_ld = cdiv(N, 4) * 4;
  w.bias_part = static_cast<float*>(cv.take(sizeof(float) * w.nchunks * w.bias_ld));
  // the sums per split of the two products, one after the other
  w.part = cv.take(std::max(w.dx.part_bytes, w.dw.part_bytes));
  w.bytes = cv.off;
  return w;
}

template <typename T>
int run_linear_backward(int dtype, int act, int64_t rows, int64_t K, int64_t N, const void* X, const void* W, const void* pre,
                        const void* dOut, void* dX, float* dW, float* dbias, void* ws, hipStream_t s) {
  const LinBwdWs w = lin_bwd_ws(ws, dtype, act, rows, K, N);
  const void* dp = dOut;
  if (w.pass && dW) {
    LinBwdParams p{};
    p.x = X; p.w = W; p.pre = pre; p.dout = dOut;
    p.dx = w.fused ? dX : nullptr;
    p.hi = !w.fused && dX ? w.dp : nullptr;
    p.part = static_cast<float*>(w.part); p.part_stride = w.dw.part_stride;
    p.bias_part = dbias ? w.bias_part : nullptr; p.bias_ld = w.bias_ld;
    p.T = rows; p.K = K; p.N = N; p.chunk = w.chunk; p.nchunks = w.nchunks; p.act = act;
    HIPTRY(launch_lin_bwd(p, w.kt, w.nt, w.fused, s));
    LinSumParams sums{};
    sums.job[sums.njobs++] = {p.part, p.part_stride, K * N, w.nchunks, dW};
    if (dbias) sums.job[sums.njobs++] = {w.bias_part, w.bias_ld, N, w.nchunks, dbias};
    HIPTRY(launch_lin_sum(sums, s));
    if (dX && !w.fused) {
      LinGemmParams q = lin_params(w.dx, rows, K, N, act != FLAREPP_ACT_NONE ? w.dp : dOut, W, w.part);
      q.out = dX;
      if (w.dx.strip) HIPTRY(launch_lin_rows<T>(q, kLinInput, w.dx.strip, s));
      else HIPTRY(launch_lin_gemm<T>(q, kLinInput, w.dx.tile, w.dx.direct, s));
      if (q.part) HIPTRY(launch_lin_finish<T>(q, s));
    }
    return api_ok();
  }
  if (act != FLAREPP_ACT_NONE || dbias) {
    LinSlopeParams p{};
    p.dout = dOut; p.pre = pre; p.act = act; p.T = rows; p.N = N;
    if (act != FLAREPP_ACT_NONE) {
      p.dp = w.dp;
      p.dp_lo = dW ? w.dp_lo : nullptr;
      dp = w.dp;
    }
    p.part = w.nchunks == 1 ? dbias : dbias ? w.bias_part : nullptr;
    p.part_ld = w.bias_ld; p.nchunks = w.nchunks; p.chunk = w.chunk;
    HIPTRY(launch_lin_slope<T>(p, s));
  }
  LinGemmParams px = lin_params(w.dx, rows, K, N, dp, W, w.part);
  px.out = dX;
  LinGemmParams pw = lin_params(w.dw, K, N, rows, X, dp, w.part);
  pw.r_lo = act != FLAREPP_ACT_NONE ? w.dp_lo : nullptr;
  LinSumParams sums{};
  if (dW) {
    if (pw.part) sums.job[sums.njobs++] = {pw.part, pw.part_stride, K * N, pw.splits, dW};
    else pw.part = dW;
  }
  // small products go together (the partial sums of both never share the workspace)
  if (dX && dW && !px.part && !w.dx.strip && w.dx.tile == kTile64 && w.dw.tile == kTile64) {
    HIPTRY(launch_lin_pair<T>(px, pw, w.dx.direct && w.dw.direct, s));
  } else {
    if (dX) {
      if (w.dx.strip) HIPTRY(launch_lin_rows<T>(px, kLinInput, w.dx.strip, s));
      else HIPTRY(launch_lin_gemm<T>(px, kLinInput, w.dx.tile, w.dx.direct, s));
      if (px.part) HIPTRY(launch_lin_finish<T>(px, s));
    }
    if (dW) HIPTRY(launch_lin_gemm<T>(pw, kLinWeight, w.dw.tile, w.dw.direct, s));
  }
  if (dbias && w.nchunks > 1) sums.job[sums.njobs++] = {w.bias_part, w.bias_ld, N, w.nchunks, dbias};
  if (sums.njobs) HIPTRY(launch_lin_sum(sums, s));
  return api_ok();
}

// ---- embedding ---------------------------------------------------------------------
int check_embedding_shape(int dtype, int64_t T, int64_t V, int64_t C) {
  TRY(check_dtype(dtype));
  TRY(check_size(T, "T", kMaxRows));
  TRY(check_size(V, "V", kMaxRows));
  TRY(check_size(C, "C", kMaxWidth));
  if (std::max(T, V) * C > kMaxElems) return fail(FLAREPP_ERR_UNSUPPORTED, "max(T, V) * C too large");
  return FLAREPP_OK;
}

size_t embed_ws(EmbedGradParams& p, void* base) {
  int bits = 1;
  while ((int64_t(1) << bits) <= p.V) ++bits;  // symbols 0 .. V - 1, and V for padding
  p.passes = (bits + 9) / 10;
  p.bits = (bits + p.passes - 1) / p.passes;
  if (embed_few(p.T, p.C)) return 0;
  p.chunk = embed_chunk(p.T);
  const int64_t nb = cdiv(p.T, embed_tile(p.T)), chunks = cdiv(p.T, p.chunk);
  Carver cv{static_cast<char*>(base)};
  for (int i = 0; i < 2; ++i) {
    p.key[i] = static_cast<uint32_t*>(cv.take(4 * p.T));
    p.pos[i] = static_cast<int32_t*>(cv.take(4 * p.T));
  }
  p.counts = static_cast<int32_t*>(cv.take(sizeof(int32_t) * (nb << p.bits)));
  p.totals = static_cast<int32_t*>(cv.take(sizeof(int32_t) << p.bits));
  p.part = static_cast<float*>(cv.take(sizeof(float) * 2 * chunks * p.C));
  return cv.off;
}

// ---- optimiser -----------------------------------------------------------------------
// The same for many buffers.
int check_ranges(std::vector<Range>& r) {
  std::sort(r.begin(), r.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t any = 0, written = 0;
  for (const Range& x : r) {
    if (x.from < (x.written ? any : written))
      return fail(FLAREPP_ERR_INVALID_ARG, "a buffer that the step writes overlaps another of its buffers");
    any = std::max(any, x.to);
    if (x.written) written = std::max(written, x.to);
  }
  return FLAREPP_OK;
}

bool unit_interval(double b) { return b >= 0.0 && b < 1.0; }

void adamw_schedule(AdamwSchedule& a, double lr, double beta1, double beta2, int64_t step) {
  a.lr = lr;
  a.size = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
  a.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
  a.step = (uint32_t)step;
  a.pad = 0;
}

int check_adamw_hyper(double lr, double beta1, double beta2, int64_t step) {
  if (!(lr >= 0.0) || !std::isfinite(lr)) return fail(FLAREPP_ERR_INVALID_ARG, "lr=%g must be finite and >= 0", lr);
  if (!unit_interval(beta1) || !unit_interval(beta2))
    return fail(FLAREPP_ERR_INVALID_ARG, "beta1=%g, beta2=%g must be in [0, 1)", beta1, beta2);
  return check_size(step, "step", int64_t(1) << 31);
}

int adamw_entry(int state, int64_t count, const flarepp_adamw_tensor* tensors, double lr, double beta1, double beta2, double eps,
                int64_t step, const void* schedule, void* stream) {
  if (state != FLAREPP_STATE_F32 && state != FLAREPP_STATE_E4M3)
    return fail(FLAREPP_ERR_UNSUPPORTED, "unknown state %d (FLAREPP_STATE_F32=0 or FLAREPP_STATE_E4M3=1)", state);
  const bool q8 = state == FLAREPP_STATE_E4M3;
  TRY(check_size(count, "count", 1 << 20));
  if (!tensors) return fail(FLAREPP_ERR_INVALID_ARG, "tensors is NULL");
  TRY(check_adamw_hyper(lr, beta1, beta2, step));
  if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(FLAREPP_ERR_INVALID_ARG, "eps=%g must be finite and >= 0", eps);
  TRY(check_ptr(schedule, "schedule", true));
  std::vector<Range> ranges;
  ranges.reserve(7 * count);
  for (int64_t i = 0; i < count; ++i) {
    const flarepp_adamw_tensor& t = tensors[i];
    TRY(check_size(t.n, "n", kMaxElems));
    if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.0)
      return fail(FLAREPP_ERR_INVALID_ARG, "weight_decay=%g must be finite and >= 0", t.weight_decay);
    const int64_t blocks = cdiv(t.n, kAdamwBlock);
    const struct { const void* p; const char* name; int64_t bytes; bool used, written; } bufs[] = {
        {t.p, "p", 4 * t.n, true, true},          {t.g, "g", 4 * t.n, true, false},
        {t.m, "m", (q8 ? 1 : 4) * t.n, true, true}, {t.v, "v", (q8 ? 1 : 4) * t.n, true, true},
        {t.m_scale, "m_scale", 4 * blocks, q8, true}, {t.v_scale, "v_scale", 4 * blocks, q8, true},
        {t.p_low, "p_low", 2 * t.n, t.p_low != nullptr, true}};
    for (const auto& b : bufs) {
      if (!b.used) {
        if (b.p) return fail(FLAREPP_ERR_INVALID_ARG, "%s of tensor %lld is given but the state has no scales", b.name, (long long)i);
        continue;
      }
      TRY(check_ptr(b.p, b.name));
      ranges.push_back(range(b.p, b.bytes, b.written));
    }
  }
  TRY(check_ranges(ranges));
  AdamwParams p{};
  p.b1 = (float)beta1; p.a1 = (float)(1.0 - beta1);
  p.b2 = (float)beta2; p.a2 = (float)(1.0 - beta2);
  p.eps = (float)eps;
  adamw_schedule(p.now, lr, beta1, beta2, step);
  p.schedule = static_cast<const AdamwSchedule*>(schedule);
  for (int64_t i = 0; i < count;) {
    p.count = 0;
    int64_t blocks = 0;
    for (; i < count && p.count < kAdamwPerLaunch; ++i) {
      const flarepp_adamw_tensor& t = tensors[i];
      const int64_t more = cdiv(t.n, kAdamwUnit);
      if (p.count && blocks + more > (1 << 30)) break;
      p.first[p.count] = (int)blocks;
      p.t[p.count++] = {(float*)t.p, (const float*)t.g, t.m, t.v, (float*)t.m_scale, (float*)t.v_scale, t.p_low,
                        t.n, t.weight_decay};
      blocks += more;
    }
    p.blocks = (int)blocks;
    HIPTRY(launch_adamw(p, q8, static_cast<hipStream_t>(stream)));
  }
  return api_ok();
}

}  // namespace

extern "C" {

size_t flarepp_linear_workspace_bytes(int dtype, int64_t T, int64_t K, int64_t N) {
  if (check_linear_shape(dtype, FLAREPP_ACT_NONE, T, K, N) != FLAREPP_OK) return 0;
  return std::max<size_t>(256, lin_plan(kLinForward, dtype == FLAREPP_F32 ? 4 : 2, T, N, K).part_bytes);
}

int flarepp_linear_forward(int dtype, int act, int64_t T, int64_t K, int64_t N, const void* X, const void* W, const void* bias,
                           const void* residual, void* out, void* pre, void* ws, size_t ws_bytes, void* stream) {
  TRY(check_linear_shape(dtype, act, T, K, N));
  TRY(check_ptr(X, "X"));
  TRY(check_ptr(W, "W"));
  TRY(check_ptr(bias, "bias", true));
  TRY(check_ptr(residual, "residual", true));
  TRY(check_ptr(out, "out"));
  TRY(check_ptr(pre, "pre", true));
  const int64_t bs = dtype == FLAREPP_F32 ? 4 : 2;
  const size_t need = lin_plan(kLinForward, (int)bs, T, N, K).part_bytes;
  TRY(check_ws(ws, ws_bytes, need));
  TRY(check_disjoint({range(X, bs * T * K, false), range(W, bs * K * N, false), range(bias, bs * N, false),
                      range(residual == out ? nullptr : residual, bs * T * N, false), range(out, bs * T * N, true),
                      range(pre, bs * T * N, true), range(need ? ws : nullptr, need, true)}));
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == FLAREPP_F32 ? run_linear<float>(act, T, K, N, X, W, bias, residual, out, pre, ws, s)
                              : run_linear<__bf16>(act, T, K, N, X, W, bias, residual, out, pre, ws, s);
}

size_t flarepp_linear_backward_workspace_bytes(int dtype, int act, int64_t T, int64_t K, int64_t N) {
  if (check_linear_shape(dtype, act, T, K, N) != FLAREPP_OK) return 0;
  return lin_bwd_ws(nullptr, dtype, act, T, K, N).bytes;
}

int flarepp_linear_backward(int dtype, int act, int64_t T, int64_t K, int64_t N, const void* X, const void* W, const void* pre,
                            const void* dOut, void* dX, float* dW, float* dbias, void* ws, size_t ws_bytes, void* stream) {
  TRY(check_linear_shape(dtype, act, T, K, N));
  if (!dX && !dW && !dbias) return fail(FLAREPP_ERR_INVALID_ARG, "dX, dW and dbias are all NULL");
  TRY(check_ptr(X, "X", !dW));
  TRY(check_ptr(W, "W", !dX));
  TRY(check_ptr(pre, "pre", act == FLAREPP_ACT_NONE));
  TRY(check_ptr(dOut, "dOut"));
  TRY(check_ptr(dX, "dX", true));
  TRY(check_ptr(dW, "dW", true));
  TRY(check_ptr(dbias, "dbias", true));
  const int64_t bs = dtype == FLAREPP_F32 ? 4 : 2;
  const size_t need = flarepp_linear_backward_workspace_bytes(dtype, act, T, K, N);
  TRY(check_ws(ws, ws_bytes, need));
  TRY(check_disjoint({range(dW ? X : nullptr, bs * T * K, false), range(dX ? W : nullptr, bs * K * N, false),
                      range(act != FLAREPP_ACT_NONE ? pre : nullptr, bs * T * N, false), range(dOut, bs * T * N, false),
                      range(dX, bs * T * K, true), range(dW, 4 * K * N, true), range(dbias, 4 * N, true),
                      range(ws, need, true)}));
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dtype == FLAREPP_F32 ? run_linear_backward<float>(dtype, act, T, K, N, X, W, pre, dOut, dX, dW, dbias, ws, s)
                              : run_linear_backward<__bf16>(dtype, act, T, K, N, X, W, pre, dOut, dX, dW, dbias, ws, s);
}

int flarepp_embedding_forward(int dtype, int64_t T, int64_t V, int64_t C, const int64_t* ids, const void* table, float scale,
                              void* out, void* stream) {
  TRY(check_embedding_shape(dtype, T, V, C));
  TRY(check_ptr(ids, "ids"));
  TRY(check_ptr(table, "table"));
  TRY(check_ptr(out, "out"));
  const int64_t bs = dtype == FLAREPP_F32 ? 4 : 2;
  TRY(check_disjoint({range(ids, 8 * T, false), range(table, bs * V * C, false), range(out, bs * T * C, true)}));
  EmbedParams p{ids, table, out, T, V, C, scale};
  hipStream_t s = static_cast<hipStream_t>(stream);
  HIPTRY(dtype == FLAREPP_F32 ? launch_embed<float>(p, s) : launch_embed<__bf16>(p, s));
  return api_ok();
}

size_t flarepp_embedding_backward_workspace_bytes(int64_t T, int64_t V, int64_t C) {
  if (check_embedding_shape(FLAREPP_F32, T, V, C) != FLAREPP_OK) return 0;
  EmbedGradParams p{};
  p.T = T; p.V = V; p.C = C;
  return std::max<size_t>(256, embed_ws(p, nullptr));
}

int flarepp_embedding_backward(int dtype, int64_t T, int64_t V, int64_t C, const int64_t* ids, const void* dOut, float scale,
                               float* dTable, void* ws, size_t ws_bytes, void* stream) {
  TRY(check_embedding_shape(dtype, T, V, C));
  TRY(check_ptr(ids, "ids"));
  TRY(check_ptr(dOut, "dOut"));
  TRY(check_ptr(dTable, "dTable"));
  EmbedGradParams p{};
  p.ids = ids; p.dout = dOut; p.T = T; p.V = V; p.C = C; p.scale = scale; p.dtable = dTable;
  const size_t need = embed_ws(p, ws);
  TRY(check_ws(ws, ws_bytes, need));
  TRY(check_disjoint({range(ids, 8 * T, false), range(dOut, (dtype == FLAREPP_F32 ? 4 : 2) * T * C, false),
                      range(dTable, 4 * V * C, true), range(need ? ws : nullptr, need, true)}));
  hipStream_t s = static_cast<hipStream_t>(stream);
  HIPTRY(dtype == FLAREPP_F32 ? launch_embed_grad<float>(p, s) : launch_embed_grad<__bf16>(p, s));
  return api_ok();
}

int flarepp_adamw_schedule(double lr, double beta1, double beta2, int64_t step, void* out) {
  TRY(check_adamw_hyper(lr, beta1, beta2, step));
  if (!out) return fail(FLAREPP_ERR_INVALID_ARG, "out is NULL");
  AdamwSchedule a;
  static_assert(sizeof(a) == FLAREPP_ADAMW_SCHEDULE_BYTES, "stated in the header");
  adamw_schedule(a, lr, beta1, beta2, step);
  __builtin_memcpy(out, &a, sizeof(a));
  return api_ok();
}

int flarepp_adamw_step(int state, int64_t count, const flarepp_adamw_tensor* tensors, double lr, double beta1, double beta2,
                       double eps, int64_t step, const void* schedule, void* stream) {
  try {
    return adamw_entry(state, count, tensors, lr, beta1, beta2, eps, step, schedule, stream);
  } catch (const std::bad_alloc&) {
    return fail(FLAREPP_ERR_UNSUPPORTED, "no host memory for the check of %lld tensors", (long long)count);
  }
}

}  // extern "C"
