// Log-probabilities of given tokens, with entropies, top alternatives and
// the gradient of the logits.
#include <limits.h>
#include <math.h>

#include "common.h"

namespace foremoe {
namespace {

constexpr int kLpThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;

struct LogprobArgs {
  const void* logits;
  int64_t ld;
  int32_t N, V;
  const int32_t* targets;
  float c, inv_temperature;  // c: log2(e) / temperature
  int32_t n_top;
  float *logp, *entropy, *lse;
  int32_t* top_ids;
  float* top_logp;
};

template <bool BF16>
__device__ __forceinline__ float load_lp(const void* p, int64_t i) {
  if constexpr (BF16) return bf2f(((const uint16_t*)p)[i]);
  return ((const float*)p)[i];
}

// Running maximum m of the logits x, s = sum e, t = sum (x - m) e with
// e = 2^((x - m) c), so that lse = m / temperature + ln2 log2 s and
// entropy = ln2 log2 s - t / (s temperature), both terms >= 0. Subtracting
// before scaling keeps logits up to the type's ends apart. m starts at the
// lowest finite number, so an x of -inf adds nothing to s.
struct Sums {
  float m, s, t;
};

__device__ __forceinline__ float rebased(float t, float d, float s) { return t + fmaxf(d, kLowest) * s; }

__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.m - m, db = b.m - m;
  const float ea = exp2f(da * c), eb = exp2f(db * c);
  Sums r;
  r.m = m;
  r.s = a.s * ea + b.s * eb;
  // an e of 0 takes what was below along, however large (d s may overflow)
  r.t = (ea == 0.0f ? 0.0f : ea * rebased(a.t, da, a.s)) + (eb == 0.0f ? 0.0f : eb * rebased(b.t, db, b.s));
  return r;
}

__device__ __forceinline__ Sums add(Sums a, float x, float c) {
  if (x > a.m) {
    const float d = a.m - x, e = exp2f(d * c);
    a.t = e == 0.0f ? 0.0f : e * rebased(a.t, d, a.s);
    a.s *= e;
    a.m = x;
  }
  const float d = x - a.m, e = exp2f(d * c);
  a.s += e;
  a.t += fmaxf(d, kLowest) * e;
  return a;
}

__device__ __forceinline__ bool better(float v, int id, float w, int jd) { return v > w || (v == w && id < jd); }

// One workgroup per row; the top alternatives one after another, each a pass
// over the row.
template <bool BF16>
__global__ __launch_bounds__(kLpThreads) void logprobs_kernel(LogprobArgs a) {
  __shared__ Sums sh[kLpThreads / 64];
  __shared__ float sh_v[kLpThreads / 64];
  __shared__ int sh_i[kLpThreads / 64];
  const int64_t row = blockIdx.x, base = row * a.ld;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  const int target = a.targets ? a.targets[row] : 0;
  if ((unsigned)target >= (unsigned)a.V) {
    if (tid == 0) {
      if (a.logp) a.logp[row] = 0.0f;
      if (a.entropy) a.entropy[row] = 0.0f;
      if (a.lse) a.lse[row] = 0.0f;
    }
    for (int k = tid; k < a.n_top; k += kLpThreads) {
      a.top_ids[row * a.n_top + k] = -1;
      a.top_logp[row * a.n_top + k] = -INFINITY;
    }
    return;
  }
  Sums r{kLowest, 0.0f, 0.0f};
  for (int j = tid; j < a.V; j += kLpThreads) r = add(r, load_lp<BF16>(a.logits, base + j), a.c);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1)
    r = join(r, Sums{__shfl_xor(r.m, o, 64), __shfl_xor(r.s, o, 64), __shfl_xor(r.t, o, 64)}, a.c);
  if (lane == 0) sh[wave] = r;
  __syncthreads();
  r = sh[0];
  for (int w = 1; w < kLpThreads / 64; ++w) r = join(r, sh[w], a.c);
  const float ls = kLn2 * log2f(r.s);
  const bool none = r.s == 0.0f;
  if (tid == 0) {
    if (a.lse) a.lse[row] = r.m * a.inv_temperature + ls;
    if (a.entropy) a.entropy[row] = none ? 0.0f : ls - r.t / r.s * a.inv_temperature;
    if (a.logp)
      a.logp[row] = none ? -INFINITY : (load_lp<BF16>(a.logits, base + target) - r.m) * a.inv_temperature - ls;
  }
  float last = INFINITY;
  int last_id = -1;
  for (int k = 0; k < a.n_top; ++k) {
    float v = -INFINITY;
    int id = INT_MAX;
    for (int j = tid; j < a.V; j += kLpThreads) {
      const float x = load_lp<BF16>(a.logits, base + j);
      if (x > -INFINITY && better(last, last_id, x, j) && better(x, j, v, id)) v = x, id = j;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      const float w = __shfl_xor(v, o, 64);
      const int jd = __shfl_xor(id, o, 64);
      if (better(w, jd, v, id)) v = w, id = jd;
    }
    __syncthreads();
    if (lane == 0) sh_v[wave] = v, sh_i[wave] = id;
    __syncthreads();
    v = sh_v[0], id = sh_i[0];
    for (int w = 1; w < kLpThreads / 64; ++w)
      if (better(sh_v[w], sh_i[w], v, id)) v = sh_v[w], id = sh_i[w];
    if (tid == 0) {
      const bool left = id == INT_MAX;
      a.top_ids[row * a.n_top + k] = left ? -1 : id;
      a.top_logp[row * a.n_top + k] = left ? -INFINITY : (v - r.m) * a.inv_temperature - ls;
    }
    last = v, last_id = id;
  }
}

struct LogprobBwdArgs {
  const void* logits;
  int64_t ld;
  int32_t N, V;
  const int32_t* targets;
  float inv_temperature;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dlogits;
  int64_t ld_out;
};

template <bool BF16>
__global__ __launch_bounds__(kLpThreads) void logprobs_bwd_kernel(LogprobBwdArgs a) {
  const int64_t row = blockIdx.y;
  const int target = a.targets ? a.targets[row] : -1;
  const bool keep = !a.targets || (unsigned)target < (unsigned)a.V;
  // a row of -inf only: every p is 0
  const float lse = a.lse[row] == -INFINITY ? INFINITY : a.lse[row];
  const float dlp = a.dlogp ? a.dlogp[row] * a.inv_temperature : 0.0f;
  const float dh = a.dentropy ? a.dentropy[row] * a.inv_temperature : 0.0f;
  const float h = a.dentropy ? a.entropy[row] : 0.0f;
  for (int j = blockIdx.x * kLpThreads + threadIdx.x; j < a.V; j += gridDim.x * kLpThreads) {
    float d = 0.0f;
    if (keep) {
      const float y = fmaf(load_lp<BF16>(a.logits, row * a.ld + j), a.inv_temperature, -lse);
      const float p = exp2f(y * kLog2e);
      if (!(p == 0.0f)) d = -p * (dlp + dh * (y + h));
      if (j == target) d += dlp;
    }
    if constexpr (BF16)
      ((uint16_t*)a.dlogits)[row * a.ld_out + j] = (uint16_t)pack_bf2(d, 0.0f);
    else
      ((float*)a.dlogits)[row * a.ld_out + j] = d;
  }
}

constexpr size_t kLpWsBytes = 256;

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static int check_logprobs(const char* who, const void* logits, foremoe_dtype dtype, int64_t ld, int64_t N, int64_t V,
                          float temperature) {
  REQUIRE(dtype == FOREMOE_BF16 || dtype == FOREMOE_F32, "%s: bad dtype", who);
  REQUIRE(N >= 0 && N < INT_MAX, "%s: N=%lld outside [0, 2^31)", who, (long long)N);
  REQUIRE(V >= 1 && V < INT_MAX, "%s: V=%lld outside [1, 2^31)", who, (long long)V);
  REQUIRE(ld >= V && ld <= (int64_t)1 << 32, "%s: ld=%lld outside [V, 2^32]", who, (long long)ld);
  REQUIRE(temperature > 0.0f && isfinite(temperature) && isfinite(kLog2e / temperature) && 1.0f / temperature > 0.0f,
          "%s: temperature must be positive and finite", who);
  REQUIRE(logits || N == 0, "%s: logits is NULL", who);
  REQUIRE(((uintptr_t)logits & (dtype == FOREMOE_BF16 ? 1 : 3)) == 0, "%s: logits misaligned", who);
  return FOREMOE_OK;
}

extern "C" {

size_t foremoe_logprobs_workspace_size(void) { return kLpWsBytes; }

int foremoe_token_logprobs(const void* logits, foremoe_dtype dtype, int64_t ld, int64_t N, int64_t V,
                           const int32_t* targets, float temperature, int32_t n_top, float* logp, float* entropy,
                           float* lse, int32_t* top_ids, float* top_logp, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_logprobs("token_logprobs", logits, dtype, ld, N, V, temperature);
  if (rc) return rc;
  REQUIRE(n_top >= 0 && n_top <= FOREMOE_MAX_TOP && n_top <= V, "token_logprobs: n_top=%d outside [0, min(V, %d)]",
          n_top, FOREMOE_MAX_TOP);
  REQUIRE(n_top == 0 || N == 0 || (top_ids && top_logp), "token_logprobs: top_ids or top_logp is NULL");
  REQUIRE(!logp || targets || N == 0, "token_logprobs: logp needs targets");
  REQUIRE(ws || ws_bytes == 0, "token_logprobs: workspace NULL with ws_bytes > 0");
  if (ws) {
    REQUIRE(((uintptr_t)ws & 255) == 0, "token_logprobs: workspace not 256-byte aligned");
    REQUIRE(ws_bytes >= kLpWsBytes, "token_logprobs: workspace too small (%zu < %zu)", ws_bytes, kLpWsBytes);
  }
  if (N == 0) return FOREMOE_OK;
  LogprobArgs a{logits, ld, (int32_t)N, (int32_t)V, targets, kLog2e / temperature, 1.0f / temperature, n_top, logp, entropy, lse, top_ids,
                top_logp};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == FOREMOE_BF16)
    hipLaunchKernelGGL(logprobs_kernel<true>, dim3((unsigned)N), dim3(kLpThreads), 0, st, a);
  else
    hipLaunchKernelGGL(logprobs_kernel<false>, dim3((unsigned)N), dim3(kLpThreads), 0, st, a);
  return check_launch("token_logprobs");
}

int foremoe_token_logprobs_bwd(const void* logits, foremoe_dtype dtype, int64_t ld, int64_t N, int64_t V,
                               const int32_t* targets, float temperature, const float* lse, const float* entropy,
                               const float* dlogp, const float* dentropy, void* dlogits, int64_t ld_out,
                               void* stream) {
  int rc = check_logprobs("token_logprobs_bwd", logits, dtype, ld, N, V, temperature);
  if (rc) return rc;
  REQUIRE(ld_out >= V && ld_out <= (int64_t)1 << 32, "token_logprobs_bwd: ld_out=%lld outside [V, 2^32]",
          (long long)ld_out);
  REQUIRE(dlogits != logits || ld == ld_out || N == 0, "token_logprobs_bwd: in place needs ld_out == ld");
  if (N == 0) return FOREMOE_OK;
  REQUIRE(lse && dlogits, "token_logprobs_bwd: lse or dlogits is NULL");
  REQUIRE(!dlogp || targets, "token_logprobs_bwd: dlogp needs targets");
  REQUIRE(!dentropy || entropy, "token_logprobs_bwd: dentropy needs entropy");
  REQUIRE(((uintptr_t)dlogits & (dtype == FOREMOE_BF16 ? 1 : 3)) == 0, "token_logprobs_bwd: dlogits misaligned");
  hipStream_t st = (hipStream_t)stream;
  // the grid's second dimension ends at 65535 rows
  const size_t item = dtype == FOREMOE_BF16 ? 2 : 4;
  for (int64_t r = 0; r < N; r += 65535) {
    const int64_t n = N - r < 65535 ? N - r : 65535;
    LogprobBwdArgs a{(const char*)logits + (size_t)r * ld * item, ld, (int32_t)n, (int32_t)V,
                     targets ? targets + r : nullptr, 1.0f / temperature, lse + r,
                     entropy ? entropy + r : nullptr, dlogp ? dlogp + r : nullptr, dentropy ? dentropy + r : nullptr,
                     (char*)dlogits + (size_t)r * ld_out * item, ld_out};
    const unsigned gx = (unsigned)((V + kLpThreads * 8 - 1) / (kLpThreads * 8));
    const dim3 grid(gx < 64 ? gx : 64, (unsigned)n);
    if (dtype == FOREMOE_BF16)
      hipLaunchKernelGGL(logprobs_bwd_kernel<true>, grid, dim3(kLpThreads), 0, st, a);
    else
      hipLaunchKernelGGL(logprobs_bwd_kernel<false>, grid, dim3(kLpThreads), 0, st, a);
  }
  return check_launch("token_logprobs_bwd");
}

}  // extern "C"
