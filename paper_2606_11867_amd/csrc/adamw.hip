// One AdamW step over many tensors, with first and second moments in 32 or
// 8 bits (App. A.4: the accumulated fp32 gradients and the bf16 weights that
// it joins).
#include <limits.h>
#include <math.h>

#include "common.h"

// 8-bit states round what the formulas give, operation by operation: a
// product fused into a sum would move values across a rounding boundary.
#pragma clang fp contract(off)

namespace foremoe {
namespace {

constexpr int kAdamThreads = FOREMOE_ADAMW_BLOCK;
// elements of a record that one launch takes: fewer than 2^32 threads
constexpr int64_t kAdamPiece = (int64_t)1 << 30;

struct AdamRecord {
  void* param;
  void* grad;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int64_t n;
  float decay;
  uint32_t first;  // its first workgroup
};

struct AdamArgs {
  AdamRecord rec[FOREMOE_ADAMW_LAUNCH];
  int32_t n_rec;
  int32_t zero_grads;
  float beta1, one_beta1, beta2, one_beta2, eps, alpha, root;
  const float* grad_scale;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// ---------------------------------------------------------------------------
// 8-bit codes: x in [0, 1] as the top bits of its fp32 pattern, rounded to
// nearest even, counted so that 1.0 is the largest code.
// ---------------------------------------------------------------------------
template <int SHIFT, int ONE>
__device__ __forceinline__ int top_bits(float x) {
  const uint32_t b = __float_as_uint(x);
  return (int)((b + ((1u << (SHIFT - 1)) - 1) + ((b >> SHIFT) & 1)) >> SHIFT) - ((0x3F800000 >> SHIFT) - ONE);
}
template <int SHIFT, int ONE>
__device__ __forceinline__ float of_top_bits(uint32_t c) {
  return c ? __uint_as_float((c + ((0x3F800000u >> SHIFT) - ONE)) << SHIFT) : 0.0f;
}
// |m|: 3 bits of fraction under a sign; sqrt(v): 4 bits, a value above 0
// keeps a code above 0 (the step divides by it)
__device__ __forceinline__ uint32_t encode_m(float m, float inv) {
  const uint32_t c = (uint32_t)min(max(top_bits<20, 127>(fabsf(m) * inv), 0), 127);
  return c | (c && m < 0.0f ? 128u : 0u);
}
__device__ __forceinline__ uint32_t encode_v(float u, float inv) {
  const float x = u * inv;
  return x > 0.0f ? (uint32_t)min(max(top_bits<19, 255>(x), 1), 255) : 0u;
}
__device__ __forceinline__ float decode_m(uint32_t c, float scale) {
  const float x = of_top_bits<20, 127>(c & 127) * scale;
  return c & 128 ? -x : x;
}
__device__ __forceinline__ float decode_v(uint32_t c, float scale) {
  const float u = of_top_bits<19, 255>(c) * scale;
  return u * u;
}
__device__ __forceinline__ float inverse(float scale) { return scale >= 0x1p-126f ? 1.0f / scale : 0.0f; }

// The largest of non-negative values over the workgroup, by their patterns:
// a NaN is above every number, so it wins.
__device__ __forceinline__ float block_max(float v, uint32_t* sh) {
  uint32_t b = __float_as_uint(v) & 0x7fffffffu;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) b = max(b, (uint32_t)__shfl_xor((int)b, o, 64));
  __syncthreads();
  if (lane_id() == 0) sh[threadIdx.x >> 6] = b;
  __syncthreads();
  for (int w = 0; w < kAdamThreads / 64; ++w) b = max(b, sh[w]);
  return __uint_as_float(b);
}

template <bool PBF16, bool GBF16, bool BITS8>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamArgs a) {
  __shared__ uint32_t sh[kAdamThreads / 64];
  int r = 0;
  while (r + 1 < a.n_rec && a.rec[r + 1].first <= blockIdx.x) ++r;
  const AdamRecord& rec = a.rec[r];
  const int64_t block = blockIdx.x - rec.first, i = block * kAdamThreads + threadIdx.x;
  const bool in = i < rec.n;
  float m = 0.0f, v = 0.0f;
  if (in) {
    float g = GBF16 ? bf2f(((uint16_t*)rec.grad)[i]) : ((float*)rec.grad)[i];
    if (a.grad_scale) g = g * *a.grad_scale;
    if constexpr (BITS8) {
      m = decode_m(((uint8_t*)rec.m)[i], rec.m_scale[block]);
      v = decode_v(((uint8_t*)rec.v)[i], rec.v_scale[block]);
    } else {
      m = ((float*)rec.m)[i];
      v = ((float*)rec.v)[i];
    }
    m = m * a.beta1 + g * a.one_beta1;
    v = v * a.beta2 + g * g * a.one_beta2;
  }
  const float u = sqrtf(v);
  if (in) {
    float p = rec.master ? rec.master[i] : PBF16 ? bf2f(((uint16_t*)rec.param)[i]) : ((float*)rec.param)[i];
    const float den = u * a.root + a.eps;
    p = p * rec.decay - (den == 0.0f ? 0.0f : m / den) * a.alpha;
    if (rec.master) rec.master[i] = p;
    if constexpr (PBF16)
      ((uint16_t*)rec.param)[i] = (uint16_t)pack_bf2(p, 0.0f);
    else
      ((float*)rec.param)[i] = p;
    if (a.zero_grads) {
      if constexpr (GBF16)
        ((uint16_t*)rec.grad)[i] = 0;
      else
        ((float*)rec.grad)[i] = 0.0f;
    }
  }
  if constexpr (BITS8) {
    const float ms = block_max(m, sh), vs = block_max(u, sh);
    if (in) {
      ((uint8_t*)rec.m)[i] = (uint8_t)encode_m(m, inverse(ms));
      ((uint8_t*)rec.v)[i] = (uint8_t)encode_v(u, inverse(vs));
    }
    __syncthreads();  // every thread has read the old scales
    if (threadIdx.x == 0) rec.m_scale[block] = ms, rec.v_scale[block] = vs;
  } else if (in) {
    ((float*)rec.m)[i] = m;
    ((float*)rec.v)[i] = v;
  }
}

__global__ __launch_bounds__(kAdamThreads) void adamw_values_kernel(const uint8_t* m, const float* m_scale,
                                                                    const uint8_t* v, const float* v_scale, int64_t n,
                                                                    float* m_out, float* v_out) {
  const int64_t block = blockIdx.x + (int64_t)blockIdx.y * gridDim.x, i = block * kAdamThreads + threadIdx.x;
  if (i >= n) return;
  m_out[i] = decode_m(m[i], m_scale[block]);
  v_out[i] = decode_v(v[i], v_scale[block]);
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

template <bool PBF16, bool GBF16>
static void launch_adamw(const AdamArgs& a, unsigned blocks, int bits, hipStream_t st) {
  if (bits == 8)
    hipLaunchKernelGGL((adamw_kernel<PBF16, GBF16, true>), dim3(blocks), dim3(kAdamThreads), 0, st, a);
  else
    hipLaunchKernelGGL((adamw_kernel<PBF16, GBF16, false>), dim3(blocks), dim3(kAdamThreads), 0, st, a);
}

extern "C" {

int foremoe_adamw_step(const foremoe_adamw_tensor* tensors, int32_t n_tensors, foremoe_dtype param_dtype,
                       foremoe_dtype grad_dtype, int32_t state_bits, double lr, double beta1, double beta2,
                       double eps, int64_t step, const float* grad_scale, int32_t zero_grads, void* stream) {
  REQUIRE(param_dtype == FOREMOE_BF16 || param_dtype == FOREMOE_F32, "adamw_step: bad parameter dtype");
  REQUIRE(grad_dtype == FOREMOE_BF16 || grad_dtype == FOREMOE_F32, "adamw_step: bad gradient dtype");
  REQUIRE(state_bits == 8 || state_bits == 32, "adamw_step: state_bits=%d is neither 8 nor 32", state_bits);
  REQUIRE(n_tensors >= 0 && (tensors || n_tensors == 0), "adamw_step: n_tensors < 0 or tensors NULL");
  REQUIRE(isfinite(lr) && lr >= 0, "adamw_step: lr must be finite and not negative");
  REQUIRE(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1, "adamw_step: betas outside [0, 1)");
  REQUIRE(isfinite(eps) && eps >= 0, "adamw_step: eps must be finite and not negative");
  REQUIRE(step >= 1, "adamw_step: step=%lld, the first is 1", (long long)step);
  const uintptr_t pb = param_dtype == FOREMOE_BF16 ? 2 : 4, gb = grad_dtype == FOREMOE_BF16 ? 2 : 4;
  const uintptr_t sb = state_bits == 8 ? 1 : 4;
  REQUIRE(!misaligned(grad_scale, 4), "adamw_step: grad_scale misaligned");
  for (int i = 0; i < n_tensors; ++i) {
    const foremoe_adamw_tensor& t = tensors[i];
    REQUIRE(t.n >= 0 && t.n <= (int64_t)1 << 40, "adamw_step: tensor %d: n=%lld outside [0, 2^40]", i, (long long)t.n);
    if (t.n == 0) continue;
    REQUIRE(t.param && t.grad && t.m && t.v, "adamw_step: tensor %d: NULL pointer", i);
    REQUIRE(state_bits == 32 || (t.m_scale && t.v_scale), "adamw_step: tensor %d: 8-bit states without scales", i);
    REQUIRE(!t.master || param_dtype == FOREMOE_BF16, "adamw_step: tensor %d: a master goes with bf16 parameters", i);
    REQUIRE(isfinite(t.weight_decay), "adamw_step: tensor %d: weight decay is not finite", i);
    REQUIRE(!misaligned(t.param, pb) && !misaligned(t.grad, gb) && !misaligned(t.master, 4) && !misaligned(t.m, sb) &&
                !misaligned(t.v, sb) && !misaligned(t.m_scale, 4) && !misaligned(t.v_scale, 4),
            "adamw_step: tensor %d: misaligned pointer", i);
  }
  AdamArgs a{};
  a.zero_grads = zero_grads, a.grad_scale = grad_scale;
  a.beta1 = (float)beta1, a.one_beta1 = (float)(1 - beta1), a.beta2 = (float)beta2, a.one_beta2 = (float)(1 - beta2);
  a.eps = (float)eps, a.alpha = (float)(lr / (1 - pow(beta1, (double)step)));
  a.root = (float)(1 / sqrt(1 - pow(beta2, (double)step)));
  uint64_t blocks = 0;
  int rc = FOREMOE_OK;
  auto flush = [&] {
    if (!a.n_rec) return;
    hipStream_t st = (hipStream_t)stream;
    const bool p = param_dtype == FOREMOE_BF16, g = grad_dtype == FOREMOE_BF16;
    if (p && g) launch_adamw<true, true>(a, (unsigned)blocks, state_bits, st);
    else if (p) launch_adamw<true, false>(a, (unsigned)blocks, state_bits, st);
    else if (g) launch_adamw<false, true>(a, (unsigned)blocks, state_bits, st);
    else launch_adamw<false, false>(a, (unsigned)blocks, state_bits, st);
    if (rc == FOREMOE_OK) rc = check_launch("adamw_step");
    a.n_rec = 0, blocks = 0;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const foremoe_adamw_tensor& t = tensors[i];
    for (int64_t at = 0; at < t.n; at += kAdamPiece) {
      const int64_t n = t.n - at < kAdamPiece ? t.n - at : kAdamPiece;
      const uint64_t nb = (uint64_t)(n + kAdamThreads - 1) / kAdamThreads;
      if (a.n_rec == FOREMOE_ADAMW_LAUNCH || (blocks + nb) * kAdamThreads > (uint64_t)2 * kAdamPiece) flush();
      AdamRecord& r = a.rec[a.n_rec++];
      r.param = (char*)t.param + at * pb, r.grad = (char*)t.grad + at * gb;
      r.master = t.master ? t.master + at : nullptr;
      r.m = (char*)t.m + at * sb, r.v = (char*)t.v + at * sb;
      r.m_scale = state_bits == 8 ? t.m_scale + at / FOREMOE_ADAMW_BLOCK : nullptr;
      r.v_scale = state_bits == 8 ? t.v_scale + at / FOREMOE_ADAMW_BLOCK : nullptr;
      r.n = n, r.decay = (float)(1 - lr * t.weight_decay), r.first = (uint32_t)blocks;
      blocks += nb;
    }
  }
  flush();
  return rc;
}

int foremoe_adamw_state_values(const uint8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale,
                               int64_t n, float* m_out, float* v_out, void* stream) {
  REQUIRE(n >= 0 && n <= (int64_t)1 << 40, "adamw_state_values: n=%lld outside [0, 2^40]", (long long)n);
  if (n == 0) return FOREMOE_OK;
  REQUIRE(m && m_scale && v && v_scale && m_out && v_out, "adamw_state_values: NULL pointer");
  REQUIRE(!misaligned(m_scale, 4) && !misaligned(v_scale, 4) && !misaligned(m_out, 4) && !misaligned(v_out, 4),
          "adamw_state_values: misaligned pointer");
  const int64_t nb = (n + kAdamThreads - 1) / kAdamThreads;
  const int64_t gx = nb < (1 << 20) ? nb : 1 << 20, gy = (nb + gx - 1) / gx;
  hipLaunchKernelGGL(adamw_values_kernel, dim3((unsigned)gx, (unsigned)gy), dim3(kAdamThreads), 0,
                     (hipStream_t)stream, m, m_scale, v, v_scale, n, m_out, v_out);
  return check_launch("adamw_state_values");
}

}  // extern "C"
