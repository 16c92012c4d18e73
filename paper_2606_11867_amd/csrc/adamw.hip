// One AdamW step over many tensors, with first and second moments in 32 or
// 8 bits (App. A.4: the accumulated fp32 gradients and the bf16 weights that
// it joins). Every element is read and written once, so the step is bound by
// HBM: 34 bytes an element with fp32 masters, bf16 copies, fp32 moments and
// cleared fp32 gradients, 16 with 8-bit moments and bf16 gradients. There the
// vector units come near as well: about 60 instruction slots an element for
// decoding, an exact square root, two maxima and encoding. Measured on MI355X:
//   75.5 M elements, 32 bits, masters, cleared gradients  450-466 us, 5.5-5.7 TB/s
//   the same with 8-bit states                            255-261 us, 6.4-6.5 TB/s
//   68.9 M in 60 tensors, 8 bits, bf16 gradients          173-185 us, 6.0-6.4 TB/s, two launches
//   40 tensors of 64 to 40000 elements                    4.9 us, one launch
// Records travel in the kernel's arguments (4 KiB hold 48), so a step needs
// no table in device memory; a workgroup finds its record by bisection.
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "common.h"

// 8-bit states round what the formulas give, operation by operation: a
// product fused into a sum would move values across a rounding boundary.
#pragma clang fp contract(off)

namespace foremoe {
namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamBlocks = 2;  // blocks of 256 elements that a wavefront takes, 4 elements a lane
constexpr int kAdamChunk = kAdamThreads / 64 * kAdamBlocks * FOREMOE_ADAMW_BLOCK;  // elements of a workgroup
static_assert(FOREMOE_ADAMW_BLOCK == 64 * 4);
// elements of a record that one launch takes: fewer than 2^32 threads
constexpr int64_t kAdamPiece = (int64_t)1 << 30;
static_assert(kAdamPiece % kAdamChunk == 0);

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
};

struct AdamArgs {
  AdamRecord rec[FOREMOE_ADAMW_LAUNCH];
  uint32_t first[FOREMOE_ADAMW_LAUNCH];  // a record's first workgroup
  int32_t n_rec;
  int32_t zero_grads;
  float beta1, one_beta1, beta2, one_beta2, eps, alpha, root;
  const float* grad_scale;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

// A lane's four elements of a block, as they lie in memory. Tensors may start
// at any element, so the vectors have the alignment of the type only. Every
// byte is read once and written once: both carry the nontemporal hint.
// `block` is uniform; `left` elements of the block exist (FULL: all).
template <class T>
struct Four {
  typedef T any __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  T e[4];
  template <bool FULL>
  __device__ __forceinline__ void load(const void* block, int lane, int left) {
    const T* at = (const T*)block + (uint32_t)lane * 4;
    if (FULL || lane * 4 + 4 <= left) {
      const any x = __builtin_nontemporal_load((const any*)at);
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = x[k];
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) e[k] = lane * 4 + k < left ? at[k] : T(0);
    }
  }
  template <bool FULL>
  __device__ __forceinline__ void store(void* block, int lane, int left) const {
    T* at = (T*)block + (uint32_t)lane * 4;
    if (FULL || lane * 4 + 4 <= left) {
      const any x = {e[0], e[1], e[2], e[3]};
      __builtin_nontemporal_store(x, (any*)at);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (lane * 4 + k < left) at[k] = e[k];
    }
  }
};

// ---------------------------------------------------------------------------
// 8-bit codes: x in [0, 1] as the top bits of its fp32 pattern, rounded to
// nearest even, counted so that 1.0 is the largest code.
// ---------------------------------------------------------------------------
template <int SHIFT, int ONE>
__device__ __forceinline__ int top_bits(float x) {
  const uint32_t b = __float_as_uint(x);
  constexpr uint32_t kZero = ((0x3F800000u >> SHIFT) - ONE) << SHIFT;  // the pattern of code 0
  return (int)(b + ((b >> SHIFT) & 1) + (((1u << (SHIFT - 1)) - 1) - kZero)) >> SHIFT;
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
// Correctly rounded square root and reciprocal of numbers from 2^-90 on (the
// reciprocal to 2^120): the hardware's, within a unit in the last place,
// corrected once by a residual that a fused multiply-add gives exactly (P.
// Markstein's method), in 11 and 7 instruction slots where the compiler's take
// 18 and 15. For a reciprocal the method proves all but the significand of all
// ones, where it depends on the estimate; with this hardware's it is right
// there too. The tests go over every significand of both.
constexpr float kExactFrom = 0x1p-90f, kExactTo = 0x1p120f;
__device__ __forceinline__ float exact_sqrt(float x) {
  const float s = __builtin_amdgcn_sqrtf(x), h = 0.5f * __builtin_amdgcn_rsqf(x);
  return fmaf(fmaf(-s, s, x), h, s);
}
__device__ __forceinline__ float exact_reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  return fmaf(fmaf(-x, r, 1.0f), r, r);
}
// Within a unit in the last place, where no code depends on it. The
// hardware's square root does not take subnormal numbers, so small ones are
// scaled first, without a branch (75.5 M elements with masters: 455 us, 459
// with a branch to sqrtf, 450 where subnormal v count as 0).
__device__ __forceinline__ float near_sqrt(float x) {
  const bool tiny = x < kExactFrom;
  return __builtin_amdgcn_sqrtf(tiny ? x * 0x1p64f : x) * (tiny ? 0x1p-32f : 1.0f);
}
// What a block's values are multiplied by; x is uniform.
__device__ __forceinline__ float inverse(float x) {
  if (__builtin_expect(x >= kExactFrom && x <= kExactTo, 1)) return exact_reciprocal(x);
  return x >= 0x1p-126f ? 1.0f / x : 0.0f;
}

// The largest of the wavefront's patterns. Of non-negative floats: a NaN is
// above every number, so it wins.
__device__ __forceinline__ float wave_max_pattern(uint32_t b) {
  // within rows of 16 lanes, then the rows' last lanes onwards: lane 63 has it
#define FOREMOE_DPP_MAX(ctrl, rows) b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, ctrl, rows, 0xf, true))
  FOREMOE_DPP_MAX(0x111, 0xf);  // row_shr:1
  FOREMOE_DPP_MAX(0x112, 0xf);  // row_shr:2
  FOREMOE_DPP_MAX(0x114, 0xf);  // row_shr:4
  FOREMOE_DPP_MAX(0x118, 0xf);  // row_shr:8
  FOREMOE_DPP_MAX(0x142, 0xa);  // row_bcast:15
  FOREMOE_DPP_MAX(0x143, 0xc);  // row_bcast:31
#undef FOREMOE_DPP_MAX
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)b, 63));
}

// One wavefront's kAdamBlocks blocks of 256 elements, 4 consecutive ones a
// lane: all are loaded, then worked on one after another; a block's scale is
// then one maximum over the wavefront. left: elements from its first block on.
template <bool PBF16, bool GBF16, bool BITS8, bool FULL>
__device__ __forceinline__ void adamw_blocks(const AdamArgs& a, const AdamRecord& rec, int64_t block0, int left) {
  typedef typename std::conditional<PBF16, uint16_t, float>::type P;
  typedef typename std::conditional<GBF16, uint16_t, float>::type G;
  typedef typename std::conditional<BITS8, uint8_t, float>::type S;
  constexpr int B = FOREMOE_ADAMW_BLOCK;
  const int lane = lane_id();
  const bool master = PBF16 && rec.master;
  const int64_t i0 = block0 * B;
  G* const grad0 = (G*)rec.grad + i0;
  P* const param0 = (P*)rec.param + i0;
  float* const master0 = master ? rec.master + i0 : nullptr;
  S* const m0 = (S*)rec.m + i0;
  S* const v0 = (S*)rec.v + i0;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  Four<G> g[kAdamBlocks];
  Four<P> p[kAdamBlocks];
  Four<float> w[kAdamBlocks];
  Four<S> m[kAdamBlocks], v[kAdamBlocks];
  float m_scale[kAdamBlocks], v_scale[kAdamBlocks];
#pragma unroll
  for (int q = 0; q < kAdamBlocks; ++q) {
    if (!FULL && q * B >= left) break;
    g[q].template load<FULL>(grad0 + q * B, lane, left - q * B);
    if (master)
      w[q].template load<FULL>(master0 + q * B, lane, left - q * B);
    else
      p[q].template load<FULL>(param0 + q * B, lane, left - q * B);
    m[q].template load<FULL>(m0 + q * B, lane, left - q * B);
    v[q].template load<FULL>(v0 + q * B, lane, left - q * B);
    if constexpr (BITS8) m_scale[q] = rec.m_scale[block0 + q], v_scale[q] = rec.v_scale[block0 + q];
  }
#pragma unroll
  for (int q = 0; q < kAdamBlocks; ++q) {
    if (!FULL && q * B >= left) break;
    float mm[4], vv[4], u[4];
    bool ends = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float grad;
      if constexpr (GBF16) grad = bf2f(g[q].e[k]);
      else grad = g[q].e[k];
      if (a.grad_scale) grad = grad * gs;
      if constexpr (BITS8) {
        mm[k] = decode_m(m[q].e[k], m_scale[q]);
        vv[k] = decode_v(v[q].e[k], v_scale[q]);
      } else {
        mm[k] = m[q].e[k];
        vv[k] = v[q].e[k];
      }
      mm[k] = mm[k] * a.beta1 + grad * a.one_beta1;
      vv[k] = vv[k] * a.beta2 + grad * grad * a.one_beta2;
      if constexpr (BITS8) {
        // exact, since it makes the code; neither subnormal numbers nor an
        // infinity (a NaN by the residual) are for the method
        u[k] = exact_sqrt(vv[k]);
        ends |= !(vv[k] >= kExactFrom && vv[k] < INFINITY);
      } else {
        u[k] = near_sqrt(vv[k]);
      }
    }
    if (BITS8 && __any(ends)) {
#pragma unroll
      for (int k = 0; k < 4; ++k) u[k] = sqrtf(vv[k]);
    }
    uint32_t m_most = 0, u_most = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float wk;
      if (master) wk = w[q].e[k];
      else if constexpr (PBF16) wk = bf2f(p[q].e[k]);
      else wk = p[q].e[k];
      // the reciprocal is within a unit in the last place; den is 0 or normal:
      // eps is, and the root of the least v is
      const float den = u[k] * a.root + a.eps;
      wk = wk * rec.decay - (den == 0.0f ? 0.0f : mm[k] * __builtin_amdgcn_rcpf(den)) * a.alpha;
      if (master) w[q].e[k] = wk;
      if constexpr (!PBF16) p[q].e[k] = wk;
      else p[q].e[k] = (uint16_t)pack_bf2(wk, 0.0f);
      if constexpr (BITS8) {
        m_most = max(m_most, __float_as_uint(mm[k]) & 0x7fffffffu);
        u_most = max(u_most, __float_as_uint(u[k]) & 0x7fffffffu);
      } else {
        m[q].e[k] = mm[k], v[q].e[k] = vv[k];
      }
    }
    if constexpr (BITS8) {
      const float ms = wave_max_pattern(m_most), us = wave_max_pattern(u_most);
      const float mi = inverse(ms), ui = inverse(us);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[q].e[k] = (uint8_t)encode_m(mm[k], mi);
        v[q].e[k] = (uint8_t)encode_v(u[k], ui);
      }
      if (lane == 0) rec.m_scale[block0 + q] = ms, rec.v_scale[block0 + q] = us;
    }
    if (master) w[q].template store<FULL>(master0 + q * B, lane, left - q * B);
    p[q].template store<FULL>(param0 + q * B, lane, left - q * B);
    m[q].template store<FULL>(m0 + q * B, lane, left - q * B);
    v[q].template store<FULL>(v0 + q * B, lane, left - q * B);
    if (a.zero_grads) {
      Four<G> z{};
      z.template store<FULL>(grad0 + q * B, lane, left - q * B);
    }
  }
}

template <bool PBF16, bool GBF16, bool BITS8>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(AdamArgs a) {
  int r = 0;
#pragma unroll
  for (int step = 32; step; step >>= 1)
    if (r + step < a.n_rec && a.first[r + step] <= blockIdx.x) r += step;
  const AdamRecord& rec = a.rec[r];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t block0 = ((int64_t)(blockIdx.x - a.first[r]) * (kAdamThreads / 64) + wave) * kAdamBlocks;
  const int64_t left = rec.n - block0 * FOREMOE_ADAMW_BLOCK;
  if (left >= kAdamBlocks * FOREMOE_ADAMW_BLOCK)
    adamw_blocks<PBF16, GBF16, BITS8, true>(a, rec, block0, kAdamBlocks * FOREMOE_ADAMW_BLOCK);
  else if (left > 0)
    adamw_blocks<PBF16, GBF16, BITS8, false>(a, rec, block0, (int)left);
}

__global__ __launch_bounds__(kAdamThreads) void adamw_values_kernel(const uint8_t* m, const float* m_scale,
                                                                    const uint8_t* v, const float* v_scale, int64_t n,
                                                                    float* m_out, float* v_out) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  const int64_t block = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kAdamThreads / 64) + wave;
  const int64_t i0 = block * FOREMOE_ADAMW_BLOCK;
  if (i0 >= n) return;
  const int left = (int)(n - i0 < FOREMOE_ADAMW_BLOCK ? n - i0 : FOREMOE_ADAMW_BLOCK);
  Four<uint8_t> cm, cv;
  Four<float> fm, fv;
  cm.load<false>(m + i0, lane, left);
  cv.load<false>(v + i0, lane, left);
  const float ms = m_scale[block], vs = v_scale[block];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    fm.e[k] = decode_m(cm.e[k], ms);
    fv.e[k] = decode_v(cv.e[k], vs);
  }
  fm.store<false>(m_out + i0, lane, left);
  fv.store<false>(v_out + i0, lane, left);
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
  a.eps = eps < 0x1p-126 ? 0.0f : (float)eps, a.alpha = (float)(lr / (1 - pow(beta1, (double)step)));
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
      const uint64_t nb = (uint64_t)(n + kAdamChunk - 1) / kAdamChunk;
      if (a.n_rec == FOREMOE_ADAMW_LAUNCH || (blocks + nb) * kAdamThreads > (uint64_t)2 * kAdamPiece) flush();
      a.first[a.n_rec] = (uint32_t)blocks;
      AdamRecord& r = a.rec[a.n_rec++];
      r.param = (char*)t.param + at * pb, r.grad = (char*)t.grad + at * gb;
      r.master = t.master ? t.master + at : nullptr;
      r.m = (char*)t.m + at * sb, r.v = (char*)t.v + at * sb;
      r.m_scale = state_bits == 8 ? t.m_scale + at / FOREMOE_ADAMW_BLOCK : nullptr;
      r.v_scale = state_bits == 8 ? t.v_scale + at / FOREMOE_ADAMW_BLOCK : nullptr;
      r.n = n, r.decay = (float)(1 - lr * t.weight_decay);
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
  const int64_t nb = (n + kAdamThreads * 4 - 1) / (kAdamThreads * 4);
  const int64_t gx = nb < (1 << 20) ? nb : 1 << 20, gy = (nb + gx - 1) / gx;
  hipLaunchKernelGGL(adamw_values_kernel, dim3((unsigned)gx, (unsigned)gy), dim3(kAdamThreads), 0,
                     (hipStream_t)stream, m, m_scale, v, v_scale, n, m_out, v_out);
  return check_launch("adamw_state_values");
}

}  // extern "C"
