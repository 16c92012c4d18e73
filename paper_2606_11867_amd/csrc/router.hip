// The router around the expert layer (Sec. 2.1; replay of recorded ids,
// Sec. 5): ids and gates from logits, the balance loss with its counts, and
// the gradient of the logits.
#include <limits.h>
#include <math.h>

#include "common.h"

namespace foremoe {
namespace {

constexpr int kRouterThreads = 256;
constexpr int kRouterWaves = kRouterThreads / 64;
constexpr int kRouterBlocks = 512;  // most workgroups that leave partial statistics
constexpr float kNegInf = -INFINITY;

struct RouterArgs {
  const void* logits;
  int64_t ld, T;
  int32_t E, K;
  int32_t sigmoid, renorm;
  float scale;
  const float* bias;
  const uint8_t* mask;
  const int32_t* ids_in;
  int32_t* ids;
  float* gates;
  // statistics: prob_part [blocks, E], count_part [blocks, E], token_part [blocks]
  float* prob_part;
  int32_t* count_part;
  int32_t* token_part;
  // backward
  const float* dgates;
  const int32_t* counts;
  const int32_t* n_tokens;
  float coef;
  void* dlogits;
  int64_t ld_out;
};

template <bool BF16>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  if constexpr (BF16) return bf2f(((const uint16_t*)p)[i]);
  return ((const float*)p)[i];
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return v;
}

__device__ __forceinline__ float sigmoid(float v) { return 1.0f / (1.0f + expf(-v)); }

// One token's scores: s[j] (softmax numerators or sigmoids) of the experts
// lane + 64 j, and their sum.
template <int VPL>
__device__ __forceinline__ float token_scores(const float (&v)[VPL], bool sig, float (&s)[VPL]) {
  float m = kNegInf;
#pragma unroll
  for (int j = 0; j < VPL; ++j) m = fmaxf(m, v[j]);
  m = wave_max(m);
  if (m == kNegInf) m = 0.0f;
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    s[j] = sig ? sigmoid(v[j]) : expf(v[j] - m);
    sum += s[j];
  }
  return wave_sum(sum);
}

// The score of a picked place (x its logit) over the sum that its gate
// divides by, for the place this lane holds; `empty` places give 0.
__device__ __forceinline__ float place_gate(float x, bool empty, bool sig, bool renorm, float row_max,
                                            float row_sum, float* denom) {
  float q;
  if (sig) {
    q = empty ? 0.0f : sigmoid(x);
    *denom = renorm ? wave_sum(q) : 1.0f;
  } else if (renorm) {
    float mx = wave_max(empty ? kNegInf : x);
    if (mx == kNegInf) mx = 0.0f;
    q = empty ? 0.0f : expf(x - mx);
    *denom = wave_sum(q);
  } else {
    q = empty ? 0.0f : expf(x - row_max);
    *denom = row_sum;
  }
  return *denom == 0.0f ? 0.0f : q / *denom;
}

// One wavefront per token, expert e = lane + 64 j in register j.
template <bool BF16, int VPL>
__global__ __launch_bounds__(kRouterThreads) void router_fwd_kernel(RouterArgs a) {
  extern __shared__ char smem[];
  float* sh_prob = (float*)smem;                             // [waves][E]
  int32_t* sh_count = (int32_t*)(sh_prob + kRouterWaves * a.E);  // [E]
  int32_t* sh_tokens = sh_count + a.E;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const bool stats = a.prob_part != nullptr;
  if (stats) {
    for (int e = threadIdx.x; e < a.E; e += kRouterThreads) sh_count[e] = 0;
    if (threadIdx.x == 0) *sh_tokens = 0;
    __syncthreads();
  }
  float acc[VPL] = {};
  int tokens = 0;
  const bool sig = a.sigmoid != 0;
  for (int64_t t = (int64_t)blockIdx.x * kRouterWaves + wave; t < a.T; t += (int64_t)gridDim.x * kRouterWaves) {
    float v[VPL], s[VPL];
    bool some = false;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int e = lane + 64 * j;
      v[j] = e < a.E ? load_logit<BF16>(a.logits, t * a.ld + e) : kNegInf;
      some |= v[j] != kNegInf;  // true for a NaN
    }
    const bool alive = __any(some) && (!a.mask || a.mask[t]);
    const float sum = token_scores<VPL>(v, sig, s);
    int id = -1;  // this lane's place, k = lane
    if (a.ids_in) {
      if (lane < a.K) id = a.ids_in[t * a.K + lane];
      if ((unsigned)id >= (unsigned)a.E) id = -1;
    } else {
      float key[VPL];
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        const int e = lane + 64 * j;
        key[j] = v[j];
        if (a.bias && e < a.E) key[j] = s[j] + a.bias[e];
        if (!(v[j] > kNegInf) || !(key[j] > kNegInf)) key[j] = kNegInf;
      }
      for (int k = 0; k < a.K; ++k) {
        float best = kNegInf;
#pragma unroll
        for (int j = 0; j < VPL; ++j) best = fmaxf(best, key[j]);
        best = wave_max(best);
        if (best == kNegInf) break;
        int at = INT_MAX;
#pragma unroll
        for (int j = VPL - 1; j >= 0; --j)
          if (key[j] == best) at = lane + 64 * j;
        at = wave_min(at);
        if (lane == k) id = at;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
          if (lane + 64 * j == at) key[j] = kNegInf;
      }
    }
    if (!alive) id = -1;
    const float x = id >= 0 ? load_logit<BF16>(a.logits, t * a.ld + id) : kNegInf;
    if (x == kNegInf) id = -1;
    float m = kNegInf;
#pragma unroll
    for (int j = 0; j < VPL; ++j) m = fmaxf(m, v[j]);
    m = wave_max(m);
    float denom;
    const float g = place_gate(x, id < 0, sig, a.renorm != 0, m == kNegInf ? 0.0f : m, sum, &denom);
    if (lane < a.K) {
      a.ids[t * a.K + lane] = id;
      a.gates[t * a.K + lane] = id < 0 ? 0.0f : a.scale * g;
    }
    if (stats && alive) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int j = 0; j < VPL; ++j) acc[j] += s[j] * inv;
      ++tokens;
      if (lane < a.K && id >= 0) atomicAdd(&sh_count[id], 1);
    }
  }
  if (!stats) return;
#pragma unroll
  for (int j = 0; j < VPL; ++j) {
    const int e = lane + 64 * j;
    if (e < a.E) sh_prob[wave * a.E + e] = acc[j];
  }
  if (lane == 0) atomicAdd(sh_tokens, tokens);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouterThreads) {
    float p = 0.0f;
    for (int w = 0; w < kRouterWaves; ++w) p += sh_prob[w * a.E + e];
    a.prob_part[(size_t)blockIdx.x * a.E + e] = p;
    a.count_part[(size_t)blockIdx.x * a.E + e] = sh_count[e];
  }
  if (threadIdx.x == 0) a.token_part[blockIdx.x] = *sh_tokens;
}

// The workgroups' partial statistics summed in their order.
__global__ __launch_bounds__(1024) void router_stats_kernel(int E, int blocks, const float* prob_part,
                                                            const int32_t* count_part, const int32_t* token_part,
                                                            int32_t* counts, int32_t* n_tokens, float* prob_mean,
                                                            float* loss) {
  __shared__ float sh_loss[16];
  __shared__ int sh_total[16];
  const int e = threadIdx.x, lane = lane_id(), wave = threadIdx.x >> 6;
  int n = 0, c = 0;
  float p = 0.0f;
  for (int b = 0; b < blocks; ++b) {
    n += token_part[b];
    if (e < E) {
      p += prob_part[(size_t)b * E + e];
      c += count_part[(size_t)b * E + e];
    }
  }
  const float mean = p / (float)max(n, 1);
  if (e < E) {
    counts[e] = c;
    prob_mean[e] = mean;
  }
  const float part = wave_sum((float)c * mean);
  int total = c;
  for (int o = 32; o >= 1; o >>= 1) total += __shfl_xor(total, o, 64);
  if (lane == 0) {
    sh_loss[wave] = part;
    sh_total[wave] = total;
  }
  __syncthreads();
  if (e == 0) {
    float l = 0.0f;
    int all = 0;
    for (int w = 0; w < 16; ++w) {
      l += sh_loss[w];
      all += sh_total[w];
    }
    *n_tokens = n;
    *loss = (float)E * (l / (float)max(all, 1));
  }
}

template <bool BF16, int VPL>
__global__ __launch_bounds__(kRouterThreads) void router_bwd_kernel(RouterArgs a) {
  __shared__ int sh_total;
  const int lane = lane_id(), wave = threadIdx.x >> 6;
  const bool sig = a.sigmoid != 0, renorm = a.renorm != 0, balance = a.coef != 0.0f;
  float c[VPL] = {};
  if (balance) {
    if (threadIdx.x == 0) sh_total = 0;
    __syncthreads();
    int mine = 0;
    for (int e = threadIdx.x; e < a.E; e += kRouterThreads) mine += a.counts[e];
    atomicAdd(&sh_total, mine);
    __syncthreads();
    const float k = a.coef * (float)a.E / (float)max(*a.n_tokens, 1) / (float)max(sh_total, 1);
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int e = lane + 64 * j;
      if (e < a.E) c[j] = k * (float)a.counts[e];
    }
  }
  for (int64_t t = (int64_t)blockIdx.x * kRouterWaves + wave; t < a.T; t += (int64_t)gridDim.x * kRouterWaves) {
    float v[VPL], s[VPL], d[VPL];
    bool some = false;
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int e = lane + 64 * j;
      v[j] = e < a.E ? load_logit<BF16>(a.logits, t * a.ld + e) : kNegInf;
      some |= v[j] != kNegInf;
      d[j] = 0.0f;
    }
    if (__any(some) && (!a.mask || a.mask[t])) {
      const float sum = token_scores<VPL>(v, sig, s);
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      float w = 0.0f;
      int id = -1;
      if (a.dgates) {
        if (lane < a.K) id = a.ids[t * a.K + lane];
        if ((unsigned)id >= (unsigned)a.E) id = -1;
        const float x = id >= 0 ? load_logit<BF16>(a.logits, t * a.ld + id) : kNegInf;
        const float dg = id >= 0 ? a.scale * a.dgates[t * a.K + lane] : 0.0f;
        w = dg;
        if (renorm) {
          float denom;
          const float q = place_gate(x, id < 0, sig, true, 0.0f, 0.0f, &denom);
          const float dot = wave_sum(q * dg);
          w = id < 0 || denom == 0.0f ? 0.0f : sig ? (dg - dot) / denom : q * (dg - dot);
        }
      }
      float ds[VPL] = {};  // what the gates give: of the score, or of the logit (softmax renormalised)
      if (a.dgates)
        for (int k = 0; k < a.K; ++k) {
          const int ik = __shfl(id, k, 64);
          const float wk = __shfl(w, k, 64);
#pragma unroll
          for (int j = 0; j < VPL; ++j)
            if (lane + 64 * j == ik) ds[j] += wk;
        }
      float pc = 0.0f;  // sum of pi times its gradient
      const bool through_pi = !sig && !renorm;
#pragma unroll
      for (int j = 0; j < VPL; ++j) pc += s[j] * inv * (c[j] + (through_pi ? ds[j] : 0.0f));
      if (balance || through_pi) pc = wave_sum(pc);
#pragma unroll
      for (int j = 0; j < VPL; ++j) {
        const float pi = s[j] * inv;
        float r = 0.0f;
        if (through_pi) {
          r = pi * (c[j] + ds[j] - pc);
        } else if (sig) {
          r = s[j] * (1.0f - s[j]) * ds[j];
          if (balance) r += pi * (1.0f - s[j]) * (c[j] - pc);
        } else {
          r = ds[j];
          if (balance) r += pi * (c[j] - pc);
        }
        d[j] = r;
      }
    }
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
      const int e = lane + 64 * j;
      if (e >= a.E) continue;
      if constexpr (BF16)
        ((uint16_t*)a.dlogits)[t * a.ld_out + e] = (uint16_t)pack_bf2(d[j], 0.0f);
      else
        ((float*)a.dlogits)[t * a.ld_out + e] = d[j];
    }
  }
}

size_t router_ws_bytes(int32_t E) {
  return align_up(256 + sizeof(int32_t) * (size_t)kRouterBlocks * (2 * (size_t)E + 1), 256);
}

// launch(VPL as a constant): registers for E experts over 64 lanes.
template <class Launch>
void by_experts(int E, Launch&& launch) {
  if (E <= 64) launch(std::integral_constant<int, 1>{});
  else if (E <= 128) launch(std::integral_constant<int, 2>{});
  else if (E <= 256) launch(std::integral_constant<int, 4>{});
  else if (E <= 512) launch(std::integral_constant<int, 8>{});
  else launch(std::integral_constant<int, 16>{});
}

unsigned router_grid(int64_t T, int64_t most) {
  const int64_t g = (T + kRouterWaves - 1) / kRouterWaves;
  return (unsigned)(g < 1 ? 1 : g < most ? g : most);
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static int check_router(const char* who, const void* logits, foremoe_dtype dtype, int64_t ld, int64_t T, int32_t E,
                        int32_t K, foremoe_score score, float scale) {
  REQUIRE(dtype == FOREMOE_BF16 || dtype == FOREMOE_F32, "%s: bad dtype", who);
  REQUIRE(E >= 1 && E <= FOREMOE_MAX_EXPERTS, "%s: E=%d outside [1, %d]", who, E, FOREMOE_MAX_EXPERTS);
  REQUIRE(K >= 1 && K <= FOREMOE_MAX_TOPK && K <= E, "%s: K=%d outside [1, min(E, %d)]", who, K, FOREMOE_MAX_TOPK);
  REQUIRE(T >= 0 && T <= INT_MAX && T * (int64_t)K < (int64_t)INT_MAX, "%s: T*K must be in [0, 2^31)", who);
  REQUIRE(ld >= E && ld <= (int64_t)1 << 31, "%s: ld=%lld outside [E=%d, 2^31]", who, (long long)ld, E);
  REQUIRE(score == FOREMOE_SOFTMAX || score == FOREMOE_SIGMOID, "%s: bad score function", who);
  REQUIRE(isfinite(scale), "%s: scale is not finite", who);
  REQUIRE(logits || T == 0, "%s: logits is NULL", who);
  REQUIRE(((uintptr_t)logits & (dtype == FOREMOE_BF16 ? 1 : 3)) == 0, "%s: logits misaligned", who);
  return FOREMOE_OK;
}

extern "C" {

size_t foremoe_router_workspace_size(int32_t E) {
  if (E < 1 || E > FOREMOE_MAX_EXPERTS) return 0;
  return router_ws_bytes(E);
}

int foremoe_router_fwd(const void* logits, foremoe_dtype dtype, int64_t ld, int64_t T, int32_t E, int32_t K,
                       foremoe_score score, int32_t renorm, float scale, const float* bias, const uint8_t* mask,
                       const int32_t* ids_in, int32_t* ids, float* gates, int32_t* counts, int32_t* n_tokens,
                       float* prob_mean, float* balance_loss, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_router("router_fwd", logits, dtype, ld, T, E, K, score, scale);
  if (rc) return rc;
  REQUIRE((ids && gates) || T == 0, "router_fwd: ids or gates is NULL");
  REQUIRE(!bias || score == FOREMOE_SIGMOID, "router_fwd: a bias goes with sigmoid scores only");
  const int n_stats = !!counts + !!n_tokens + !!prob_mean + !!balance_loss;
  REQUIRE(n_stats == 0 || n_stats == 4, "router_fwd: all four statistics or none");
  if (n_stats) {
    REQUIRE(ws && ((uintptr_t)ws & 255) == 0, "router_fwd: workspace NULL or not 256-byte aligned");
    REQUIRE(ws_bytes >= router_ws_bytes(E), "router_fwd: workspace too small (%zu < %zu)", ws_bytes,
            router_ws_bytes(E));
  } else if (T == 0) {
    return FOREMOE_OK;
  }
  RouterArgs a{};
  a.logits = logits, a.ld = ld, a.T = T, a.E = E, a.K = K;
  a.sigmoid = score == FOREMOE_SIGMOID, a.renorm = renorm, a.scale = scale;
  a.bias = ids_in ? nullptr : bias, a.mask = mask, a.ids_in = ids_in, a.ids = ids, a.gates = gates;
  const unsigned grid = router_grid(T, n_stats ? kRouterBlocks : 1 << 16);
  size_t smem = 0;
  if (n_stats) {
    a.prob_part = (float*)((char*)ws + 256);
    a.count_part = (int32_t*)(a.prob_part + (size_t)kRouterBlocks * E);
    a.token_part = a.count_part + (size_t)kRouterBlocks * E;
    smem = sizeof(float) * ((size_t)(kRouterWaves + 1) * E + 1);
  }
  hipStream_t st = (hipStream_t)stream;
  by_experts(E, [&](auto vpl) {
    if (dtype == FOREMOE_BF16)
      hipLaunchKernelGGL((router_fwd_kernel<true, decltype(vpl)::value>), dim3(grid), dim3(kRouterThreads), smem, st, a);
    else
      hipLaunchKernelGGL((router_fwd_kernel<false, decltype(vpl)::value>), dim3(grid), dim3(kRouterThreads), smem, st,
                         a);
  });
  if (n_stats)
    hipLaunchKernelGGL(router_stats_kernel, dim3(1), dim3(1024), 0, st, E, (int)grid, a.prob_part, a.count_part,
                       a.token_part, counts, n_tokens, prob_mean, balance_loss);
  return check_launch("router_fwd");
}

int foremoe_router_bwd(const void* logits, foremoe_dtype dtype, int64_t ld, int64_t T, int32_t E, int32_t K,
                       foremoe_score score, int32_t renorm, float scale, const uint8_t* mask, const int32_t* ids,
                       const float* dgates, const int32_t* counts, const int32_t* n_tokens, float balance_coef,
                       void* dlogits, int64_t ld_out, void* stream) {
  int rc = check_router("router_bwd", logits, dtype, ld, T, E, K, score, scale);
  if (rc) return rc;
  REQUIRE(isfinite(balance_coef), "router_bwd: balance_coef is not finite");
  REQUIRE(balance_coef == 0.0f || (counts && n_tokens), "router_bwd: a balance gradient needs counts and n_tokens");
  REQUIRE(ld_out >= E && ld_out <= (int64_t)1 << 31, "router_bwd: ld_out=%lld outside [E=%d, 2^31]",
          (long long)ld_out, E);
  REQUIRE(dlogits != logits || ld == ld_out || T == 0, "router_bwd: in place needs ld_out == ld");
  if (T == 0) return FOREMOE_OK;
  REQUIRE(dlogits && (!dgates || ids), "router_bwd: NULL buffer");
  REQUIRE(((uintptr_t)dlogits & (dtype == FOREMOE_BF16 ? 1 : 3)) == 0, "router_bwd: dlogits misaligned");
  RouterArgs a{};
  a.logits = logits, a.ld = ld, a.T = T, a.E = E, a.K = K;
  a.sigmoid = score == FOREMOE_SIGMOID, a.renorm = renorm, a.scale = scale;
  a.mask = mask, a.ids = const_cast<int32_t*>(ids), a.dgates = dgates, a.counts = counts, a.n_tokens = n_tokens;
  a.coef = balance_coef, a.dlogits = dlogits, a.ld_out = ld_out;
  const unsigned grid = router_grid(T, 4096);
  hipStream_t st = (hipStream_t)stream;
  by_experts(E, [&](auto vpl) {
    if (dtype == FOREMOE_BF16)
      hipLaunchKernelGGL((router_bwd_kernel<true, decltype(vpl)::value>), dim3(grid), dim3(kRouterThreads), 0, st, a);
    else
      hipLaunchKernelGGL((router_bwd_kernel<false, decltype(vpl)::value>), dim3(grid), dim3(kRouterThreads), 0, st, a);
  });
  return check_launch("router_bwd");
}

}  // extern "C"
