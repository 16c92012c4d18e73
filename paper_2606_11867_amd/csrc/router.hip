// The router around the expert layer (Sec. 2.1; replay of recorded ids,
// Sec. 5): ids and gates from logits, the balance loss with its counts, and
// the gradient of the logits.
//
// A row of logits is one load of 16 lanes (64 above 256 experts) and stays in
// their registers: scores, picks, gates and statistics need no second pass.
// The bytes (32768 x 256 bf16: 17 MB, 3 us) are not what bounds it; the picks
// are, K maxima over a token's lanes one after another, and below some
// thousand tokens a launch's round trips to memory. The picked logits are
// read again by id, from cache, so that replayed and picked ids take one path.
// Kernels' times on MI355X (us):
//   24 x 128 bf16, 8 picks 3.5; 16384 x 128 fp32: 7.8 picked, 3.3-3.7 replayed
//   32768 x 256 bf16: 12.1, with sigmoid scores and bias 22; replayed 4.7
//   statistics: 2 to 5 more in the kernel and one of 5.4-5.7 behind it
//   backward: 16384 x 128 fp32 6.4-7.3, 32768 x 256 bf16 13.0-14.1
// Statistics: a workgroup sums its tokens' distributions in registers (fp32) and
// counts picks in LDS, leaves them in the workspace, and router_stats_kernel
// adds the workgroups' parts in a fixed order: no floating-point atomics. At
// most 512 workgroups (us, forward with statistics at 256, 512, 1024: 32768 x 256
// bf16 22.9, 21.7, 25.3; 16384 x 128 fp32 16.5, 15.3, 15.1).
#include <limits.h>
#include <math.h>

#include "common.h"

namespace foremoe {
namespace {

constexpr int kRouterThreads = 512;
constexpr int kRouterWaves = kRouterThreads / 64;
constexpr int kRouterBlocks = 512;  // most workgroups that leave partial statistics
constexpr int kStatColumns = 16;    // experts that a workgroup of the statistics kernel sums
constexpr int kStatThreads = 1024;
constexpr float kNegInf = -INFINITY;
constexpr float kLog2e = 1.4426950408889634f;

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

// ---------------------------------------------------------------------------
// A token is worked on by L lanes, 16 (four tokens to a wavefront) up to 256
// experts and all 64 above. Register j of lane l holds expert
// 4 (L (j / 4) + l) + j % 4, so that four registers are one load.
// ---------------------------------------------------------------------------
template <int L>
__device__ __forceinline__ int expert_of(int lane, int j) {
  return 4 * (L * (j / 4) + lane) + j % 4;
}

// Reductions over a token's lanes; every lane gets the same bits. Within 16
// lanes by rotations, which cost no more than the operation itself.
template <int CTRL>
__device__ __forceinline__ int rotated(int v) {
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
// v of the other 16 lanes of a pair of rows, or of the other half, combined.
template <class Op>
__device__ __forceinline__ int across_rows(int v, Op&& op) {
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = op((int)a[0], (int)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return op((int)b[0], (int)b[1]);
}
template <int L, class Op>
__device__ __forceinline__ float reduce(float v, Op&& op) {
  v = op(v, __int_as_float(rotated<0x128>(__float_as_int(v))));  // row_ror:8, 4, 2, 1
  v = op(v, __int_as_float(rotated<0x124>(__float_as_int(v))));
  v = op(v, __int_as_float(rotated<0x122>(__float_as_int(v))));
  v = op(v, __int_as_float(rotated<0x121>(__float_as_int(v))));
  if constexpr (L == 64)
    v = __int_as_float(across_rows(__float_as_int(v), [&](int a, int b) {
      return __float_as_int(op(__int_as_float(a), __int_as_float(b)));
    }));
  return v;
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  return reduce<L>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  return reduce<L>(v, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ uint32_t lanes_max_uint(uint32_t v) {
  v = max(v, (uint32_t)rotated<0x128>((int)v));
  v = max(v, (uint32_t)rotated<0x124>((int)v));
  v = max(v, (uint32_t)rotated<0x122>((int)v));
  v = max(v, (uint32_t)rotated<0x121>((int)v));
  if constexpr (L == 64)
    v = (uint32_t)across_rows((int)v, [](int a, int b) { return (int)max((uint32_t)a, (uint32_t)b); });
  return v;
}
template <int L>
__device__ __forceinline__ int lanes_min(int v) {
  v = min(v, rotated<0x128>(v));
  v = min(v, rotated<0x124>(v));
  v = min(v, rotated<0x122>(v));
  v = min(v, rotated<0x121>(v));
  if constexpr (L == 64) v = across_rows(v, [](int a, int b) { return min(a, b); });
  return v;
}

typedef float f32x4_a __attribute__((ext_vector_type(4)));

// Orders a wavefront's own LDS accesses.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// e^d for d <= 0, and the sigmoid: within |d| 2^-24 + 2 units in the last
// place. For sums over all experts (shares, the softmax's denominator), where an
// error counts by its term: sum p |d|, from the maximum, is at most log E.
__device__ __forceinline__ float fast_exp(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float fast_sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -kLog2e));
}
// e^d for d <= 0 within two units in the last place at any distance: for the
// gates, of which there are few.
__device__ __forceinline__ float near_exp(float d) {
  d = d < -200.0f ? -200.0f : d;  // keeps a NaN
  const float n = rintf(d * kLog2e);
  constexpr float kLog2eRest = 1.92596299e-8f;  // log2(e) minus its fp32 value
  const float f = fmaf(d, kLog2eRest, fmaf(d, kLog2e, -n));
  return __builtin_amdgcn_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
}
// The sigmoid of the definition's four fp32 operations, each rounded, where a
// score plus a bias decides. The quotient is the hardware's reciprocal
// corrected by its residual, correctly rounded up to 2^120 as the optimizer's
// (P. Markstein's method; adamw.hip has what holds for a significand of all
// ones).
template <int V>
__device__ __forceinline__ void exact_sigmoids(const float (&v)[V], float (&s)[V]) {
  bool far = false;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const float d = 1.0f + expf(-v[j]), r = __builtin_amdgcn_rcpf(d);
    s[j] = d > 0x1p120f ? 0.0f : fmaf(fmaf(-d, r, 1.0f), r, r);
    far |= d > 0x1p120f && d < INFINITY;
  }
  if (__any(far)) {
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = 1.0f / (1.0f + expf(-v[j]));
  }
}

// Whole numbers or floats [E] of a lane's experts, 0 beyond the last.
template <int L, int V, class T>
__device__ __forceinline__ void load_experts(const T* p, int E, int lane, T (&out)[V]) {
  typedef T four __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int j = 0; j < V; j += 4) {
    const int e = expert_of<L>(lane, j);
    four x = {0, 0, 0, 0};
    if (e + 4 <= E) {
      x = *(const four*)(p + e);
    } else if (E % 4 != 0) {
#pragma unroll
      for (int i = 0; i < 3; ++i)
        if (e + i < E) x[i] = p[e + i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) out[j + i] = x[i];
  }
}

// A token's row of logits, -inf beyond the last expert.
template <bool BF16, int L, int V>
__device__ __forceinline__ void load_row(const RouterArgs& a, int64_t t, int lane, float (&v)[V]) {
  typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
  const char* row = (const char*)a.logits + (size_t)t * a.ld * (BF16 ? 2 : 4);
  auto four = [&](int j, int e) {
    if constexpr (BF16) {
      const u16x4 x = *(const u16x4*)(row + 2 * e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[j + i] = bf2f(x[i]);
    } else {
      const f32x4 x = *(const f32x4*)(row + 4 * e);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[j + i] = x[i];
    }
  };
  if (a.E == L * V) {
#pragma unroll
    for (int j = 0; j < V; j += 4) four(j, expert_of<L>(lane, j));
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = kNegInf;
    if (a.E % 4 == 0) {
#pragma unroll
      for (int j = 0; j < V; j += 4)
        if (expert_of<L>(lane, j) < a.E) four(j, expert_of<L>(lane, j));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (expert_of<L>(lane, j) < a.E) v[j] = load_logit<BF16>(row, expert_of<L>(lane, j));
    }
  }
}

template <int L, int V>
__device__ __forceinline__ float row_max(const float (&v)[V]) {
  float most = v[0];
#pragma unroll
  for (int j = 1; j < V; ++j) most = fmaxf(most, v[j]);
  return lanes_max<L>(most);
}

// Whether some logit is not -inf (a NaN is not), the row's maximum (0 where
// there is none), its scores s and their sum. exact: sigmoids that decide.
template <int L, int V>
__device__ __forceinline__ bool row_scores(const float (&v)[V], bool sig, bool exact, float (&s)[V], float& top,
                                           float& sum) {
  bool some = false;
#pragma unroll
  for (int j = 0; j < V; ++j) some |= v[j] != kNegInf;
  top = 0.0f;
  if (exact) {
    exact_sigmoids<V>(v, s);
  } else if (sig) {
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = fast_sigmoid(v[j]);
  } else {
    const float m = row_max<L, V>(v);
    top = m > kNegInf ? m : 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] = fast_exp(v[j] - top);
  }
  sum = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j) sum += s[j];
  sum = lanes_sum<L>(sum);
  return lanes_max<L>(some ? 1.0f : 0.0f) != 0.0f;
}

// Sigmoid scores whose sum lies below this are all e^l to the last bit. Their
// shares of the sum come from e^(l - max): the scores themselves may be too
// small for fp32.
constexpr float kFarSum = 0x1p-60f;

// Adds the shares of such tokens (`far`).
template <int L, int V>
__device__ __forceinline__ void add_far_shares(const float (&v)[V], bool far, float (&acc)[V]) {
  float most = row_max<L, V>(v), all = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j) all += fast_exp(v[j] - most);
  all = lanes_sum<L>(all);
  asm volatile("" : "+v"(most));  // exponentials once more, not V registers that hold them
  const float inv = 1.0f / all;
#pragma unroll
  for (int j = 0; j < V; ++j) acc[j] += far ? fast_exp(v[j] - most) * inv : 0.0f;
}
// Puts e^(l - max) in the place of their scores, and its sum; returns what s
// is to be multiplied by to be the score again.
template <int L, int V>
__device__ __forceinline__ float far_scores(const float (&v)[V], bool far, float (&s)[V], float& sum) {
  const float most = row_max<L, V>(v);
  float all = 0.0f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    s[j] = far ? fast_exp(v[j] - most) : s[j];
    all += s[j];
  }
  all = lanes_sum<L>(all);
  sum = far ? all : sum;
  return far ? fast_exp(most) : 1.0f;
}

// The C * L places of a token, place lane + c L in register c: the scores q
// of the picked logits x over the sum that the gates divide by. Renormalised
// ones are scaled by the largest, so that small ones are not lost.
template <int L, int C>
__device__ __forceinline__ float place_scores(const float (&x)[C], const int (&id)[C], bool sig, bool renorm,
                                              float top, float sum, float (&q)[C]) {
  if (renorm) {
    top = kNegInf;
#pragma unroll
    for (int c = 0; c < C; ++c) top = fmaxf(top, id[c] < 0 ? kNegInf : x[c]);
    top = lanes_max<L>(top);
    if (!(top > kNegInf)) top = 0.0f;
  }
  const float up = renorm ? fminf(top, 0.0f) : 0.0f;
  float total = 0.0f;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    // the sigmoid is e^min(x, 0) / (1 + e^-|x|)
    q[c] = id[c] < 0 ? 0.0f
           : sig     ? near_exp(fminf(x[c], 0.0f) - up) * fast_sigmoid(fabsf(x[c]))
                     : near_exp(x[c] - top);
    total += q[c];
  }
  if (renorm) return lanes_sum<L>(total);
  return sig ? 1.0f : sum;
}

// The K largest keys in descending order, ties to the lower id; place k goes
// to lane k % L. Every pick compares and takes out one key by one.
template <int L, int V, int C>
__device__ __forceinline__ void pick_keys(float (&key)[V], int K, int lane, int (&id)[C]) {
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll 1
    for (int k = 0; k < L && c * L + k < K; ++k) {
      float best = key[0];
#pragma unroll
      for (int j = 1; j < V; ++j) best = fmaxf(best, key[j]);
      best = lanes_max<L>(best);
      int at = INT_MAX;
#pragma unroll
      for (int j = V - 1; j >= 0; --j) at = key[j] == best ? expert_of<L>(lane, j) : at;
      at = lanes_min<L>(at);
#pragma unroll
      for (int j = 0; j < V; ++j) key[j] = expert_of<L>(lane, j) == at ? kNegInf : key[j];
      if (lane == k) id[c] = best > kNegInf ? at : -1;
    }
  }
}

// The same for keys of 16 bits, each in one 32-bit integer with its expert:
// the key's bits in the order of the floats, the expert's complement below; 0
// for a key that is never picked. All of a token's integers differ, so the
// next one below the last pick is last + max(p - last) modulo 2^32 (what is
// not below wraps round to less): a subtraction and half a maximum for each,
// and nothing to take out. (32768 x 256: 19.7 -> 15.3 us. The leading 24 bits
// of fp32 keys, with pick_keys where those do not decide, were tried while one
// kernel found ids in every way, and its registers spilled; not since.)
template <int L, int V, int C>
__device__ __forceinline__ void pick_packed(const float (&key)[V], int K, int lane, int (&id)[C]) {
  constexpr uint32_t kIds = L == 16 ? 0xff : 0x3ff;
  static_assert(L * V <= kIds + 1);
  uint32_t p[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int32_t b = __float_as_int(key[j] + 0.0f);  // 0.0 and -0.0 tie
    const uint32_t o = (uint32_t)b ^ ((uint32_t)(b >> 31) | 0x80000000u);
    p[j] = key[j] > kNegInf ? (o & ~kIds) | (kIds - expert_of<L>(lane, j)) : 0;
  }
  uint32_t last = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
#pragma unroll 1
    for (int k = 0; k < L && c * L + k < K; ++k) {
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) most = max(most, p[j] - last);
      const uint32_t best = last + lanes_max_uint<L>(most);
      if (lane == k) id[c] = best ? (int)(kIds - (best & kIds)) : -1;
      last = best ? best : 1;  // from 1 the next is 0 again
    }
  }
}

// How a kernel finds its ids; each its own kernel, for the registers.
enum Pick { kReplay, kLogits, kBiased };

template <bool BF16, int PICK, int L, int V, int C>
__global__ __launch_bounds__(kRouterThreads, 4) void router_fwd_kernel(RouterArgs a) {
  constexpr int kTokens = 64 / L;  // of a wavefront
  extern __shared__ char smem[];
  float* sh_prob = (float*)smem;                                // [waves, E]
  int32_t* sh_count = (int32_t*)(sh_prob + kRouterWaves * a.E);  // [E]
  int32_t* sh_tokens = sh_count + a.E;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x % L, sub = lane_id() / L;
  const bool stats = a.prob_part != nullptr, sig = a.sigmoid != 0, renorm = a.renorm != 0;
  // replayed gates that need the picked logits alone
  const bool rows = stats || PICK != kReplay || (!sig && !renorm);
  if (stats) {
    for (int e = threadIdx.x; e < a.E; e += kRouterThreads) sh_count[e] = 0;
    if (threadIdx.x == 0) *sh_tokens = 0;
    __syncthreads();
  }
  float acc[V] = {}, bias[V] = {};
  int tokens = 0;
  if constexpr (PICK == kBiased) load_experts<L, V>(a.bias, a.E, lane, bias);
  // every lane of a wavefront stays in the loop while one of its tokens is left
  for (int64_t t0 = ((int64_t)blockIdx.x * kRouterWaves + wave) * kTokens; t0 < a.T;
       t0 += (int64_t)gridDim.x * kRouterWaves * kTokens) {
    const bool in = t0 + sub < a.T;
    const int64_t t = in ? t0 + sub : a.T - 1;
    bool alive = in && (!a.mask || a.mask[t]);
    float v[V], s[V], top = 0.0f, sum = 1.0f;
    int id[C];
    if constexpr (PICK == kReplay) {
#pragma unroll
      for (int c = 0; c < C; ++c) id[c] = lane + c * L < a.K ? a.ids_in[t * a.K + lane + c * L] : -1;
    }
    if (rows) {
      load_row<BF16, L, V>(a, t, lane, v);
      alive &= row_scores<L, V>(v, sig, PICK == kBiased, s, top, sum);
    }
    if (stats) {
      const bool far = sig && alive && !(sum >= kFarSum);
      if (__builtin_expect(__any(far), 0)) add_far_shares<L, V>(v, far, acc);
      if (alive) {
        const float inv = far ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] += s[j] * inv;
        ++tokens;
      }
    }
    if constexpr (PICK != kReplay) {
#pragma unroll
      for (int c = 0; c < C; ++c) id[c] = -1;
      float key[V];
      if constexpr (PICK == kBiased) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          key[j] = s[j] + bias[j];
          if (!(v[j] > kNegInf) || !(key[j] > kNegInf)) key[j] = kNegInf;
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) key[j] = v[j] > kNegInf ? v[j] : kNegInf;
      }
      if constexpr (BF16 && PICK == kLogits)
        pick_packed<L, V, C>(key, a.K, lane, id);
      else
        pick_keys<L, V, C>(key, a.K, lane, id);
    }
    float x[C], q[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      if (!alive || (unsigned)id[c] >= (unsigned)a.E) id[c] = -1;
      x[c] = id[c] >= 0 ? load_logit<BF16>(a.logits, t * a.ld + id[c]) : kNegInf;
      if (x[c] == kNegInf) id[c] = -1;
    }
    const float denom = place_scores<L, C>(x, id, sig, renorm, top, sum, q);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int k = lane + c * L;
      if (!in || k >= a.K) continue;
      a.ids[t * a.K + k] = id[c];
      a.gates[t * a.K + k] = id[c] < 0 || denom == 0.0f ? 0.0f : a.scale * (q[c] / denom);
      if (stats && id[c] >= 0) atomicAdd(&sh_count[id[c]], 1);
    }
  }
  if (!stats) return;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    if constexpr (L == 16) {
      acc[j] += __shfl_xor(acc[j], 16, 64);
      acc[j] += __shfl_xor(acc[j], 32, 64);
    }
    const int e = expert_of<L>(lane, j);
    if (sub == 0 && e < a.E) sh_prob[wave * a.E + e] = acc[j];
  }
  if (lane == 0) atomicAdd(sh_tokens, tokens);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouterThreads) {
    float p = 0.0f;
#pragma unroll
    for (int w = 0; w < kRouterWaves; ++w) p += sh_prob[w * a.E + e];
    a.prob_part[(size_t)blockIdx.x * a.E + e] = p;
    a.count_part[(size_t)blockIdx.x * a.E + e] = sh_count[e];
  }
  if (threadIdx.x == 0) a.token_part[blockIdx.x] = *sh_tokens;
}

// The workgroups' partial statistics summed in a fixed order: 16 experts to a
// workgroup, 64 threads to an expert, so that all loads of 512 workgroups'
// parts are under way at once. The last workgroup to finish adds up the
// balance loss; the results that it reads have reached memory before their
// workgroup took its ticket, past the XCDs' caches.
__global__ __launch_bounds__(kStatThreads) void router_stats_kernel(int E, int blocks, const float* prob_part,
                                                                    const int32_t* count_part,
                                                                    const int32_t* token_part, int32_t* counts,
                                                                    int32_t* n_tokens, float* prob_mean, float* loss,
                                                                    uint32_t* ticket) {
  constexpr int kRows = kStatThreads / kStatColumns, kWaves = kStatThreads / 64;
  __shared__ float sh_p[kWaves][kStatColumns];
  __shared__ int sh_c[kWaves][kStatColumns], sh_n[kWaves];
  __shared__ bool sh_last;
  const int tid = threadIdx.x, wave = tid >> 6;
  const int column = tid % kStatColumns, e = blockIdx.x * kStatColumns + column;
  int c = 0, n = 0;
  float p = 0.0f;
  for (int b = tid; b < blocks; b += kStatThreads) n += token_part[b];
  if (e < E) {
#pragma unroll 8
    for (int b = tid / kStatColumns; b < blocks; b += kRows) {
      p += prob_part[(size_t)b * E + e];
      c += count_part[(size_t)b * E + e];
    }
  }
#pragma unroll
  for (int o = kStatColumns; o < 64; o <<= 1) {
    p += __shfl_xor(p, o, 64);
    c += __shfl_xor(c, o, 64);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) n += __shfl_xor(n, o, 64);
  if (lane_id() == 0) sh_n[wave] = n;
  if (lane_id() < kStatColumns) sh_p[wave][column] = p, sh_c[wave][column] = c;
  __syncthreads();
  n = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) n += sh_n[w];
  if (tid < kStatColumns && e < E) {
    p = 0.0f, c = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) p += sh_p[w][tid], c += sh_c[w][tid];
    __hip_atomic_store(counts + e, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(prob_mean + e, p / (float)max(n, 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): they have reached memory
  }
  __syncthreads();
  if (tid == 0) sh_last = atomicAdd(ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!sh_last || wave != 0) return;
  float l = 0.0f;
  int all = 0;
#pragma unroll 4
  for (int i = tid; i < E; i += 64) {
    const int ci = __hip_atomic_load(counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    l += (float)ci * __hip_atomic_load(prob_mean + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    all += ci;
  }
  l = wave_sum(l);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) all += __shfl_xor(all, o, 64);
  if (tid == 0) {
    *n_tokens = n;
    *loss = (float)E * (l / (float)max(all, 1));
    __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

template <bool BF16, int L, int V, int C>
__global__ __launch_bounds__(kRouterThreads) void router_bwd_kernel(RouterArgs a) {
  constexpr int kTokens = 64 / L;
  typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
  __shared__ f32x4_a sh_w[C == 1 && L == 16 ? kRouterWaves : 1][kTokens][L * V / 4];  // a token's gradients by expert
  const int wave = threadIdx.x >> 6, lane = threadIdx.x % L, sub = lane_id() / L;
  const bool sig = a.sigmoid != 0, renorm = a.renorm != 0, balance = a.coef != 0.0f;
  const bool through_pi = !sig && !renorm;  // the gates' gradient goes through the whole softmax
  float push[V] = {};  // balance gradient of pi
  if (balance) {
    // a token's lanes hold all the counts; the total of many ranks' may pass 32
    // bits as a whole number
    int count[V];
    load_experts<L, V>(a.counts, a.E, lane, count);
    float total = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) total += (float)count[j];
    const int n = *a.n_tokens;
    total = lanes_sum<L>(total);
    const float k = a.coef * (float)a.E / (float)max(n, 1) / fmaxf(total, 1.0f);
#pragma unroll
    for (int j = 0; j < V; ++j) push[j] = k * (float)count[j];
  }
  for (int64_t t0 = ((int64_t)blockIdx.x * kRouterWaves + wave) * kTokens; t0 < a.T;
       t0 += (int64_t)gridDim.x * kRouterWaves * kTokens) {
    const bool in = t0 + sub < a.T;
    const int64_t t = in ? t0 + sub : a.T - 1;
    float v[V], s[V], top, sum;
    int id[C];
    float dg[C], x[C], w[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      id[c] = -1, dg[c] = w[c] = 0.0f;
      if (a.dgates && lane + c * L < a.K) {
        id[c] = a.ids[t * a.K + lane + c * L];
        dg[c] = a.scale * a.dgates[t * a.K + lane + c * L];
      }
      if ((unsigned)id[c] >= (unsigned)a.E) id[c] = -1;
    }
    load_row<BF16, L, V>(a, t, lane, v);
    const bool alive = row_scores<L, V>(v, sig, false, s, top, sum) && (!a.mask || a.mask[t]);
    float unit = 1.0f;  // the score over s
    const bool far = sig && alive && !(sum >= kFarSum);
    if (__builtin_expect(__any(far), 0)) unit = far_scores<L, V>(v, far, s, sum);
    const float inv = alive ? 1.0f / sum : 0.0f;
    float ds[V] = {};  // of the score, or, renormalised, of the logit (a sigmoid's over 1 - s)
    if (a.dgates) {
      if (renorm) {
        float q[C], dot = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) x[c] = id[c] >= 0 ? load_logit<BF16>(a.logits, t * a.ld + id[c]) : kNegInf;
        const float denom = place_scores<L, C>(x, id, sig, true, 0.0f, 0.0f, q);
        const float over = denom == 0.0f ? 0.0f : 1.0f / denom;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          q[c] *= over;
          if (id[c] >= 0) dot += q[c] * dg[c];
        }
        dot = lanes_sum<L>(dot);
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = id[c] < 0 ? 0.0f : q[c] * (dg[c] - dot);
      } else {
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = id[c] < 0 ? 0.0f : dg[c];
      }
      // every place's w to its expert's register: through LDS, or, where an
      // id comes twice in a token (the sum's order has to be the same every
      // time) or places take several registers, one place after another
      bool twice = C > 1 || L > 16;
      if constexpr (C == 1 && L == 16) {
        const int mine = id[0] >= 0 ? id[0] : -1 - lane;  // no two empty places alike
        twice |= mine == rotated<0x121>(mine) || mine == rotated<0x122>(mine) || mine == rotated<0x123>(mine) ||
                 mine == rotated<0x124>(mine) || mine == rotated<0x125>(mine) || mine == rotated<0x126>(mine) ||
                 mine == rotated<0x127>(mine) || mine == rotated<0x128>(mine);
      }
      if (C > 1 || L > 16 || __any(twice)) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
#pragma unroll 1
          for (int k = 0; k < L && c * L + k < a.K; ++k) {
            const int ik = __shfl(id[c], k, L);
            const float wk = __shfl(w[c], k, L);
#pragma unroll
            for (int j = 0; j < V; ++j) ds[j] += expert_of<L>(lane, j) == ik ? wk : 0.0f;
          }
        }
      } else {
        f32x4_a* mine = sh_w[C == 1 && L == 16 ? wave : 0][sub];
#pragma unroll
        for (int j = 0; j < V / 4; ++j) mine[L * j + lane] = f32x4_a{0.0f, 0.0f, 0.0f, 0.0f};
        wave_fence();
        if (id[0] >= 0) ((float*)mine)[id[0]] = w[0];
        wave_fence();
#pragma unroll
        for (int j = 0; j < V / 4; ++j) {
          const f32x4_a x4 = mine[L * j + lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) ds[4 * j + i] = x4[i];
        }
        wave_fence();
      }
    }
    float pc = 0.0f;  // sum of pi times its gradient
    if (balance || through_pi) {
#pragma unroll
      for (int j = 0; j < V; ++j) pc += s[j] * push[j];
      if (through_pi) {
#pragma unroll
        for (int j = 0; j < V; ++j) pc += s[j] * ds[j];
      }
      pc = lanes_sum<L>(pc) * inv;
    }
    if (through_pi) {
#pragma unroll
      for (int j = 0; j < V; ++j) ds[j] = s[j] * inv * (push[j] + ds[j] - pc);
    } else if (sig && renorm) {
#pragma unroll
      for (int j = 0; j < V; ++j) ds[j] = fmaf(-unit, s[j], 1.0f) * (ds[j] + s[j] * inv * (push[j] - pc));
    } else if (sig) {
#pragma unroll
      for (int j = 0; j < V; ++j)
        ds[j] = fmaf(-unit, s[j], 1.0f) * s[j] * (unit * ds[j] + inv * (push[j] - pc));
    } else if (balance) {
#pragma unroll
      for (int j = 0; j < V; ++j) ds[j] += s[j] * inv * (push[j] - pc);
    }
    if (!alive) {
#pragma unroll
      for (int j = 0; j < V; ++j) ds[j] = 0.0f;
    }
    if (!in) continue;
    char* row = (char*)a.dlogits + (size_t)t * a.ld_out * (BF16 ? 2 : 4);
    auto four = [&](int j, int e) {
      if constexpr (BF16)
        *(u32x2*)(row + 2 * e) = u32x2{pack_bf2(ds[j], ds[j + 1]), pack_bf2(ds[j + 2], ds[j + 3])};
      else
        *(f32x4*)(row + 4 * e) = f32x4{ds[j], ds[j + 1], ds[j + 2], ds[j + 3]};
    };
    if (a.E % 4 == 0) {
#pragma unroll
      for (int j = 0; j < V; j += 4)
        if (expert_of<L>(lane, j) < a.E) four(j, expert_of<L>(lane, j));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const int e = expert_of<L>(lane, j);
        if (e >= a.E) continue;
        if constexpr (BF16)
          ((uint16_t*)row)[e] = (uint16_t)pack_bf2(ds[j], 0.0f);
        else
          ((float*)row)[e] = ds[j];
      }
    }
  }
}

size_t router_ws_bytes(int32_t E) {
  return align_up(256 + sizeof(int32_t) * (size_t)kRouterBlocks * (2 * (size_t)E + 1), 256);
}

template <int L_, int V_, int C_>
struct Shape {
  static constexpr int L = L_, V = V_, C = C_;
};

// launch(the lanes of a token, registers for E experts and K places over them)
template <class Launch>
void by_shape(int E, int K, Launch&& launch) {
  if (E > 512) launch(Shape<64, 16, 1>{});
  else if (E > 256) launch(Shape<64, 8, 1>{});
  else if (K > 16) E <= 128 ? launch(Shape<16, 8, 4>{}) : launch(Shape<16, 16, 4>{});
  else if (E <= 64) launch(Shape<16, 4, 1>{});
  else if (E <= 128) launch(Shape<16, 8, 1>{});
  else launch(Shape<16, 16, 1>{});
}

unsigned router_grid(int64_t T, int L, int64_t most) {
  const int64_t tokens = kRouterWaves * (64 / L), g = (T + tokens - 1) / tokens;
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
  size_t smem = 0;
  if (n_stats) {
    a.prob_part = (float*)((char*)ws + 256);
    a.count_part = (int32_t*)(a.prob_part + (size_t)kRouterBlocks * E);
    a.token_part = a.count_part + (size_t)kRouterBlocks * E;
    smem = sizeof(float) * ((size_t)(kRouterWaves + 1) * E + 1);
  }
  hipStream_t st = (hipStream_t)stream;
  by_shape(E, K, [&](auto s) {
    constexpr int L = decltype(s)::L, V = decltype(s)::V, C = decltype(s)::C;
    const unsigned grid = router_grid(T, L, n_stats ? kRouterBlocks : 1 << 16);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(kRouterThreads), smem, st, a); };
    if (dtype == FOREMOE_BF16)
      ids_in ? launch(router_fwd_kernel<true, kReplay, L, V, C>)
      : bias ? launch(router_fwd_kernel<true, kBiased, L, V, C>)
             : launch(router_fwd_kernel<true, kLogits, L, V, C>);
    else
      ids_in ? launch(router_fwd_kernel<false, kReplay, L, V, C>)
      : bias ? launch(router_fwd_kernel<false, kBiased, L, V, C>)
             : launch(router_fwd_kernel<false, kLogits, L, V, C>);
    if (n_stats)
      hipLaunchKernelGGL(router_stats_kernel, dim3((E + kStatColumns - 1) / kStatColumns), dim3(kStatThreads), 0, st, E,
                         (int)grid, a.prob_part, a.count_part, a.token_part, counts, n_tokens, prob_mean, balance_loss,
                         (uint32_t*)ws);
  });
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
  hipStream_t st = (hipStream_t)stream;
  by_shape(E, K, [&](auto s) {
    constexpr int L = decltype(s)::L, V = decltype(s)::V, C = decltype(s)::C;
    const unsigned grid = router_grid(T, L, 4096);
    if (dtype == FOREMOE_BF16)
      hipLaunchKernelGGL((router_bwd_kernel<true, L, V, C>), dim3(grid), dim3(kRouterThreads), 0, st, a);
    else
      hipLaunchKernelGGL((router_bwd_kernel<false, L, V, C>), dim3(grid), dim3(kRouterThreads), 0, st, a);
  });
  return check_launch("router_bwd");
}

}  // extern "C"
