// The expert layer for a few tokens: from ids and gates to the output in two
// launches. Both stream the picked experts' weights once from memory straight
// into registers as the first operand of the matrix instructions (16 rows of
// weights by up to 16 tokens); nothing else is worth counting.
//
//   gate/up: a workgroup takes 8 hidden columns (8 rows of Wg, 8 of Wu) of one
//     expert, its wavefronts the k axis; H in fp32, as two bf16 planes (its
//     rounding, and what that leaves) where the weights are bf16 or 4 bits.
//   down: a workgroup takes 8 output columns of every expert, its wavefronts
//     the experts, or parts of their k axis where experts are few. So it holds
//     a token's sum over its experts alone: no partial sums in memory, no
//     counters, a fixed order.
#include "common.h"
#include "mx.h"

namespace foremoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

enum Weights { kBf16 = 0, kF32 = 1, kFp4 = 2 };

struct FewArgs {
  const void* x;  // [T, d], rows ld elements apart
  int64_t ld;
  int T, K, E, W, d, F, Fp;  // Fp: row length of h, F rounded up
  const int32_t* ids;
  const float* gates;
  const int32_t* widx;
  const char *gu, *dn;               // weights or codes
  const uint8_t *gu_scales, *dn_scales;
  char* h;                           // bf16: planes [2][pairs][Fp]; fp32: [pairs][Fp]
  void* y;
  int y_f32;
};

// The weights that pair p goes to, or -1.
__device__ __forceinline__ int pair_weights(const FewArgs& a, int p) {
  const int id = a.ids[p];
  if (id < 0 || id >= a.E) return -1;
  const int w = a.widx ? a.widx[id] : id;
  return w >= 0 && w < a.W ? w : -1;
}

// A chunk is 64 bytes of a row of weights: 16 bytes for each of four lanes.
template <int WT>
struct Chunk {
  static constexpr int PER_LANE = WT == kBf16 ? 8 : (WT == kF32 ? 4 : 32);  // elements
  static constexpr int K = 4 * PER_LANE;
  static constexpr int OPERANDS = WT == kFp4 ? 4 : 1;  // 16-byte operands of tokens per lane
  static constexpr int ES = WT == kF32 ? 4 : 2;        // bytes of a token's element
};

struct WeightFrag {
  uint4 v;
  float scale;
};

// This lane's part of chunk c of a row (zeros past its end). VEC: the row
// starts on 16 bytes and its length is a multiple of them.
template <int WT, bool VEC>
__device__ __forceinline__ WeightFrag load_weights(const char* row, const uint8_t* scales, int n, int c, int g) {
  using C = Chunk<WT>;
  WeightFrag f;
  f.v = uint4{0, 0, 0, 0}, f.scale = 0.0f;
  const int k = c * C::K + g * C::PER_LANE;
  if (k >= n) return f;
  if constexpr (VEC) {
    f.v = *(const uint4*)(row + (size_t)c * 64 + g * 16);
    if constexpr (WT == kFp4) f.scale = mx_scale_operand(scales[k / kMxBlock]);
  } else if constexpr (WT == kBf16) {
    const uint16_t* p = (const uint16_t*)row + k;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (k + i < n) w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    f.v = uint4{w[0], w[1], w[2], w[3]};
  } else {
    const uint32_t* p = (const uint32_t*)row + k;
    f.v.x = p[0];
    if (k + 1 < n) f.v.y = p[1];
    if (k + 2 < n) f.v.z = p[2];
    if (k + 3 < n) f.v.w = p[3];
  }
  return f;
}

template <int WT>
struct TokenFrag {
  uint4 v[Chunk<WT>::OPERANDS];
};

// The same k of a token's row (of n elements, readable in 16 bytes if VEC).
template <int WT, bool VEC>
__device__ __forceinline__ TokenFrag<WT> load_token(const char* row, int n, int c, int g, bool there) {
  using C = Chunk<WT>;
  TokenFrag<WT> f;
#pragma unroll
  for (int i = 0; i < C::OPERANDS; ++i) f.v[i] = uint4{0, 0, 0, 0};
  const int k = c * C::K + g * C::PER_LANE;
  if (!there || k >= n) return f;
  if constexpr (VEC) {
#pragma unroll
    for (int i = 0; i < C::OPERANDS; ++i) f.v[i] = *(const uint4*)(row + (size_t)k * C::ES + 16 * i);
  } else {
    f.v[0] = load_weights<WT == kFp4 ? kBf16 : WT, false>(row, nullptr, n, c, g).v;
  }
  return f;
}

// acc[row of weights][token] += weights x tokens; PLANES of the tokens add up.
template <int WT, int PLANES>
__device__ __forceinline__ f32x4 multiply(const WeightFrag& w, const TokenFrag<WT>* t, f32x4 acc) {
  if constexpr (WT == kF32) {
    const float a[4] = {__uint_as_float(w.v.x), __uint_as_float(w.v.y), __uint_as_float(w.v.z), __uint_as_float(w.v.w)};
    const uint4 u = t[0].v[0];
    const float b[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
  } else if constexpr (WT == kBf16) {
#pragma unroll
    for (int p = 0; p < PLANES; ++p)
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.v),
                                                    __builtin_bit_cast(bf16x8, t[p].v[0]), acc, 0, 0, 0);
  } else {
    const uint32_t q[4] = {w.v.x, w.v.y, w.v.z, w.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 a = {mx_get2_bf16<0>(q[i], w.scale), mx_get2_bf16<1>(q[i], w.scale), mx_get2_bf16<2>(q[i], w.scale),
                       mx_get2_bf16<3>(q[i], w.scale)};
#pragma unroll
      for (int p = 0; p < PLANES; ++p)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                      __builtin_bit_cast(bf16x8, t[p].v[i]), acc, 0, 0, 0);
    }
  }
  return acc;
}

// ---------------------------------------------------------------------------
// gate/up. Grid: (tiles of 8 hidden columns, candidates): with more pairs than
// matrices a candidate is a matrix, else a pair, the first of those that share
// its matrix.
// ---------------------------------------------------------------------------
constexpr int kUpThreads = 256, kUpWaves = kUpThreads / 64;

template <int WT, bool VEC, int NG>
__device__ __forceinline__ void up_groups(const FewArgs& a, const uint16_t* list, int first, int count, const char* row,
                                          const uint8_t* scales, float (*red)[4][16][16]) {
  using C = Chunk<WT>;
  constexpr int U = 4;
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, col = lane & 15;
  const char* tok[NG];
  bool there[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int q = first + 16 * i + col;
    there[i] = q < count;
    tok[i] = (const char*)a.x + (there[i] ? (int64_t)(list[q] / a.K) * a.ld * C::ES : 0);
  }
  f32x4 acc[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) acc[i] = f32x4{0, 0, 0, 0};
  const int nc = (a.d + C::K - 1) / C::K;
  for (int c0 = wave; c0 < nc; c0 += U * kUpWaves) {
    WeightFrag w[U];
    TokenFrag<WT> t[U][NG];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = load_weights<WT, VEC>(row, scales, a.d, c0 + u * kUpWaves, g);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NG; ++i) t[u][i] = load_token<WT, VEC>(tok[i], a.d, c0 + u * kUpWaves, g, there[i]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NG; ++i) acc[i] = multiply<WT, 1>(w[u], &t[u][i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) red[wave][i][4 * g + q][col] = acc[i][q];
}

template <int WT, bool VEC>
__global__ __launch_bounds__(kUpThreads) void few_up_kernel(FewArgs a) {
  __shared__ uint16_t list[FOREMOE_FEW_PAIRS];
  __shared__ int s_count, s_earlier;
  __shared__ float red[kUpWaves][4][16][16];
  const int pairs = a.T * a.K, tid = threadIdx.x;
  const bool by_pair = pairs <= a.W;
  const int w = by_pair ? pair_weights(a, blockIdx.y) : (int)blockIdx.y;
  if (w < 0) return;
  if (tid == 0) s_count = 0, s_earlier = 0;
  __syncthreads();
  // the order of the list does not matter: a token's column is its own
  for (int p = tid; p < pairs; p += kUpThreads) {
    if (pair_weights(a, p) == w) {
      if (by_pair && p < (int)blockIdx.y) s_earlier = 1;
      list[atomicAdd(&s_count, 1)] = (uint16_t)p;
    }
  }
  __syncthreads();
  const int count = s_count;
  if (count == 0 || s_earlier) return;

  using C = Chunk<WT>;
  const int f0 = blockIdx.x * 8, r = lane_id() & 15;
  // rows 0-7: Wg, 8-15: Wu; those past F repeat the last and are not used
  const int f = f0 + (r & 7) < a.F ? f0 + (r & 7) : a.F - 1;
  const int64_t row = (int64_t)w * 2 * a.F + (r < 8 ? f : a.F + f);
  const char* rp = a.gu + (WT == kFp4 ? row * (a.d / 2) : row * a.d * C::ES);
  const uint8_t* sp = WT == kFp4 ? a.gu_scales + row * (a.d / kMxBlock) : nullptr;
  const int64_t plane = (int64_t)pairs * a.Fp;
  for (int first = 0; first < count; first += 64) {
    const int left = count - first;
    if (left <= 16) up_groups<WT, VEC, 1>(a, list, first, count, rp, sp, red);
    else if (left <= 32) up_groups<WT, VEC, 2>(a, list, first, count, rp, sp, red);
    else up_groups<WT, VEC, 4>(a, list, first, count, rp, sp, red);
    __syncthreads();
    const int n = left < 64 ? left : 64;
    for (int o = tid; o < n * 8; o += kUpThreads) {
      const int j = o & 7, q = o >> 3;
      float ga = 0, up = 0;
#pragma unroll
      for (int v = 0; v < kUpWaves; ++v) ga += red[v][q >> 4][j][q & 15], up += red[v][q >> 4][j + 8][q & 15];
      if (f0 + j < a.F) {
        const float h = ga / (1.0f + expf(-ga)) * up;
        const int64_t at = (int64_t)list[first + q] * a.Fp + f0 + j;
        if constexpr (WT == kF32) {
          ((float*)a.h)[at] = h;
        } else {
          const uint32_t hi = pack_bf2(h, 0.0f) & 0xffffu;
          ((uint16_t*)a.h)[at] = (uint16_t)hi;
          // (an infinite h leaves NaN: nothing)
          const float rest = h - bf2f(hi);
          ((uint16_t*)a.h)[plane + at] = rest == rest ? (uint16_t)pack_bf2(rest, 0.0f) : (uint16_t)0;
        }
      }
    }
    // the last tile also clears what the rows are longer than F
    if (blockIdx.x == gridDim.x - 1) {
      const int extra = a.Fp - a.F;
      for (int o = tid; o < n * extra; o += kUpThreads) {
        const int64_t at = (int64_t)list[first + o / extra] * a.Fp + a.F + o % extra;
        if constexpr (WT == kF32) ((float*)a.h)[at] = 0.0f;
        else ((uint16_t*)a.h)[at] = 0, ((uint16_t*)a.h)[plane + at] = 0;
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// down and the sum over a token's experts. The 16 rows of an instruction are 8
// output columns at two chunks of the k axis, and its 16 columns 8 tokens at
// the same two: the two diagonal quarters are the products.
// ---------------------------------------------------------------------------
constexpr int kDownThreads = 1024, kDownWaves = kDownThreads / 64;

template <int WT, bool VEC, int NG>
__device__ __forceinline__ void down_groups(const FewArgs& a, const uint16_t* list, int first, int count,
                                            const char* row, const uint8_t* scales, int part, int parts, float* yp) {
  using C = Chunk<WT>;
  constexpr int U = NG == 1 ? 4 : 2, PLANES = WT == kF32 ? 1 : 2;
  const int lane = lane_id(), g = lane >> 4, r = lane & 15, odd = r >> 3;
  const int64_t plane = (int64_t)a.T * a.K * a.Fp * C::ES;
  const char* tok[NG];
  bool there[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int q = first + 8 * i + (r & 7);
    there[i] = q < count;
    tok[i] = a.h + (there[i] ? (int64_t)list[q] * a.Fp * C::ES : 0);
  }
  f32x4 acc[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) acc[i] = f32x4{0, 0, 0, 0};
  const int nc = (a.F + 2 * C::K - 1) / (2 * C::K);  // pairs of chunks
  for (int c0 = part; c0 < nc; c0 += U * parts) {
    WeightFrag w[U];
    TokenFrag<WT> t[U][NG][PLANES];
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = load_weights<WT, VEC>(row, scales, a.F, 2 * (c0 + u * parts) + odd, g);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NG; ++i)
#pragma unroll
        for (int p = 0; p < PLANES; ++p)
          t[u][i][p] = load_token<WT, true>(tok[i] + p * plane, a.Fp, 2 * (c0 + u * parts) + odd, g, there[i]);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < NG; ++i) acc[i] = multiply<WT, PLANES>(w[u], t[u][i], acc[i]);
  }
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      // row 4 g + q and column r of the even chunks, row + 8 and column + 8 of the odd
      const float v = acc[i][q] + __shfl(acc[i][q], (lane + 40) & 63, 64);
      const int at = first + 8 * i + r;
      if (r < 8 && g < 2 && at < count) yp[((size_t)part * a.T * a.K + list[at]) * 8 + 4 * g + q] = v;
    }
}

template <int WT, bool VEC, int CAP>
__global__ __launch_bounds__(kDownThreads) void few_down_kernel(FewArgs a) {
  __shared__ float yp[CAP * 8];              // [parts][pairs][8]
  __shared__ uint16_t list[FOREMOE_FEW_PAIRS];  // pairs by matrix
  __shared__ int16_t of_pair[FOREMOE_FEW_PAIRS];
  __shared__ int begin[FOREMOE_MAX_SLOTS + 1];
  __shared__ uint16_t used[FOREMOE_MAX_SLOTS];
  __shared__ int wave_pairs[kDownWaves], wave_used[kDownWaves];
  const int pairs = a.T * a.K, tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // group the pairs by matrix; the order within a group does not matter
  begin[tid] = 0;
  __syncthreads();
  int w_of[2], rank[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int p = tid + i * kDownThreads;
    w_of[i] = p < pairs ? pair_weights(a, p) : -1;
    if (p < pairs) of_pair[p] = (int16_t)w_of[i];
    if (w_of[i] >= 0) rank[i] = atomicAdd(&begin[w_of[i]], 1);
  }
  __syncthreads();
  const int mine = begin[tid];
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  const uint64_t any = __ballot(mine > 0);
  if (lane == 63) wave_pairs[wave] = upto;
  if (lane == 0) wave_used[wave] = __popcll(any);
  __syncthreads();
  int base = 0, ubase = 0, n_used = 0;
  for (int v = 0; v < kDownWaves; ++v) {
    if (v < wave) base += wave_pairs[v], ubase += wave_used[v];
    n_used += wave_used[v];
  }
  begin[tid] = base + upto - mine;
  if (tid == kDownThreads - 1) begin[FOREMOE_MAX_SLOTS] = base + upto;
  if (mine > 0) used[ubase + lanes_below(any)] = (uint16_t)tid;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (w_of[i] >= 0) list[begin[w_of[i]] + rank[i]] = (uint16_t)(tid + i * kDownThreads);
  __syncthreads();

  // parts of the k axis where experts are fewer than wavefronts
  int parts = 1;
  while (n_used > 0 && 2 * parts * n_used <= kDownWaves && 2 * parts * pairs <= CAP) parts *= 2;

  using C = Chunk<WT>;
  const int c0 = blockIdx.x * 8, r = lane & 15;
  const int out = c0 + (r & 7) < a.d ? c0 + (r & 7) : a.d - 1;
  for (int u = wave; u < n_used * parts; u += kDownWaves) {
    const int w = __builtin_amdgcn_readfirstlane(used[u / parts]), part = u % parts;
    const int first = __builtin_amdgcn_readfirstlane(begin[w]), count = __builtin_amdgcn_readfirstlane(begin[w + 1]);
    const int64_t row = (int64_t)w * a.d + out;
    const char* rp = a.dn + (WT == kFp4 ? row * (a.F / 2) : row * a.F * C::ES);
    const uint8_t* sp = WT == kFp4 ? a.dn_scales + row * (a.F / kMxBlock) : nullptr;
    for (int at = first; at < count; at += 32) {
      const int left = count - at;
      if (left <= 8) down_groups<WT, VEC, 1>(a, list, at, count, rp, sp, part, parts, yp);
      else if (left <= 16) down_groups<WT, VEC, 2>(a, list, at, count, rp, sp, part, parts, yp);
      else down_groups<WT, VEC, 4>(a, list, at, count, rp, sp, part, parts, yp);
    }
  }
  __syncthreads();
  for (int o = tid; o < a.T * 8; o += kDownThreads) {
    const int t = o >> 3, j = o & 7;
    if (c0 + j >= a.d) continue;
    float s = 0.0f;
    for (int k = 0; k < a.K; ++k) {
      const int p = t * a.K + k;
      if (of_pair[p] < 0) continue;
      float v = 0.0f;
      for (int q = 0; q < parts; ++q) v += yp[((size_t)q * pairs + p) * 8 + j];
      s += a.gates[p] * v;
    }
    const int64_t at = (int64_t)t * a.d + c0 + j;
    if (a.y_f32) ((float*)a.y)[at] = s;
    else ((uint16_t*)a.y)[at] = (uint16_t)pack_bf2(s, 0.0f);
  }
}

template <int WT, bool UP_VEC, bool DOWN_VEC>
void launch_few(const FewArgs& a, hipStream_t st) {
  const int pairs = a.T * a.K;
  hipLaunchKernelGGL((few_up_kernel<WT, UP_VEC>), dim3((a.F + 7) / 8, pairs < a.W ? pairs : a.W), dim3(kUpThreads), 0,
                     st, a);
  const dim3 grid((a.d + 7) / 8);
  if (pairs <= 512) hipLaunchKernelGGL((few_down_kernel<WT, DOWN_VEC, 512>), grid, dim3(kDownThreads), 0, st, a);
  else hipLaunchKernelGGL((few_down_kernel<WT, DOWN_VEC, 2048>), grid, dim3(kDownThreads), 0, st, a);
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

// h rows: whole pairs of chunks of the type with the most elements a chunk
static int64_t few_row(int64_t F) { return (F + 255) / 256 * 256; }

static int few_check(const char* name, const FewArgs& a, int64_t T, int64_t x_bytes, foremoe_dtype out_dtype,
                     const void* ws, size_t ws_bytes) {
  REQUIRE(out_dtype == FOREMOE_BF16 || out_dtype == FOREMOE_F32, "%s: bad output dtype", name);
  REQUIRE(T >= 0 && T <= FOREMOE_FEW_TOKENS, "%s: T=%lld outside [0, %d]", name, (long long)T, FOREMOE_FEW_TOKENS);
  REQUIRE(a.K >= 1 && a.K <= FOREMOE_MAX_TOPK && T * a.K <= FOREMOE_FEW_PAIRS, "%s: K=%d outside [1, %d], or T*K above %d",
          name, a.K, FOREMOE_MAX_TOPK, FOREMOE_FEW_PAIRS);
  REQUIRE(a.E >= 1 && a.E <= FOREMOE_MAX_EXPERTS, "%s: E=%d outside [1, %d]", name, a.E, FOREMOE_MAX_EXPERTS);
  REQUIRE(a.W >= 1 && a.W <= FOREMOE_MAX_SLOTS, "%s: W=%d outside [1, %d]", name, a.W, FOREMOE_MAX_SLOTS);
  REQUIRE(a.widx || a.E <= a.W, "%s: E=%d above W=%d without expert_widx", name, a.E, a.W);
  REQUIRE(a.d >= 1 && a.F >= 1 && 2 * (int64_t)a.d * a.F < (int64_t)1 << 31, "%s: d=%d, F=%d: 2 d F outside [1, 2^31)",
          name, a.d, a.F);
  REQUIRE(a.ld >= a.d && a.ld <= (int64_t)1 << 40, "%s: ld=%lld below d or above 2^40", name, (long long)a.ld);
  if (T == 0) return FOREMOE_OK;
  REQUIRE(a.x && a.ids && a.gates && a.gu && a.dn && a.y && ws, "%s: NULL pointer", name);
  REQUIRE(!misaligned(a.x, x_bytes) && !misaligned(a.ids, 4) && !misaligned(a.gates, 4) && !misaligned(a.widx, 4) &&
              !misaligned(a.gu, 16) && !misaligned(a.dn, 16) && !misaligned(a.y, out_dtype == FOREMOE_F32 ? 4 : 2),
          "%s: misaligned pointer", name);
  const size_t need = foremoe_few_workspace_size(T, a.K, a.F);
  REQUIRE(ws_bytes >= need, "%s: workspace too small (%zu < %zu bytes)", name, ws_bytes, need);
  REQUIRE(!misaligned(ws, 256), "%s: workspace misaligned", name);
  return FOREMOE_OK;
}

extern "C" {

size_t foremoe_few_workspace_size(int64_t T, int32_t K, int32_t F) {
  if (T < 0 || T > FOREMOE_FEW_TOKENS || K < 1 || K > FOREMOE_MAX_TOPK || T * K > FOREMOE_FEW_PAIRS || F < 1) return 0;
  const size_t n = (size_t)(T * K) * (size_t)few_row(F) * 4;
  return n < 256 ? 256 : n;
}

int foremoe_few_tokens_ffn(const void* x, foremoe_dtype dtype, int64_t ld, int64_t T, int32_t d, int32_t F,
                           const int32_t* ids, const float* gates, int32_t K, int32_t E, const int32_t* expert_widx,
                           int32_t W, const void* w_gate_up, const void* w_down, void* y, foremoe_dtype out_dtype,
                           void* ws, size_t ws_bytes, void* stream) {
  REQUIRE(dtype == FOREMOE_BF16 || dtype == FOREMOE_F32, "few_tokens_ffn: bad dtype");
  FewArgs a{};
  a.x = x, a.ld = ld, a.T = (int)T, a.K = K, a.E = E, a.W = W, a.d = d, a.F = F, a.Fp = (int)few_row(F);
  a.ids = ids, a.gates = gates, a.widx = expert_widx, a.gu = (const char*)w_gate_up, a.dn = (const char*)w_down;
  a.h = (char*)ws, a.y = y, a.y_f32 = out_dtype == FOREMOE_F32;
  const int64_t b = dtype == FOREMOE_BF16 ? 2 : 4;
  const int rc = few_check("few_tokens_ffn", a, T, b, out_dtype, ws, ws_bytes);
  if (rc != FOREMOE_OK || T == 0) return rc;
  const bool up = d * b % 16 == 0 && ld * b % 16 == 0 && !misaligned(x, 16), down = F * b % 16 == 0;
  hipStream_t st = (hipStream_t)stream;
#define LAUNCH(WT)                                          \
  do {                                                      \
    if (up && down) launch_few<WT, true, true>(a, st);      \
    else if (up) launch_few<WT, true, false>(a, st);        \
    else if (down) launch_few<WT, false, true>(a, st);      \
    else launch_few<WT, false, false>(a, st);               \
  } while (0)
  if (dtype == FOREMOE_BF16) LAUNCH(kBf16);
  else LAUNCH(kF32);
#undef LAUNCH
  return check_launch("few_tokens_ffn");
}

int foremoe_few_tokens_ffn_mxfp4(const void* x, int64_t ld, int64_t T, int32_t d, int32_t F, const int32_t* ids,
                                 const float* gates, int32_t K, int32_t E, const int32_t* expert_widx, int32_t W,
                                 const uint8_t* gate_up_codes, const uint8_t* gate_up_scales,
                                 const uint8_t* down_codes, const uint8_t* down_scales, void* y,
                                 foremoe_dtype out_dtype, void* ws, size_t ws_bytes, void* stream) {
  FewArgs a{};
  a.x = x, a.ld = ld, a.T = (int)T, a.K = K, a.E = E, a.W = W, a.d = d, a.F = F, a.Fp = (int)few_row(F);
  a.ids = ids, a.gates = gates, a.widx = expert_widx, a.gu = (const char*)gate_up_codes, a.dn = (const char*)down_codes;
  a.gu_scales = gate_up_scales, a.dn_scales = down_scales;
  a.h = (char*)ws, a.y = y, a.y_f32 = out_dtype == FOREMOE_F32;
  const int rc = few_check("few_tokens_ffn_mxfp4", a, T, 2, out_dtype, ws, ws_bytes);
  if (rc != FOREMOE_OK) return rc;
  if (d % kMxBlock || F % kMxBlock)
    return set_error(FOREMOE_EUNSUPPORTED, "few_tokens_ffn_mxfp4: d=%d and F=%d must be multiples of %d", d, F, kMxBlock);
  if (T == 0) return FOREMOE_OK;
  REQUIRE(gate_up_scales && down_scales, "few_tokens_ffn_mxfp4: NULL pointer");
  REQUIRE(!misaligned(x, 16) && ld % 8 == 0, "few_tokens_ffn_mxfp4: x must start its rows on 16 bytes");
  launch_few<kFp4, true, true>(a, (hipStream_t)stream);
  return check_launch("few_tokens_ffn_mxfp4");
}

}  // extern "C"
