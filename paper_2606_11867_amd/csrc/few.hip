// The expert layer for a few tokens: from ids and gates to the output in two
// launches. Both stream the picked experts' weights once from memory straight
// into registers as the first operand of the matrix instructions (16 rows of
// weights by up to 16 tokens); nothing else is worth counting.
//
//   gate/up: a unit is 8 hidden columns (8 rows of Wg, 8 of Wu) of one matrix in
//     use; a workgroup to a CU takes its even share of all units, a wavefront a
//     unit or, where they are few, a part of its k axis.
//   down: a workgroup takes its even share of the output columns, of every
//     matrix in use, a wavefront up to 16 columns of one, or a part of their k
//     axis. So it holds a token's sum over its experts alone: no partial sums in
//     memory, no counters, a fixed order.
//
// Bound by memory where many experts are picked: 64 tokens over 32 experts of
// 7168 x 2048 in bf16 pick 28 of them, 2.45 GB, and take 313 and 169 us (5.2 and
// 4.8 TB/s); 24 tokens of 8 of 128 experts of 2048 x 768 in 4 bits, 0.25 GB, 37 and
// 33 us, of which a good part is each wavefront's wait for a unit's first weights.
// One token of 8 experts of 2048 x 768 takes 16 and 12 us, of which 12
// would be its 75 MB: there the latency of a launch, of the ids and of the first
// weights counts.
#include <type_traits>

#include "common.h"
#include "mx.h"

namespace foremoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;

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
  char* h;                           // bf16: planes [2 or 3][pairs][Fp]; fp32: [pairs][Fp]
  void* y;
  int y_f32;
  int planes;        // of the hidden rows
  int width, tiles;  // of the second product: output columns of a tile, tiles of a workgroup
};

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
  uint32_t scale;  // 4 bits: the block's scale byte
};

// The scale bytes of CHUNKS chunks from c on of a row of nb blocks, in one
// load (a load a byte took 17 of 101 us of 24 tokens in 4 bits). CHECKED: some
// may be past the row's end.
template <int CHUNKS, bool CHECKED>
__device__ __forceinline__ uint64_t load_scales(const uint8_t* scales, int nb, int c) {
  typedef typename std::conditional<CHUNKS == 2, uint64_t, uint32_t>::type Word;
  constexpr int N = 4 * CHUNKS;
  const int at = 4 * c;
  Word v = 0;
  if constexpr (CHECKED) {
    if (nb >= N) {  // the row's last ones, moved down
      const int from = at + N <= nb ? at : nb - N;
      __builtin_memcpy(&v, scales + from, N);
      v = at < nb ? v >> (8 * (at - from)) : 0;
    } else {
      for (int i = 0; i < N; ++i)
        if (at + i < nb) v |= (Word)scales[at + i] << (8 * i);
    }
  } else {
    __builtin_memcpy(&v, scales + at, N);
  }
  return v;
}

// This lane's part of chunk c of a row of n elements. CHECKED: zeros past its
// end. VEC: the row starts on 16 bytes and its length is a multiple of them.
template <int WT, bool VEC, bool CHECKED>
__device__ __forceinline__ uint4 load_weights(const char* row, int n, int c, int g) {
  using C = Chunk<WT>;
  const int k = c * C::K + g * C::PER_LANE;
  if constexpr (VEC) {
    if (CHECKED && k >= n) return uint4{0, 0, 0, 0};
    return *(const uint4*)(row + (size_t)c * 64 + g * 16);
  } else if constexpr (WT == kBf16) {
    const uint16_t* p = (const uint16_t*)row + k;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!CHECKED || k + i < n) w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
    return uint4{w[0], w[1], w[2], w[3]};
  } else {
    const uint32_t* p = (const uint32_t*)row + k;
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!CHECKED || k + i < n) w[i] = p[i];
    return uint4{w[0], w[1], w[2], w[3]};
  }
}

template <int WT>
struct TokenFrag {
  uint4 v[Chunk<WT>::OPERANDS];
};

// Tokens (or hidden rows) of a matrix, one to a column of a product. VEC: read
// through a range-checked buffer, in which a column without a token lies
// outside: it reads zeros, without a branch and without touching memory (lanes
// that read another's address again took a third of the gate/up product of 24
// tokens in 4 bits).
struct Tokens {
  __amdgpu_buffer_rsrc_t buffer;
  const char* base;  // (in LDS where they are staged)
};
constexpr uint32_t kOutside = 0xF0000000u;  // more than a buffer has, and room for a row behind it
constexpr int kFewSide = 1 << 25;           // longest row: 2^27 bytes

__device__ __forceinline__ Tokens tokens_at(const void* base, uint32_t bytes) {
  return Tokens{__builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000), (const char*)base};
}

// The same k of the token at offset `at`. STAGED: in LDS, whole chunks long.
template <int WT, bool VEC, bool STAGED, bool HIDDEN, bool CHECKED>
__device__ __forceinline__ TokenFrag<WT> load_token(const Tokens& tokens, uint32_t at, int n, int c, int g) {
  using C = Chunk<WT>;
  TokenFrag<WT> f;
  const int k = c * C::K + g * C::PER_LANE;
  if constexpr (STAGED) {
#pragma unroll
    for (int i = 0; i < C::OPERANDS; ++i)
      f.v[i] = __builtin_bit_cast(uint4, *(const lds_u32x4*)(uintptr_t)(at + (uint32_t)(k * C::ES + 16 * i)));
  } else if constexpr (VEC) {
    constexpr bool APART = HIDDEN && WT == kFp4;  // see h_place
    const uint32_t o = CHECKED && k >= n ? kOutside : at + (uint32_t)((APART ? c * C::K + g * 8 : k) * C::ES);
#pragma unroll
    for (int i = 0; i < C::OPERANDS; ++i)
      f.v[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(tokens.buffer, o, (APART ? 64 : 16) * i, 0));
  } else {
    f.v[0] = uint4{0, 0, 0, 0};
    if (at < kOutside) f.v[0] = load_weights<WT == kFp4 ? kBf16 : WT, false, CHECKED>(tokens.base + at, n, c, g);
  }
  return f;
}

// acc[row of weights][token] += weights x tokens.
template <int WT>
__device__ __forceinline__ f32x4 multiply(const WeightFrag& w, const TokenFrag<WT>& t, f32x4 acc) {
  if constexpr (WT == kF32) {
    const float a[4] = {__uint_as_float(w.v.x), __uint_as_float(w.v.y), __uint_as_float(w.v.z), __uint_as_float(w.v.w)};
    const uint4 u = t.v[0];
    const float b[4] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc, 0, 0, 0);
  } else if constexpr (WT == kBf16) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w.v), __builtin_bit_cast(bf16x8, t.v[0]),
                                                  acc, 0, 0, 0);
  } else {
    const uint32_t q[4] = {w.v.x, w.v.y, w.v.z, w.v.w};
    const float s = mx_scale_operand(w.scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 a = {mx_get2_bf16<0>(q[i], s), mx_get2_bf16<1>(q[i], s), mx_get2_bf16<2>(q[i], s),
                       mx_get2_bf16<3>(q[i], s)};
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, t.v[i]),
                                                    acc, 0, 0, 0);
    }
  }
  return acc;
}

// ---------------------------------------------------------------------------
// The pairs of a call by the matrix that they go to, in LDS: every workgroup
// finds them by itself.
// ---------------------------------------------------------------------------
struct Groups {
  uint16_t list[FOREMOE_FEW_PAIRS];      // pairs, matrix by matrix
  int16_t place[FOREMOE_FEW_PAIRS];      // of a pair in the list, or -1
  uint16_t used[FOREMOE_MAX_SLOTS];      // the matrices that have pairs
  uint16_t begin_used[FOREMOE_MAX_SLOTS + 1];  // their first places, and the end
  int begin[FOREMOE_MAX_SLOTS];          // (while grouping) pairs of a matrix, then its first place
  int waves[32];
  int n_used, most;                      // most: pairs of a matrix
};

// The order of the pairs within a matrix is whatever the atomics make it; no
// result depends on it, as a token's column of a product is its own.
template <int THREADS>
__device__ __forceinline__ void group_pairs(const FewArgs& a, Groups& G) {
  if (a.T * a.K <= 64) {
    // one wavefront, a lane to a pair, without the tables and the scan over all
    // matrices that more pairs need
    if (threadIdx.x < 64) {
      const int pairs = a.T * a.K, lane = lane_id();
      int w = lane < pairs ? a.ids[lane] : -1;
      if ((unsigned)w >= (unsigned)a.E) w = -1;
      if (w >= 0 && a.widx) w = a.widx[w];
      if ((unsigned)w >= (unsigned)a.W) w = -1;
      uint64_t left = __ballot(w >= 0);
      int at = 0, n = 0, most = 0;
      while (left) {
        const int p = __builtin_ctzll(left), v = __builtin_amdgcn_readlane(w, p);
        const uint64_t same = __ballot(w == v);
        const int m = __popcll(same);
        if (lane == 0) G.used[n] = (uint16_t)v, G.begin_used[n] = (uint16_t)at;
        if (w == v) G.list[at + lanes_below(same)] = (uint16_t)lane, G.place[lane] = (int16_t)(at + lanes_below(same));
        at += m, ++n, most = m > most ? m : most;
        left &= ~same;
      }
      if (lane < pairs && w < 0) G.place[lane] = -1;
      if (lane == 0) G.n_used = n, G.most = most, G.begin_used[n] = (uint16_t)at;
    }
    __syncthreads();
    return;
  }
  constexpr int WAVES = THREADS / 64, PER = FOREMOE_FEW_PAIRS / THREADS, WPER = FOREMOE_MAX_SLOTS / THREADS;
  const int pairs = a.T * a.K, tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int w[PER], rank[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * THREADS;
    w[i] = p < pairs ? a.ids[p] : -1;
    if ((unsigned)w[i] >= (unsigned)a.E) w[i] = -1;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (w[i] >= 0 && a.widx) w[i] = a.widx[w[i]];
    if ((unsigned)w[i] >= (unsigned)a.W) w[i] = -1;
  }
#pragma unroll
  for (int i = 0; i < WPER; ++i) G.begin[tid + i * THREADS] = 0;
  if (tid == 0) G.most = 16;  // (or less)
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) rank[i] = w[i] >= 0 ? atomicAdd(&G.begin[w[i]], 1) : 0;
  __syncthreads();
  // a thread's matrices are neighbours: tid * WPER ..
  int mine[WPER], sum = 0, some = 0;
#pragma unroll
  for (int i = 0; i < WPER; ++i) {
    mine[i] = G.begin[tid * WPER + i], sum += mine[i], some += mine[i] > 0;
    if (mine[i] > 16) atomicMax(&G.most, mine[i]);
  }
  int upto = sum | some << 16;  // at most 2048 pairs, 1024 matrices
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  if (lane == 63) G.waves[wave] = upto;
  __syncthreads();
  int before = upto - (sum | some << 16), all = 0;
#pragma unroll
  for (int v = 0; v < WAVES; ++v) {
    const int x = G.waves[v];
    if (v < wave) before += x;
    all += x;
  }
  int at = before & 0xffff, u = before >> 16;
#pragma unroll
  for (int i = 0; i < WPER; ++i) {
    G.begin[tid * WPER + i] = at;
    if (mine[i] > 0) G.begin_used[u] = (uint16_t)at, G.used[u++] = (uint16_t)(tid * WPER + i);
    at += mine[i];
  }
  if (tid == 0) G.n_used = all >> 16, G.begin_used[all >> 16] = (uint16_t)(all & 0xffff);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * THREADS, to = w[i] >= 0 ? G.begin[w[i]] + rank[i] : -1;
    if (p < pairs) G.place[p] = (int16_t)to;
    if (to >= 0) G.list[to] = (uint16_t)p;
  }
  __syncthreads();
}

// Parts that the k axis (nc steps) of each of n units is cut into for 16
// wavefronts, with `each` of `slots` partial sums for a part of all units: the
// shortest time, a unit or part costing four steps besides its own.
__device__ __forceinline__ int parts_for(int n, int nc, int each, int slots) {
  int best = 1, cost = (n + 15) / 16 * (nc + 4);
  for (int p = 2; p <= 16 && p <= nc && p * each <= slots; p *= 2) {
    const int c = (n * p + 15) / 16 * ((nc + p - 1) / p + 4);
    if (c < cost) cost = c, best = p;
  }
  return best;
}

// ---------------------------------------------------------------------------
// gate/up. A unit is 8 hidden columns of a matrix in use; a workgroup to a CU
// takes its even share of them, a wavefront a unit or a part of its k axis.
// ---------------------------------------------------------------------------
constexpr int kFewThreads = 1024, kFewWaves = 16, kUpSlots = 1024, kUpStage = 72 << 10;
static_assert(FOREMOE_FEW_PAIRS % kFewThreads == 0 && FOREMOE_MAX_SLOTS % kFewThreads == 0, "group_pairs");
// Steps of weights in flight behind those that are multiplied: as many as the
// registers of 16 wavefronts a CU hold beside NG groups of tokens.
template <int WT, int NG>
constexpr int kAhead = WT == kFp4 ? 1 : (NG == 4 ? 2 : 4);
template <int WT, int NG>
constexpr int kAheadStaged = NG == 1 ? 4 : 2;  // (4 for both spills registers: 51 us of 24 tokens in 4 bits, 37 so)
template <int WT, int NG>
constexpr int kAheadDown = WT == kFp4 ? (NG == 1 ? 2 : 1) : (NG == 4 ? 2 : 4);
// Groups of tokens that a step of weights is multiplied with, at most.
template <int WT>
constexpr int kGroups = WT == kFp4 ? 2 : 4;

// Rows of a unit, chunks [c0, c1) of them.
struct Stretch {
  const char* row;
  const uint8_t* scales;
  int c0, c1;
};
// U steps of weights on their way.
template <int WT, int U, int S>
struct Ahead {
  uint4 v[U];
  typename std::conditional<S == 2, uint64_t, uint32_t>::type scales[WT == kFp4 ? U : 1];
};
template <int WT, bool WVEC, int U, int S>
__device__ __forceinline__ void load_ahead(Ahead<WT, U, S>& to, const Stretch& s, int n, int c, int odd, int g) {
#pragma unroll
  for (int u = 0; u < U; ++u) to.v[u] = load_weights<WT, WVEC, false>(s.row, n, c + u * S + odd, g);
  if constexpr (WT == kFp4) {
#pragma unroll
    for (int u = 0; u < U; ++u) to.scales[u] = load_scales<S, false>(s.scales, 0, c + u * S);
  }
}

// sums[i] = rows of weights x the tokens at offsets tok[i] over a stretch, in
// steps of S chunks (lane: chunk c + odd where S is 2). U steps at a time
// without a branch, the weights of the next on their way while these are
// multiplied; then the steps that are left, one of which may end in the row's
// last, short chunk.
template <int WT, bool WVEC, bool TVEC, bool STAGED, bool HIDDEN, int NG, int U, int S>
__device__ __forceinline__ void stream_rows(const Stretch& s, int n, const Tokens& tokens, const uint32_t* tok, int nt,
                                            int odd, int g, f32x4* sums) {
#pragma unroll
  for (int i = 0; i < NG; ++i) sums[i] = f32x4{0, 0, 0, 0};
  const int by = 8 * g + (S == 2 ? 32 * odd : 0);  // bit of this lane's scale
  const int whole = min(s.c1, n / (Chunk<WT>::K * S) * S) - s.c0, blocks = whole > 0 ? whole / (U * S) : 0;
  if (blocks > 0) {
    Ahead<WT, U, S> next;
    load_ahead<WT, WVEC, U, S>(next, s, n, s.c0, odd, g);
    for (int b = 0; b < blocks; ++b) {
      const int c = s.c0 + b * U * S;
      WeightFrag w[U];
      TokenFrag<WT> t[STAGED ? 1 : U][NG];  // (from LDS a step at a time)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        w[u].v = next.v[u];
        if constexpr (WT == kFp4) w[u].scale = (uint32_t)(next.scales[u] >> by) & 0xffu;
      }
      auto load_t = [&](int to, int u) {
#pragma unroll
        for (int i = 0; i < NG; ++i)
          t[to][i] = load_token<WT, TVEC, STAGED, HIDDEN, false>(tokens, tok[i], nt, c + u * S + odd, g);
      };
      if constexpr (!STAGED) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_t(u, u);
      }
      load_ahead<WT, WVEC, U, S>(next, s, n, b + 1 < blocks ? c + U * S : c, odd, g);  // (the last again: no branch)
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if constexpr (STAGED) load_t(0, u);
#pragma unroll
        for (int i = 0; i < NG; ++i) sums[i] = multiply<WT>(w[u], t[STAGED ? 0 : u][i], sums[i]);
      }
    }
  }
  for (int c = s.c0 + blocks * U * S; c < s.c1; c += S) {
    WeightFrag w;
    w.v = load_weights<WT, WVEC, true>(s.row, n, c + odd, g);
    w.scale = WT == kFp4 ? (uint32_t)(load_scales<S, true>(s.scales, n / kMxBlock, c) >> by) & 0xffu : 0;
#pragma unroll
    for (int i = 0; i < NG; ++i)
      sums[i] = multiply<WT>(w, load_token<WT, TVEC, STAGED, HIDDEN, true>(tokens, tok[i], nt, c + odd, g), sums[i]);
  }
}

// Both products of up to 16 NG pairs from place `first` on, over a stretch.
// STAGED: the token of place q is at stage + (q - q0) * stride in LDS.
template <int WT, bool VEC, bool STAGED, int NG>
__device__ __forceinline__ void up_groups(const FewArgs& a, const Groups& G, uint32_t stage, int stride, int q0,
                                          int first, int end, const Stretch& s, f32x4* sums) {
  using C = Chunk<WT>;
  const int lane = lane_id(), g = lane >> 4, col = lane & 15;
  uint32_t tok[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int q = first + 16 * i + col;
    // (staged, a column without a token reads another's: no product of it is used)
    if constexpr (STAGED) tok[i] = stage + (uint32_t)(((q < end ? q : first) - q0) * stride);
    else tok[i] = q < end ? (uint32_t)(G.list[q] / a.K * a.ld * C::ES) : kOutside;
  }
  const Tokens x = tokens_at(a.x, (uint32_t)(((a.T - 1) * a.ld + a.d) * C::ES));
  constexpr int U = STAGED ? kAheadStaged<WT, NG> : kAhead<WT, NG>;
  stream_rows<WT, VEC, VEC, STAGED, false, NG, U, 1>(s, a.d, x, tok, a.d, 0, g, sums);
}

// The same of all pairs of one matrix, up to 16 kGroups at a time; done(sums,
// q) takes those of the 16 from place q on.
template <int WT, bool VEC, bool STAGED, class Done>
__device__ __forceinline__ void up_unit(const FewArgs& a, const Groups& G, uint32_t stage, int stride, int q0, int first,
                                        int end, const Stretch& s, Done&& done) {
  for (int at = first; at < end; at += 16 * kGroups<WT>) {
    f32x4 sums[4];
    if (end - at <= 16) {
      up_groups<WT, VEC, STAGED, 1>(a, G, stage, stride, q0, at, end, s, sums);
      done(sums[0], at);
    } else if (kGroups<WT> == 2 || end - at <= 32) {
      up_groups<WT, VEC, STAGED, 2>(a, G, stage, stride, q0, at, end, s, sums);
#pragma unroll
      for (int k = 0; k < 2; ++k) done(sums[k], at + 16 * k);
    } else {
      up_groups<WT, VEC, STAGED, kGroups<WT>>(a, G, stage, stride, q0, at, end, s, sums);
#pragma unroll
      for (int k = 0; k < kGroups<WT>; ++k) done(sums[k], at + 16 * k);
    }
  }
}

// Where element f of a hidden row lies. With 4-bit weights a lane takes 32
// neighbours of a chunk, eight at a time: the eights that the four lanes take
// together lie together.
template <int WT>
__device__ __forceinline__ int h_place(int f) {
  return WT == kFp4 ? (f & ~127) | (f >> 3 & 3) << 5 | (f >> 5 & 3) << 3 | (f & 7) : f;
}

// An element of the hidden rows: fp32, or a bf16 plane for its rounding and one
// or two for what the planes before leave.
template <int WT>
__device__ __forceinline__ void put_h(const FewArgs& a, int pair, int f, float gate, float up) {
  const float h = f < a.F ? gate / (1.0f + expf(-gate)) * up : 0.0f;
  const int64_t at = (int64_t)pair * a.Fp + h_place<WT>(f), plane = (int64_t)a.T * a.K * a.Fp;
  if constexpr (WT == kF32) {
    ((float*)a.h)[at] = h;
  } else {
    float left = h;
    for (int p = 0; p < a.planes; ++p) {
      const uint32_t b = pack_bf2(left, 0.0f) & 0xffffu;
      ((uint16_t*)a.h)[p * plane + at] = (uint16_t)b;
      left -= bf2f(b);
      if (!(fabsf(left) < INFINITY)) left = 0.0f;  // an infinite h leaves NaN: nothing
    }
  }
}

template <int WT, bool VEC>
__global__ __launch_bounds__(kFewThreads) void few_up_kernel(FewArgs a) {
  __shared__ Groups G;
  __shared__ float partial[kUpSlots][16];  // [unit][part][pair][row]
  __shared__ __attribute__((aligned(16))) char stage[WT == kFp4 ? kUpStage : 16];
  group_pairs<kFewThreads>(a, G);
  using C = Chunk<WT>;
  const int lane = lane_id(), g = lane >> 4, r = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // units are numbered matrix by matrix, so that a workgroup's are neighbours
  // in memory and have the same tokens
  const int n_used = G.n_used, tiles = (a.F + 7) / 8;
  const int64_t units = (int64_t)tiles * n_used;
  const int64_t u0 = units * blockIdx.x / gridDim.x;
  const int n = (int)(units * (blockIdx.x + 1) / gridDim.x - u0);
  if (n == 0) return;
  const int nc = (a.d + C::K - 1) / C::K;
  // In 4 bits the tokens of this workgroup's matrices are staged where they fit:
  // from memory they take four times as many loads as the weights (24 tokens:
  // 68 -> 57 us, 37 with what came after; with 16-bit weights, where they take as many, the wait for the
  // staging costs more than it saves, 298 -> 352).
  const int m0 = (int)(u0 / tiles), m1 = (int)((u0 + n - 1) / tiles);
  const int q0 = G.begin_used[m0], staged_pairs = G.begin_used[m1 + 1] - q0;
  const int stride = nc * C::K * C::ES + 16;  // rows 4 banks apart
  const bool staged = WT == kFp4 && staged_pairs * (int64_t)stride <= kUpStage;
  const uint32_t stage0 = (uint32_t)(uintptr_t)stage;
  if (staged) {
    const int per_row = nc * C::K * C::ES / 16, have = a.d * C::ES / 16;  // 16-byte pieces, and those before the end
    for (int o = threadIdx.x; o < staged_pairs * per_row; o += kFewThreads) {
      const int q = o / per_row, j = o % per_row;
      const char* from = (const char*)a.x + (int64_t)(G.list[q0 + q] / a.K) * a.ld * C::ES;
      *(uint4*)(stage + q * stride + 16 * j) = j < have ? ((const uint4*)from)[j] : uint4{0, 0, 0, 0};
    }
    __syncthreads();
  }
  const int parts = G.most <= 16 ? parts_for(n, nc, n * 16, kUpSlots) : 1;
  for (int i = wave; i < n * parts; i += kFewWaves) {
    const int unit = i / parts, part = i % parts;
    const int c = __builtin_amdgcn_readfirstlane((int)((u0 + unit) / tiles));
    const int tile = __builtin_amdgcn_readfirstlane((int)((u0 + unit) % tiles));
    const int k0 = nc * part / parts, k1 = nc * (part + 1) / parts;
    const int w = __builtin_amdgcn_readfirstlane(G.used[c]);
    const int first = __builtin_amdgcn_readfirstlane(G.begin_used[c]), end = __builtin_amdgcn_readfirstlane(G.begin_used[c + 1]);
    // rows 0-7: Wg, 8-15: Wu; those past F repeat the last and are not used
    const int f0 = tile * 8, f = f0 + (r & 7) < a.F ? f0 + (r & 7) : a.F - 1;
    const int64_t row = (int64_t)w * 2 * a.F + (r < 8 ? f : a.F + f);
    const char* rp = a.gu + (WT == kFp4 ? row * (a.d / 2) : row * a.d * C::ES);
    const uint8_t* sp = WT == kFp4 ? a.gu_scales + row * (a.d / kMxBlock) : nullptr;
    auto done = [&](f32x4 sums, int at) {
      // this lane: rows 4 g .. of column r; the up's are 8 rows below the gate's
      const int q = at + r;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v = sums[e], up = __shfl_xor(v, 32, 64);
        if (q >= end) continue;
        if (parts > 1) partial[(unit * parts + part) * 16 + r][4 * g + e] = v;
        else if (g < 2) put_h<WT>(a, G.list[q], f0 + 4 * g + e, v, up);
      }
    };
    if (WT == kFp4 && staged) up_unit<WT, VEC, WT == kFp4>(a, G, stage0, stride, q0, first, end, Stretch{rp, sp, k0, k1}, done);
    else up_unit<WT, VEC, false>(a, G, 0, 0, 0, first, end, Stretch{rp, sp, k0, k1}, done);
  }
  if (parts > 1) {
    __syncthreads();
    for (int o = threadIdx.x; o < n * 128; o += kFewThreads) {
      const int unit = o >> 7, q = (o >> 3) & 15, j = o & 7;
      const int c = (int)((u0 + unit) / tiles), first = G.begin_used[c];
      if (first + q >= G.begin_used[c + 1]) continue;
      float gate = 0, up = 0;
      for (int p = 0; p < parts; ++p) {
        const float* v = partial[(unit * parts + p) * 16 + q];
        gate += v[j], up += v[j + 8];
      }
      put_h<WT>(a, G.list[first + q], (int)((u0 + unit) % tiles) * 8 + j, gate, up);
    }
  }
  // what the rows of h are longer than F's whole tiles is cleared by the
  // workgroup of a matrix's last unit
  const int past = tiles * 8, extra = a.Fp - past;
  for (int c = (int)((u0 + tiles) / tiles - 1); (int64_t)(c + 1) * tiles <= u0 + n; ++c) {
    const int first = G.begin_used[c], m = G.begin_used[c + 1] - first;
    for (int o = threadIdx.x; o < m * extra; o += kFewThreads)
      put_h<WT>(a, G.list[first + o / extra], past + o % extra, 0.0f, 0.0f);
  }
}

// ---------------------------------------------------------------------------
// down and the sum over a token's experts. The 16 rows of an instruction are
// ROWS output columns: 16, or where a workgroup has no more than 8, those at two
// chunks of the k axis. Its 16 columns are PL planes of ROWS / PL pairs (fp32 one
// plane; bf16 two, or for an fp32 output three and an empty one), at the same two
// chunks where ROWS is 8: then of its products one row half by one column half
// each is wanted.
// ---------------------------------------------------------------------------
template <int WT, bool VEC, int ROWS, int PL, int NG>
__device__ __forceinline__ void down_groups(const FewArgs& a, const Groups& G, int first, int end, const Stretch& s,
                                            float* yp) {
  using C = Chunk<WT>;
  constexpr int S = 16 / ROWS, P = ROWS / PL;  // pairs of a group
  const int lane = lane_id(), g = lane >> 4, r = lane & 15;
  const int plane = (r & (ROWS - 1)) / P;
  const uint32_t plane_bytes = (uint32_t)(a.T * a.K * a.Fp * C::ES);
  uint32_t tok[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int q = first + P * i + (r & (P - 1));
    tok[i] = q < end && plane < 3 ? (uint32_t)(G.list[q] * a.Fp * C::ES) + plane * plane_bytes : kOutside;
  }
  const Tokens h = tokens_at(a.h, plane_bytes * (WT == kF32 ? 1 : a.planes));
  f32x4 acc[NG];
  stream_rows<WT, VEC, true, false, true, NG, kAheadDown<WT, NG>, S>(s, a.F, h, tok, a.Fp, S == 2 ? r >> 3 : 0, g, acc);
#pragma unroll
  for (int i = 0; i < NG; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float v = acc[i][e];  // row 4 g + e, column r
      if constexpr (S == 2) v += __shfl(v, (lane + 40) & 63, 64);  // of the odd chunks: row + 8, column + 8
      if constexpr (PL >= 2) {  // and the other planes, but for those of an infinite sum, which hold infinity times 0
        float all = v + __shfl(v, (lane + ROWS / 2) & 63, 64);
        if constexpr (PL == 4) all += __shfl(all, (lane + ROWS / 4) & 63, 64);
        v = fabsf(v) < INFINITY ? all : v;
      }
      const int q = first + P * i + r;
      if (r < P && 4 * g < ROWS && q < end) yp[q * ROWS + 4 * g + e] = v;
    }
}

template <int WT, bool VEC, int ROWS, int PL, int CAP>
__global__ __launch_bounds__(kFewThreads) void few_down_kernel(FewArgs a) {
  __shared__ Groups G;
  __shared__ float yp[CAP * ROWS];  // [tile][part][place][ROWS]
  group_pairs<kFewThreads>(a, G);
  const int tid = threadIdx.x, lane = lane_id();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_used = G.n_used, count = G.begin_used[n_used];
  using C = Chunk<WT>;
  constexpr int S = 16 / ROWS, P = ROWS / PL;
  const int r = lane & 15, nc = (a.F + S * C::K - 1) / (S * C::K);  // steps of S chunks
  // this workgroup's tiles of a.width columns, as many at a time as their
  // sums have room
  const int t0 = a.tiles * (int)blockIdx.x, t1 = min(t0 + a.tiles, (a.d + a.width - 1) / a.width);
  const int room = count > 0 ? CAP / count : t1 - t0;
  for (int tile0 = t0; tile0 < t1; tile0 += room) {
    const int nt = min(room, t1 - tile0);
    const int parts = parts_for(n_used * nt, nc, count * nt, CAP);
    for (int u = wave; u < n_used * nt * parts; u += kFewWaves) {
      const int part = u % parts, tile = u / parts % nt, c = u / parts / nt;
      const int w = __builtin_amdgcn_readfirstlane(G.used[c]);
      const int first = __builtin_amdgcn_readfirstlane(G.begin_used[c]), end = __builtin_amdgcn_readfirstlane(G.begin_used[c + 1]);
      const int col = (tile0 + tile) * a.width, cols = min(a.width, a.d - col);
      const int64_t row = (int64_t)w * a.d + col + min(r & (ROWS - 1), cols - 1);
      const char* rp = a.dn + (WT == kFp4 ? row * (a.F / 2) : row * a.F * C::ES);
      const uint8_t* sp = WT == kFp4 ? a.dn_scales + row * (a.F / kMxBlock) : nullptr;
      const Stretch s{rp, sp, nc * part / parts * S, nc * (part + 1) / parts * S};
      float* to = yp + (size_t)(tile * parts + part) * count * ROWS;
      for (int at = first; at < end; at += kGroups<WT> * P) {
        if (end - at <= P) down_groups<WT, VEC, ROWS, PL, 1>(a, G, at, end, s, to);
        else if (kGroups<WT> == 2 || end - at <= 2 * P) down_groups<WT, VEC, ROWS, PL, 2>(a, G, at, end, s, to);
        else down_groups<WT, VEC, ROWS, PL, kGroups<WT>>(a, G, at, end, s, to);
      }
    }
    __syncthreads();
    const int c0 = tile0 * a.width, cols = min(nt * a.width, a.d - c0);
    for (int o = tid; o < a.T * cols; o += kFewThreads) {
      const int t = o / cols, j = o % cols;
      const float* from = yp + (size_t)(j / a.width * parts) * count * ROWS + j % a.width;
      float s = 0.0f;
      for (int k = 0; k < a.K; ++k) {
        const int q = G.place[t * a.K + k];
        if (q < 0) continue;
        float v = 0.0f;
        for (int p = 0; p < parts; ++p) v += from[((size_t)p * count + q) * ROWS];
        s = fmaf(a.gates[t * a.K + k], v, s);
      }
      const int64_t at = (int64_t)t * a.d + c0 + j;
      if (a.y_f32) ((float*)a.y)[at] = s;
      else ((uint16_t*)a.y)[at] = (uint16_t)pack_bf2(s, 0.0f);
    }
    if (tile0 + room < t1) __syncthreads();
  }
}

template <int WT, bool VEC, int ROWS>
void launch_down(FewArgs a, int share, hipStream_t st) {
  const int pairs = a.T * a.K;
  a.tiles = (share + ROWS - 1) / ROWS;
  a.width = (share + a.tiles - 1) / a.tiles;
  const dim3 grid((a.d + a.tiles * a.width - 1) / (a.tiles * a.width));
#define DOWN(PL, CAP) \
  hipLaunchKernelGGL((few_down_kernel<WT, VEC, ROWS, PL, CAP>), grid, dim3(kFewThreads), 0, st, a)
  if constexpr (WT == kF32) {
    if (pairs <= 512) DOWN(1, 512);
    else DOWN(1, 2048);
  } else if (a.planes == 2) {
    if (pairs <= 512) DOWN(2, 512);
    else DOWN(2, 2048);
  } else {
    if (pairs <= 512) DOWN(4, 512);
    else DOWN(4, 2048);
  }
#undef DOWN
}

template <int WT, bool UP_VEC, bool DOWN_VEC>
void launch_few(FewArgs a, hipStream_t st) {
  const int pairs = a.T * a.K, cus = num_cus();
  const int64_t units = (int64_t)((a.F + 7) / 8) * (pairs < a.W ? pairs : a.W);
  hipLaunchKernelGGL((few_up_kernel<WT, UP_VEC>), dim3((unsigned)(units < cus ? units : cus)), dim3(kFewThreads), 0, st,
                     a);
  // an even share of the columns to every CU, in tiles of 16 at most, or of 8
  // where it has no more: a tile's rows of weights are multiplied with every
  // hidden row of their matrix, which come from the L2 again for each tile (us, 8
  // / 16: 64 tokens over 28 experts of 7168 x 2048 209 / 169, 32 places of each of
  // 8 such experts 297 / 164)
  const int share = (a.d + cus - 1) / cus;
  if (share > 8) launch_down<WT, DOWN_VEC, 16>(a, share, st);
  else launch_down<WT, DOWN_VEC, 8>(a, share, st);
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
  if (a.d >= kFewSide || a.F >= kFewSide || (T * a.ld + a.d) * 4 >= kOutside || T * a.K * few_row(a.F) * 8 >= kOutside)
    return set_error(FOREMOE_EUNSUPPORTED, "%s: d=%d or F=%d not below 2^25, or x or the hidden rows past 3.7 GB", name, a.d,
                     a.F);
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
  const size_t n = (size_t)(T * K) * (size_t)few_row(F) * 6;  // three bf16 planes, or fp32
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
  a.h = (char*)ws, a.y = y, a.y_f32 = out_dtype == FOREMOE_F32, a.planes = a.y_f32 ? 3 : 2;
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
  a.h = (char*)ws, a.y = y, a.y_f32 = out_dtype == FOREMOE_F32, a.planes = a.y_f32 ? 3 : 2;
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
