// Log-probabilities of given tokens, with entropies, top alternatives and
// the gradient of the logits: what recompute computes of every rollout token
// and where the policy update's backward starts (Sec. 2.3).
//
// Forward: one pass over a row keeps the running maximum, the sum of
// exponentials and their first moment in the log domain (struct Sums), in
// fp32, and the candidates for the top places (struct TopList). A row of N x V
// logits is read once: HBM-bound where rows fill the GPU, about 9 vector
// instruction slots an element (4 of them the exponential) against 13 that
// fit in the time of 2 bytes. Measured on MI355X:
//   8192 x 131072 bf16, a fifth ignored   258-270 us, 6.4-6.6 TB/s
//   2045 x 32003 fp32                     47 us, 5.1 TB/s
//   8192 x 131072 bf16, 20 alternatives   420 us, 5.1 TB/s
//   1 x 131072 bf16: 7.2 us, with 20 alternatives 15.2 us: latency (pieces, their
//   join and two rankings)
// A row of few is cut into pieces; each leaves its sums and its sorted top
// places in the workspace, and the last to finish, by a ticket, joins them in
// their order, so that results do not depend on the run.
//
// Backward: every gradient from its logit and four numbers of the row, one
// read and one write: HBM-bound, forward and backward of 4096 x 131072 bf16
// 456-467 us (2.8 GB, 6.0-6.1 TB/s).
#include <limits.h>
#include <math.h>

#include "common.h"

// Fused multiply-adds are written out: a product that is rounded once and
// used twice has to be the same both times.
#pragma clang fp contract(off)

namespace foremoe {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
// A row may start at any element, so its 16-byte vectors have the alignment
// of the type only; the hardware takes those.
typedef u32x4 u32x4_any __attribute__((aligned(2)));

constexpr int kLpThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kTile = 4;         // vectors that a lane holds at a time
constexpr int kBwdTile = 4;      // the same in the backward
// A gradient of this many bytes does not stay in the Infinity Cache (256 MB)
// until it is used, and is better kept out of it, and its logits' last read
// with it: forward and backward of 2045 x 32003 fp32 152 -> 123 us, of 4096 x
// 131072 bf16 518 -> 468. A smaller one is used from there: 512 x 32000 bf16 (33
// MB) with a product behind it 136 -> 153 us with the hint, 300 x 131072 (79
// MB) 308 -> 307.
constexpr size_t kStreamBytes = (size_t)128 << 20;
// The forward keeps logits of this many bytes out too, where no top places are
// wanted (their candidates are read again): 8192 x 131072 bf16 302 -> 270 us,
// with the backward 937 -> 926. Of smaller ones a backward that follows finds
// part there: forward and backward of 4096 x 131072 (1 GB) 467 us, 474 with
// the hint, of 2045 x 32003 fp32 123 and 136.
constexpr size_t kStreamLogits = (size_t)3 << 29;
constexpr int kBuf = 512;        // candidates for the top places that a wavefront keeps
// pieces of one row (us at 64 and 16, with 20 places: 1 x 131072 14.1 and
// 14.2, 4 x 131072 15.8 and 14.3)
constexpr int kMaxPieces = 16;
constexpr int kFewRows = 256;    // fewer rows than this are cut into pieces
// and into about so many of all rows (us at 256, 512, 1024: 64 x 131072 bf16
// 10.5, 10.8, 13.4, with 20 places 23.0, 22.1, 22.1; 130 x 70001 fp32 with 20
// places 32.2, 27.9, 30.9; 200 x 131072 16.5, 18.5, 22.1): the rows with places
// decide, those without would like fewer
constexpr int kSplit = 512;
constexpr int kMaxSplit = kSplit + kFewRows;
static_assert(kMaxSplit >= kMaxPieces * (kFewRows / kMaxPieces));
constexpr int kJoin = kMaxPieces * FOREMOE_MAX_TOP / kLpThreads;  // candidates a lane takes when pieces are joined
static_assert(kJoin * 64 <= kBuf);

struct Sums {
  float m, s, t;
};

struct LogprobArgs {
  const void* logits;
  int64_t ld;
  int32_t first, V;  // first: the launch's first row
  const int32_t* targets;
  float c, inv_temperature;  // c: log2(e) / temperature
  int32_t n_top;
  float *logp, *entropy, *lse;
  int32_t* top_ids;
  float* top_logp;
  int32_t pieces, piece_vectors;
  uint32_t* ticket;     // [N]
  Sums* part;           // [N, pieces]
  uint64_t* part_top;   // [N, pieces, n_top]
};

template <bool BF16>
constexpr int kVec = BF16 ? 8 : 4;  // elements of a 16-byte vector

template <bool BF16>
__device__ __forceinline__ float load_lp(const void* p, int64_t i) {
  if constexpr (BF16) return bf2f(((const uint16_t*)p)[i]);
  return ((const float*)p)[i];
}

template <bool STREAM>
__device__ __forceinline__ u32x4 load_vec(const void* row, uint32_t vector) {
  const u32x4_any* p = (const u32x4_any*)((const char*)row + (size_t)vector * 16);
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}

template <bool BF16>
__device__ __forceinline__ void unpack(u32x4 v, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    } else {
      x[i] = __uint_as_float(v[i]);
    }
  }
}

// Running sums of a row: the maximum m of its logits x, and with
// y = (x - m) c in base 2, s = sum 2^y and t = sum y 2^y, so that
//   lse = ln2 (m c + log2 s),  entropy = ln2 (log2 s - t / s),
// both terms of the entropy >= 0. y is one fused multiply-add, x c - m c with
// m c rounded once: the same reference everywhere, so that its rounding
// cancels. m starts at the lowest finite number, so an x of -inf adds nothing
// to s. Where m c is so large that its rounding is no small part of a y (a row
// that a mask fills with -1e9, or the type's ends), x - m is taken first and
// then scaled: m c itself is the reference. Powers and logarithms are the
// hardware's, within a unit in the last place; a y is within |y| 2^-24 of its
// value, as a scaled logit is in fp32.
__device__ __forceinline__ bool huge(float mc) { return !(fabsf(mc) < 0x1p24f); }

// Either kind of reference, exactly.
__device__ __forceinline__ double reference(float m, float c) {
  const float mc = m * c;
  return huge(mc) ? (double)m * (double)c : (double)mc;
}

// The sums seen from a reference that lies -y above their own.
__device__ __forceinline__ void lower(Sums& a, float y) {
  const float e = __builtin_amdgcn_exp2f(y);
  a.t = e == 0.0f ? 0.0f : e * (a.t + y * a.s);
  a.s = e == 0.0f ? a.s * 0.0f : a.s * e;  // keeps a NaN
}

__device__ __forceinline__ void rebase(Sums& a, float m, float c) {
  const float from = a.m * c, to = m * c;
  float y = from - to;
  if (a.s == 0.0f) {
    y = -INFINITY;  // nothing yet: under the lowest number
  } else if (__builtin_expect(huge(from) || huge(to), 0)) {
    y = (float)(reference(a.m, c) - reference(m, c));
  }
  lower(a, y);
  a.m = m;
}

// (In 64 bits for every join: branches as in rebase would cost one 0.1 us.)
__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  if (b.m > a.m) {
    const Sums x = a;
    a = b, b = x;
  }
  lower(b, (float)(reference(b.m, c) - reference(a.m, c)));
  return Sums{a.m, a.s + b.s, a.t + b.t};
}

// Adds n elements of one lane.
template <int n>
__device__ __forceinline__ void add(Sums& a, const float* x, float c) {
  float top = x[0];
#pragma unroll
  for (int i = 1; i < n; ++i) top = fmaxf(top, x[i]);
  if (top > a.m) rebase(a, top, c);
  const float mc = a.m * c;
  float s[2] = {0.0f, 0.0f}, t[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < n; ++i) {
    const float y = fmaf(x[i], c, -mc), e = __builtin_amdgcn_exp2f(y);
    s[i & 1] += e;
    t[i & 1] = fmaf(y, e, t[i & 1]);
  }
  s[0] += s[1];
  t[0] += t[1];
  // a y of -inf (a masked logit) has made a NaN of y 2^y: again with care
  if (__builtin_expect(t[0] != t[0] || huge(mc), 0)) {
    s[0] = t[0] = 0.0f;
    const bool far = huge(mc);
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float y = far ? (x[i] - a.m) * c : fmaf(x[i], c, -mc), e = __builtin_amdgcn_exp2f(y);
      s[0] += e;
      t[0] += fmaxf(y, kLowest) * e;
    }
  }
  a.s += s[0];
  a.t += t[0];
}

// A logit and its id as one integer in the order of the top places: larger
// logits first, among equals (0.0 and -0.0 too) the lower id. 0 for a NaN and
// -inf, which have no place.
__device__ __forceinline__ uint64_t place_key(float x, uint32_t id) {
  const uint32_t b = __float_as_uint(x + 0.0f);
  const uint32_t o = b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
  return x > -INFINITY ? (uint64_t)o << 32 | (uint32_t)~id : 0;
}
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t key_id(uint64_t k) { return (int32_t)~(uint32_t)k; }

// A threshold that at least n lanes' values reach, bit by bit from the top:
// the first that just n reach, or else the n-th largest value.
__device__ __forceinline__ uint32_t nth_largest(uint32_t value, int n) {
  uint32_t k = 0;
#pragma unroll 1
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    const int reach = __popcll(__ballot(value >= (k | bit)));
    if (reach >= n) k |= bit;
    if (reach == n) break;
  }
  return k;
}

// The candidates of a wavefront for the n top places: every element it has
// seen whose key is at least its threshold, in any order.
//
// The threshold is the n-th largest of the 64 lanes' own maxima, so n
// elements reach it: of the first elements, then of the kept candidates
// whenever the buffer is full. A lane holds kBuf / 64 = 8 candidates then, so
// at most 8 n <= 256 of them pass, and a ballot's 64 always fit behind them.
struct TopList {
  uint64_t* buf;  // [kBuf] in LDS
  int n, count;
  uint64_t least;  // the threshold, > 0
  float x;         // its logit

  __device__ __forceinline__ void start(uint64_t* b, int places) {
    buf = b, n = places, count = 0, least = 1, x = -INFINITY;
  }
  // Before anything is offered: the lanes' largest elements so far.
  __device__ __forceinline__ void first_threshold(float lane_max) {
    const uint32_t o = nth_largest((uint32_t)(place_key(lane_max, 0) >> 32), n);
    if (o) least = (uint64_t)o << 32, x = key_logit(least);
  }
  __device__ __forceinline__ void fence() const {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  __device__ __forceinline__ void put(uint64_t key) {
    const bool pass = key >= least;
    const uint64_t mask = __ballot(pass);
    if (pass) buf[count + lanes_below(mask)] = key;
    count += __popcll(mask);
  }
  __device__ __forceinline__ void prune() {
    const int lane = lane_id();
    fence();
    uint64_t e[kBuf / 64], best = 0;
#pragma unroll
    for (int q = 0; q < kBuf / 64; ++q) {
      const int at = lane + 64 * q;
      e[q] = at < count ? buf[at] : 0;
      best = e[q] > best ? e[q] : best;
    }
    // n lanes reach t: those above o, and of those at o the ones with the lowest ids
    const uint32_t hi = (uint32_t)(best >> 32), o = nth_largest(hi, n);
    const uint32_t lo = nth_largest(hi == o ? (uint32_t)best : 0, n - __popcll(__ballot(hi > o)));
    const uint64_t t = (uint64_t)o << 32 | lo;
    if (t > least) least = t, x = key_logit(t);
    fence();
    count = 0;
#pragma unroll
    for (int q = 0; q < kBuf / 64; ++q) put(e[q]);
    fence();
  }
  // The elements whose bit is set in `mine`; key(bit) gives one's key. All
  // lanes of the wavefront together.
  template <class Key>
  __device__ __forceinline__ void offer(uint32_t mine, Key&& key) {
    while (__any(mine != 0)) {
      const uint64_t k = mine ? key(__builtin_ctz(mine)) : 0;
      mine &= mine - 1;
      if (count + __popcll(__ballot(k >= least)) > kBuf) prune();
      put(k);
    }
  }
};

// Sums of the workgroup, in every thread; the order of the joins is fixed.
template <int WAVES>
__device__ __forceinline__ Sums join_block(Sums r, Sums* sh, float c) {
#pragma unroll 1
  for (int o = 32; o >= 1; o >>= 1)
    r = join(r, Sums{__shfl_xor(r.m, o, 64), __shfl_xor(r.s, o, 64), __shfl_xor(r.t, o, 64)}, c);
  if constexpr (WAVES > 1) {
    if (lane_id() == 0) sh[threadIdx.x >> 6] = r;
    __syncthreads();
    r = sh[0];
#pragma unroll 1
    for (int w = 1; w < WAVES; ++w) r = join(r, sh[w], c);
  }
  return r;
}

// The workgroup's candidates by rank: out(place, key) for the places below n,
// and how many there are. A thread counts what is before its candidate.
template <int WAVES, class Out>
__device__ __forceinline__ int rank_block(TopList& top, const uint64_t* buf, int* sh_count, Out&& out) {
  constexpr int kStep = 8;
  if (top.count > 64) top.prune();
  // filled up to a multiple of kStep with keys that are behind every other
  if (lane_id() < kStep && top.count + lane_id() < kBuf) top.buf[top.count + lane_id()] = 0;
  if (lane_id() == 0) sh_count[threadIdx.x >> 6] = top.count;
  if constexpr (WAVES > 1) __syncthreads();
  else top.fence();
  int all = 0;
  for (int w = 0; w < WAVES; ++w) all += sh_count[w];
#pragma unroll 1
  for (int j = threadIdx.x; j < all; j += 64 * WAVES) {
    int w = 0, i = j;
    while (i >= sh_count[w]) i -= sh_count[w++];
    const uint64_t me = buf[w * kBuf + i];
    int rank = 0;
#pragma unroll 1
    for (int q = 0; q < WAVES; ++q) {
      const int cq = sh_count[q];
#pragma unroll 1
      for (int o = 0; o < cq; o += kStep) {
#pragma unroll
        for (int z = 0; z < kStep; ++z) rank += buf[q * kBuf + o + z] > me;
      }
    }
    if (rank < top.n) out(rank, me);
  }
  return min(all, top.n);
}

// A workgroup of WAVES wavefronts takes a piece of a row; where a row has
// several, the last one to finish joins them. STREAM: its loads carry the
// nontemporal hint.
template <bool BF16, bool TOP, int WAVES, bool STREAM>
__global__ __launch_bounds__(64 * WAVES) void logprobs_kernel(LogprobArgs a) {
  constexpr int kThreads = 64 * WAVES, VEC = kVec<BF16>;
  __shared__ uint64_t buf[TOP ? WAVES * kBuf : 1];
  __shared__ Sums sh[WAVES];
  __shared__ int sh_count[WAVES];
  __shared__ bool sh_last;
  const int tid = threadIdx.x, wave = tid >> 6;
  const int64_t row = a.first + (int64_t)(a.pieces > 1 ? blockIdx.x / (unsigned)a.pieces : blockIdx.x);
  const int piece = a.pieces > 1 ? (int)(blockIdx.x % (unsigned)a.pieces) : 0;
  const int target = a.targets ? a.targets[row] : 0;
  if ((unsigned)target >= (unsigned)a.V) {
    if (piece != 0) return;
    if (tid == 0) {
      if (a.logp) a.logp[row] = 0.0f;
      if (a.entropy) a.entropy[row] = 0.0f;
      if (a.lse) a.lse[row] = 0.0f;
    }
    for (int k = tid; k < a.n_top; k += kThreads) {
      a.top_ids[row * a.n_top + k] = -1;
      a.top_logp[row * a.n_top + k] = -INFINITY;
    }
    return;
  }
  const char* x0 = (const char*)a.logits + (size_t)row * a.ld * (BF16 ? 2 : 4);
  TopList top;
  if constexpr (TOP) top.start(buf + wave * kBuf, a.n_top);

  Sums r{kLowest, 0.0f, 0.0f};
  const uint32_t vectors = (uint32_t)a.V / VEC, beg = (uint32_t)piece * a.piece_vectors;
  const uint32_t end = min(vectors, beg + a.piece_vectors);
  if (end == vectors) {  // the row's last elements, less than a vector
    const uint32_t id = vectors * VEC + tid;
    float x = -INFINITY;
    if (id < (uint32_t)a.V) {
      x = load_lp<BF16>(x0, id);
      add<1>(r, &x, a.c);
    }
    if constexpr (TOP) top.put(place_key(x, id));
  }
  bool first = true;
  uint32_t at = beg;  // the workgroup's next vector
  // a lane's elements x of the vectors at, at + kThreads, ...
  auto consider = [&](const auto& x) {
    constexpr int n = sizeof(x) / sizeof(float);
    float most = x[0];
#pragma unroll
    for (int i = 1; i < n; ++i) most = fmaxf(most, x[i]);
    if (first) top.first_threshold(most), first = false;
    if (__any(most >= top.x)) {
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < n; ++i) mine |= x[i] > -INFINITY && x[i] >= top.x ? 1u << i : 0u;
      top.offer(mine, [&](int i) {
        const uint32_t id = (at + (i / VEC) * kThreads + tid) * VEC + i % VEC;
        if constexpr (n > VEC) return place_key(load_lp<BF16>(x0, id), id);
        float v = x[0];
#pragma unroll
        for (int j = 1; j < VEC; ++j) v = j == i ? x[j] : v;
        return place_key(v, id);
      });
    }
  };
  u32x4 next[kTile];  // under way while a tile is summed
  const uint32_t whole = end - (end - beg) % (kTile * kThreads);
#pragma unroll
  for (int u = 0; u < kTile; ++u)
    if (at < whole) next[u] = load_vec<STREAM>(x0, at + u * kThreads + tid);
#pragma unroll 1
  for (; at < whole; at += kTile * kThreads) {
    float x[kTile * VEC];
#pragma unroll
    for (int u = 0; u < kTile; ++u) unpack<BF16>(next[u], x + u * VEC);
    if (at + kTile * kThreads < whole) {
#pragma unroll
      for (int u = 0; u < kTile; ++u) next[u] = load_vec<STREAM>(x0, at + (kTile + u) * kThreads + tid);
    }
    add<kTile * VEC>(r, x, a.c);
    if constexpr (TOP) consider(x);
  }
  // what is left of the piece, at most kTile vectors for a thread
  u32x4 one;
  if (at + tid < end) one = load_vec<STREAM>(x0, at + tid);
#pragma unroll 1
  for (; at < end; at += kThreads) {
    float x[VEC];
    unpack<BF16>(one, x);
    if (at + kThreads + tid < end) one = load_vec<STREAM>(x0, at + kThreads + tid);
    if (at + tid < end) {
      add<VEC>(r, x, a.c);
    } else if constexpr (TOP) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = -INFINITY;  // has no place
    }
    if constexpr (TOP) consider(x);
  }
  r = join_block<WAVES>(r, sh, a.c);

  // pieces are taken by workgroups (of a part of a row: WAVES > 1)
  if (WAVES > 1 && a.pieces > 1) {
    const int64_t me = row * a.pieces + piece;
    auto keep = [](auto* p, auto v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    auto fetch = [](const auto* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
    if constexpr (TOP) {
      uint64_t* mine = a.part_top + me * a.n_top;
      const int got = rank_block<WAVES>(top, buf, sh_count, [&](int k, uint64_t key) { keep(&mine[k], key); });
      for (int k = got + tid; k < a.n_top; k += kThreads) keep(&mine[k], (uint64_t)0);
    }
    if (tid == 0) {
      keep(&a.part[me].m, r.m);
      keep(&a.part[me].s, r.s);
      keep(&a.part[me].t, r.t);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wavefront's part has reached memory
    __syncthreads();
    if (tid == 0) sh_last = atomicAdd(a.ticket + row, 1u) == (unsigned)a.pieces - 1;
    __syncthreads();
    if (!sh_last) return;
    // every piece's part is in memory: join them
    r = Sums{kLowest, 0.0f, 0.0f};
    if (tid < a.pieces) {
      const Sums* p = a.part + row * a.pieces + tid;
      r = Sums{fetch(&p->m), fetch(&p->s), fetch(&p->t)};
    }
    if constexpr (TOP) {
      const uint64_t* p = a.part_top + row * a.pieces * a.n_top;
      const int n = a.pieces * a.n_top;
      uint64_t e[kJoin], best = 0;
#pragma unroll
      for (int q = 0; q < kJoin; ++q) {
        e[q] = tid + q * kThreads < n ? fetch(p + tid + q * kThreads) : 0;
        best = e[q] > best ? e[q] : best;
      }
      top.start(buf + wave * kBuf, a.n_top);
      const uint32_t o = nth_largest((uint32_t)(best >> 32), a.n_top);
      if (o) top.least = (uint64_t)o << 32;
#pragma unroll
      for (int q = 0; q < kJoin; ++q) top.put(e[q]);  // kJoin x 64: they all fit
    }
    r = join_block<WAVES>(r, sh, a.c);
    if (tid == 0) __hip_atomic_store(a.ticket + row, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }

  const bool none = r.s == 0.0f;  // nothing but -inf
  const float mc = r.m * a.c, ls = __builtin_amdgcn_logf(r.s);
  // log2 of the probability of a logit x
  auto lp = [&](float x) { return (huge(mc) ? (x - r.m) * a.c : fmaf(x, a.c, -mc)) - ls; };
  if (tid == 0) {
    if (a.lse) a.lse[row] = huge(mc) ? r.m * a.inv_temperature + kLn2 * ls : kLn2 * (mc + ls);
    if (a.entropy) a.entropy[row] = none ? 0.0f : kLn2 * (ls - r.t / r.s);
    if (a.logp) a.logp[row] = none ? -INFINITY : kLn2 * lp(load_lp<BF16>(x0, target));
  }
  if constexpr (TOP) {
    const int got = rank_block<WAVES>(top, buf, sh_count, [&](int k, uint64_t key) {
      a.top_ids[row * a.n_top + k] = key_id(key);
      a.top_logp[row * a.n_top + k] = kLn2 * lp(key_logit(key));
    });
    for (int k = got + tid; k < a.n_top; k += kThreads) {
      a.top_ids[row * a.n_top + k] = -1;
      a.top_logp[row * a.n_top + k] = -INFINITY;
    }
  }
}

constexpr size_t kLpTicketBytes = sizeof(uint32_t) * kMaxSplit;
constexpr size_t kLpPartBytes = sizeof(Sums) * kMaxSplit;
constexpr size_t kLpWsBytes = kLpTicketBytes + kLpPartBytes + sizeof(uint64_t) * FOREMOE_MAX_TOP * kMaxSplit;

template <bool BF16, bool TOP>
void launch_logprobs(LogprobArgs a, int64_t N, int waves, hipStream_t st) {
  const bool stream_through = !TOP && (size_t)N * a.V * (BF16 ? 2 : 4) >= kStreamLogits;
  // a launch has fewer than 2^32 threads
  constexpr int64_t kRows = 1 << 22;
  for (int64_t r = 0; r < N; r += kRows) {
    a.first = (int32_t)r;
    const dim3 grid((unsigned)((N - r < kRows ? N - r : kRows) * a.pieces));
    auto launch = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, st, a); };
    constexpr int kWaves = kLpThreads / 64;
    if (waves == 1)
      stream_through ? launch(logprobs_kernel<BF16, TOP, 1, !TOP>, 64)
                     : launch(logprobs_kernel<BF16, TOP, 1, false>, 64);
    else
      stream_through ? launch(logprobs_kernel<BF16, TOP, kWaves, !TOP>, kLpThreads)
                     : launch(logprobs_kernel<BF16, TOP, kWaves, false>, kLpThreads);
  }
}

struct LogprobBwdArgs {
  const void* logits;
  int64_t ld;
  int32_t V;
  const int32_t* targets;
  float inv_temperature;
  const float *lse, *entropy, *dlogp, *dentropy;
  void* dlogits;
  int64_t ld_out;
};

// One row's gradient: d = -p (a + b (y + h)), y = x / temperature - lse. An
// lse that rounding has left below the largest x / temperature, by 32 at 1e9,
// gives no p above 1.
struct RowGrad {
  float it, lse, a, b, h;
  __device__ __forceinline__ float operator()(float x) const {
    float y = fmaf(x, it, -lse);
    y = y > 0.0f ? 0.0f : y;  // keeps a NaN
    const float p = __builtin_amdgcn_exp2f(y * kLog2e);
    const float d = -p * fmaf(b, y + h, a);
    return p == 0.0f ? 0.0f : d;  // y is -inf where the logit is
  }
};

// A workgroup takes kBwdTile vectors per thread of one row; every element is
// read and then written by one thread, so the gradient may replace the logits.
// STREAM: its accesses carry the nontemporal hint.
template <bool BF16, bool STREAM>
__global__ __launch_bounds__(kLpThreads) void logprobs_bwd_kernel(LogprobBwdArgs a) {
  constexpr int VEC = kVec<BF16>;
  const int64_t row = blockIdx.y;
  const int tid = threadIdx.x;
  const char* x0 = (const char*)a.logits + (size_t)row * a.ld * (BF16 ? 2 : 4);
  char* d0 = (char*)a.dlogits + (size_t)row * a.ld_out * (BF16 ? 2 : 4);
  const uint32_t vectors = (uint32_t)a.V / VEC, at = blockIdx.x * (kBwdTile * kLpThreads) + tid;
  const int target = a.targets ? a.targets[row] : -1;
  const bool keep = !a.targets || (unsigned)target < (unsigned)a.V;
  u32x4 held[kBwdTile];
  if (keep) {
#pragma unroll
    for (int u = 0; u < kBwdTile; ++u)
      if (at + u * kLpThreads < vectors) held[u] = load_vec<STREAM>(x0, at + u * kLpThreads);
  }
  RowGrad g;
  // a row of -inf only: every p is 0
  g.it = a.inv_temperature, g.lse = a.lse[row] == -INFINITY ? INFINITY : a.lse[row];
  const float dlp = a.dlogp ? a.dlogp[row] * a.inv_temperature : 0.0f;
  g.a = dlp;
  g.b = a.dentropy ? a.dentropy[row] * a.inv_temperature : 0.0f;
  g.h = a.dentropy ? a.entropy[row] : 0.0f;
#pragma unroll
  for (int u = 0; u < kBwdTile; ++u) {
    const uint32_t v = at + u * kLpThreads;
    if (v >= vectors) continue;
    u32x4 out = {0, 0, 0, 0};
    if (keep) {
      float x[VEC];
      unpack<BF16>(held[u], x);
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = g(x[i]);
      if (a.dlogp && (uint32_t)target / VEC == v) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[i] += (uint32_t)target % VEC == i ? dlp : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = BF16 ? pack_bf2(x[2 * i % VEC], x[(2 * i + 1) % VEC]) : __float_as_uint(x[i]);
    }
    u32x4_any* to = (u32x4_any*)(d0 + (size_t)v * 16);
    if constexpr (STREAM)
      __builtin_nontemporal_store(out, to);
    else
      *to = out;
  }
  const uint32_t id = vectors * VEC + tid;  // the row's last elements, less than a vector
  if (blockIdx.x == 0 && id < (uint32_t)a.V) {
    float d = 0.0f;
    if (keep) d = g(load_lp<BF16>(x0, id)) + (a.dlogp && target == (int)id ? dlp : 0.0f);
    if constexpr (BF16)
      ((uint16_t*)d0)[id] = (uint16_t)pack_bf2(d, 0.0f);
    else
      ((float*)d0)[id] = d;
  }
}

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
  const int vec = dtype == FOREMOE_BF16 ? kVec<true> : kVec<false>;
  const int64_t vectors = V / vec;
  // A wavefront for a row, or a workgroup: a workgroup's barriers and joins
  // cost more than they give where rows are short, or many and wanted with
  // top places (us, workgroup -> wavefront: 16384 x 8000 bf16 81 -> 54, 600 x
  // 4096 5.3 -> 4.5, 16384 x 16000 123 -> 101, 8192 x 131072 with 20 places
  // 494 -> 415; without places 365 -> 378, 2048 x 131072 with 5 118 -> 143).
  // Rows that do not fill the GPU are cut into pieces.
  const int waves = vectors <= 1024 || (N >= 4096 && (n_top || vectors <= 2048)) ? 1 : kLpThreads / 64;
  int64_t pieces = 1;
  if (ws && waves > 1 && N < kFewRows) {
    // at least a vector for every thread, where there are more rows a tile
    // (without top places two)
    const bool few = N <= kFewRows / kMaxPieces;
    const int64_t most = vectors / (kLpThreads * (few ? 1 : n_top ? kTile : 2 * kTile));
    pieces = (kSplit + N - 1) / N;
    if (pieces > most) pieces = most;
    if (pieces > kMaxPieces) pieces = kMaxPieces;
    if (pieces < 1) pieces = 1;
  }
  LogprobArgs a{};
  a.logits = logits, a.ld = ld, a.V = (int32_t)V, a.targets = targets;
  a.c = kLog2e / temperature, a.inv_temperature = 1.0f / temperature, a.n_top = n_top;
  a.logp = logp, a.entropy = entropy, a.lse = lse, a.top_ids = top_ids, a.top_logp = top_logp;
  const int64_t per = (vectors + pieces - 1) / pieces;
  a.piece_vectors = (int32_t)((per + kLpThreads - 1) / kLpThreads * kLpThreads);
  if (pieces > 1) pieces = (vectors + a.piece_vectors - 1) / a.piece_vectors;
  a.pieces = (int32_t)pieces;
  a.ticket = (uint32_t*)ws;
  a.part = (Sums*)((char*)ws + kLpTicketBytes);
  a.part_top = (uint64_t*)((char*)ws + kLpTicketBytes + kLpPartBytes);
  hipStream_t st = (hipStream_t)stream;
  if (dtype == FOREMOE_BF16)
    n_top ? launch_logprobs<true, true>(a, N, waves, st) : launch_logprobs<true, false>(a, N, waves, st);
  else
    n_top ? launch_logprobs<false, true>(a, N, waves, st) : launch_logprobs<false, false>(a, N, waves, st);
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
    LogprobBwdArgs a{(const char*)logits + (size_t)r * ld * item, ld, (int32_t)V,
                     targets ? targets + r : nullptr, 1.0f / temperature, lse + r,
                     entropy ? entropy + r : nullptr, dlogp ? dlogp + r : nullptr, dentropy ? dentropy + r : nullptr,
                     (char*)dlogits + (size_t)r * ld_out * item, ld_out};
    const int64_t per = kLpThreads * kBwdTile, vectors = V / (dtype == FOREMOE_BF16 ? kVec<true> : kVec<false>);
    const dim3 grid((unsigned)(vectors < 1 ? 1 : (vectors + per - 1) / per), (unsigned)n);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kLpThreads), 0, st, a); };
    const bool stream_through = (size_t)N * V * item >= kStreamBytes;
    if (dtype == FOREMOE_BF16)
      stream_through ? launch(logprobs_bwd_kernel<true, true>) : launch(logprobs_bwd_kernel<true, false>);
    else
      stream_through ? launch(logprobs_bwd_kernel<false, true>) : launch(logprobs_bwd_kernel<false, false>);
  }
  return check_launch("token_logprobs_bwd");
}

}  // extern "C"
