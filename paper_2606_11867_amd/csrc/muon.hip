// One Muon step over batches of matrices: momentum, Newton-Schulz products on
// the fp16 matrix cores, update (include/foremoe.h).
//
// A matrix lies in the workspace with its smaller side as rows (transposed
// where it is tall), padded with zeros to whole tiles: X, m x n with m <= n.
// A step of the iteration is three products, each one launch for all matrices:
//   G = X X^T, P = b G + c G G (symmetric: half of the tiles, each written
//   twice), X = a X + P X.
// X is held as two fp16 numbers, its rounding and 2^10 times what that
// leaves; the products take the first, a X takes both. So a product's factors
// are within 2^-11 of themselves, and directions that u does not have stay
// at the size that fp32 leaves there: P X alone would fill them with the
// rounding of X, which each step multiplies by a. (The last step does without the
// second numbers: that is one factor a.) Off the exact X by, of its norm, the plain
// iteration in fp32 beside it (simulated, 130 x 300): Gaussian 2^-9.2 after 5
// steps and 2^-7.7 after 16, 2^-19 and 2^-18; rank 5, 2^-10.3 after 5 steps and
// 2^-15, 2^-9.7 after 8 and 2^-9.6, 2^-7.2 after 10 and 2^-6.1, and from 12 on
// either has filled the empty directions.
// X, G and P are held 2^8 times as large, which keeps entries of large, even
// matrices (1/sqrt(m n) and less) above fp16's subnormal numbers.
//
// The passes over the tensors are bound by memory, the products by the matrix
// cores and, of X, by the 8 bytes an element that its two numbers are read and
// written with: 48 matrices of 768 x 2048 (75 M elements) take 165 us for the
// momentum (5.5 TB/s), 250 for X0 (4.8), five times 100 for G and 49 for P, four
// times 218 for X (0.53 PFLOP/s), 315 for the last X and the update.
#include <math.h>

#include "common.h"
#include "mfma_tiles.h"

namespace foremoe {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kMuonBK = 64;
// Elements of a matrix to a workgroup of the momentum pass: 4096, more where
// that would leave over 1024 sums to add up.
constexpr int kMomentThreads = 256, kMomentChunk = 4096, kMomentMost = 1024;
constexpr float kHeld = 256.0f, kRest = 1024.0f;

struct MuonRec {
  void* param;
  void* grad;
  float* master;
  float* m;
  int64_t batch;
  int32_t rows, cols;
  int32_t mm, nn;          // padded sides, mm the smaller one's
  uint32_t chunks;         // of a matrix, in the momentum pass
  int32_t chunk;           // elements of one
  float decay, move;       // 1 - lr weight_decay, lr scale
  int32_t wide;            // the tensors' rows start on 16 bytes: read and written so
  union {
    struct {
      uint16_t *x[2], *rest[2];  // [batch, mm, nn]
      uint16_t *gram, *poly;     // [batch, mm, mm]
      double* squares;           // [batch, chunks]
    };
    struct {  // small matrices (m <= 64)
      double* part;     // [batch, chunks, tiles of 16 x 16 on and above the diagonal]: of each chunk of columns u u^T
      double* q;        // [batch, whole tiles of rows and columns]: Q
      double* inverse;  // [batch]: 1 / max(|u|, eps)
      double* held;     // [batch, m, n]: X between two stages
    };
  };
};

// First workgroup of every record in a launch.
struct Firsts {
  uint32_t at[FOREMOE_MUON_LAUNCH];
};

struct MuonArgs {
  Firsts first;  // of this launch
  MuonRec rec[FOREMOE_MUON_LAUNCH];
  int n_rec, nesterov, zero_grads, from;  // from: which X the launch reads
  int has_rest, put_rest;  // whether that X has its second numbers, and the written one
  uint32_t n_work;         // workgroups with work in a product's launch
  int steps;               // (of a stage, for small matrices)
  int from_u, to_params;   // small matrices: whether the stage starts from u, and ends in the parameters
  double coef[3];
  float momentum, a, b, c;
  double eps;
  const float* grad_scale;
};
static_assert(sizeof(MuonArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ uint16_t half_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ float half_value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

// Two values as the fp16 numbers next to them, and 2^10 times what those leave.
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& rest) {
  const uint32_t ha = half_bits(a), hb = half_bits(b);
  hi = ha | hb << 16;
  rest = (uint32_t)half_bits((a - half_value(ha)) * kRest) | (uint32_t)half_bits((b - half_value(hb)) * kRest) << 16;
}
__device__ __forceinline__ float join(uint32_t hi, uint32_t rest, int second) {
  return half_value(hi >> (16 * second) & 0xffffu) + half_value(rest >> (16 * second) & 0xffffu) * (1.0f / kRest);
}

__device__ __forceinline__ int find_rec(const MuonArgs& a, uint32_t b) {
  int r = 0;
#pragma unroll
  for (int i = 1; i < FOREMOE_MUON_LAUNCH; ++i) r += i < a.n_rec && a.first.at[i] <= b;
  return r;
}

// 1 / max(norm, eps). Nothing in the matrix: no move, also where 1 / eps is
// infinite; not finite: NaN everywhere.
__device__ __forceinline__ double inverse_norm(double norm, double eps) {
  if (norm == 0) return 0.0;
  return norm < INFINITY ? 1.0 / fmax(norm, eps) : (double)NAN;
}

// Four neighbours of a tensor, from element i on: at once (wide), or those
// of them that are below n.
template <bool BF16_T>
__device__ __forceinline__ void get4(const void* p, int64_t i, int64_t left, bool wide, float* v) {
  if constexpr (BF16_T) {
    const uint16_t* q = (const uint16_t*)p + i;
    if (wide && left >= 4) {
      const uint2 w = *(const uint2*)q;
      v[0] = bf2f(w.x & 0xffffu), v[1] = __uint_as_float(w.x & 0xffff0000u);
      v[2] = bf2f(w.y & 0xffffu), v[3] = __uint_as_float(w.y & 0xffff0000u);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < left ? bf2f(q[e]) : 0.0f;
    }
  } else {
    const float* q = (const float*)p + i;
    if (wide && left >= 4) {
      const float4 w = *(const float4*)q;
      v[0] = w.x, v[1] = w.y, v[2] = w.z, v[3] = w.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = e < left ? q[e] : 0.0f;
    }
  }
}
template <bool BF16_T>
__device__ __forceinline__ void put4(void* p, int64_t i, int64_t left, bool wide, const float* v) {
  if constexpr (BF16_T) {
    uint16_t* q = (uint16_t*)p + i;
    const uint2 w = {pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])};
    if (wide && left >= 4) {
      *(uint2*)q = w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) q[e] = (uint16_t)((e < 2 ? w.x : w.y) >> (16 * (e & 1)));
    }
  } else {
    float* q = (float*)p + i;
    if (wide && left >= 4) {
      *(float4*)q = float4{v[0], v[1], v[2], v[3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (e < left) q[e] = v[e];
    }
  }
}

// m and the squares of u, a workgroup to a chunk of a matrix (12 bytes an
// element: see above).
template <bool GBF16>
__global__ __launch_bounds__(kMomentThreads) void muon_moment_kernel(MuonArgs a) {
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = blockIdx.x - a.first.at[ri];
  const int64_t matrix = b / r.chunks, chunk = b % r.chunks;
  const int64_t n = (int64_t)r.rows * r.cols, base = matrix * n;
  const int64_t lo = chunk * r.chunk, hi = lo + r.chunk < n ? lo + r.chunk : n;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const bool wide = r.wide;
  double s = 0;
#pragma unroll 4
  for (int64_t i = lo + threadIdx.x * 4; i < hi; i += kMomentThreads * 4) {
    float g[4], m[4];
    get4<GBF16>(r.grad, base + i, hi - i, wide, g);
    get4<false>(r.m, base + i, hi - i, wide, m);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      g[e] *= gs;
      m[e] = fmaf(a.momentum, m[e], g[e]);
      const float u = a.nesterov ? fmaf(a.momentum, m[e], g[e]) : m[e];
      s += (double)u * u;
    }
    put4<false>(r.m, base + i, hi - i, wide, m);
  }
  __shared__ double part[kMomentThreads / 64];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0;
    for (int w = 0; w < kMomentThreads / 64; ++w) t += part[w];
    r.squares[matrix * r.chunks + chunk] = t;
  }
}

// X = u / max(|u|, eps), 64 x 64 of the padded matrix to a workgroup.
template <bool GBF16>
__global__ __launch_bounds__(256) void muon_scale_kernel(MuonArgs a) {
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = blockIdx.x - a.first.at[ri];
  const uint32_t tn = r.nn / 64, tiles = (uint32_t)(r.mm / 64) * tn;
  const int64_t matrix = b / tiles;
  const int i0 = (int)(b % tiles / tn) * 64, j0 = (int)(b % tiles % tn) * 64;
  const bool tall = r.rows > r.cols, wide = r.wide;
  const int tid = threadIdx.x;
  __shared__ float tile[64][65];
  // the matrix's norm, summed in the same order by every wavefront
  double s = 0;
  for (uint32_t i = tid & 63; i < r.chunks; i += 64) s += r.squares[matrix * r.chunks + i];
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
  const double inv = inverse_norm(sqrt(s), a.eps);
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  // read along the source's rows
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int tr = k * 16 + (tid >> 4), tc = (tid & 15) * 4;
    const int rr = r0 + tr, cc = c0 + tc, left = r.cols - cc;
    float u[4] = {0, 0, 0, 0};
    if (rr < r.rows && left > 0) {
      const int64_t i = base + (int64_t)rr * r.cols + cc;
      get4<false>(r.m, i, left, wide, u);
      if (a.nesterov) {
        float g[4];
        get4<GBF16>(r.grad, i, left, wide, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = fmaf(a.momentum, u[e], g[e] * gs);
      }
      if (a.zero_grads) {
        const float z[4] = {0, 0, 0, 0};
        put4<GBF16>(r.grad, i, left, wide, z);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = e < left ? (float)((double)u[e] * inv) * kHeld : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[tr][tc + e] = u[e];
  }
  __syncthreads();
  const int64_t at = matrix * (int64_t)r.mm * r.nn;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = k * 32 + (tid >> 3), j = (tid & 7) * 8;
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v0 = tall ? tile[j + 2 * e][i] : tile[i][j + 2 * e];
      const float v1 = tall ? tile[j + 2 * e + 1][i] : tile[i][j + 2 * e + 1];
      split2(v0, v1, h[e], l[e]);
    }
    const int64_t o = at + (int64_t)(i0 + i) * r.nn + j0 + j;
    *(uint4*)(r.x[0] + o) = uint4{h[0], h[1], h[2], h[3]};
    *(uint4*)(r.rest[0] + o) = uint4{l[0], l[1], l[2], l[3]};
  }
}

enum Product { kGram = 0, kPoly = 1, kApply = 2, kUpdate = 3 };

// p = p (1 - lr weight_decay) - lr scale X at N places of four neighbours:
// place(k, i, left) gives the element and how many of its row are left there
// (none: not a place), x(k, v) the values of 2^8 X. All reads come first, as
// the compiler cannot move one past a store.
template <bool PBF16, int N, class Place>
__device__ __forceinline__ void update_read(const MuonRec& r, Place place, float (*p)[4]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    int64_t i;
    int left;
    place(k, i, left);
    if (left <= 0) continue;
    if (PBF16 && !r.master) get4<true>(r.param, i, left, r.wide, p[k]);
    else get4<false>(PBF16 ? r.master : r.param, i, left, r.wide, p[k]);
  }
}
template <bool PBF16, int N, class Place, class X>
__device__ __forceinline__ void update_write(const MuonRec& r, Place place, X x, float (*p)[4]) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    int64_t i;
    int left;
    place(k, i, left);
    if (left <= 0) continue;
    float v[4];
    x(k, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) p[k][e] = fmaf(-r.move, v[e] * (1.0f / kHeld), p[k][e] * r.decay);
    if (r.master) put4<false>(r.master, i, left, r.wide, p[k]);
    put4<PBF16>(r.param, i, left, r.wide, p[k]);
  }
}
template <bool PBF16, int N, class Place, class X>
__device__ __forceinline__ void update_n(const MuonRec& r, Place place, X x) {
  float p[N][4];
  update_read<PBF16, N>(r, place, p);
  update_write<PBF16, N>(r, place, x, p);
}

// One T x T tile of one matrix's product, by wavefronts of 64 x 64 (T = 128) or
// 64 x 128 (T = 256). The workgroups of an XCD have neighbouring tiles, whose
// operands its L2 then holds once (48 matrices of 768 x 2048, G: 135 -> 100 us).
// The sums go through LDS, so that memory is read and written in whole lines
// (X of the same: 412 -> 219 us). kUpdate is the last step's kApply: its X
// goes into the parameters at once. Two stages of 64 of the k axis; four take
// as long, also where a CU has one small tile alone. With T = 256, kUpdate has more
// alive than the registers hold and spills, outside the k loop, 25 of a lane for
// fp32 parameters and 6 for bf16 ones (48 matrices of 768 x 2048, the whole step:
// 2189 us in fp32, 2205 in bf16 with masters).
template <int P, bool PBF16, int T>
__global__ __launch_bounds__(T * 2) void muon_product_kernel(MuonArgs a) {
  constexpr int NS = 2, BK = kMuonBK, NW = T / 32, NT = 64 * NW, WN = T / 2;
  constexpr bool SYM = P == kGram || P == kPoly;
  using CoreT = Core<T, T, T / 64, 2, false, Fp16>;
  using AT = KTile<T, BK, NW>;
  using BT = typename std::conditional<SYM, KTile<T, BK, NW>, MTile<T, BK, NW>>::type;
  constexpr int STAGE = AT::BYTES + BT::BYTES;
  constexpr int LD = T + 4;  // floats of a row of sums: rows 4 banks apart
  constexpr int H = 64;      // the sums go through LDS by the rows of a wavefront
  constexpr int LDS_BYTES = NS * STAGE > H * LD * 4 ? NS * STAGE : H * LD * 4;
  __shared__ __attribute__((aligned(1024))) char lds[LDS_BYTES];
  const uint32_t bid = (uint32_t)xcd_virtual_id();
  if (bid >= a.n_work) return;
  const int ri = find_rec(a, bid);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = bid - a.first.at[ri];
  const uint32_t tm = (uint32_t)r.mm / T, tn = (uint32_t)r.nn / T;
  const uint32_t tiles = SYM ? tm * (tm + 1) / 2 : tm * tn;
  const int64_t matrix = b / tiles;
  uint32_t ti, tj, t = b % tiles;
  if constexpr (SYM) {  // row by row of the upper triangle
    ti = 0;
    while (t >= tm - ti) t -= tm - ti, ++ti;
    tj = ti + t;
  } else {
    ti = t % tm, tj = t / tm;
  }
  const int i0 = __builtin_amdgcn_readfirstlane((int)ti) * T, j0 = __builtin_amdgcn_readfirstlane((int)tj) * T;
  const int lane = lane64(), wave = wave_id(), wm = wave / 2, wn = wave % 2;
  const int64_t xat = matrix * (int64_t)r.mm * r.nn;
  const uint16_t* X = r.x[a.from] + xat;
  uint16_t* G = r.gram + matrix * (int64_t)r.mm * r.mm;
  uint16_t* Q = r.poly + matrix * (int64_t)r.mm * r.mm;
  const int lda = P == kGram ? r.nn : r.mm, ldb = P == kPoly ? r.mm : r.nn;
  const int KT = (P == kGram ? r.nn : r.mm) / BK;
  const uint16_t* abase = (P == kGram ? X : P == kPoly ? G : Q) + (int64_t)i0 * lda;
  const uint16_t* bbase = SYM ? (P == kGram ? X : G) + (int64_t)j0 * ldb : X + j0;
  const uint32_t lda2 = (uint32_t)lda * 2, ldb2 = (uint32_t)ldb * 2;
  const uint32_t lds0 = lds_addr(lds);
  auto off_a = [&](int q) -> uint32_t { return (uint32_t)q * lda2; };
  auto off_b = [&](int q) -> uint32_t { return (uint32_t)q * ldb2; };
  const uint32_t va0 = AT::voff(lane, off_a, 0), vb0 = BT::voff(lane, off_b, 0);
  uint32_t sa[AT::PER_WAVE], sb[BT::PER_WAVE];
#pragma unroll
  for (int i = 0; i < AT::PER_WAVE; ++i) sa[i] = __builtin_amdgcn_readfirstlane(AT::voff(lane, off_a, i) - va0);
#pragma unroll
  for (int i = 0; i < BT::PER_WAVE; ++i) sb[i] = __builtin_amdgcn_readfirstlane(BT::voff(lane, off_b, i) - vb0);
  auto issue = [&](int kt, int p) {  // stages past the last load nothing
    const bool live = kt < KT;
    const uint32_t st = lds0 + (uint32_t)((kt % NS) * STAGE);
    const int k0 = live ? kt * BK : 0;
    if (p < AT::PER_WAVE) {
      AT::issue_s(buf_rsrc(abase + k0, live ? (uint32_t)T * lda2 - 2u * k0 : 0u), st, va0, sa[p], p);
    } else if constexpr (SYM) {
      BT::issue_s(buf_rsrc(bbase + k0, live ? (uint32_t)T * ldb2 - 2u * k0 : 0u), st + AT::BYTES, vb0,
                  sb[p - AT::PER_WAVE], p - AT::PER_WAVE);
    } else {
      BT::issue_s(buf_rsrc(bbase + (int64_t)k0 * ldb, live ? (uint32_t)BK * ldb2 - 2u * j0 : 0u), st + AT::BYTES, vb0,
                  sb[p - AT::PER_WAVE], p - AT::PER_WAVE);
    }
  };
  // What the epilogue reads of X or G, 16 bytes at a time, is on its way a
  // part ahead, the first under the k loop where the registers hold it.
  const int tid = threadIdx.x, ei = tid / (T / 8), ej = tid % (T / 8) * 8;  // row (+ 16 k) and column
  constexpr bool OF_X = P == kApply || P == kUpdate;
  uint4 old[2][4], rest[2][4];
  auto fetch = [&](int part) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = i0 + part * H + k * 16 + ei;
      if constexpr (OF_X) {
        const int64_t o = xat + (int64_t)row * r.nn + j0 + ej;
        old[part & 1][k] = *(const uint4*)(r.x[a.from] + o);
        if (a.has_rest) rest[part & 1][k] = *(const uint4*)(r.rest[a.from] + o);
      } else if constexpr (P == kPoly) {
        old[part & 1][k] = *(const uint4*)(G + (int64_t)row * r.mm + j0 + ej);
      }
    }
  };
  if constexpr (T == 128) fetch(0);
  CoreT core;
  const typename CoreT::template Offsets<AT, BT, BK> offs(lane, wm, wn);
  core.zero();
  pipelined_k_loop<CoreT, AT, BT, BK, NS, T == 256 ? 2 : 1>(core, lds, KT, offs, issue, false, [] {});
  if constexpr (T != 128) fetch(0);

  float(*sum)[LD] = (float(*)[LD])lds;
  const bool tall = r.rows > r.cols;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  static_for<0, T / H>([&](auto partc) {
    constexpr int part = decltype(partc)::value;
    __syncthreads();  // every wavefront has read its last fragments, or the sums before
    if (wm == part) {
#pragma unroll
      for (int i = 0; i < CoreT::MB; ++i)
#pragma unroll
        for (int j = 0; j < CoreT::NB; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = core.acc[i][j][4 * q + e] * (1.0f / kHeld);
            *(float4*)&sum[32 * i + (lane & 31)][wn * WN + 32 * j + 8 * q + 4 * (lane >> 5)] =
                float4{v[0], v[1], v[2], v[3]};
          }
    }
    const int ih = i0 + part * H;  // their first row
    // kUpdate: H rows of X by T columns are so many of the parameters, or T
    // rows by H columns; of a small tile they are read here already
    const int r0 = tall ? j0 : ih, c0 = tall ? ih : j0;
    const int pi = tall ? tid / 16 : tid / (T / 4), pk = tall ? NT / 16 : 8, pj = (tall ? tid % 16 : tid % (T / 4)) * 4;
    auto place = [&](int k, int64_t& o, int& left) {
      const int row = r0 + pi + pk * k;
      o = base + (int64_t)row * r.cols + c0 + pj, left = row < r.rows ? r.cols - (c0 + pj) : 0;
    };
    float param[P == kUpdate ? 8 : 1][4];
    if constexpr (P == kUpdate && T == 128) update_read<PBF16, 8>(r, place, param);
    __syncthreads();
    if constexpr (part + 1 < T / H) fetch(part + 1);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = k * 16 + ei, j = ej;
      float v[8];
      *(float4*)v = *(const float4*)&sum[i][j];
      *(float4*)(v + 4) = *(const float4*)&sum[i][j + 4];
      const uint4 h4 = old[part & 1][k];
      const uint32_t h[4] = {h4.x, h4.y, h4.z, h4.w};
      if constexpr (OF_X) {
        const int64_t o = xat + (int64_t)(ih + i) * r.nn + j0 + j;
        const uint4 l4 = a.has_rest ? rest[part & 1][k] : uint4{0, 0, 0, 0};
        const uint32_t l[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(a.a, join(h[e / 2], l[e / 2], e & 1), v[e]);
        if constexpr (P == kApply) {
          uint32_t nh[4], nl[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) split2(v[2 * e], v[2 * e + 1], nh[e], nl[e]);
          *(uint4*)(r.x[a.from ^ 1] + o) = uint4{nh[0], nh[1], nh[2], nh[3]};
          if (a.put_rest) *(uint4*)(r.rest[a.from ^ 1] + o) = uint4{nl[0], nl[1], nl[2], nl[3]};
        } else {
          *(float4*)&sum[i][j] = *(const float4*)v;
          *(float4*)&sum[i][j + 4] = *(const float4*)(v + 4);
        }
      } else {
        const int64_t o = (int64_t)(ih + i) * r.mm + j0 + j;
        if constexpr (P == kPoly) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = fmaf(a.c, v[e], a.b * half_value(h[e / 2] >> (16 * (e & 1)) & 0xffffu));
          *(float4*)&sum[i][j] = *(const float4*)v;
          *(float4*)&sum[i][j + 4] = *(const float4*)(v + 4);
        }
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (uint32_t)half_bits(v[2 * e]) | (uint32_t)half_bits(v[2 * e + 1]) << 16;
        *(uint4*)((P == kGram ? G : Q) + o) = uint4{w[0], w[1], w[2], w[3]};
      }
    }
    if (P != kApply && !(SYM && ti == tj)) {
      __syncthreads();
      if constexpr (SYM) {  // the same on the other side of the diagonal
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = k * (NT / 8) + (tid >> 3), i = (tid & 7) * 8;
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            w[e] = (uint32_t)half_bits(sum[i + 2 * e][j]) | (uint32_t)half_bits(sum[i + 2 * e + 1][j]) << 16;
          *(uint4*)((P == kGram ? G : Q) + (int64_t)(j0 + j) * r.mm + ih + i) = uint4{w[0], w[1], w[2], w[3]};
        }
      } else {
        if constexpr (T != 128) update_read<PBF16, 8>(r, place, param);
        update_write<PBF16, 8>(
            r, place,
            [&](int k, float* v) {
              const int i = pi + pk * k;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = tall ? sum[pj + e][i] : sum[i][pj + e];
            },
            param);
      }
    }
  });
}

// The update without any step of the iteration: 64 x 64 of X to a workgroup.
template <bool PBF16>
__global__ __launch_bounds__(256) void muon_update_kernel(MuonArgs a) {
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = blockIdx.x - a.first.at[ri];
  const uint32_t tn = r.nn / 64, tiles = (uint32_t)(r.mm / 64) * tn;
  const int64_t matrix = b / tiles;
  const int i0 = (int)(b % tiles / tn) * 64, j0 = (int)(b % tiles % tn) * 64;
  const bool tall = r.rows > r.cols;
  const int tid = threadIdx.x;
  __shared__ float tile[64][65];
  const int64_t at = matrix * (int64_t)r.mm * r.nn;
  for (int e = tid; e < 4096; e += 256) {
    const int i = e >> 6, j = e & 63;
    const int64_t o = at + (int64_t)(i0 + i) * r.nn + j0 + j;
    const float x = join(r.x[0][o], r.rest[0][o], 0);
    if (tall) tile[j][i] = x;
    else tile[i][j] = x;
  }
  __syncthreads();
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0, j = (tid & 15) * 4;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  update_n<PBF16, 4>(
      r,
      [&](int k, int64_t& o, int& left) {
        const int row = r0 + (tid >> 4) + 16 * k;
        o = base + (int64_t)row * r.cols + c0 + j, left = row < r.rows ? r.cols - (c0 + j) : 0;
      },
      [&](int k, float* v) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = tile[(tid >> 4) + 16 * k][j + e];
      });
}

// ---------------------------------------------------------------------------
// Matrices with a side of at most 64. With M = a I + b G + c G G, all of G, M
// and Q are symmetric polynomials of the first G and commute: X = Q X0 with Q = M
// .. M, and the next G is M G M. So X is read twice, for the first G and for
// Q X0, and the rest happens in the LDS of one workgroup a matrix.
//
// All of it is fp64, and only so many steps at a time (a stage, see
// small_stages): what G is off by where u has nothing, or next to nothing, is an
// eigenvalue near 0 of either sign, which a step multiplies by a^2, where X itself
// would have no such eigenvalue and grow by a. Once a negative one is no longer
// small, M runs away with it. From an fp32 G that takes 8 to 10 steps of the
// usual coefficients; from an fp64 one it stays below 2^-53 2^24, and the next
// stage forms G again from X, which is held in fp64 in between. X comes out within
// the rounding of fp32 whatever the rank of u and the number of steps (simulated:
// 2^-24 of its norm after 16 steps, where the plain iteration in fp32 has filled
// the empty directions). Latency bounds it: the small ones of six matrices with
// sides of 24 to 400 take 8, 25 and 13 us (in fp32 9, 27 and 13).
// ---------------------------------------------------------------------------
constexpr int kSmall = 64, kSmallChunks = 64;
constexpr int kSmallLD = 68;       // doubles of a row in LDS: 16 rows of 4 are 2 to a bank
constexpr int kSmallThreads = 512; // of a matrix's steps: two wavefronts a SIMD

typedef double f64x4 __attribute__((ext_vector_type(4)));
typedef double SmallRow[kSmallLD];

// 16 x 16 tiles along a side of m, and of the upper triangle.
__host__ __device__ __forceinline__ int small_tiles(int m) { return (m + 15) / 16; }
__host__ __device__ __forceinline__ int small_upper(int m) { return small_tiles(m) * (small_tiles(m) + 1) / 2; }

// Tile t of the upper triangle, column by column: those of a smaller matrix come first.
__device__ __forceinline__ void small_tile(int t, int& ti, int& tj) {
  tj = t < 1 ? 0 : t < 3 ? 1 : t < 6 ? 2 : 3;
  ti = t - tj * (tj + 1) / 2;
}

// acc += that tile of A B^T, k below n (a multiple of 4). The matrix
// instruction leaves row 4 q + lane / 16, column lane % 16 in element q.
__device__ __forceinline__ f64x4 small_product(const SmallRow* A, const SmallRow* B, int ti, int tj, int n, f64x4 acc) {
  const int lane = lane64(), l = lane & 15, h = lane >> 4;
#pragma unroll 4
  for (int k = 0; k < n; k += 4)
    acc = __builtin_amdgcn_mfma_f64_16x16x4f64(A[16 * ti + l][k + h], B[16 * tj + l][k + h], acc, 0, 0, 0);
  return acc;
}

// A tile of a symmetric matrix, on both sides of the diagonal: f(q, i, j) gives
// element q. Of a tile on the diagonal the upper half counts, so that the matrix
// is symmetric to the last bit and its rows serve as its columns.
template <class F>
__device__ __forceinline__ void small_put(SmallRow* M, int ti, int tj, F&& f) {
  const int lane = lane64(), j = 16 * tj + (lane & 15);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int i = 16 * ti + 4 * q + (lane >> 4);
    const double v = f(q, i, j);
    if (i <= j) M[i][j] = v, M[j][i] = v;
  }
}

// The 64 x 64 tile of the matrix whose first long index is l0, the small side as
// rows, into LDS; zeros past the ends. In the first stage it is u, times inv,
// otherwise X. MOMENT: m is updated on the way, and nothing is scaled.
template <bool GBF16, bool MOMENT>
__device__ __forceinline__ void small_x(const MuonArgs& a, const MuonRec& r, int64_t matrix, int l0, double inv,
                                        SmallRow* u) {
  const bool tall = r.rows > r.cols;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  if (!a.from_u) {
    const int m = tall ? r.cols : r.rows, n = tall ? r.rows : r.cols;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int i = k * 4 + (threadIdx.x >> 6), j = threadIdx.x & 63;
      u[i][j] = i < m && l0 + j < n ? r.held[base + (int64_t)i * n + l0 + j] : 0.0;
    }
    return;
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const int r0 = tall ? l0 : 0, c0 = tall ? 0 : l0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int tr = k * 16 + (threadIdx.x >> 4), tc = (threadIdx.x & 15) * 4;
    const int rr = r0 + tr, cc = c0 + tc, left = r.cols - cc;
    float v[4] = {0, 0, 0, 0};
    if (rr < r.rows && left > 0) {
      const int64_t i = base + (int64_t)rr * r.cols + cc;
      float g[4] = {0, 0, 0, 0};
      get4<false>(r.m, i, left, r.wide, v);
      if (MOMENT || a.nesterov) {
        get4<GBF16>(r.grad, i, left, r.wide, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] *= gs;
      }
      if constexpr (MOMENT) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(a.momentum, v[e], g[e]);
        put4<false>(r.m, i, left, r.wide, v);
      } else if (a.zero_grads) {
        const float z[4] = {0, 0, 0, 0};
        put4<GBF16>(r.grad, i, left, r.wide, z);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (a.nesterov) v[e] = fmaf(a.momentum, v[e], g[e]);
        if (e >= left) v[e] = 0.0f;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double x = MOMENT ? (double)v[e] : (double)v[e] * inv;
      if (tall) u[tc + e][tr] = x;
      else u[tr][tc + e] = x;
    }
  }
}

// A chunk's part of u u^T (squares of fp32 numbers are far inside fp64's range),
// with m on the way, or of X X^T.
template <bool GBF16>
__global__ __launch_bounds__(256) void muon_small_gram_kernel(MuonArgs a) {
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = blockIdx.x - a.first.at[ri];
  const int64_t matrix = b / r.chunks, chunk = b % r.chunks;
  const bool tall = r.rows > r.cols;
  const int n = tall ? r.rows : r.cols;
  const int blocks = (n + 63) / 64;  // of the long side
  const int b0 = (int)(blocks * chunk / r.chunks), b1 = (int)(blocks * (chunk + 1) / r.chunks);
  const int wave = wave_id(), tiles = small_upper(tall ? r.cols : r.rows);
  __shared__ SmallRow u[kSmall];
  f64x4 acc[3];
#pragma unroll
  for (int p = 0; p < 3; ++p) acc[p] = f64x4{0, 0, 0, 0};
  for (int t = b0; t < b1; ++t) {
    __syncthreads();
    small_x<GBF16, true>(a, r, matrix, t * 64, 1.0, u);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      int ti, tj;
      small_tile(wave + 4 * p, ti, tj);
      if (wave + 4 * p < tiles) acc[p] = small_product(u, u, ti, tj, kSmall, acc[p]);
    }
  }
  double* to = r.part + (matrix * r.chunks + chunk) * (tiles * 256) + lane64();
#pragma unroll
  for (int p = 0; p < 3; ++p)
    if (wave + 4 * p < tiles)
#pragma unroll
      for (int q = 0; q < 4; ++q) to[(wave + 4 * p) * 256 + q * 64] = acc[p][q];
}

// Q of a stage, and in the first one 1 / max(|u|, eps).
__global__ __launch_bounds__(kSmallThreads) void muon_small_steps_kernel(MuonArgs a) {
  constexpr int NW = kSmallThreads / 64;
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const int64_t matrix = blockIdx.x - a.first.at[ri];
  const int m = r.rows < r.cols ? r.rows : r.cols, n = (m + 3) & ~3, side = 16 * small_tiles(m);
  const int tiles = small_upper(m);
  const int tid = threadIdx.x, lane = lane64(), wave = wave_id();
  __shared__ SmallRow G[kSmall], M[kSmall], S[kSmall], Q[kSmall];
  const double* part = r.part + matrix * r.chunks * (tiles * 256);
  for (int o = tid; o < tiles * 256; o += kSmallThreads) {
    double s = 0;
#pragma unroll 8
    for (int c = 0; c < (int)r.chunks; ++c) s += part[c * (tiles * 256) + o];
    int ti, tj;
    small_tile(o >> 8, ti, tj);
    const int i = 16 * ti + (o >> 6 & 3) * 4 + (lane >> 4), j = 16 * tj + (lane & 15);
    if (i <= j) G[i][j] = s, G[j][i] = s;
  }
  for (int o = tid; o < side * side; o += kSmallThreads) Q[o / side][o % side] = o / side == o % side ? 1.0 : 0.0;
  __syncthreads();
  if (a.from_u) {
    // |u|^2, summed in the same order by every wavefront
    double s = lane < m ? G[lane][lane] : 0.0;
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
    const double inv = inverse_norm(sqrt(s), a.eps);
    __syncthreads();
    for (int o = tid; o < side * side; o += kSmallThreads) G[o / side][o % side] *= inv * inv;
    if (tid == 0) r.inverse[matrix] = inv;
    __syncthreads();
  }
  for (int t = 0; t < a.steps; ++t) {
    const bool more = t + 1 < a.steps;
    f64x4 q[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      int ti, tj;
      small_tile(wave + NW * p, ti, tj);
      if (wave + NW * p >= tiles) continue;
      const f64x4 s = small_product(G, G, ti, tj, n, f64x4{0, 0, 0, 0});
      small_put(M, ti, tj, [&](int e, int i, int j) {
        return (i == j ? a.coef[0] : 0.0) + fma(a.coef[1], G[i][j], a.coef[2] * s[e]);
      });
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      int ti, tj;
      small_tile(wave + NW * p, ti, tj);
      if (wave + NW * p >= tiles) continue;
      if (more) {
        const f64x4 s = small_product(M, G, ti, tj, n, f64x4{0, 0, 0, 0});
        small_put(S, ti, tj, [&](int e, int, int) { return s[e]; });
      }
      q[p] = small_product(M, Q, ti, tj, n, f64x4{0, 0, 0, 0});
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      int ti, tj;
      small_tile(wave + NW * p, ti, tj);
      if (wave + NW * p >= tiles) continue;
      small_put(Q, ti, tj, [&](int e, int, int) { return q[p][e]; });
      if (more) {
        const f64x4 g = small_product(S, M, ti, tj, n, f64x4{0, 0, 0, 0});
        small_put(G, ti, tj, [&](int e, int, int) { return g[e]; });
      }
    }
    __syncthreads();
  }
  for (int o = tid; o < side * side; o += kSmallThreads) r.q[matrix * (side * side) + o] = Q[o / side][o % side];
}

// X = Q X for 64 of the long side: into the parameters, or held for the next
// stage in place of what it was.
template <bool GBF16, bool PBF16>
__global__ __launch_bounds__(256) void muon_small_apply_kernel(MuonArgs a) {
  const int ri = find_rec(a, blockIdx.x);
  const MuonRec& r = a.rec[ri];
  const uint32_t b = blockIdx.x - a.first.at[ri];
  const bool tall = r.rows > r.cols;
  const int m = tall ? r.cols : r.rows, n = tall ? r.rows : r.cols;
  const int blocks = (n + 63) / 64, tid = threadIdx.x, lane = lane64(), wave = wave_id();
  const int64_t matrix = b / blocks;
  const int l0 = (int)(b % blocks) * 64;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  __shared__ SmallRow u[kSmall], Q[kSmall];
  const int side = 16 * small_tiles(m);
  for (int i = tid; i < side * side; i += 256) Q[i / side][i % side] = r.q[matrix * (side * side) + i];
  small_x<GBF16, false>(a, r, matrix, l0, a.from_u ? r.inverse[matrix] : 1.0, u);
  __syncthreads();
  // rows 16 wave .. of X, all 64 columns
  const int l = lane & 15, h = lane >> 4;
  f64x4 x[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) x[c] = f64x4{0, 0, 0, 0};
  if (16 * wave < m) {
#pragma unroll 2
    for (int k = 0; k < m; k += 4) {  // (u is zero past m)
      const double q = Q[16 * wave + l][k + h];
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = __builtin_amdgcn_mfma_f64_16x16x4f64(q, u[k + h][16 * c + l], x[c], 0, 0, 0);
    }
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int q = 0; q < 4; ++q) u[16 * wave + 4 * q + h][16 * c + l] = x[c][q];
  __syncthreads();
  if (!a.to_params) {
    for (int o = tid; o < m * 64; o += 256) {
      const int i = o >> 6, j = o & 63;
      if (l0 + j < n) r.held[base + (int64_t)i * n + l0 + j] = u[i][j];
    }
    return;
  }
  const int r0 = tall ? l0 : 0, c0 = tall ? 0 : l0, i0 = tid >> 4, j = (tid & 15) * 4;
  update_n<PBF16, 4>(
      r,
      [&](int k, int64_t& at, int& left) {
        const int row = r0 + i0 + 16 * k;
        at = base + (int64_t)row * r.cols + c0 + j, left = row < r.rows ? r.cols - (c0 + j) : 0;
      },
      [&](int k, float* v) {
        const int i = i0 + 16 * k;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)(tall ? u[j + e][i] : u[i][j + e]) * kHeld;
      });
}

// ---------------------------------------------------------------------------
// What the coefficients make of singular values, and the stages that follow.
// ---------------------------------------------------------------------------
// The largest |p + q l + r l^2| for l in [0, top].
double most_of(double p, double q, double r, double top) {
  const double v = fmax(fabs(p), fabs(p + (q + r * top) * top)), at = -q / (2 * r);
  return at > 0 && at < top ? fmax(v, fabs(p + 0.5 * q * at)) : v;
}

// One step on an X whose singular values are at most s.
struct Reach {
  double s;     // what they are at most afterwards: the largest |s M(s^2)|
  double poly;  // the largest |b s^2 + c s^4|
  double off;   // an eigenvalue l of G becomes f(l) = l M(l)^2: the largest |f'| = |M(l)| |a + 3 b l + 5 c l^2|, or 1
};
Reach reach(const double* coef, double s) {
  const double a = coef[0], b = coef[1], c = coef[2], top = s * s;
  Reach r;
  r.poly = most_of(0.0, b, c, top);
  r.off = fmax(1.0, most_of(a, b, c, top) * most_of(a, 3 * b, 5 * c, top));
  // s M(s^2) is largest at an end, or where a + 3 b l + 5 c l^2 is 0
  r.s = s * fabs(a + (b + c * top) * top);
  const double h = 1.5 * b, t = -(h + copysign(sqrt(h * h - 5 * c * a), h));
  for (double l : {t / (5 * c), a / t})
    if (l > 0 && l < top) r.s = fmax(r.s, sqrt(l) * fabs(a + (b + c * l) * l));
  return r;
}

// Stages of small matrices: what G is off by is multiplied by `off` each step (a^2
// near 0). A stage ends before their product passes 2^24.
struct Stages {
  int n, steps[16];
};
Stages small_stages(const double* coef, int ns_steps) {
  Stages g{};
  g.n = 1;
  double s = 1.0, off = 1.0;  // (|X| is 1 at first)
  for (int t = 0; t < ns_steps; ++t) {
    const Reach r = reach(coef, s);
    if (g.steps[g.n - 1] > 0 && !(off * r.off <= (double)(1 << 24))) ++g.n, off = 1.0;
    off *= r.off, s = r.s, ++g.steps[g.n - 1];
  }
  return g;
}

// Whether G and P of large matrices stay within fp16, 2^8 times as large as they
// are held: below 255.8, of which the format's roundings may take some.
constexpr double kHalfMost = 250.0;
bool within_half(const double* coef, int ns_steps) {
  double s = 1.0;
  for (int t = 0; t < ns_steps; ++t) {
    const Reach r = reach(coef, s);
    if (!(s * s <= kHalfMost && r.poly <= kHalfMost)) return false;
    s = r.s;
  }
  return true;
}

int64_t pad_side(int64_t n, int tile) { return (n + tile - 1) / tile * tile; }

bool is_small(const foremoe_muon_tensor& t) { return t.rows <= kSmall || t.cols <= kSmall; }

// Lays a tensor's part of the workspace out from `at` (bytes); returns its end.
size_t lay_out(const foremoe_muon_tensor& t, int tile, size_t at, char* ws, MuonRec* r) {
  const int64_t s = t.rows < t.cols ? t.rows : t.cols, l = t.rows < t.cols ? t.cols : t.rows;
  const int64_t mm = pad_side(s, tile), nn = pad_side(l, tile);
  const int64_t even = ((s * l + kMomentMost - 1) / kMomentMost + 1023) / 1024 * 1024;
  const int64_t chunk = even > kMomentChunk ? even : kMomentChunk, chunks = (s * l + chunk - 1) / chunk;
  auto take = [&](size_t bytes) {
    char* p = ws + at;
    at = align_up(at + bytes, 256);
    return p;
  };
  MuonRec q{};
  if (s <= kSmall) {
    const int64_t tiles = (l + 63) / 64;
    // parts of u u^T to be joined by one workgroup: 16, more for the longest
    const int64_t most = tiles < 256 ? 16 : kSmallChunks;
    q.chunks = (uint32_t)(tiles < most ? tiles : most);
    q.part = (double*)take((size_t)t.batch * q.chunks * small_upper((int)s) * 256 * 8);
    q.q = (double*)take((size_t)t.batch * small_tiles((int)s) * small_tiles((int)s) * 256 * 8);
    q.inverse = (double*)take((size_t)t.batch * 8);
    q.held = (double*)take((size_t)t.batch * s * l * 8);
    if (r) *r = q;
    return at;
  }
  for (int i = 0; i < 2; ++i) {
    q.x[i] = (uint16_t*)take((size_t)t.batch * mm * nn * 2);
    q.rest[i] = (uint16_t*)take((size_t)t.batch * mm * nn * 2);
  }
  q.gram = (uint16_t*)take((size_t)t.batch * mm * mm * 2);
  q.poly = (uint16_t*)take((size_t)t.batch * mm * mm * 2);
  q.squares = (double*)take((size_t)t.batch * chunks * 8);
  q.mm = (int)mm, q.nn = (int)nn, q.chunks = (uint32_t)chunks, q.chunk = (int32_t)chunk;
  if (r) *r = q;
  return at;
}

// 64 x 64 tiles of a tensor padded to 256: no launch over it has more workgroups.
constexpr int64_t kMuonMostTiles = (int64_t)1 << 23;
int64_t scale_tiles(const foremoe_muon_tensor& t) {
  return t.batch * (pad_side(t.rows, 256) / 64) * (pad_side(t.cols, 256) / 64);
}

// Tiles of the products' launches over the tensors [i, end), counted for 256 CUs
// whatever the device has, as the workspace's size goes by them and is asked for
// without one (with fewer CUs it is the choice that may be the slower one): of the symmetric
// ones, and of X. A k step of a 256-wide tile takes a CU about as long as one
// of two 128-wide ones, four times the work against two; one 128-wide tile
// alone on a CU about half of that. So the wide ones are faster where whole rounds of
// them fill the CUs and the padding does not take it back (us, 128 / 256: 48
// matrices of 768 x 2048, G 104 / 124, X 219 / 211; 6 of 2048 x 7168, G 246 /
// 194, X 464 / 441; the large ones of six with sides of 24 to 400, G 10 / 13, X 10
// / 20).
struct Tiles {
  int pad, sym, full;
};
Tiles choose_tiles(const foremoe_muon_tensor* tensors, int i, int end) {
  // rounds x k steps of a launch of `tile` over matrices padded to `pad`
  auto cost = [&](int tile, int pad, bool of_x) {
    double tiles = 0, steps = 0;
    for (int j = i; j < end; ++j) {
      const foremoe_muon_tensor& t = tensors[j];
      if (t.batch == 0 || is_small(t)) continue;
      const double m = (double)pad_side(t.rows < t.cols ? t.rows : t.cols, pad);
      const double n = (double)pad_side(t.rows < t.cols ? t.cols : t.rows, pad);
      const double tm = m / tile, count = t.batch * (of_x ? tm * (n / tile) : tm * (tm + 1) / 2);
      tiles += count, steps += count * (of_x ? m : n + m);
    }
    if (tiles == 0) return 0.0;
    const bool wide = tile == 256;
    return ceil(tiles / (wide ? 256 : 512)) * (steps / tiles) * (wide || tiles > 256 ? 1.0 : 0.5);
  };
  const double sym = cost(128, 256, false), full = cost(128, 256, true);
  const double wide_sym = cost(256, 256, false), wide_full = cost(256, 256, true);
  const double narrow = cost(128, 128, false) + cost(128, 128, true);
  if (narrow <= fmin(sym, wide_sym) + fmin(full, wide_full)) return {128, 128, 128};
  return {256, wide_sym < sym ? 256 : 128, wide_full < full ? 256 : 128};
}

// The end of the launches' group of tensors that starts at i.
int group_end(const foremoe_muon_tensor* tensors, int i, int n) {
  int count = 0;
  int64_t tiles = 0;
  for (; i < n; ++i) {
    if (tensors[i].batch == 0) continue;
    tiles += scale_tiles(tensors[i]);
    if (count == FOREMOE_MUON_LAUNCH || (count > 0 && tiles > kMuonMostTiles)) break;
    ++count;
  }
  return i;
}

int check_tensor(const foremoe_muon_tensor& t, int i) {
  if (t.batch < 0 || t.batch > (int64_t)1 << 30)
    return set_error(FOREMOE_EINVAL, "muon_step: tensor %d: batch=%lld outside [0, 2^30]", i, (long long)t.batch);
  if (t.batch == 0) return FOREMOE_OK;
  if (t.rows < 1 || t.cols < 1 || t.rows > FOREMOE_MUON_SIDE || t.cols > FOREMOE_MUON_SIDE ||
      (t.rows < t.cols ? t.rows : t.cols) > FOREMOE_MUON_RANK)
    return set_error(FOREMOE_EINVAL, "muon_step: tensor %d: %d x %d: sides outside [1, %d], or the smaller above %d", i,
                     t.rows, t.cols, FOREMOE_MUON_SIDE, FOREMOE_MUON_RANK);
  if (scale_tiles(t) > kMuonMostTiles)
    return set_error(FOREMOE_EUNSUPPORTED, "muon_step: tensor %d: more than 2^35 elements, padding included", i);
  return FOREMOE_OK;
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

// The grid of a launch with count(record) workgroups to a matrix.
template <class Count>
static unsigned grid_of(MuonArgs& a, Count count) {
  uint64_t n = 0;
  for (int i = 0; i < a.n_rec; ++i) {
    a.first.at[i] = (uint32_t)n;
    n += (uint64_t)a.rec[i].batch * count(a.rec[i]);
  }
  a.n_work = (uint32_t)n;
  return (unsigned)n;
}

static void launch_small(MuonArgs& a, const Stages& stages, bool pb16, bool gb16, hipStream_t st) {
  const int steps = a.steps;
  for (int k = 0; k < stages.n; ++k) {
    a.steps = stages.steps[k], a.from_u = k == 0, a.to_params = k + 1 == stages.n;
    unsigned n = grid_of(a, [](const MuonRec& r) { return (uint64_t)r.chunks; });
    if (gb16) hipLaunchKernelGGL((muon_small_gram_kernel<true>), dim3(n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((muon_small_gram_kernel<false>), dim3(n), dim3(256), 0, st, a);
    n = grid_of(a, [](const MuonRec&) { return (uint64_t)1; });
    hipLaunchKernelGGL(muon_small_steps_kernel, dim3(n), dim3(kSmallThreads), 0, st, a);
    n = grid_of(a, [](const MuonRec& r) { return (uint64_t)((r.rows > r.cols ? r.rows : r.cols) + 63) / 64; });
    if (gb16 && pb16) hipLaunchKernelGGL((muon_small_apply_kernel<true, true>), dim3(n), dim3(256), 0, st, a);
    else if (gb16) hipLaunchKernelGGL((muon_small_apply_kernel<true, false>), dim3(n), dim3(256), 0, st, a);
    else if (pb16) hipLaunchKernelGGL((muon_small_apply_kernel<false, true>), dim3(n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((muon_small_apply_kernel<false, false>), dim3(n), dim3(256), 0, st, a);
  }
  a.steps = steps;
}

// (a grid of a multiple of the XCDs: see xcd_virtual_id)
template <int P, bool PBF16>
static void launch_product(MuonArgs& a, int tile, hipStream_t st) {
  const uint64_t T = tile;
  const unsigned n = grid_of(a, [T](const MuonRec& r) {
    const uint64_t tm = r.mm / T;
    return P == kGram || P == kPoly ? tm * (tm + 1) / 2 : tm * (r.nn / T);
  });
  const dim3 grid((n + 7) / 8 * 8), threads(tile * 2);
  if (tile == 256) hipLaunchKernelGGL((muon_product_kernel<P, PBF16, 256>), grid, threads, 0, st, a);
  else hipLaunchKernelGGL((muon_product_kernel<P, PBF16, 128>), grid, threads, 0, st, a);
}

static void launch_large(MuonArgs& a, const Tiles& tiles, bool pb16, bool gb16, hipStream_t st) {
  unsigned n = grid_of(a, [](const MuonRec& r) { return (uint64_t)r.chunks; });
  if (gb16) hipLaunchKernelGGL((muon_moment_kernel<true>), dim3(n), dim3(kMomentThreads), 0, st, a);
  else hipLaunchKernelGGL((muon_moment_kernel<false>), dim3(n), dim3(kMomentThreads), 0, st, a);
  n = grid_of(a, [](const MuonRec& r) { return (uint64_t)(r.mm / 64) * (r.nn / 64); });
  if (gb16) hipLaunchKernelGGL((muon_scale_kernel<true>), dim3(n), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((muon_scale_kernel<false>), dim3(n), dim3(256), 0, st, a);
  if (a.steps == 0) {
    if (pb16) hipLaunchKernelGGL((muon_update_kernel<true>), dim3(n), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((muon_update_kernel<false>), dim3(n), dim3(256), 0, st, a);
  }
  a.from = 0;
  for (int step = 0; step < a.steps; ++step) {
    // the X before the last step has no second numbers: one more step
    // multiplies what that leaves out by a at most
    a.has_rest = step == 0 || step + 1 < a.steps, a.put_rest = step + 2 < a.steps;
    launch_product<kGram, false>(a, tiles.sym, st);
    launch_product<kPoly, false>(a, tiles.sym, st);
    if (step + 1 < a.steps) launch_product<kApply, false>(a, tiles.full, st);
    else if (pb16) launch_product<kUpdate, true>(a, tiles.full, st);
    else launch_product<kUpdate, false>(a, tiles.full, st);
    a.from ^= 1;
  }
}

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

extern "C" {

size_t foremoe_muon_workspace_size(const foremoe_muon_tensor* tensors, int32_t n_tensors) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return 0;
  for (int i = 0; i < n_tensors; ++i)
    if (check_tensor(tensors[i], i) != FOREMOE_OK) return 0;
  size_t most = 256;
  for (int i = 0, end; i < n_tensors; i = end) {
    end = group_end(tensors, i, n_tensors);
    const int pad = choose_tiles(tensors, i, end).pad;
    size_t at = 0;
    for (int j = i; j < end; ++j)
      if (tensors[j].batch) at = lay_out(tensors[j], pad, at, nullptr, nullptr);
    most = at > most ? at : most;
  }
  return most;
}

int foremoe_muon_step(const foremoe_muon_tensor* tensors, int32_t n_tensors, foremoe_dtype param_dtype,
                      foremoe_dtype grad_dtype, double lr, double momentum, int32_t nesterov, int32_t ns_steps,
                      const double* coef, double eps, const float* grad_scale, int32_t zero_grads, void* ws,
                      size_t ws_bytes, void* stream) {
  REQUIRE(param_dtype == FOREMOE_BF16 || param_dtype == FOREMOE_F32, "muon_step: bad parameter dtype");
  REQUIRE(grad_dtype == FOREMOE_BF16 || grad_dtype == FOREMOE_F32, "muon_step: bad gradient dtype");
  REQUIRE(n_tensors >= 0 && (tensors || n_tensors == 0), "muon_step: n_tensors < 0 or tensors NULL");
  REQUIRE(isfinite(lr) && lr >= 0, "muon_step: lr must be finite and not negative");
  REQUIRE(momentum >= 0 && momentum < 1, "muon_step: momentum outside [0, 1)");
  REQUIRE(ns_steps >= 0 && ns_steps <= 16, "muon_step: ns_steps=%d outside [0, 16]", ns_steps);
  REQUIRE(coef && isfinite(coef[0]) && isfinite(coef[1]) && isfinite(coef[2]), "muon_step: coef NULL or not finite");
  REQUIRE(isfinite(eps) && eps >= 0, "muon_step: eps must be finite and not negative");
  REQUIRE(!misaligned(grad_scale, 4), "muon_step: grad_scale misaligned");
  const uintptr_t pb = param_dtype == FOREMOE_BF16 ? 2 : 4, gb = grad_dtype == FOREMOE_BF16 ? 2 : 4;
  bool some = false, large = false;
  for (int i = 0; i < n_tensors; ++i) {
    const foremoe_muon_tensor& t = tensors[i];
    const int rc = check_tensor(t, i);
    if (rc != FOREMOE_OK) return rc;
    if (t.batch == 0) continue;
    some = true, large = large || !is_small(t);
    REQUIRE(t.param && t.grad && t.m, "muon_step: tensor %d: NULL pointer", i);
    REQUIRE(!t.master || param_dtype == FOREMOE_BF16, "muon_step: tensor %d: a master goes with bf16 parameters", i);
    REQUIRE(isfinite(t.weight_decay) && isfinite(t.scale), "muon_step: tensor %d: weight decay or scale is not finite",
            i);
    REQUIRE(!misaligned(t.param, pb) && !misaligned(t.grad, gb) && !misaligned(t.master, 4) && !misaligned(t.m, 4),
            "muon_step: tensor %d: misaligned pointer", i);
  }
  if (!some) return FOREMOE_OK;
  if (large && !within_half(coef, ns_steps))
    return set_error(FOREMOE_EUNSUPPORTED,
                     "muon_step: %d steps of coef (%g, %g, %g) may pass %g on the way, which matrices with both sides "
                     "above %d cannot hold",
                     ns_steps, coef[0], coef[1], coef[2], kHalfMost, kSmall);
  REQUIRE(ws, "muon_step: workspace NULL");
  const size_t need = foremoe_muon_workspace_size(tensors, n_tensors);
  REQUIRE(ws_bytes >= need, "muon_step: workspace too small (%zu < %zu bytes)", ws_bytes, need);
  REQUIRE(!misaligned(ws, 256), "muon_step: workspace misaligned");

  MuonArgs a{};
  a.nesterov = nesterov != 0, a.zero_grads = zero_grads != 0, a.grad_scale = grad_scale, a.steps = ns_steps;
  a.momentum = (float)momentum, a.a = (float)coef[0], a.b = (float)coef[1], a.c = (float)coef[2], a.eps = eps;
  for (int i = 0; i < 3; ++i) a.coef[i] = coef[i];
  const Stages stages = small_stages(coef, ns_steps);
  const bool pb16 = param_dtype == FOREMOE_BF16, gb16 = grad_dtype == FOREMOE_BF16;
  hipStream_t st = (hipStream_t)stream;
  int rc = FOREMOE_OK;
  for (int i = 0, end; i < n_tensors && rc == FOREMOE_OK; i = end) {
    end = group_end(tensors, i, n_tensors);
    const Tiles tiles = choose_tiles(tensors, i, end);
    size_t at = 0;
    for (int small = 1; small >= 0; --small) {
      a.n_rec = 0;
      for (int j = i; j < end; ++j) {
        const foremoe_muon_tensor& t = tensors[j];
        if (t.batch == 0 || is_small(t) != (small != 0)) continue;
        MuonRec& r = a.rec[a.n_rec++];
        at = lay_out(t, tiles.pad, at, (char*)ws, &r);
        r.param = t.param, r.grad = t.grad, r.master = t.master, r.m = t.m;
        r.batch = t.batch, r.rows = t.rows, r.cols = t.cols;
        r.wide = t.cols % 4 == 0 && !misaligned(t.param, 16) && !misaligned(t.grad, 16) && !misaligned(t.master, 16) &&
                 !misaligned(t.m, 16);
        r.decay = (float)(1 - lr * t.weight_decay), r.move = (float)(lr * t.scale);
      }
      if (a.n_rec == 0) continue;
      if (small) launch_small(a, stages, pb16, gb16, st);
      else launch_large(a, tiles, pb16, gb16, st);
      rc = check_launch("muon_step");
      if (rc != FOREMOE_OK) break;
    }
  }
  return rc;
}

}  // extern "C"
