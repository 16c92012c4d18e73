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
// are rounded to 2^-12 of themselves, and directions that u does not have stay
// at the size that fp32 leaves there: P X alone would fill them with the
// rounding of X, which each of the first steps multiplies by a.
// X, G and P are held 2^8 times as large, which keeps entries of large, even
// matrices (1/sqrt(m n) and less) above fp16's subnormal numbers.
#include <math.h>

#include "common.h"
#include "mfma_tiles.h"

namespace foremoe {
namespace {

constexpr int kMuonTile = 128, kMuonBK = 64, kMuonNS = 2, kMuonWaves = 4;
constexpr int kMomentThreads = 256, kMomentChunk = 16384;  // elements of a matrix per workgroup
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
  float decay, move;       // 1 - lr weight_decay, lr scale
  uint16_t *x[2], *rest[2];  // [batch, mm, nn]
  uint16_t *gram, *poly;     // [batch, mm, mm]
  double* squares;           // [batch, chunks]
  // first workgroup of the record in each kind of launch
  uint32_t at_moment, at_scale, at_sym, at_full;
};

struct MuonArgs {
  MuonRec rec[FOREMOE_MUON_LAUNCH];
  int n_rec, nesterov, zero_grads, from;  // from: which X the launch reads
  float momentum, a, b, c;
  double eps;
  const float* grad_scale;
};
static_assert(sizeof(MuonArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ uint16_t half_bits(float v) { return __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ __forceinline__ float half_value(uint32_t b) { return (float)__builtin_bit_cast(_Float16, (uint16_t)b); }

template <class At>
__device__ __forceinline__ int find_rec(const MuonArgs& a, At at) {
  int r = 0;
  for (int i = 1; i < a.n_rec; ++i)
    if (at(a.rec[i]) <= blockIdx.x) r = i;
  return r;
}

template <bool BF16_IN>
__device__ __forceinline__ float element(const void* p, int64_t i) {
  if constexpr (BF16_IN) return bf2f(((const uint16_t*)p)[i]);
  else return ((const float*)p)[i];
}

// m and the squares of u, a workgroup to a chunk of a matrix.
template <bool GBF16>
__global__ __launch_bounds__(kMomentThreads) void muon_moment_kernel(MuonArgs a) {
  const MuonRec& r = a.rec[find_rec(a, [](const MuonRec& q) { return q.at_moment; })];
  const uint32_t b = blockIdx.x - r.at_moment;
  const int64_t matrix = b / r.chunks, chunk = b % r.chunks;
  const int64_t n = (int64_t)r.rows * r.cols, base = matrix * n;
  const int64_t lo = chunk * kMomentChunk, hi = lo + kMomentChunk < n ? lo + kMomentChunk : n;
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  double s = 0;
  for (int64_t i = lo + threadIdx.x; i < hi; i += kMomentThreads) {
    const float g = element<GBF16>(r.grad, base + i) * gs;
    const float m = fmaf(a.momentum, r.m[base + i], g);
    r.m[base + i] = m;
    const float u = a.nesterov ? fmaf(a.momentum, m, g) : m;
    s += (double)u * u;
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
  const MuonRec& r = a.rec[find_rec(a, [](const MuonRec& q) { return q.at_scale; })];
  const uint32_t b = blockIdx.x - r.at_scale;
  const uint32_t tn = r.nn / 64, tiles = (uint32_t)(r.mm / 64) * tn;
  const int64_t matrix = b / tiles;
  const int i0 = (int)(b % tiles / tn) * 64, j0 = (int)(b % tiles % tn) * 64;
  const bool tall = r.rows > r.cols;
  const int tid = threadIdx.x;
  // the matrix's norm, summed in the same order by every workgroup
  __shared__ double part[256];
  __shared__ float tile[64][65];
  double s = 0;
  for (uint32_t i = tid; i < r.chunks; i += 256) s += r.squares[matrix * r.chunks + i];
  part[tid] = s;
  __syncthreads();
  for (int o = 128; o; o >>= 1) {
    if (tid < o) part[tid] += part[tid + o];
    __syncthreads();
  }
  const double norm = sqrt(part[0]);
  const double den = !(norm <= a.eps) ? norm : a.eps;
  // nothing in it: no move; not finite: NaN everywhere
  const double inv = den == 0 ? 0.0 : (isinf(den) ? (double)NAN : 1.0 / den);
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  // read along the source's rows
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  for (int e = tid; e < 4096; e += 256) {
    const int rr = r0 + (e >> 6), cc = c0 + (e & 63);
    float v = 0.0f;
    if (rr < r.rows && cc < r.cols) {
      const int64_t i = base + (int64_t)rr * r.cols + cc;
      float u = r.m[i];
      if (a.nesterov) u = fmaf(a.momentum, u, element<GBF16>(r.grad, i) * gs);
      if (a.zero_grads) {
        if constexpr (GBF16) ((uint16_t*)r.grad)[i] = 0;
        else ((float*)r.grad)[i] = 0.0f;
      }
      v = (float)((double)u * inv) * kHeld;
    }
    tile[e >> 6][e & 63] = v;
  }
  __syncthreads();
  const int64_t at = matrix * (int64_t)r.mm * r.nn;
  for (int e = tid; e < 4096; e += 256) {
    const int i = e >> 6, j = e & 63;
    const float v = tall ? tile[j][i] : tile[i][j];
    const uint16_t h = half_bits(v);
    const int64_t o = at + (int64_t)(i0 + i) * r.nn + j0 + j;
    r.x[0][o] = h;
    r.rest[0][o] = half_bits((v - half_value(h)) * kRest);
  }
}

enum Product { kGram = 0, kPoly = 1, kApply = 2 };

// One 128 x 128 tile of one matrix's product.
template <Product P>
__global__ __launch_bounds__(64 * kMuonWaves) void muon_product_kernel(MuonArgs a) {
  constexpr int T = kMuonTile, BK = kMuonBK, NS = kMuonNS, NW = kMuonWaves;
  constexpr bool SYM = P != kApply;
  using CoreT = Core<T, T, 2, 2, false, Fp16>;
  using AT = KTile<T, BK, NW>;
  using BT = typename std::conditional<SYM, KTile<T, BK, NW>, MTile<T, BK, NW>>::type;
  constexpr int STAGE = AT::BYTES + BT::BYTES;
  __shared__ __attribute__((aligned(1024))) char lds[NS * STAGE];
  const MuonRec& r = a.rec[find_rec(a, [](const MuonRec& q) { return SYM ? q.at_sym : q.at_full; })];
  const uint32_t b = blockIdx.x - (SYM ? r.at_sym : r.at_full);
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
  const uint16_t* X = r.x[a.from] + matrix * (int64_t)r.mm * r.nn;
  const uint16_t* G = r.gram + matrix * (int64_t)r.mm * r.mm;
  uint16_t* Q = r.poly + matrix * (int64_t)r.mm * r.mm;
  const int lda = P == kGram ? r.nn : r.mm, ldb = P == kPoly ? r.mm : r.nn;
  const int KT = (P == kGram ? r.nn : r.mm) / BK;
  const uint16_t* abase = (P == kGram ? X : P == kPoly ? G : Q) + (int64_t)i0 * lda;
  const uint16_t* bbase = P == kApply ? X + j0 : (P == kGram ? X : G) + (int64_t)j0 * ldb;
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
  CoreT core;
  const typename CoreT::template Offsets<AT, BT, BK> offs(lane, wm, wn);
  core.zero();
  pipelined_k_loop<CoreT, AT, BT, BK, NS, 1>(core, lds, KT, offs, issue, false, [] {});

  const int64_t xat = matrix * (int64_t)r.mm * r.nn;
#pragma unroll
  for (int i = 0; i < CoreT::MB; ++i)
#pragma unroll
    for (int j = 0; j < CoreT::NB; ++j) {
      const int row = i0 + wm * 64 + 32 * i + (lane & 31);
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        const int col = j0 + wn * 64 + 32 * j + 8 * q4 + 4 * (lane >> 5);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = core.acc[i][j][4 * q4 + e] * (1.0f / kHeld);
        if constexpr (P == kApply) {
          const int64_t o = xat + (int64_t)row * r.nn + col;
          const uint2 h = *(const uint2*)(r.x[a.from] + o), l = *(const uint2*)(r.rest[a.from] + o);
          const uint32_t hw[2] = {h.x, h.y}, lw[2] = {l.x, l.y};
          uint32_t nh[2] = {0, 0}, nl[2] = {0, 0};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int s = 16 * (e & 1);
            const float old = half_value(hw[e / 2] >> s & 0xffffu) + half_value(lw[e / 2] >> s & 0xffffu) * (1.0f / kRest);
            const float x = fmaf(a.a, old, v[e]);
            const uint32_t hb = half_bits(x);
            nh[e / 2] |= hb << s;
            nl[e / 2] |= (uint32_t)half_bits((x - half_value(hb)) * kRest) << s;
          }
          *(uint2*)(r.x[a.from ^ 1] + o) = uint2{nh[0], nh[1]};
          *(uint2*)(r.rest[a.from ^ 1] + o) = uint2{nl[0], nl[1]};
        } else {
          uint16_t* out = P == kGram ? (uint16_t*)G : Q;
          if constexpr (P == kPoly) {
            const uint2 h = *(const uint2*)(G + (int64_t)row * r.mm + col);
            const uint32_t hw[2] = {h.x, h.y};
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fmaf(a.c, v[e], a.b * half_value(hw[e / 2] >> (16 * (e & 1)) & 0xffffu));
          }
          uint16_t hb[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) hb[e] = half_bits(v[e]);
          *(uint2*)(out + (int64_t)row * r.mm + col) =
              uint2{(uint32_t)hb[0] | (uint32_t)hb[1] << 16, (uint32_t)hb[2] | (uint32_t)hb[3] << 16};
          if (ti != tj) {
#pragma unroll
            for (int e = 0; e < 4; ++e) out[(int64_t)(col + e) * r.mm + row] = hb[e];
          }
        }
      }
    }
}

// p = p (1 - lr weight_decay) - lr scale X, 64 x 64 of X to a workgroup.
template <bool PBF16>
__global__ __launch_bounds__(256) void muon_update_kernel(MuonArgs a) {
  const MuonRec& r = a.rec[find_rec(a, [](const MuonRec& q) { return q.at_scale; })];
  const uint32_t b = blockIdx.x - r.at_scale;
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
    const float x = (half_value(r.x[a.from][o]) + half_value(r.rest[a.from][o]) * (1.0f / kRest)) * (1.0f / kHeld);
    if (tall) tile[j][i] = x;
    else tile[i][j] = x;
  }
  __syncthreads();
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0;
  const int64_t base = matrix * (int64_t)r.rows * r.cols;
  for (int e = tid; e < 4096; e += 256) {
    const int rr = r0 + (e >> 6), cc = c0 + (e & 63);
    if (rr >= r.rows || cc >= r.cols) continue;
    const int64_t o = base + (int64_t)rr * r.cols + cc;
    const float old = PBF16 && !r.master ? bf2f(((const uint16_t*)r.param)[o])
                                         : (r.master ? r.master[o] : ((const float*)r.param)[o]);
    const float p = fmaf(-r.move, tile[e >> 6][e & 63], old * r.decay);
    if (r.master) r.master[o] = p;
    if constexpr (PBF16) ((uint16_t*)r.param)[o] = (uint16_t)pack_bf2(p, 0.0f);
    else ((float*)r.param)[o] = p;
  }
}

int64_t pad_side(int64_t n) { return (n + kMuonTile - 1) / kMuonTile * kMuonTile; }

// Lays a tensor's part of the workspace out from `at` (bytes); returns its end.
size_t lay_out(const foremoe_muon_tensor& t, size_t at, char* ws, MuonRec* r) {
  const int64_t s = t.rows < t.cols ? t.rows : t.cols, l = t.rows < t.cols ? t.cols : t.rows;
  const int64_t mm = pad_side(s), nn = pad_side(l);
  const int64_t chunks = (s * l + kMomentChunk - 1) / kMomentChunk;
  auto take = [&](size_t bytes) {
    char* p = ws + at;
    at = align_up(at + bytes, 256);
    return p;
  };
  MuonRec q{};
  for (int i = 0; i < 2; ++i) {
    q.x[i] = (uint16_t*)take((size_t)t.batch * mm * nn * 2);
    q.rest[i] = (uint16_t*)take((size_t)t.batch * mm * nn * 2);
  }
  q.gram = (uint16_t*)take((size_t)t.batch * mm * mm * 2);
  q.poly = (uint16_t*)take((size_t)t.batch * mm * mm * 2);
  q.squares = (double*)take((size_t)t.batch * chunks * 8);
  q.mm = (int)mm, q.nn = (int)nn, q.chunks = (uint32_t)chunks;
  if (r) *r = q;
  return at;
}

// 64 x 64 tiles of a tensor: no launch over it has more workgroups.
constexpr int64_t kMuonMostTiles = (int64_t)1 << 23;
int64_t scale_tiles(const foremoe_muon_tensor& t) {
  return t.batch * (pad_side(t.rows) / 64) * (pad_side(t.cols) / 64);
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

// Whether a tensor starts another launch behind n others of `tiles` tiles.
bool starts_launch(const foremoe_muon_tensor& t, int n, int64_t tiles) {
  return n == FOREMOE_MUON_LAUNCH || (n > 0 && tiles + scale_tiles(t) > kMuonMostTiles);
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

extern "C" {

size_t foremoe_muon_workspace_size(const foremoe_muon_tensor* tensors, int32_t n_tensors) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors)) return 0;
  size_t most = 256, at = 0;
  int64_t tiles = 0;
  int n = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (check_tensor(tensors[i], i) != FOREMOE_OK) return 0;
    if (tensors[i].batch == 0) continue;
    if (starts_launch(tensors[i], n, tiles)) n = 0, at = 0, tiles = 0;
    at = lay_out(tensors[i], at, nullptr, nullptr);
    most = at > most ? at : most;
    tiles += scale_tiles(tensors[i]);
    ++n;
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
  bool some = false;
  for (int i = 0; i < n_tensors; ++i) {
    const foremoe_muon_tensor& t = tensors[i];
    const int rc = check_tensor(t, i);
    if (rc != FOREMOE_OK) return rc;
    if (t.batch == 0) continue;
    some = true;
    REQUIRE(t.param && t.grad && t.m, "muon_step: tensor %d: NULL pointer", i);
    REQUIRE(!t.master || param_dtype == FOREMOE_BF16, "muon_step: tensor %d: a master goes with bf16 parameters", i);
    REQUIRE(isfinite(t.weight_decay) && isfinite(t.scale), "muon_step: tensor %d: weight decay or scale is not finite",
            i);
    REQUIRE(!misaligned(t.param, pb) && !misaligned(t.grad, gb) && !misaligned(t.master, 4) && !misaligned(t.m, 4),
            "muon_step: tensor %d: misaligned pointer", i);
  }
  if (!some) return FOREMOE_OK;
  REQUIRE(ws, "muon_step: workspace NULL");
  const size_t need = foremoe_muon_workspace_size(tensors, n_tensors);
  REQUIRE(ws_bytes >= need, "muon_step: workspace too small (%zu < %zu bytes)", ws_bytes, need);
  REQUIRE(!misaligned(ws, 256), "muon_step: workspace misaligned");

  MuonArgs a{};
  a.nesterov = nesterov != 0, a.zero_grads = zero_grads != 0, a.grad_scale = grad_scale;
  a.momentum = (float)momentum, a.a = (float)coef[0], a.b = (float)coef[1], a.c = (float)coef[2], a.eps = eps;
  hipStream_t st = (hipStream_t)stream;
  uint64_t moment = 0, scale = 0, sym = 0, full = 0;
  size_t at = 0;
  int rc = FOREMOE_OK;
  auto flush = [&] {
    if (!a.n_rec || rc != FOREMOE_OK) return;
    a.from = 0;
    const dim3 gm((unsigned)moment), gsc((unsigned)scale), gsy((unsigned)sym), gf((unsigned)full), pt(64 * kMuonWaves);
    if (grad_dtype == FOREMOE_BF16) {
      hipLaunchKernelGGL((muon_moment_kernel<true>), gm, dim3(kMomentThreads), 0, st, a);
      hipLaunchKernelGGL((muon_scale_kernel<true>), gsc, dim3(256), 0, st, a);
    } else {
      hipLaunchKernelGGL((muon_moment_kernel<false>), gm, dim3(kMomentThreads), 0, st, a);
      hipLaunchKernelGGL((muon_scale_kernel<false>), gsc, dim3(256), 0, st, a);
    }
    for (int i = 0; i < ns_steps; ++i) {
      hipLaunchKernelGGL((muon_product_kernel<kGram>), gsy, pt, 0, st, a);
      hipLaunchKernelGGL((muon_product_kernel<kPoly>), gsy, pt, 0, st, a);
      hipLaunchKernelGGL((muon_product_kernel<kApply>), gf, pt, 0, st, a);
      a.from ^= 1;
    }
    if (param_dtype == FOREMOE_BF16) hipLaunchKernelGGL((muon_update_kernel<true>), gsc, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((muon_update_kernel<false>), gsc, dim3(256), 0, st, a);
    rc = check_launch("muon_step");
    a.n_rec = 0, at = 0, moment = scale = sym = full = 0;
  };
  for (int i = 0; i < n_tensors; ++i) {
    const foremoe_muon_tensor& t = tensors[i];
    if (t.batch == 0) continue;
    if (starts_launch(t, a.n_rec, (int64_t)scale)) flush();
    MuonRec& r = a.rec[a.n_rec++];
    at = lay_out(t, at, (char*)ws, &r);
    r.param = t.param, r.grad = t.grad, r.master = t.master, r.m = t.m;
    r.batch = t.batch, r.rows = t.rows, r.cols = t.cols;
    r.decay = (float)(1 - lr * t.weight_decay), r.move = (float)(lr * t.scale);
    const uint64_t tm = r.mm / kMuonTile, tn = r.nn / kMuonTile;
    r.at_moment = (uint32_t)moment, r.at_scale = (uint32_t)scale, r.at_sym = (uint32_t)sym, r.at_full = (uint32_t)full;
    moment += (uint64_t)t.batch * r.chunks, scale += (uint64_t)t.batch * tm * tn * 4;
    sym += (uint64_t)t.batch * (tm * (tm + 1) / 2), full += (uint64_t)t.batch * tm * tn;
  }
  flush();
  return rc;
}

}  // extern "C"
