// Microscaled 4-bit floats: quantisation of rows, the values that codes stand
// for, and the grouped SwiGLU expert FFN (forward) with operands in 4 bits.
#include "common.h"
#include "mfma_tiles.h"
#include "mx.h"

namespace foremoe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// Quantisation. Four lanes share a block, eight elements each: HBM-bound.
// ---------------------------------------------------------------------------
constexpr int kQuantThreads = 256;

struct QuantArgs {
  const void* x;
  int64_t ld;
  int64_t rows;
  uint32_t cols, per_row;  // per_row: groups of eight in a row, the last block's padding included
  const int32_t* n_rows;
  uint8_t* codes;
  uint8_t* scales;
};

template <bool BF16_IN, bool VEC>
__device__ __forceinline__ void load8(const void* x, int64_t at, int64_t left, float* v) {
  if constexpr (BF16_IN) {
    const uint16_t* p = (const uint16_t*)x + at;
    if (VEC && left >= 8) {
      const uint4 w = *(const uint4*)p;
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) v[2 * i] = bf2f(u[i] & 0xffffu), v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? bf2f(p[i]) : 0.0f;
    }
  } else {
    const float* p = (const float*)x + at;
    if (VEC && left >= 8) {
      const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.0f;
    }
  }
}

template <bool BF16_IN, bool VEC>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(QuantArgs a) {
  const int64_t rows = a.n_rows ? (*a.n_rows < a.rows ? *a.n_rows : a.rows) : a.rows;
  // the four lanes of a block take part in its maximum together: units are
  // whole blocks, and a lane past the end has no other lane of its block before it
  const int64_t n = rows * a.per_row;
  for (int64_t u = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x; u < n; u += (int64_t)gridDim.x * kQuantThreads) {
    const int64_t row = u / a.per_row;
    const uint32_t c = (uint32_t)(u - row * a.per_row) * 8;
    float v[8];
    load8<BF16_IN, VEC>(a.x, row * a.ld + c, (int64_t)a.cols - c, v);
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
      most = b > most ? b : most;
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const uint32_t other = __shfl_xor(most, o, 64);
      most = other > most ? other : most;
    }
    const uint32_t s = mx_scale_of(most);
    const float inv = mx_inverse(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= inv;
    ((uint32_t*)a.codes)[u] = s == 255 ? 0u : mx_put8(v);
    if ((u & 3) == 0) a.scales[u >> 2] = (uint8_t)s;
  }
}

template <bool BF16_OUT, bool VEC>
__global__ __launch_bounds__(kQuantThreads) void values_kernel(QuantArgs a, void* out) {
  const int64_t n = a.rows * a.per_row;
  for (int64_t u = (int64_t)blockIdx.x * kQuantThreads + threadIdx.x; u < n; u += (int64_t)gridDim.x * kQuantThreads) {
    const int64_t row = u / a.per_row;
    const uint32_t c = (uint32_t)(u - row * a.per_row) * 8;
    const uint32_t w = ((const uint32_t*)a.codes)[u];
    const float s = mx_scale_operand(a.scales[u >> 2]);
    const int64_t at = row * a.ld + c, left = (int64_t)a.cols - c;
    if constexpr (BF16_OUT) {
      const uint4 v = {mx_get2_bf16<0>(w, s), mx_get2_bf16<1>(w, s), mx_get2_bf16<2>(w, s), mx_get2_bf16<3>(w, s)};
      uint16_t* p = (uint16_t*)out + at;
      if (VEC && left >= 8) {
        *(uint4*)p = v;
      } else {
        const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) p[i] = (uint16_t)(q[i / 2] >> (16 * (i & 1)));
      }
    } else {
      const f32x2_t q[4] = {mx_get2<0>(w, s), mx_get2<1>(w, s), mx_get2<2>(w, s), mx_get2<3>(w, s)};
      float* p = (float*)out + at;
      if (VEC && left >= 8) {
        *(float4*)p = float4{q[0].x, q[0].y, q[1].x, q[1].y};
        *(float4*)(p + 4) = float4{q[2].x, q[2].y, q[3].x, q[3].y};
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < left) p[i] = i & 1 ? q[i / 2].y : q[i / 2].x;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Grouped FFN. Both products are C = A W^T over the rows of a slot with codes
// as operands of v_mfma_scale_f32_32x32x64_f8f6f4: a lane of a fragment holds
// one block of 32 codes, and its scale. A tile is BM rows of a slot by BN rows
// of a weight matrix; a stage is 128 of the k axis.
// ---------------------------------------------------------------------------
struct Ffn4Args {
  const uint8_t *a_codes, *a_scales;  // [n_cap, K / 2], [n_cap, K / 32]
  const uint8_t *b_codes, *b_scales;  // [W, N, K / 2], [W, N, K / 32]
  int K, N;
  int F;               // gate/up: N = 2F
  uint16_t* y;         // down: [n_cap, N] bf16
  uint8_t *h_codes, *h_scales;  // gate/up: [n_cap, F / 2], [n_cap, F / 32]
  const int32_t* slot_offset;
  const int32_t* slot_widx;
  int S, W, n_tiles;   // n_tiles: tiles along N
  int64_t n_cap;
};

struct SlotTile {
  int64_t row0, end;  // rows of the tile: [row0, min(row0 + BM, end))
  int w;
};

// The slot and rows of row tile t (tiles numbered slot by slot), found by
// every wavefront alone. False past the last.
template <int BM>
__device__ __forceinline__ bool find_row_tile(const Ffn4Args& a, int t, SlotTile& r) {
  const int lane = lane64();
  for (int j0 = 0; j0 < a.S; j0 += 64) {
    const int j = j0 + lane;
    int64_t beg = 0, end = 0;
    if (j < a.S) {
      beg = a.slot_offset[j], end = a.slot_offset[j + 1];
      beg = beg < 0 ? 0 : (beg > a.n_cap ? a.n_cap : beg);
      end = end > a.n_cap ? a.n_cap : end;
    }
    const int mine = end > beg ? (int)((end - beg + BM - 1) / BM) : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o, 64);
      if (lane >= o) upto += v;
    }
    const uint64_t hit = __ballot(upto > t);
    if (hit) {
      const int who = __builtin_ctzll(hit);
      const int before = __shfl(upto - mine, who, 64);
      const int b = __shfl((int)beg, who, 64), e = __shfl((int)end, who, 64);
      r.row0 = __builtin_amdgcn_readfirstlane(b + (t - before) * BM);
      r.end = __builtin_amdgcn_readfirstlane(e);
      r.w = __builtin_amdgcn_readfirstlane(a.slot_widx[j0 + who]);
      return true;
    }
    t -= __shfl(upto, 63, 64);
  }
  return false;
}

// One wavefront moves 64 x 4 bytes: lane l's word lands at lds_wave_base + 4 l.
__device__ __forceinline__ void dma4(i32x4 rs, uint32_t lds_wave_base, uint32_t voff) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds_wave_base);
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(m0v), "v"(voff), "s"(rs) : "memory");
}

constexpr int kMxM = 128, kMxN = 256, kMxStages = 3, kMxWaves = 4;

template <bool GATE_UP>
__global__ __launch_bounds__(64 * kMxWaves, 2) void ffn4_kernel(Ffn4Args a) {
  constexpr int BM = kMxM, BN = kMxN, NS = kMxStages, NW = kMxWaves;
  // 128 codes are 64 bytes: the geometry of a tile of 32 16-bit elements
  using AT = KTile<BM, 32, NW>;
  using BT = KTile<BN, 32, NW>;
  constexpr int SCALES = (BM + BN) * 4;  // a word (four blocks) per row
  constexpr int STAGE = AT::BYTES + BT::BYTES + SCALES;
  constexpr int NSC = (BM + BN) / 64;    // wavefront loads of scales
  constexpr int SC_PER_WAVE = (NSC + NW - 1) / NW;
  constexpr int PER = AT::PER_WAVE + BT::PER_WAVE + SC_PER_WAVE;
  constexpr int WM = 64, WN = 128, MB = WM / 32, NB = WN / 32;
  __shared__ __attribute__((aligned(1024))) char lds[NS * STAGE + 256];  // the last 256: loads of nothing

  SlotTile r;
  if (!find_row_tile<BM>(a, (int)(blockIdx.x / (unsigned)a.n_tiles), r)) return;
  if (r.w < 0 || r.w >= a.W) return;
  const int nt = blockIdx.x % (unsigned)a.n_tiles;
  const int lane = lane64(), wave = wave_id(), half = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t lds0 = lds_addr(lds);
  const uint32_t kb = (uint32_t)a.K / 2, ks = (uint32_t)a.K / 32;  // bytes of a row of codes, of scales
  const int KT = a.K / 128;

  const int64_t rows = r.end - r.row0 < BM ? r.end - r.row0 : BM;
  const uint8_t* abase = a.a_codes + r.row0 * (int64_t)kb;
  const uint8_t* asbase = a.a_scales + r.row0 * (int64_t)ks;
  const uint32_t abytes = (uint32_t)rows * kb, asbytes = (uint32_t)rows * ks;
  const uint8_t* bbase = a.b_codes + (int64_t)r.w * a.N * kb;
  const uint8_t* bsbase = a.b_scales + (int64_t)r.w * a.N * ks;
  const uint32_t bbytes = (uint32_t)a.N * kb, bsbytes = (uint32_t)a.N * ks;
  // row of the weight matrix that LDS row i of the tile holds
  const int n0 = GATE_UP ? nt * (BN / 2) : nt * BN;
  auto wrow = [&](int i) -> uint32_t {
    return (uint32_t)(GATE_UP ? (i < BN / 2 ? n0 + i : a.F + n0 + i - BN / 2) : n0 + i);
  };
  uint32_t va[AT::PER_WAVE], vb[BT::PER_WAVE], vs[SC_PER_WAVE];
#pragma unroll
  for (int i = 0; i < AT::PER_WAVE; ++i) va[i] = AT::voff(lane, [&](int q) { return (uint32_t)q * kb; }, i);
#pragma unroll
  for (int i = 0; i < BT::PER_WAVE; ++i) vb[i] = BT::voff(lane, [&](int q) { return wrow(q) * kb; }, i);
#pragma unroll
  for (int i = 0; i < SC_PER_WAVE; ++i) {
    const int q = (wave + NW * i) * 64 + lane;  // row of the A tile, then of the B tile
    vs[i] = q < BM ? (uint32_t)q * ks : wrow(q - BM) * ks;
  }
  auto issue = [&](int kt) {
    const bool live = kt < KT;
    const uint32_t at = lds0 + (uint32_t)((kt % NS) * STAGE);
    const uint32_t kc = live ? (uint32_t)kt * 64u : 0u, kw = live ? (uint32_t)kt * 4u : 0u;
    const i32x4 ra = buf_rsrc(abase + kc, live ? abytes - kc : 0u), rb = buf_rsrc(bbase + kc, live ? bbytes - kc : 0u);
#pragma unroll
    for (int i = 0; i < AT::PER_WAVE; ++i) AT::issue(ra, at, va[i], i);
#pragma unroll
    for (int i = 0; i < BT::PER_WAVE; ++i) BT::issue(rb, at + AT::BYTES, vb[i], i);
#pragma unroll
    for (int i = 0; i < SC_PER_WAVE; ++i) {
      const int q = wave + NW * i;
      const bool some = live && q < NSC, is_a = q * 64 < BM;
      dma4(buf_rsrc((is_a ? asbase : bsbase) + kw, some ? (is_a ? asbytes : bsbytes) - kw : 0u),
           q < NSC ? at + AT::BYTES + BT::BYTES + q * 256 : lds0 + NS * STAGE, vs[i]);
    }
  };

  f32x16 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  // LDS row that block j of this wavefront's columns starts at: with SwiGLU
  // the gate's columns, then the up's columns of the same outputs
  auto bcol = [&](int j) {
    return GATE_UP ? (j < NB / 2 ? wn * (WN / 2) + j * 32 : BN / 2 + wn * (WN / 2) + (j - NB / 2) * 32)
                   : wn * WN + j * 32;
  };
  uint32_t oa[MB], ob[NB], ka[2];
#pragma unroll
  for (int i = 0; i < MB; ++i) oa[i] = AT::lane_off(lane, wm * WM + i * 32);
#pragma unroll
  for (int j = 0; j < NB; ++j) ob[j] = AT::BYTES + BT::lane_off(lane, bcol(j));
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) ka[kk] = AT::kstep_off(lane, kk);

#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue(s);
  for (int kt = 0; kt < KT; ++kt) {
    wait_vm<(NS - 2) * PER>();  // stage kt has landed
    __syncthreads();            // for every wavefront, and stage kt - 1 has been read
    issue(kt + NS - 1);
    const char* st = lds + (kt % NS) * STAGE;
    const uint32_t* sc = (const uint32_t*)(st + AT::BYTES + BT::BYTES);
    uint32_t sa[MB], sb[NB];  // this lane's blocks are 2 kk + half: their bytes 2 kk after the shift
#pragma unroll
    for (int i = 0; i < MB; ++i) sa[i] = sc[wm * WM + i * 32 + (lane & 31)] >> (8 * half);
#pragma unroll
    for (int j = 0; j < NB; ++j) sb[j] = sc[BM + bcol(j) + (lane & 31)] >> (8 * half);
    static_for<0, 2>([&](auto kkc) {
      constexpr int kk = decltype(kkc)::value;
      i32x4 fa[MB], fb[NB];
#pragma unroll
      for (int i = 0; i < MB; ++i) fa[i] = *(const i32x4*)(st + oa[i] + ka[kk]);
#pragma unroll
      for (int j = 0; j < NB; ++j) fb[j] = *(const i32x4*)(st + ob[j] + ka[kk]);
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(
              __builtin_shufflevector(fb[j], fb[j], 0, 1, 2, 3, -1, -1, -1, -1),
              __builtin_shufflevector(fa[i], fa[i], 0, 1, 2, 3, -1, -1, -1, -1), acc[i][j], 4, 4, 2 * kk, sb[j], 2 * kk,
              sa[i]);
    });
  }
  wait_vm<0>();  // the loads of nothing, before the workgroup's LDS is another's

  // block (i, j), register q: row 32 i + lane % 32, column 32 j + 8 (q / 4) + 4 half + q % 4
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int64_t row = r.row0 + wm * WM + i * 32 + (lane & 31);
    const bool there = row < r.end;
    if constexpr (GATE_UP) {
      const int64_t hrow = row * (a.F / 32);
#pragma unroll
      for (int j = 0; j < NB / 2; ++j) {
        float g[16], h[16];
#pragma unroll
        for (int q = 0; q < 16; ++q) g[q] = acc[i][j][q];
        silu_n<16>(g, h);
        uint32_t most = 0;
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          h[q] *= acc[i][j + NB / 2][q];
          const uint32_t b = __float_as_uint(h[q]) & 0x7fffffffu;
          most = b > most ? b : most;
        }
        const uint32_t other = __shfl_xor(most, 32, 64);
        most = other > most ? other : most;
        const uint32_t s = mx_scale_of(most);
        const float inv = mx_inverse(s);
#pragma unroll
        for (int q = 0; q < 16; ++q) h[q] *= inv;
        // codes of the four columns of each group of eight that this lane
        // has; the other half's lane has the other four
        uint32_t c[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] = mx_put2<1>(mx_put2<0>(0u, h[4 * q], h[4 * q + 1]), h[4 * q + 2], h[4 * q + 3]);
        const int f = n0 + wn * (WN / 2) + j * 32;
        uint32_t word[2];  // of groups 0, 1 in the lower half's lanes, of 2, 3 in the upper's
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint32_t give = half ? c[q] : c[q + 2], keep = half ? c[q + 2] : c[q];
          const uint32_t got = __shfl_xor(give, 32, 64);
          word[q] = half ? (got & 0xffffu) | keep << 16 : (keep & 0xffffu) | got << 16;
        }
        if (there) {
          if (s == 255) word[0] = word[1] = 0;
          *(uint2*)(a.h_codes + row * (a.F / 2) + f / 2 + 8 * half) = uint2{word[0], word[1]};
          if (half == 0) a.h_scales[hrow + f / 32] = (uint8_t)s;
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int c = n0 + wn * WN + j * 32 + 4 * half;
        if (there && c < a.N) {  // N is a multiple of 128: a block is in or out
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *(uint2*)(a.y + row * a.N + c + 8 * q) = uint2{pack_bf2(acc[i][j][4 * q], acc[i][j][4 * q + 1]),
                                                           pack_bf2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3])};
        }
      }
    }
  }
}

}  // namespace
}  // namespace foremoe

using namespace foremoe;

#define REQUIRE(cond, ...)                                      \
  do {                                                          \
    if (!(cond)) return set_error(FOREMOE_EINVAL, __VA_ARGS__); \
  } while (0)

static bool misaligned(const void* p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) != 0; }

static unsigned quant_blocks(int64_t units) {
  const int64_t nb = (units + kQuantThreads - 1) / kQuantThreads;
  return (unsigned)(nb < (1 << 20) ? nb : 1 << 20);
}

extern "C" {

int foremoe_mxfp4_quantize(const void* x, foremoe_dtype dtype, int64_t ld, int64_t rows, int64_t cols,
                           const int32_t* n_rows, uint8_t* codes, uint8_t* scales, void* stream) {
  REQUIRE(dtype == FOREMOE_BF16 || dtype == FOREMOE_F32, "mxfp4_quantize: bad dtype");
  REQUIRE(rows >= 0 && rows < (int64_t)1 << 31, "mxfp4_quantize: rows=%lld outside [0, 2^31)", (long long)rows);
  REQUIRE(cols >= 1 && cols < (int64_t)1 << 31, "mxfp4_quantize: cols=%lld outside [1, 2^31)", (long long)cols);
  REQUIRE(ld >= cols && ld <= (int64_t)1 << 32, "mxfp4_quantize: ld=%lld below cols or above 2^32", (long long)ld);
  if (rows == 0) return FOREMOE_OK;
  REQUIRE(x && codes && scales, "mxfp4_quantize: NULL pointer");
  const uintptr_t b = dtype == FOREMOE_BF16 ? 2 : 4;
  REQUIRE(!misaligned(x, b) && !misaligned(codes, 16) && !misaligned(n_rows, 4), "mxfp4_quantize: misaligned pointer");
  QuantArgs a{};
  a.x = x, a.ld = ld, a.rows = rows, a.cols = (uint32_t)cols;
  a.per_row = (uint32_t)((cols + kMxBlock - 1) / kMxBlock * 4);
  a.n_rows = n_rows, a.codes = codes, a.scales = scales;
  const unsigned blocks = quant_blocks(rows * a.per_row);
  const bool vec = !misaligned(x, 16) && ld * (int64_t)b % 16 == 0;
  hipStream_t st = (hipStream_t)stream;
#define LAUNCH(BF, V) hipLaunchKernelGGL((quantize_kernel<BF, V>), dim3(blocks), dim3(kQuantThreads), 0, st, a)
  if (dtype == FOREMOE_BF16) {
    if (vec) LAUNCH(true, true);
    else LAUNCH(true, false);
  } else {
    if (vec) LAUNCH(false, true);
    else LAUNCH(false, false);
  }
#undef LAUNCH
  return check_launch("mxfp4_quantize");
}

int foremoe_mxfp4_values(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out,
                         foremoe_dtype dtype, int64_t ld, void* stream) {
  REQUIRE(dtype == FOREMOE_BF16 || dtype == FOREMOE_F32, "mxfp4_values: bad dtype");
  REQUIRE(rows >= 0 && rows < (int64_t)1 << 31, "mxfp4_values: rows=%lld outside [0, 2^31)", (long long)rows);
  REQUIRE(cols >= 1 && cols < (int64_t)1 << 31, "mxfp4_values: cols=%lld outside [1, 2^31)", (long long)cols);
  REQUIRE(ld >= cols && ld <= (int64_t)1 << 32, "mxfp4_values: ld=%lld below cols or above 2^32", (long long)ld);
  if (rows == 0) return FOREMOE_OK;
  REQUIRE(codes && scales && out, "mxfp4_values: NULL pointer");
  const uintptr_t b = dtype == FOREMOE_BF16 ? 2 : 4;
  REQUIRE(!misaligned(out, b) && !misaligned(codes, 16), "mxfp4_values: misaligned pointer");
  QuantArgs a{};
  a.ld = ld, a.rows = rows, a.cols = (uint32_t)cols;
  a.per_row = (uint32_t)((cols + kMxBlock - 1) / kMxBlock * 4);
  a.codes = (uint8_t*)codes, a.scales = (uint8_t*)scales;
  const unsigned blocks = quant_blocks(rows * a.per_row);
  const bool vec = !misaligned(out, 16) && ld * (int64_t)b % 16 == 0;
  hipStream_t st = (hipStream_t)stream;
#define LAUNCH(BF, V) hipLaunchKernelGGL((values_kernel<BF, V>), dim3(blocks), dim3(kQuantThreads), 0, st, a, out)
  if (dtype == FOREMOE_BF16) {
    if (vec) LAUNCH(true, true);
    else LAUNCH(true, false);
  } else {
    if (vec) LAUNCH(false, true);
    else LAUNCH(false, false);
  }
#undef LAUNCH
  return check_launch("mxfp4_values");
}

size_t foremoe_ffn_mxfp4_workspace_size(int64_t n_cap, int32_t F) {
  if (n_cap < 0 || n_cap >= (int64_t)1 << 31 || F < 1 || F % 128) return 0;
  const size_t codes = align_up((size_t)n_cap * (F / 2), 256), scales = align_up((size_t)n_cap * (F / 32), 256);
  return codes + scales + 256;
}

int foremoe_grouped_ffn_mxfp4_fwd(const uint8_t* x_codes, const uint8_t* x_scales, int32_t d, int32_t F, int32_t S,
                                  const int32_t* slot_offset, const int32_t* slot_widx, int32_t W,
                                  const uint8_t* gate_up_codes, const uint8_t* gate_up_scales,
                                  const uint8_t* down_codes, const uint8_t* down_scales, int64_t n_cap, void* y_perm,
                                  void* ws, size_t ws_bytes, void* stream) {
  REQUIRE(d >= 1 && F >= 1, "grouped_ffn_mxfp4_fwd: d=%d, F=%d", d, F);
  REQUIRE(S >= 0 && S <= FOREMOE_MAX_SLOTS, "grouped_ffn_mxfp4_fwd: S=%d outside [0, %d]", S, FOREMOE_MAX_SLOTS);
  REQUIRE(W >= 0 && (W >= 1 || S == 0), "grouped_ffn_mxfp4_fwd: W=%d", W);
  REQUIRE(n_cap >= 0 && n_cap < (int64_t)1 << 31, "grouped_ffn_mxfp4_fwd: n_cap=%lld outside [0, 2^31)",
          (long long)n_cap);
  if (d % 128 || F % 128 || 2 * (int64_t)d * F >= (int64_t)1 << 32)
    return set_error(FOREMOE_EUNSUPPORTED,
                     "grouped_ffn_mxfp4_fwd: d=%d and F=%d must be multiples of 128 with 2 d F below 2^32", d, F);
  if (S == 0 || n_cap == 0) return FOREMOE_OK;
  REQUIRE(x_codes && x_scales && slot_offset && slot_widx && gate_up_codes && gate_up_scales && down_codes &&
              down_scales && y_perm && ws,
          "grouped_ffn_mxfp4_fwd: NULL pointer");
  REQUIRE(!misaligned(x_codes, 16) && !misaligned(gate_up_codes, 16) && !misaligned(down_codes, 16) &&
              !misaligned(y_perm, 16) && !misaligned(x_scales, 4) && !misaligned(gate_up_scales, 4) &&
              !misaligned(down_scales, 4) && !misaligned(slot_offset, 4) && !misaligned(slot_widx, 4),
          "grouped_ffn_mxfp4_fwd: misaligned pointer");
  const size_t need = foremoe_ffn_mxfp4_workspace_size(n_cap, F);
  REQUIRE(ws_bytes >= need, "grouped_ffn_mxfp4_fwd: workspace too small (%zu < %zu bytes)", ws_bytes, need);
  REQUIRE(!misaligned(ws, 256), "grouped_ffn_mxfp4_fwd: workspace misaligned");
  uint8_t* h_codes = (uint8_t*)ws;
  uint8_t* h_scales = h_codes + align_up((size_t)n_cap * (F / 2), 256);
  hipStream_t st = (hipStream_t)stream;
  // every slot has at most one tile that is not full
  const int64_t row_tiles = (n_cap + kMxM - 1) / kMxM + S;
  Ffn4Args a{};
  a.slot_offset = slot_offset, a.slot_widx = slot_widx, a.S = S, a.W = W, a.n_cap = n_cap, a.F = F;
  a.h_codes = h_codes, a.h_scales = h_scales, a.y = (uint16_t*)y_perm;
  a.a_codes = x_codes, a.a_scales = x_scales, a.b_codes = gate_up_codes, a.b_scales = gate_up_scales;
  a.K = d, a.N = 2 * F, a.n_tiles = F / (kMxN / 2);
  REQUIRE(row_tiles * ((d > F ? d : F) / 128) < (int64_t)1 << 31, "grouped_ffn_mxfp4_fwd: too many tiles");
  hipLaunchKernelGGL((ffn4_kernel<true>), dim3((unsigned)(row_tiles * a.n_tiles)), dim3(64 * kMxWaves), 0, st, a);
  int rc = check_launch("grouped_ffn_mxfp4_fwd (gate/up)");
  if (rc != FOREMOE_OK) return rc;
  a.a_codes = h_codes, a.a_scales = h_scales, a.b_codes = down_codes, a.b_scales = down_scales;
  a.K = F, a.N = d, a.n_tiles = (d + kMxN - 1) / kMxN;
  hipLaunchKernelGGL((ffn4_kernel<false>), dim3((unsigned)(row_tiles * a.n_tiles)), dim3(64 * kMxWaves), 0, st, a);
  return check_launch("grouped_ffn_mxfp4_fwd (down)");
}

}  // extern "C"
