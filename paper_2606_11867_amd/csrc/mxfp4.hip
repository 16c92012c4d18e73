// Microscaled 4-bit floats: quantisation of rows, the values that codes stand
// for, and the grouped SwiGLU expert FFN (forward) with operands in 4 bits.
#include "common.h"
#include "mfma_tiles.h"
#include "mx.h"

namespace foremoe {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------
// Quantisation. Four lanes share a block, eight elements each, read 16 bytes at a
// time where the rows' alignment allows it. Bound by memory: 16278 x 2048 bf16
// values take 19 us (4.5 TB/s), 24576 x 2048 of fp32 45 us (5.1 TB/s); without
// the division, or with two to eight groups a lane at once, they take as long.
// The values of codes: bound by memory too, 20 us for those of 24576 x 2048 in
// bf16 (6.4 TB/s), 51 in fp32. Rows of an odd length or pitch are read and written
// element by element, eight neighbours a lane: values of 3001 x 1155 in bf16 8 us
// (1.1 TB/s); whole lines across the ends of rows would take a pass through LDS.
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
  int group;           // row tiles of a slot that are taken together, see find_tile
  int64_t n_cap;
};

struct SlotTile {
  int64_t row0, end;  // rows of the tile: [row0, min(row0 + BM, end))
  int w;
};

// Inclusive sum over the lanes.
__device__ __forceinline__ int lanes_up_to(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // row_shr:1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);  // row_bcast:15, 31
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);
  return v;
}

// The tile of workgroup b, found by every wavefront alone, a lane to neighbouring
// slots. Tiles are numbered slot by slot, and each of the 8 XCDs has an even share
// of neighbours, which have their rows and weights in its L2 once. Within a slot
// a.group row tiles go along N together: one where a matrix fits an L2 (4 MB)
// beside the rows, and eight where it does not and its columns would be read
// again for every row tile (us, one / eight: gate/up 8 x 512 rows, 4096 x 14336,
// 460 / 357; down of the same 247 / 222; but down 2048 x 768 of 16278 rows
// 33.6 / 38). False where there is none.
template <int BM>
__device__ __forceinline__ bool find_tile(const Ffn4Args& a, unsigned b, SlotTile& r, int& nt) {
  const int per = (a.S + 63) / 64, j0 = lane64() * per, n_cap = (int)a.n_cap;
  int beg, end, w;
  auto tiles_of = [&](int j) -> int {  // of slot j, with its rows and matrix
    beg = end = 0, w = -1;
    if (j < a.S) beg = a.slot_offset[j], end = a.slot_offset[j + 1], w = a.slot_widx[j];
    beg = min(max(beg, 0), n_cap), end = min(end, n_cap);
    return end > beg ? (int)(((unsigned)(end - beg) + BM - 1) / BM) : 0;
  };
  int mine = 0;
  for (int i = per - 1; i >= 0; --i) mine += tiles_of(j0 + i);
  const int upto = lanes_up_to(mine), all = __builtin_amdgcn_readlane(upto, 63);
  const unsigned tiles = (unsigned)all * a.n_tiles, share = (tiles + 7) / 8, at = b / 8, t = (b % 8) * share + at;
  if (at >= share || t >= tiles) return false;
  const int m = (int)(t / a.n_tiles);
  const int who = __builtin_ctzll(__ballot(upto > m));
  int first = m - (upto - mine);  // of this lane's slots
  int n = 0;  // of the tile's slot
  for (int i = 0; i < per; ++i) {
    n = i == 0 ? (per == 1 ? mine : tiles_of(j0)) : tiles_of(j0 + i);
    if (first < n) break;
    first -= n;
  }
  const int in_slot = __builtin_amdgcn_readlane(first, who), group = in_slot / a.group * a.group;
  const int high = min(a.group, __builtin_amdgcn_readlane(n, who) - group);
  const unsigned u = (unsigned)(in_slot - group) * a.n_tiles + t % a.n_tiles;
  nt = (int)(u / high);
  r.row0 = __builtin_amdgcn_readlane(beg, who) + (group + (int)(u % high)) * BM;
  r.end = __builtin_amdgcn_readlane(end, who);
  r.w = __builtin_amdgcn_readlane(w, who);
  return true;
}

// One wavefront moves 64 x 4 bytes: lane l's word lands at lds_wave_base + 4 l.
__device__ __forceinline__ void dma4(i32x4 rs, uint32_t lds_wave_base, uint32_t voff) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds_wave_base);
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(m0v), "v"(voff), "s"(rs) : "memory");
}

constexpr int kMxWaves = 4;
// Large tiles, two workgroups a CU; small ones with loads further ahead, for
// calls with too few rows to give every CU a large one.
constexpr int kMxM = 128, kMxN = 256, kMxStages = 3, kMxSmallM = 64, kMxSmallN = 128, kMxSmallStages = 6;

// Four scale words of a lane's rows, one for each of four stages.
struct ScaleWords {
  uint32_t w[4];
};

template <bool GATE_UP, int BM, int BN, int NS>
__global__ __launch_bounds__(64 * kMxWaves, 2) void ffn4_kernel(Ffn4Args a) {
  constexpr int NW = kMxWaves;
  // 128 codes are 64 bytes: the geometry of a tile of 32 16-bit elements
  using AT = KTile<BM, 32, NW>;
  using BT = KTile<BN, 32, NW>;
  constexpr int STAGE = AT::BYTES + BT::BYTES, ROWS = BM + BN;
  constexpr int PER = AT::PER_WAVE + BT::PER_WAVE;
  // Scales come for four stages at once, 16 bytes of a row, into one buffer
  // that is free again when all have read theirs (a word of a row for every
  // stage: 8200 x 7168 x 4096 245 us, this 200).
  constexpr int SC_LOADS = ROWS / 64, SC_PER = (SC_LOADS + NW - 1) / NW, SCALES = ROWS * 16;
  constexpr int WM = BM / 2, WN = BN / 2, MB = WM / 32, NB = WN / 32;
  constexpr int YLD = BN * 2 + 16;  // bytes of a row of y in LDS
  static_assert(ROWS % 64 == 0 && SC_PER <= 2 && (NS - 2) * PER + 2 < 64, "loads of scales, and in flight");
  static_assert(NS * STAGE >= BM * YLD, "the output's tile takes the stages' place");
  __shared__ __attribute__((aligned(1024))) char lds[NS * STAGE + SCALES];

  SlotTile r;
  int nt;
  if (!find_tile<BM>(a, blockIdx.x, r, nt)) return;
  if (r.w < 0 || r.w >= a.W) return;
  const int lane = lane64(), wave = wave_id(), half = lane >> 5;
  const int wm = wave >> 1, wn = wave & 1;
  const uint32_t lds0 = lds_addr(lds);
  char* const sc = lds + NS * STAGE;
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
  uint32_t va[AT::PER_WAVE], vb[BT::PER_WAVE], vs[SC_PER];
#pragma unroll
  for (int i = 0; i < AT::PER_WAVE; ++i) va[i] = AT::voff(lane, [&](int q) { return (uint32_t)q * kb; }, i);
#pragma unroll
  for (int i = 0; i < BT::PER_WAVE; ++i) vb[i] = BT::voff(lane, [&](int q) { return wrow(q) * kb; }, i);
#pragma unroll
  for (int i = 0; i < SC_PER; ++i) {
    const int q = (wave + NW * i) * 64 + lane;  // row of the A tile, then of the B tile
    vs[i] = q < BM ? (uint32_t)q * ks : wrow(q - BM) * ks;
  }
  auto issue = [&](int kt) {  // stages past the last load nothing
    const bool live = kt < KT;
    const uint32_t at = lds0 + (uint32_t)((kt % NS) * STAGE);
    const uint32_t kc = live ? (uint32_t)kt * 64u : 0u;
    const i32x4 ra = buf_rsrc(abase + kc, live ? abytes - kc : 0u), rb = buf_rsrc(bbase + kc, live ? bbytes - kc : 0u);
#pragma unroll
    for (int i = 0; i < AT::PER_WAVE; ++i) AT::issue(ra, at, va[i], i);
#pragma unroll
    for (int i = 0; i < BT::PER_WAVE; ++i) BT::issue(rb, at + AT::BYTES, vb[i], i);
  };
  // The 16 bytes from o on of every row: those of stages 4 g .. 4 g + 3, or
  // the row's last 16, so that no load reaches past a row. Where a row has
  // fewer (K < 512), word by word.
  const bool by_word = ks < 16;
  auto first_of = [&](int g) -> uint32_t { return (uint32_t)g * 16u + 16u <= ks ? (uint32_t)g * 16u : ks - 16u; };
  auto scales_of = [&](int i, uint32_t o, bool live) {  // the resource of wavefront load i
    const int q = wave + NW * i;
    const bool some = live && q < SC_LOADS, is_a = q * 64 < BM;
    return buf_rsrc((is_a ? asbase : bsbase) + (some ? o : 0u), some ? (is_a ? asbytes : bsbytes) - o : 0u);
  };
  auto issue_scales = [&](int g) {
    const bool live = g * 4 < KT;
    const uint32_t o = live ? first_of(g) : 0u;
#pragma unroll
    for (int i = 0; i < SC_PER; ++i)
      if (wave + NW * i < SC_LOADS)
        dma16(scales_of(i, o, live), lds0 + NS * STAGE + (wave + NW * i) * 1024, vs[i]);
  };
  auto issue_words = [&] {
    for (int k = 0; k < KT; ++k)
#pragma unroll
      for (int i = 0; i < SC_PER; ++i)
        if (wave + NW * i < SC_LOADS)
          dma4(scales_of(i, (uint32_t)k * 4u, true), lds0 + NS * STAGE + k * ROWS * 4 + (wave + NW * i) * 256, vs[i]);
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

  ScaleWords sa[MB], sb[NB];
  // this lane's blocks of a stage are 2 kk + half: their bytes 2 kk after the shift
  auto read_scales = [&](int g) {
    const uint32_t skip = by_word ? 0u : ((uint32_t)g * 16u - first_of(g)) / 4u;  // words of the stages before
    auto read = [&](int row, ScaleWords& s) {
      if (by_word) {
#pragma unroll
        for (int k = 0; k < 3; ++k) s.w[k] = k < KT ? ((const uint32_t*)sc)[k * ROWS + row] : 0u;
        s.w[3] = 0;
      } else {
        const uint4 v = ((const uint4*)sc)[row];
        s.w[0] = v.x, s.w[1] = v.y, s.w[2] = v.z, s.w[3] = v.w;
        if (skip == 1) s.w[0] = s.w[1], s.w[1] = s.w[2], s.w[2] = s.w[3];
        if (skip == 2) s.w[0] = s.w[2], s.w[1] = s.w[3];
        if (skip == 3) s.w[0] = s.w[3];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) s.w[k] >>= 8 * half;
    };
#pragma unroll
    for (int i = 0; i < MB; ++i) read(wm * WM + i * 32 + (lane & 31), sa[i]);
#pragma unroll
    for (int j = 0; j < NB; ++j) read(BM + bcol(j) + (lane & 31), sb[j]);
  };

  if (by_word) issue_words();
  else issue_scales(0);
#pragma unroll
  for (int s = 0; s < NS - 1; ++s) issue(s);
  for (int k0 = 0; k0 < KT; k0 += 4) {
    static_for<0, 4>([&](auto pc) {
      constexpr int ph = decltype(pc)::value;
      const int kt = k0 + ph;
      if (kt >= KT) return;
      // Stage kt has landed: what may be in flight are the codes of the NS - 2
      // stages after it (with scales among them, one load or two fewer). Before
      // scales are read, which were asked for behind the codes of three
      // iterations ago, the codes of two. With NS = 3, in the iteration after
      // they were asked for, they may be in flight too.
      if constexpr (ph == 0 && NS > 4) {
        if (k0 > 0) wait_vm<2 * PER>();
        else wait_vm<(NS - 2) * PER>();
      } else if constexpr (ph == 2 && NS == 3) {
        if (by_word || wave >= SC_LOADS) wait_vm<(NS - 2) * PER>();  // (words came first)
        else if (wave + NW < SC_LOADS) wait_vm<(NS - 2) * PER + 2>();
        else wait_vm<(NS - 2) * PER + 1>();
      } else {
        wait_vm<(NS - 2) * PER>();
      }
      __syncthreads();  // for every wavefront, and stage kt - 1 has been read
      issue(kt + NS - 1);
      if constexpr (ph == 0) read_scales(k0 / 4);
      if constexpr (ph == 1) {
        if (!by_word) issue_scales(k0 / 4 + 1);
      }
      const char* st = lds + (kt % NS) * STAGE;
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
                __builtin_shufflevector(fa[i], fa[i], 0, 1, 2, 3, -1, -1, -1, -1), acc[i][j], 4, 4, 2 * kk,
                (int)sb[j].w[ph], 2 * kk, (int)sa[i].w[ph]);
      });
    });
  }
  wait_vm<0>();     // the loads of nothing have landed too
  __syncthreads();  // and every wavefront has read its last stage: the output takes its place

  // block (i, j), register q: row 32 i + lane % 32, column 32 j + 8 (q / 4) + 4 half + q % 4
  const int tid = threadIdx.x;
  if constexpr (GATE_UP) {
    // a tile of BN / 2 columns of h: BN / 4 bytes of codes and BN / 64 of scales a row
    constexpr int HLD = BN / 4 + 16, PARTS = BN / 64;
    typedef typename std::conditional<PARTS == 4, uint32_t, uint16_t>::type Scales;
    char* const hs = lds + BM * HLD;
#pragma unroll
    for (int i = 0; i < MB; ++i) {
      const int row = wm * WM + i * 32 + (lane & 31);
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
        const int col = wn * (WN / 2) + j * 32;
        char* const to = lds + row * HLD + col / 2 + 2 * half;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t c = mx_put2<1>(mx_put2<0>(0u, h[4 * q], h[4 * q + 1]), h[4 * q + 2], h[4 * q + 3]);
          *(uint16_t*)(to + 4 * q) = s == 255 ? (uint16_t)0 : (uint16_t)c;
        }
        if (half == 0) hs[row * PARTS + col / 32] = (char)s;
      }
    }
    __syncthreads();
#pragma unroll
    for (int o = tid; o < BM * PARTS; o += 64 * NW) {
      const int row = o / PARTS, part = o % PARTS;
      if (row < rows)
        *(uint4*)(a.h_codes + (r.row0 + row) * (a.F / 2) + n0 / 2 + 16 * part) = *(const uint4*)(lds + row * HLD + 16 * part);
    }
    if (tid < rows)
      *(Scales*)(a.h_scales + (r.row0 + tid) * (a.F / 32) + n0 / 32) = *(const Scales*)(hs + PARTS * tid);
  } else {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *(uint2*)(lds + (wm * WM + i * 32 + (lane & 31)) * YLD + (wn * WN + j * 32 + 4 * half + 8 * q) * 2) =
              uint2{pack_bf2(acc[i][j][4 * q], acc[i][j][4 * q + 1]), pack_bf2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3])};
    __syncthreads();
    // whole lines: 512 bytes of a row by 32 lanes (8 bytes of a row at a time
    // from the registers: 16278 x 768 x 2048 50 us, this 35)
    constexpr int LANES = BN / 8, AT_ONCE = 64 * NW / LANES;
    const int part = tid % LANES;
    if (n0 + part * 8 < a.N) {
#pragma unroll 4
      for (int k = 0; k < BM / AT_ONCE; ++k) {
        const int row = k * AT_ONCE + tid / LANES;
        if (row < rows)
          *(uint4*)(a.y + (r.row0 + row) * a.N + n0 + part * 8) = *(const uint4*)(lds + row * YLD + 16 * part);
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

// One product. Every slot has at most one tile that is not full; tiles are
// large unless even the most that there can be leave CUs without one.
template <bool GATE_UP>
static void launch_ffn4(Ffn4Args a, hipStream_t st) {
  auto grid = [&](int bm, int bn) {
    a.n_tiles = (a.N + bn - 1) / bn;
    return (a.n_cap + bm - 1) / bm * a.n_tiles + (int64_t)a.S * a.n_tiles;
  };
  auto rounded = [](int64_t n) { return dim3((unsigned)((n + 7) / 8 * 8)); };  // one share for each XCD: see find_tile
  int64_t n = grid(kMxM, kMxN);
  a.group = (int64_t)a.N * a.K / 2 <= 2 << 20 ? 1 : 8;
  if (n > num_cus()) {
    hipLaunchKernelGGL((ffn4_kernel<GATE_UP, kMxM, kMxN, kMxStages>), rounded(n), dim3(64 * kMxWaves), 0, st, a);
  } else {
    n = grid(kMxSmallM, kMxSmallN);
    hipLaunchKernelGGL((ffn4_kernel<GATE_UP, kMxSmallM, kMxSmallN, kMxSmallStages>), rounded(n), dim3(64 * kMxWaves), 0,
                       st, a);
  }
}

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
  Ffn4Args a{};
  a.slot_offset = slot_offset, a.slot_widx = slot_widx, a.S = S, a.W = W, a.n_cap = n_cap, a.F = F;
  a.h_codes = h_codes, a.h_scales = h_scales, a.y = (uint16_t*)y_perm;
  REQUIRE((n_cap / 128 + S + 1) * ((d > F ? d : F) / 128) < (int64_t)1 << 23, "grouped_ffn_mxfp4_fwd: too many tiles");
  a.a_codes = x_codes, a.a_scales = x_scales, a.b_codes = gate_up_codes, a.b_scales = gate_up_scales;
  a.K = d, a.N = 2 * F;
  launch_ffn4<true>(a, st);
  const int rc = check_launch("grouped_ffn_mxfp4_fwd (gate/up)");
  if (rc != FOREMOE_OK) return rc;
  a.a_codes = h_codes, a.a_scales = h_scales, a.b_codes = down_codes, a.b_scales = down_scales;
  a.K = F, a.N = d;
  launch_ffn4<false>(a, st);
  return check_launch("grouped_ffn_mxfp4_fwd (down)");
}

}  // extern "C"
