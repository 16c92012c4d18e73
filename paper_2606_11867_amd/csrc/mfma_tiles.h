// Building blocks of the MFMA kernels: range-checked buffer loads into LDS,
// swizzled operand tiles and their fragment reads, the tile core and its
// software-pipelined k loop, SiLU and its derivative.
#pragma once

#include <type_traits>

#include "common.h"

namespace foremoe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// k-steps over which one stage's loads are spread (capped at the k-steps of a stage)
#ifndef FM_LOAD_SPREAD
#define FM_LOAD_SPREAD 2
#endif
// Wave priority while a k-step's MFMAs issue (0: leave it): the wave that
// is multiplying wins the SIMD's issue arbitration over the other wave on
// that SIMD, whose reads and loads then fill the gaps.
#ifndef FM_SETPRIO
#define FM_SETPRIO 1
#endif

// SiLU a / D and sigmoid 1 / D with D = 1 + exp(-a), correctly rounded in fp32.
// The hardware reciprocal alone is 1 ulp off; one Newton step on it (on the
// quotient) gives the division's bits for every fp32 number a where neither
// D nor |a| reaches 2^126 (all of them were compared), in a third of its
// instructions. Beyond, where the reciprocal flushes its subnormal result (a
// below -87.3, with SiLU near 1e-37 in bf16) or the step has infinities, the
// division itself; one check for the N values of every lane. Down input
// gradient of 8 slots of 512 rows (d = 1024, F = 512), us: reciprocal alone
// 20.9, this 21.2, divisions 22.7; Qwen3 share's gate/up forward 115.2 / 117.2
// / 119.8.
constexpr float kDivideFrom = 0x1p126f;

template <int N>
__device__ __forceinline__ void silu_n(const float* a, float* s) {
  float D[N], m = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    D[e] = 1.0f + __expf(-a[e]);
    m = fmaxf(m, fmaxf(D[e], fabsf(a[e])));
    const float r = __builtin_amdgcn_rcpf(D[e]), q = a[e] * r;
    s[e] = copysignf(fmaf(fmaf(-q, D[e], a[e]), r, q), a[e]);  // (a zero's sign)
  }
  if (__builtin_expect(__ballot(m >= kDivideFrom) != 0, 0)) {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = a[e] / D[e];
  }
}
template <int N>
__device__ __forceinline__ void sigmoid_n(const float* a, float* s) {
  float D[N], m = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    D[e] = 1.0f + __expf(-a[e]);
    m = fmaxf(m, D[e]);
    const float r = __builtin_amdgcn_rcpf(D[e]);
    s[e] = fmaf(fmaf(-D[e], r, 1.0f), r, r);
  }
  if (__builtin_expect(__ballot(m >= kDivideFrom) != 0, 0)) {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = 1.0f / D[e];
  }
}

__device__ __forceinline__ int lane64() { return threadIdx.x & 63; }
// The same, recomputed where it stands: a kernel with several tile shapes in
// one loop would otherwise keep the lane offsets of all of them in registers
// across the loop (and spill).
__device__ __forceinline__ int lane64_here() {
  int l = threadIdx.x & 63;
  asm volatile("" : "+v"(l));
  return l;
}
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Virtual workgroup id: workgroups are dispatched round-robin over the 8 XCDs,
// so give the workgroups of one XCD consecutive ids (they then share tiles
// that reuse the same operand rows in that XCD's L2).
#ifndef FM_XCD_MAP
#define FM_XCD_MAP 1
#endif
__device__ __forceinline__ int xcd_virtual_id() {
  const int b = blockIdx.x, n = gridDim.x;
  if (!FM_XCD_MAP || n % 8 != 0) return b;
  return (b % 8) * (n / 8) + b / 8;
}

// ---------------------------------------------------------------------------
// Range-checked buffer loads straight into LDS
// ---------------------------------------------------------------------------
// A buffer resource over [base, base + bytes): a load at an offset >= bytes
// returns zeros, so ragged tile edges read as zero and no load can leave the
// operand.
__device__ __forceinline__ i32x4 buf_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = (uint64_t)base;
  i32x4 r;
  r.x = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
  r.y = __builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xFFFFu));
  r.z = __builtin_amdgcn_readfirstlane((int)bytes);
  r.w = 0x00020000;
  return r;
}

// One wavefront moves 64 x 16 bytes: lane l's bytes land at LDS address
// lds_wave_base + 16 l. The load is issued asynchronously; completion is
// awaited with wait_vm() before the workgroup barrier that publishes it.
__device__ __forceinline__ void dma16(i32x4 rs, uint32_t lds_wave_base, uint32_t voff) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds_wave_base);
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m0v), "v"(voff), "s"(rs)
               : "memory");
}

// The same with lane offset voff0 + soff (soff wave-uniform): the add sits
// in the asm so that one temporary serves every load instead of one
// precomputed offset register per load.
__device__ __forceinline__ void dma16s(i32x4 rs, uint32_t lds_wave_base, uint32_t voff0, uint32_t soff) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane(lds_wave_base);
  uint32_t t;
  asm volatile(
      "v_add_u32 %0, %1, %2\n\ts_mov_b32 m0, %3\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds"
      : "=&v"(t)
      : "s"(soff), "v"(voff0), "s"(m0v), "s"(rs)
      : "memory");
}

// Wait until at most N vector-memory operations of this wavefront are in flight.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | (7 << 4) | (15 << 8) | ((N >> 4) << 14));
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) { return (uint32_t)(uintptr_t)p; }

// ---------------------------------------------------------------------------
// LDS operand tiles. A "K-major" tile keeps ROWS rows (m or n) of BK
// contiguous k values; a "MN-major" tile keeps BK rows (k) of ROWS contiguous
// m or n values. Both are filled by dma16 and XOR-swizzled in 16-byte chunks
// so that the MFMA fragment reads hit 16 (or 32) different LDS bank groups of
// gfx950's 64 banks.
// ---------------------------------------------------------------------------
template <int ROWS, int BK, int NW>
struct KTile {
  static constexpr int CPR = BK / 8;     // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;   // rows per wavefront load
  static constexpr int NI = ROWS / RPI;  // wavefront loads per tile
  static constexpr int PER_WAVE = NI / NW;
  static constexpr int BYTES = ROWS * BK * 2;
  static_assert(NI % NW == 0, "tile must split over the wavefronts");
  __device__ __forceinline__ static int swz(int r) {
    if constexpr (CPR == 8) return (r >> 1) & 7;
    else return (r >> 2) & 3;
  }
  // This lane's source offset in load i (0 <= i < PER_WAVE) of this
  // wavefront's share of the tile, relative to the stage's first k; rowoff(r)
  // is the byte offset of tile row r. Fixed for a whole tile: each stage
  // moves the buffer resource instead.
  template <class RowOff>
  __device__ __forceinline__ static uint32_t voff(int l, RowOff rowoff, int i) {
    const int w = wave_id();
    const int r = (w + NW * i) * RPI + l / CPR;
    const int c = (l % CPR) ^ swz(r);
    return rowoff(r) + (uint32_t)c * 16u;
  }
  __device__ __forceinline__ static void issue(i32x4 rs, uint32_t lds, uint32_t voff, int i) {
    dma16(rs, lds + (wave_id() + NW * i) * 1024, voff);
  }
  // load i with lane offset voff(0) + soff_i, soff_i = voff(i) - voff(0) (the
  // same for every lane: the swizzle of a row or k row does not change by i)
  __device__ __forceinline__ static void issue_s(i32x4 rs, uint32_t lds, uint32_t voff0, uint32_t soff, int i) {
    dma16s(rs, lds + (wave_id() + NW * i) * 1024, voff0, soff);
  }
  // MFMA operand for rows mn0..mn0+31 of the tile, k-step kk (16 k values):
  // lane l gets row mn0 + l % 32, k = 16 kk + 8 (l / 32) + 0..7. The swizzle
  // only depends on l % 32 (mn0 is a multiple of 32), so the address splits
  // into a per-block lane offset and a per-k-step lane offset.
  __device__ __forceinline__ static uint32_t lane_off(int l, int mn0) {
    return (uint32_t)(mn0 + (l & 31)) * (BK * 2);
  }
  __device__ __forceinline__ static uint32_t kstep_off(int l, int kk) {
    return (uint32_t)(((2 * kk + (l >> 5)) ^ swz(l & 31)) * 16);
  }
  __device__ __forceinline__ static bf16x8 frag(const char* lds, uint32_t off, const uint32_t* koff, int kk) {
    return *reinterpret_cast<const bf16x8*>(lds + off + koff[kk]);
  }
};

template <int ROWS, int BK, int NW>
struct MTile {
  static constexpr int RB = ROWS * 2;    // bytes per k row
  static constexpr int KPI = 1024 / RB;  // k rows per wavefront load
  static constexpr int NI = BK / KPI;
  static constexpr int PER_WAVE = NI / NW;
  static constexpr int BYTES = ROWS * BK * 2;
  static_assert(NI % NW == 0 && KPI >= 1, "tile must split over the wavefronts");
  __device__ __forceinline__ static int swz(int k) { return 4 * (k & 3); }
  // This lane's source offset in load i (0 <= i < PER_WAVE) of this
  // wavefront's share of the tile; koff(k) is the byte offset of the tile's
  // k-row k (relative to the stage's first k row) at the tile's first m/n.
  template <class KOff>
  __device__ __forceinline__ static uint32_t voff(int l, KOff koff, int i) {
    const int w = wave_id();
    const int k = (w + NW * i) * KPI + (l * 16) / RB;
    const int c = ((l * 16) % RB) / 16 ^ swz(k);
    return koff(k) + (uint32_t)c * 16u;
  }
  __device__ __forceinline__ static void issue(i32x4 rs, uint32_t lds, uint32_t voff, int i) {
    dma16(rs, lds + (wave_id() + NW * i) * 1024, voff);
  }
  // load i with lane offset voff(0) + soff_i, soff_i = voff(i) - voff(0) (the
  // same for every lane: the swizzle of a row or k row does not change by i)
  __device__ __forceinline__ static void issue_s(i32x4 rs, uint32_t lds, uint32_t voff0, uint32_t soff, int i) {
    dma16s(rs, lds + (wave_id() + NW * i) * 1024, voff0, soff);
  }
  // Same operand layout as KTile::frag, assembled from two transpose reads:
  // in each 16-lane group g, lane i addresses 4 consecutive m/n of one k row
  // and lane j receives one m/n at 4 consecutive k. The k row's low two bits
  // (which pick the swizzle) come from the lane alone, so the address is a
  // per-block lane offset plus an immediate (16 kk + 4 h) * RB.
  __device__ __forceinline__ static uint32_t lane_off(int l, int mn0) {
    const int g = l >> 4, j = l & 15;
    const int krow = 8 * (g >> 1) + (j >> 2);
    const int mn = mn0 + 16 * (g & 1) + 4 * (j & 3);
    return (uint32_t)(krow * RB + (((mn >> 3) ^ swz(krow)) << 4) + (mn & 7) * 2);
  }
  __device__ __forceinline__ static uint32_t kstep_off(int, int) { return 0; }
  __device__ __forceinline__ static bf16x8 frag(const char* lds, uint32_t off, const uint32_t*, int kk) {
    s16x4 v[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      v[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + off + (kk * 16 + 4 * h) * RB));
    const s16x8 t = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, t);
  }
};

// The matrix instruction of a 16-bit type (fragments travel as bf16x8, 16 bytes a lane).
struct Bf16 {
  __device__ __forceinline__ static f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
struct Fp16 {
  __device__ __forceinline__ static f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

// ---------------------------------------------------------------------------
// MFMA tile core: WGM x WGN wavefronts, each owning (BM/WGM) x (BN/WGN) of
// the output as 32x32 blocks. The MFMA is fed the B rows as its first
// operand, so each lane ends up with 4 consecutive output columns of one
// output row: block (i, j), register q of lane l holds row
// wm*WM + 32 i + l % 32 and column bcol(j) + 8 (q / 4) + 4 (l / 32) + q % 4.
// ---------------------------------------------------------------------------
template <int BM, int BN, int WGM, int WGN, bool SWIGLU_COLS, class Mat = Bf16>
struct Core {
  static constexpr int WM = BM / WGM, WN = BN / WGN;
  static constexpr int MB = WM / 32, NB = WN / 32;
  static constexpr int GW = BN / 2 / WGN;  // SwiGLU: gate (or up) columns per wave
  static_assert(MB >= 1 && NB >= 1 && (!SWIGLU_COLS || NB % 2 == 0), "wave tile");
  f32x16 acc[MB][NB];

  // LDS row of the B tile that wave column wn's block j starts at.
  __device__ __forceinline__ static int bcol(int wn, int j) {
    if constexpr (SWIGLU_COLS) {
      // gate rows live in [0, BN/2), up rows in [BN/2, BN); the wave keeps the
      // gate block j and the up block j + NB/2 of the same output columns
      constexpr int H = NB / 2;
      return j < H ? wn * GW + j * 32 : BN / 2 + wn * GW + (j - H) * 32;
    } else {
      return wn * WN + j * 32;
    }
  }

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  }

  // Per-lane LDS offsets of every 32-row block this wave reads (fixed for
  // the whole kernel) and of every k-step.
  template <class AT, class BT, int BK>
  struct Offsets {
    uint32_t a[MB], b[NB], ka[BK / 16], kb[BK / 16];
    __device__ __forceinline__ Offsets(int lane, int wm, int wn) {
#pragma unroll
      for (int i = 0; i < MB; ++i) a[i] = AT::lane_off(lane, wm * WM + i * 32);
#pragma unroll
      for (int j = 0; j < NB; ++j) b[j] = BT::lane_off(lane, bcol(wn, j));
#pragma unroll
      for (int kk = 0; kk < BK / 16; ++kk) {
        ka[kk] = AT::kstep_off(lane, kk);
        kb[kk] = BT::kstep_off(lane, kk);
      }
    }
  };

  // Operand fragments of FS k-steps in registers (the one being multiplied
  // and the ones being read ahead).
  template <int FS>
  struct Frags {
    bf16x8 a[FS][MB], b[FS][NB];
  };

  template <class AT, class BT, int BK, class FragsT>
  __device__ __forceinline__ static void load_frags(FragsT& f, int set, const char* As, const char* Bs,
                                                    const Offsets<AT, BT, BK>& o, int kk) {
#pragma unroll
    for (int i = 0; i < MB; ++i) f.a[set][i] = AT::frag(As, o.a[i], o.ka, kk);
#pragma unroll
    for (int j = 0; j < NB; ++j) f.b[set][j] = BT::frag(Bs, o.b[j], o.kb, kk);
  }

  // The MFMAs of one k-step from register set CUR, with the LDS reads of a
  // later k-step's fragments (k-step nkk of the stage at nAs/nBs, into set
  // NXT) interleaved: one read (two in the smallest wave tiles) after each of the
  // first MFMAs, so the reads complete under the matrix work. extra(q), q < NX, runs right after
  // MFMA s when q < (s + 1) NX / (MB NB) and q >= s NX / (MB NB), evenly
  // over the k-step: the loads of a later stage, spread over the k-step so
  // that the address unit drains them while the matrix cores keep working.
  template <class AT, class BT, int BK, int NX, int CUR, int NXT, class FragsT, class Extra>
  __device__ __forceinline__ void mfma_step(FragsT& f, const char* nAs, const char* nBs, const Offsets<AT, BT, BK>& o,
                                            int nkk, Extra&& extra) {
    constexpr int NM = MB * NB;
    constexpr int RPM = (MB + NB + NM - 1) / NM;  // reads after each MFMA: one, or two in the smallest wave tiles
    static_assert(NX >= 0 && NX <= NM, "loads per k-step");
    static_assert(CUR != NXT, "the fragments being read go to another set");
    if constexpr (FM_SETPRIO > 0) __builtin_amdgcn_s_setprio(FM_SETPRIO);
#pragma unroll
    for (int s = 0; s < NM; ++s) {
      const int i = s / NB, j = s % NB;
      acc[i][j] = Mat::mfma(f.b[CUR][j], f.a[CUR][i], acc[i][j]);
      if (FM_SETPRIO > 0 && s == NM - 1) __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int t = s * RPM; t < (s + 1) * RPM && t < MB + NB; ++t) {
        if (t < MB) f.a[NXT][t] = AT::frag(nAs, o.a[t], o.ka, nkk);
        else f.b[NXT][t - MB] = BT::frag(nBs, o.b[t - MB], o.kb, nkk);
      }
      if constexpr (NX > 0) {
#pragma unroll
        for (int q = s * NX / NM; q < (s + 1) * NX / NM; ++q) extra(q);
      }
    }
#pragma unroll
    for (int s = 0; s < NM; ++s) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // one MFMA
      if (s * RPM < MB + NB) __builtin_amdgcn_sched_group_barrier(0x100, RPM, 0);  // its LDS reads
    }
  }
};

// Wait for the loads of the stage about to be computed: `ahead` younger
// stages (of PER loads each) may stay in flight.
template <int NS, int PER>
__device__ __forceinline__ void wait_stage(int ahead) {
  static_assert(NS >= 2 && NS <= 4 && (NS - 1) * PER < 64, "stages");
  if constexpr (NS >= 4) {
    if (ahead >= 3) {
      wait_vm<3 * PER>();
      return;
    }
  }
  if constexpr (NS >= 3) {
    if (ahead >= 2) {
      wait_vm<2 * PER>();
      return;
    }
  }
  if (ahead >= 1) {
    wait_vm<PER>();
    return;
  }
  wait_vm<0>();
}

// ---------------------------------------------------------------------------
// Software-pipelined K loop over an LDS ring of NS >= 2 stages.
//
// Stage kt's first fragments are already in registers when iteration kt
// starts, and every later k-step's fragments are read one k-step ahead. So
// when the last k-step of stage kt begins, every read of stage kt's buffer
// has been issued: each wavefront waits for its own loads of stage kt+1, and
// the workgroup barrier (which also retires all LDS reads) both publishes
// stage kt+1 and frees stage kt's buffer. The loads of stage kt+NS go into
// that buffer, spread over the MFMAs of the last k-step of stage kt and the
// first k-steps of stage kt+1 (issued in one burst, they would stall every
// wavefront behind the address unit at once). issue(s, p) issues load p
// (0 <= p < PER) of stage s, in increasing s, each stage whole before the
// next. Stages s >= KT must issue loads of nothing (zero-size buffer
// resources, which still write zeros to their LDS stage): every iteration
// then issues the same loads, with no branch among the MFMAs, and the
// counter waits stay exact.
// ---------------------------------------------------------------------------
template <int I, int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// Fragment read distance: 2 in the row GEMMs' 256-row tiles (gate/up forward
// 2% faster than with 1, the others the same), 1 in their smaller tiles and
// in the weight gradients (a third register set makes those spill).
#ifndef FM_FRAG_DIST
#define FM_FRAG_DIST 1
#endif
#ifndef FM_FRAG_DIST_ROWS
#define FM_FRAG_DIST_ROWS 2
#endif

// Fragments read one k-step ahead (two register sets).
template <class CoreT, class AT, class BT, int BK, int NS, class Issue, class Started>
__device__ __forceinline__ void pipelined_k_loop_d1(CoreT& core, char* lds, int KT,
                                                    const typename CoreT::template Offsets<AT, BT, BK>& o,
                                                    Issue&& issue, bool drain, Started&& started) {
  static_assert(BK % 32 == 0, "the last k-step's fragments must be read before the barrier");
  constexpr int KK = BK / 16;
  constexpr int STAGE = AT::BYTES + BT::BYTES;
  constexpr int PER = AT::PER_WAVE + BT::PER_WAVE;
  // the loads of a stage ride on SPREAD k-steps: the last one of the stage
  // before and the first SPREAD - 1 of the next; load p goes with k-step
  // j when lo(j) <= p < lo(j + 1)
  // (and no k-step carries more loads than it has MFMAs)
  constexpr int MIN_SPREAD = (PER + CoreT::MB * CoreT::NB - 1) / (CoreT::MB * CoreT::NB);
  constexpr int WANT = FM_LOAD_SPREAD > MIN_SPREAD ? FM_LOAD_SPREAD : MIN_SPREAD;
  constexpr int SPREAD = WANT < KK ? WANT : KK;
  static_assert(SPREAD >= MIN_SPREAD, "load spread");
  auto lo = [](int j) constexpr { return j * PER / SPREAD; };
  typename CoreT::template Frags<2> f;
  // stages 0 .. NS-2 whole, and the part of stage NS-1 that a previous
  // iteration's last k-step would have carried
#pragma unroll
  for (int s = 0; s < NS; ++s) {
#pragma unroll
    for (int p = 0; p < (s < NS - 1 ? PER : lo(1)); ++p) issue(s, p);
  }
  if (drain) wait_vm<0>();
  else wait_vm<(NS - 2) * PER + lo(1)>();
  __syncthreads();
  started();
  CoreT::template load_frags<AT, BT, BK>(f, 0, lds, lds + AT::BYTES, o, 0);
  for (int kt = 0; kt < KT; ++kt) {
    const char* st = lds + (kt % NS) * STAGE;
    static_for<0, KK>([&](auto kkc) {
      constexpr int kk = decltype(kkc)::value;
      constexpr int set = kk & 1;
      if constexpr (kk < KK - 1) {
        constexpr int j = kk + 1;  // position in the load window of stage kt - 1 + NS
        core.template mfma_step<AT, BT, BK, (j < SPREAD ? lo(j + 1) - lo(j) : 0), set, set ^ 1>(
            f, st, st + AT::BYTES, o, kk + 1, [&](int q) { issue(kt - 1 + NS, lo(j) + q); });
      } else {
        wait_stage<NS, PER>(NS - 2);  // stage kt+1 (past the last: empty) has landed
        __syncthreads();
        const char* nst = lds + ((kt + 1) % NS) * STAGE;
        // (after the last stage this reads a stale buffer: harmless, and no
        // branch among the MFMAs)
        core.template mfma_step<AT, BT, BK, lo(1), set, set ^ 1>(f, nst, nst + AT::BYTES, o, 0,
                                                                 [&](int q) { issue(kt + NS, q); });
      }
    });
  }
  wait_vm<0>();  // the (empty) loads of stages past the last have landed too
}

// Fragments read D k-steps ahead (D + 1 register sets), so that each LDS read
// has D k-steps of matrix work to complete under. The barrier then comes at
// k-step KK - D of stage kt, the first whose reads reach into stage kt+1: by
// then every read of stage kt's buffer has been issued, and the loads of
// stage kt+NS go into it during k-steps KK - D .. KK - D + SPREAD - 1. The
// set of global k-step g is g % (D + 1); the stage loop is unrolled U times
// so that every set index is a compile-time constant.
template <class CoreT, class AT, class BT, int BK, int NS, int D, class Issue, class Started>
__device__ __forceinline__ void pipelined_k_loop_deep(CoreT& core, char* lds, int KT,
                                                      const typename CoreT::template Offsets<AT, BT, BK>& o,
                                                      Issue&& issue, bool drain, Started&& started) {
  constexpr int KK = BK / 16;
  constexpr int FS = D + 1;
  constexpr int STAGE = AT::BYTES + BT::BYTES;
  constexpr int PER = AT::PER_WAVE + BT::PER_WAVE;
  constexpr int SPREAD = FM_LOAD_SPREAD < D ? FM_LOAD_SPREAD : D;
  static_assert(D >= 2 && KK >= D, "read distance");
  static_assert(SPREAD >= 1, "load spread");
  auto lo = [](int j) constexpr { return j * PER / SPREAD; };
  constexpr int U = [] {
    int u = 1;
    while ((u * KK) % FS) ++u;
    return u;
  }();
  typename CoreT::template Frags<FS> f;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
#pragma unroll
    for (int p = 0; p < PER; ++p) issue(s, p);
  }
  wait_stage<NS, PER>(drain ? 0 : NS - 1);  // stage 0 has landed
  __syncthreads();
  started();
  static_for<0, D>([&](auto kc) {
    constexpr int k = decltype(kc)::value;
    CoreT::template load_frags<AT, BT, BK>(f, k, lds, lds + AT::BYTES, o, k);
  });
  int kt = 0;
  while (kt < KT) {  // kt advances inside the unrolled stage loop
    static_for<0, U>([&](auto phc) {
      constexpr int ph = decltype(phc)::value;
      if (kt >= KT) return;
      const char* st = lds + (kt % NS) * STAGE;
      const char* nst = lds + ((kt + 1) % NS) * STAGE;
      static_for<0, KK>([&](auto kkc) {
        constexpr int kk = decltype(kkc)::value;
        constexpr int g = ph * KK + kk;
        constexpr int cur = g % FS, nxt = (g + D) % FS;
        constexpr int j = kk - (KK - D);  // position in the load window of stage kt + NS
        constexpr int nx = (j >= 0 && j < SPREAD) ? lo(j + 1) - lo(j) : 0;
        if constexpr (j == 0) {
          wait_stage<NS, PER>(NS - 2);  // stage kt+1 (past the last: empty) has landed
          __syncthreads();
        }
        // reads of k-step kk + D: in this stage's buffer, or in the next's
        // (after the last stage a stale buffer: harmless, and no branch among
        // the MFMAs)
        const char* rs = kk + D < KK ? st : nst;
        constexpr int rk = (kk + D) % KK;
        core.template mfma_step<AT, BT, BK, nx, cur, nxt>(f, rs, rs + AT::BYTES, o, rk, [&](int q) {
          if constexpr (j >= 0) issue(kt + NS, lo(j) + q);
        });
      });
      ++kt;
    });
  }
  wait_vm<0>();  // the (empty) loads of stages past the last have landed too
}

// drain: the first wait is for every vector-memory operation of the
// wavefront, older stores included. started() runs after the first barrier.
template <class CoreT, class AT, class BT, int BK, int NS, int D, class Issue, class Started>
__device__ __forceinline__ void pipelined_k_loop(CoreT& core, char* lds, int KT,
                                                 const typename CoreT::template Offsets<AT, BT, BK>& o,
                                                 Issue&& issue, bool drain, Started&& started) {
  if constexpr (D >= 2 && BK / 16 >= D)
    pipelined_k_loop_deep<CoreT, AT, BT, BK, NS, D>(core, lds, KT, o, issue, drain, started);
  else
    pipelined_k_loop_d1<CoreT, AT, BT, BK, NS>(core, lds, KT, o, issue, drain, started);
}

}  // namespace
}  // namespace foremoe
