// Product of 8-bit rows and 8-bit weights with a scale per block of 128 (gfx950).
//
//   y[t][n] = sum_b xs[t][b] ws[n / 128][b] sum_{k in block b} x[t][k] w[n][k]  (+ bias[n])
//
// x, w: e4m3 codes; xs: one scale per row and 128 columns of x; ws: one per 128 x 128 of w.
// The inner sums come from v_mfma_f32_16x16x128_f8f6f4, whose depth is one block: its fp32
// result is multiplied by the two scales and added to the fp32 accumulator, so the scales cost
// one multiply-add per output and block. Every output adds its blocks in ascending order,
// whatever the tile: a row's results do not depend on the other rows of the call.
//
// The instruction itself keeps, of 8 consecutive products, 13 bits below the exponent of the
// largest (measured: beside a product of 2^16 one of 2^3 counts and one of 2^2 does not, unless
// it lies in another group of 8); its sums over groups are fp32. On random codes that is 2^-19 of
// the sum of the products' magnitudes, far below the output's rounding to bf16. Products in bf16
// MFMA, which are exact, run at half its rate.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <type_traits>

#include "cw_internal.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kDepth = 128;   // columns of a block: bytes of a staged row

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

struct LinearArgs {
  const uint8_t* x;
  const float* xs;
  const uint8_t* w;
  const float* ws;
  const uint16_t* bias;   // NULL: none
  uint16_t* out;
  int rows, feats, depth, blocks;          // blocks: of 128 along depth
  int n_ftiles, n_ttiles, per_xcd;
};

// One load-to-LDS copy: lane l's 16 bytes at base + off land at dst + 16 l (base and dst
// wave-uniform, dst through M0). The compiler does not count it: the kernel's own waits
// complete it.
__device__ __forceinline__ void copy16_to_lds(const uint8_t* base, uint32_t off, uint32_t dst) {
  const uint64_t b = reinterpret_cast<uintptr_t>(base);
  const uint64_t bu = (uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(b >> 32)))) << 32) |
                      uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(b))));
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(off), "s"(bu), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory");
}

// Copies with a descriptor of a wave-uniform base and its bytes: a lane past them reads nothing.
__device__ __forceinline__ u32x4 buffer(const void* p, uint32_t bytes) {
  const uint64_t b = reinterpret_cast<uintptr_t>(p);
  return u32x4{uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(b))),
               uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(b >> 32) & 0xFFFFu)),
               uint32_t(__builtin_amdgcn_readfirstlane(bytes)), 0x00027000u};
}
__device__ __forceinline__ void buffer16_to_lds(u32x4 d, uint32_t off, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
               :: "v"(off), "s"(d), "s"(__builtin_amdgcn_readfirstlane(dst)) : "memory");
}

// s_waitcnt immediates (gfx9 encoding): vmcnt(n) with lgkmcnt(0), expcnt untouched.
constexpr int waitcnt_vm_lgkm0(int n) { return (n & 15) | (7 << 4) | ((n >> 4) << 14); }

// Workgroup barrier that no memory access or instruction group moves across.
__device__ __forceinline__ void interval_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Staged rows are 128-byte lines (a block of one row of W or x); 16-byte chunk c of row r lies at
// c ^ row_swz(r), so that the 16 rows of an operand read, two per 256 bytes of banks, take 8
// distinct positions per row parity.
__device__ __forceinline__ int row_swz(int r) { return (r >> 1) & 7; }

// Feature staged at LDS row s: within each 32 rows, block b = s / 16 of the MFMA's 16 rows holds
// features 8 g + 4 b + e at row 4 g + e, so that a lane's accumulator elements of blocks 0 and 1
// are 8 consecutive features.
__device__ __forceinline__ int staged_feature(int s) {
  return (s & ~31) | ((s & 12) << 1) | ((s & 16) >> 2) | (s & 3);
}

// First feature and token of tile L: feature tiles vary fastest in groups of eight, the token
// tiles within a group. Workgroup b runs on XCD b % 8 and takes tile (b % 8) per_xcd + b / 8, so
// the tiles that run together on one L2 share their W and x rows.
__device__ __forceinline__ void tile_origin(const LinearArgs& a, int L, int tile_f, int tile_t, int& f0, int& t0) {
  constexpr int kGroupF = 8;
  const int grp = L / (kGroupF * a.n_ttiles);
  const int gf = min(kGroupF, a.n_ftiles - grp * kGroupF);
  const int rem = L - grp * kGroupF * a.n_ttiles;
  t0 = (rem / gf) * tile_t;
  f0 = (grp * kGroupF + rem % gf) * tile_f;
}

// Zeroes an operand's columns past the end of depth: lane group g4 holds the block's columns
// 16 g4 .. + 15 and 64 + 16 g4 .. + 15, `rem` (a multiple of 16) of the block's columns exist.
__device__ __forceinline__ void cut_tail(i32x8& op, int g4, int rem) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (16 * g4 >= rem) op[i] = 0;
    if (64 + 16 * g4 >= rem) op[4 + i] = 0;
  }
}

// Bias, rounding and stores of the results of a wave: block fa (16 staged rows) and token block
// tb; first feature f of the wave's blocks and first token t.
template <int FW, int NB>
__device__ __forceinline__ void store_results(const LinearArgs& a, const f32x4 (&acc)[FW][NB], int f, int t, int lane) {
  const int l16 = lane & 15, g4 = lane >> 4;
  if constexpr (FW % 2 == 0) {
#pragma unroll
    for (int fa = 0; fa < FW; fa += 2) {
      const int n = f + 16 * fa + 8 * g4;
      if (n >= a.feats) continue;   // (a multiple of 8)
      u32x4 b{0, 0, 0, 0};
      if (a.bias) b = *reinterpret_cast<const u32x4*>(a.bias + n);
#pragma unroll
      for (int tb = 0; tb < NB; ++tb) {
        const int row = t + 16 * tb + l16;
        if (row >= a.rows) continue;
        const f32x4 lo = acc[fa][tb], hi = acc[fa + 1][tb];
        *reinterpret_cast<u32x4*>(a.out + int64_t(row) * a.feats + n) =
            u32x4{pack_bf16x2(lo[0] + bf16_lo(b[0]), lo[1] + bf16_hi(b[0])),
                  pack_bf16x2(lo[2] + bf16_lo(b[1]), lo[3] + bf16_hi(b[1])),
                  pack_bf16x2(hi[0] + bf16_lo(b[2]), hi[1] + bf16_hi(b[2])),
                  pack_bf16x2(hi[2] + bf16_lo(b[3]), hi[3] + bf16_hi(b[3]))};
      }
    }
  } else {
#pragma unroll
    for (int fa = 0; fa < FW; ++fa) {
      const int n = f + 16 * fa + 4 * g4;
      if (n >= a.feats) continue;
      u32x2 b{0, 0};
      if (a.bias) b = *reinterpret_cast<const u32x2*>(a.bias + n);
#pragma unroll
      for (int tb = 0; tb < NB; ++tb) {
        const int row = t + 16 * tb + l16;
        if (row >= a.rows) continue;
        const f32x4 v = acc[fa][tb];
        *reinterpret_cast<u32x2*>(a.out + int64_t(row) * a.feats + n) =
            u32x2{pack_bf16x2(v[0] + bf16_lo(b[0]), v[1] + bf16_hi(b[0])),
                  pack_bf16x2(v[2] + bf16_lo(b[1]), v[3] + bf16_hi(b[1]))};
      }
    }
  }
}

// ---------------------------------------------------------------------------
// One tile of TF features x TT tokens per workgroup. Waves 4-7, one on each SIMD, copy; WF x WT of
// the waves 0-3 multiply, each FW = TF / 16 / WF feature blocks x NB = TT / 16 / WT token blocks
// over all of depth. A stage is PL blocks of 128 columns of the tile's rows; a ring of ST stages.
//
// At the barrier that starts step s, stage s + 1 has landed and stage s has been read into
// registers: step s multiplies those while it reads stage s + 1 into the other register set, and
// the copies that go out after the barrier (stage s + ST) replace stage s. Columns past the end
// of depth are copied from inside the row and zeroed in registers.
// ---------------------------------------------------------------------------
template <int TF, int TT, int PL, int ST, int WF, int WT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void fp8_linear_block_kernel(const LinearArgs a) {
  constexpr int FW = TF / 16 / WF, NB = TT / 16 / WT, ROWS = TF + TT;
  constexpr int PLANE = ROWS * kDepth, STAGE = PL * PLANE;
  constexpr int CW = PL * ROWS / 8 / 4 + 1;   // copies (8 rows each, and one of scales) per stage and copying wave
  // Scales come four blocks at a time (16 bytes a token, 64 tokens a copy), with every GS-th stage, in
  // a ring of NG slots: the tokens', then the tile's feature block's. A stage's scales are copied with it
  // or before it, and slot n is copied again only for a stage that replaces one behind it.
  constexpr int GS = 4 / PL, NG = GS == 1 ? ST : 4, TC = TT > 64 ? 2 : 1, SC_SLOT = (TC + 1) * 1024;
  constexpr int SCALES = ST * STAGE, UNUSED = SCALES + NG * SC_SLOT, LDS = UNUSED + 1024;
  static_assert(FW * 16 * WF == TF && NB * 16 * WT == TT && WF * WT <= 4 && PL * ROWS % 32 == 0, "even shares");
  static_assert(PL * GS == 4 && TT <= 128 && 128 % TF == 0, "two waves copy the tokens' scales, one the features'");
  static_assert((ST + GS - 1) / GS < NG || GS == 1, "scales are not replaced before they are read");
  static_assert(CW * (ST - 1) <= 63, "outstanding copies are counted in 6 bits");
  static_assert(LDS <= 160 * 1024, "LDS of one CU");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[LDS];
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  const int tile = (blockIdx.x & 7) * a.per_xcd + (blockIdx.x >> 3);
  if (tile >= a.n_ftiles * a.n_ttiles) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int f0, t0;
  tile_origin(a, tile, TF, TT, f0, t0);
  const int nk = (a.blocks + PL - 1) / PL;
  const int rem = a.depth - (a.blocks - 1) * kDepth;   // columns of the last block

  if (wave >= 4) {
    const int cw = wave - 4;
    uint32_t off[CW - 1];
#pragma unroll
    for (int i = 0; i < CW - 1; ++i) {
      const int r8 = 8 * ((cw + 4 * i) % (ROWS / 8)), row = r8 + (lane >> 3);
      const int c = ((lane & 7) ^ row_swz(row)) * 16;
      const int src = r8 < TF ? min(FW % 2 == 0 ? staged_feature(row) : row, a.feats - 1 - f0)
                              : min(row - TF, a.rows - 1 - t0);
      off[i] = uint32_t(src) * uint32_t(a.depth) + c;
    }
    const uint8_t* const wb = a.w + int64_t(f0) * a.depth;
    const uint8_t* const xb = a.x + int64_t(t0) * a.depth;
    // Scales: copying waves 0 (and 1) bring the tokens', wave 2 the features'; in a stage without any,
    // and in the other waves, a copy that nothing reads keeps the count of copies.
    const bool mine = cw < TC || cw == 2;
    const u32x4 d_s = cw == 2 ? buffer(a.ws + int64_t(f0 / 128) * a.blocks, uint32_t(a.blocks) * 4)
                              : buffer(a.xs + int64_t(t0) * a.blocks, uint32_t(min(TT, a.rows - t0)) * a.blocks * 4);
    const uint32_t offs = cw < TC ? uint32_t(cw * 64 + lane % TT) * uint32_t(a.blocks) * 4 : 0;
    auto issue = [&](int s, int slot) __attribute__((always_inline)) {
      const bool now = mine && s % GS == 0;
      buffer16_to_lds(d_s, now ? offs + uint32_t(PL * s) * 4 : 0,
                      lds0 + (now ? SCALES + (s / GS) % NG * SC_SLOT + (cw == 2 ? TC : cw) * 1024 : UNUSED));
#pragma unroll
      for (int i = 0; i < CW - 1; ++i) {
        const int n = cw + 4 * i, pl = n / (ROWS / 8), r8 = 8 * (n % (ROWS / 8));
        const int kb = min(PL * s + pl, a.blocks - 1);   // (a block past the last: that one again, not used)
        const uint8_t* base = (r8 < TF ? wb : xb) + kb * kDepth;
        uint32_t o = off[i];
        if (rem < kDepth && kb == a.blocks - 1) {   // columns past the end: the row's last 16 instead
          const int c = ((lane & 7) ^ row_swz(r8 + (lane >> 3))) * 16;
          o -= uint32_t(max(0, c - (rem - 16)));
        }
        copy16_to_lds(base, o, lds0 + slot * STAGE + n * 1024);
      }
    };
#pragma unroll
    for (int i = 0; i < ST; ++i)
      if (i < nk) issue(i, i);
    if (nk >= ST) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(CW * (ST - 1)));
    else __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
    interval_barrier();   // stage 0 has landed
    int slot = 0;
    for (int s = 0; s < nk; ++s) {
      // stage s + 1 has landed; stages s + 2 .. s + ST - 1 stay in flight
      if (s + ST <= nk) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(CW * (ST - 2)));
      else __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
      interval_barrier();
      if (s + ST < nk) issue(s + ST, slot);
      slot = slot == ST - 1 ? 0 : slot + 1;
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
    return;
  }

  const int l16 = lane & 15, g4 = lane >> 4;
  const int wf = wave % WF, wt = wave / WF;   // (a wave with wt >= WT only takes part in the barriers)
  if (wt >= WT) {
    for (int s = -1; s < nk; ++s) interval_barrier();
    return;
  }
  const int so[2] = {l16 * kDepth + ((g4 ^ row_swz(l16)) << 4), l16 * kDepth + (((4 + g4) ^ row_swz(l16)) << 4)};
  const int frow = 16 * FW * wf, trow = TF + 16 * NB * wt;
  constexpr int NOP = FW + NB;
  i32x8 op[2][PL][NOP];   // operands of two stages: feature blocks, then token blocks
  auto read = [&](int buf, int slot, int pl, int i) __attribute__((always_inline)) {
    const uint8_t* p = lds + slot * STAGE + pl * PLANE + ((i < FW ? frow + 16 * i : trow + 16 * (i - FW)) * kDepth);
    const u32x4 lo = *reinterpret_cast<const u32x4*>(p + so[0]), hi = *reinterpret_cast<const u32x4*>(p + so[1]);
    op[buf][pl][i] = i32x8{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
  };
  float xsv[2][PL][NB], wsv[2][PL];   // scales of the lane's tokens and of the features
  auto read_scales = [&](int buf, int s) __attribute__((always_inline)) {
    const float* p = reinterpret_cast<const float*>(lds + SCALES + (s / GS) % NG * SC_SLOT) + s % GS * PL;
#pragma unroll
    for (int pl = 0; pl < PL; ++pl) {
      wsv[buf][pl] = p[TC * 256 + pl];
#pragma unroll
      for (int tb = 0; tb < NB; ++tb) xsv[buf][pl][tb] = p[(16 * (NB * wt + tb) + l16) * 4 + pl];
    }
  };
  f32x4 acc[FW][NB];
#pragma unroll
  for (int fa = 0; fa < FW; ++fa)
#pragma unroll
    for (int tb = 0; tb < NB; ++tb) acc[fa][tb] = f32x4{0.f, 0.f, 0.f, 0.f};

  interval_barrier();   // stage 0 has landed
  read_scales(0, 0);
#pragma unroll
  for (int pl = 0; pl < PL; ++pl)
#pragma unroll
    for (int i = 0; i < NOP; ++i) read(0, 0, pl, i);
  constexpr int N = PL * FW * NB;        // products of a step
  constexpr int RD = (PL * NOP + N - 1) / N;   // operand reads beside each
  constexpr int LAG = 3;                 // a product's scaling comes this many products later
  int slot = 0;
  auto step = [&](int s, auto bufc) __attribute__((always_inline)) {
    constexpr int buf = decltype(bufc)::value;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // this wave's reads of stage s are complete
    interval_barrier();
    const int next = slot == ST - 1 ? 0 : slot + 1;
    float sc[PL][NB];
#pragma unroll
    for (int pl = 0; pl < PL; ++pl)
#pragma unroll
      for (int tb = 0; tb < NB; ++tb)   // (a block past the last counts nothing)
        sc[pl][tb] = PL * s + pl < a.blocks ? xsv[buf][pl][tb] * wsv[buf][pl] : 0.f;
    read_scales(buf ^ 1, s + 1);
    if (rem < kDepth && PL * s + PL >= a.blocks) {   // (the same for the whole grid)
#pragma unroll
      for (int pl = 0; pl < PL; ++pl)
        if (PL * s + pl == a.blocks - 1) {
#pragma unroll
          for (int i = 0; i < NOP; ++i) cut_tail(op[buf][pl][i], g4, rem);
        }
    }
    f32x4 part[LAG + 1];
    auto scale = [&](int n) __attribute__((always_inline)) {
      const int pl = n / (FW * NB), tb = n / FW % NB, fa = n % FW;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[fa][tb][e] = fmaf(part[n % (LAG + 1)][e], sc[pl][tb], acc[fa][tb][e]);
      asm volatile("" : "+v"(acc[fa][tb]));   // (else the compiler scales them all at the end)
    };
#pragma unroll
    for (int n = 0; n < N + LAG; ++n) {
      if (n < N) {
        const int pl = n / (FW * NB), tb = n / FW % NB, fa = n % FW;
        part[n % (LAG + 1)] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            op[buf][pl][fa], op[buf][pl][FW + tb], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < RD; ++i)
          if (n * RD + i < PL * NOP) read(buf ^ 1, next, (n * RD + i) / NOP, (n * RD + i) % NOP);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (n >= LAG) scale(n - LAG);
      __builtin_amdgcn_sched_barrier(0);
    }
    slot = next;
  };
  int s = 0;
  for (; s + 1 < nk; s += 2) {
    step(s, std::integral_constant<int, 0>{});
    step(s + 1, std::integral_constant<int, 1>{});
  }
  if (s < nk) step(s, std::integral_constant<int, 0>{});
  store_results<FW, NB>(a, acc, f0 + frow, t0 + 16 * NB * wt, lane);
}

// ---------------------------------------------------------------------------
// Many tokens: 256 features x 128 C tokens (C = 1, 2), persistent workgroups of 8 waves, one per CU,
// walking the tiles of their XCD's range. Wave (wf, wt) owns 64 features and 64 C tokens.
//
// The two waves of a SIMD (w and w + 4) alternate: while one issues 16 products (each depth 128,
// 32 cycles), with the scaling of an earlier product beside each, the other reads its next
// operands and issues copies; a barrier ends each interval and the second group runs one
// interval behind. A step (one block of 128 columns) takes C reading intervals: c = 0 reads the
// W rows and the first 64 token rows of each group, c = 1 the other 64.
//
// LDS: a ring of nine units of 128 rows (16 KB). A step has 2 + C: two of W rows, then the token
// rows of each c. Copies run two steps ahead.
// C = 2: group 0 reads step s in intervals 4 s and 4 s + 2, group 1 in 4 s + 1 and 4 s + 3.
//  - unit 0 of step s + 2 (and its scales) is copied from interval 4 s on, in the place of unit 3 of
//    step s - 1, last read in 4 s - 1;
//  - units 1 .. 3 of step s + 2 from interval 4 s + 2 on, in the places of units 0 .. 2 of step s, last
//    read in 4 s + 1;
//  - a wave's copies of step s + 1 have landed at the end of its second reading interval of step s
//    (the nine younger copies stay in flight), at most 4 s + 3: interval 4 s + 4 may read them.
// C = 1: group 0 reads step s in interval 2 s, group 1 in 2 s + 1. Step s + 2 is copied from interval
// 2 s on in the places of step s - 1, last read in 2 s - 1; a wave's copies of step s + 1 have landed
// at the end of interval 2 s + 1 (the seven younger ones stay in flight).
// Scales come four blocks at a time (16 bytes a token) with a tile's every fourth step, in a ring of
// three slots: two steps ahead of the reads, a slot's last reader is a step behind in any case.
// The cursor of the copies runs on across tiles, so the next tile's first steps arrive during a
// tile's end.
// ---------------------------------------------------------------------------
template <int C>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
void fp8_linear_tile_kernel(const LinearArgs a) {
  constexpr int TF = 256, TT = 128 * C, UNIT = 128 * kDepth, UNITS = 9, PER = 2 + C;
  constexpr int SCALES = UNITS * UNIT, SC_SLOT = (2 * C + 1) * 1024, UNUSED = SCALES + 3 * SC_SLOT;
  constexpr int LDS = UNUSED + 1024;
  static_assert(LDS <= 160 * 1024, "LDS of one CU");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[LDS];
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
  const int xcd = blockIdx.x & 7, wg_per_xcd = gridDim.x >> 3;
  const int tile_end = min((xcd + 1) * a.per_xcd, a.n_ftiles * a.n_ttiles);
  int tile = xcd * a.per_xcd + (blockIdx.x >> 3);
  if (tile >= tile_end) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nk = a.blocks;
  const int rem = a.depth - (nk - 1) * kDepth;   // columns of the last block

  // ---- copy cursor. A wave copies 16 of the 128 rows of each unit, 8 at a time. The copies are
  // buffer loads, whose descriptor ends with the tensor: rows past the last tile's end and
  // columns behind the last row's read nothing (what lies there in LDS is not used, or cut), so
  // the lane offsets are the same for every tile and step.
  int c_tile = tile, c_step = 0, c_slot = 0, c_unit = 0;   // c_unit: ring place of the cursor's next unit
  u32x4 d_w, d_x, d_s;   // of the cursor's tile and step: W, x, and the scales that this wave copies
  uint32_t offw[2], offx[2];   // of the tile's first W unit and first x unit
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // rows 16 wave + 8 i ..
    const int r = 16 * wave + 8 * i + (lane >> 3);
    const uint32_t c = ((lane & 7) ^ row_swz(r)) * 16;
    offw[i] = uint32_t(staged_feature(r)) * uint32_t(a.depth) + c;
    offx[i] = uint32_t((r & 63) + (r >> 6) * (64 * C)) * uint32_t(a.depth) + c;
  }
  // waves 0 .. 2 C - 1 copy the tokens' scales, wave 2 C the two feature blocks' (32 lanes each); the
  // others, and all in the steps between, a line that nothing reads, to keep the count of copies
  const uint32_t offs = uint32_t(wave < 2 * C ? 64 * wave + lane : lane >> 5) * uint32_t(nk) * 4;
  auto cursor_tile = [&]() __attribute__((always_inline)) {
    int f0, t0;
    tile_origin(a, c_tile, TF, TT, f0, t0);
    const uint32_t nf = min(TF, a.feats - f0), nt = min(TT, a.rows - t0);
    d_w = buffer(a.w + int64_t(f0) * a.depth, nf * a.depth);
    d_x = buffer(a.x + int64_t(t0) * a.depth, nt * a.depth);
    if (wave < 2 * C) d_s = buffer(a.xs + int64_t(t0) * nk, nt * nk * 4);
    else d_s = buffer(a.ws + int64_t(f0 / 128) * nk, (nf + 127) / 128 * nk * 4);
  };
  cursor_tile();
  auto copy8 = [&](u32x4 d, uint32_t off, int i, int unit) __attribute__((always_inline)) {
    buffer16_to_lds(d, off, lds0 + unit * UNIT + (16 * wave + 8 * (i & 1)) * kDepth);
  };
  auto unit_add = [](int u, int n) { return u + n >= UNITS ? u + n - UNITS : u + n; };
  auto advance = [](u32x4& d, uint32_t bytes) __attribute__((always_inline)) {
    const uint64_t p = ((uint64_t(d[1]) << 32) | d[0]) + bytes;
    d[0] = uint32_t(p);
    d[1] = uint32_t(p >> 32);
    d[2] -= bytes;
  };
  auto issue_first = [&]() __attribute__((always_inline)) {   // three copies: scales, unit 0
    const bool now = wave <= 2 * C && (c_step & 3) == 0;
    buffer16_to_lds(d_s, now ? offs : 0, lds0 + (now ? SCALES + c_slot * SC_SLOT + wave * 1024 : UNUSED));
    copy8(d_w, offw[0], 0, c_unit);
    copy8(d_w, offw[1], 1, c_unit);
  };
  auto issue_rest = [&]() __attribute__((always_inline)) {    // 2 + 2 C copies; on to the next step
#pragma unroll
    for (int i = 0; i < 2; ++i) copy8(d_w, offw[i] + 128u * uint32_t(a.depth), i, unit_add(c_unit, 1));
#pragma unroll
    for (int i = 0; i < 2 * C; ++i)
      copy8(d_x, offx[i & 1] + uint32_t(i >> 1) * 64u * uint32_t(a.depth), i, unit_add(c_unit, 2 + (i >> 1)));
    c_unit = unit_add(c_unit, PER);
    ++c_step;
    if ((c_step & 3) == 0 || c_step >= nk) c_slot = c_slot == 2 ? 0 : c_slot + 1;
    if (c_step < nk) {
      advance(d_w, kDepth);
      advance(d_x, kDepth);
      if ((c_step & 3) == 0) advance(d_s, 16);
    } else if (c_tile + wg_per_xcd < tile_end) {
      c_tile += wg_per_xcd;
      c_step = 0;
      cursor_tile();
    } else {
      --c_step;   // past the last tile: its last step again, which nothing reads
    }
  };

  // ---- operand rows of this wave
  const int wf = wave & 3, wt = wave >> 2;
  const int l16 = lane & 15, g4 = lane >> 4;
  const int so[2] = {l16 * kDepth + ((g4 ^ row_swz(l16)) << 4), l16 * kDepth + (((4 + g4) ^ row_swz(l16)) << 4)};
  auto operand = [&](int unit, int row) __attribute__((always_inline)) -> i32x8 {
    const uint8_t* p = lds + unit * UNIT + row * kDepth;
    const u32x4 lo = *reinterpret_cast<const u32x4*>(p + so[0]), hi = *reinterpret_cast<const u32x4*>(p + so[1]);
    return i32x8{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
  };
  f32x4 acc[4][4 * C];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int fa = 0; fa < 4; ++fa)
#pragma unroll
      for (int tb = 0; tb < 4 * C; ++tb) acc[fa][tb] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  clear();
  constexpr int FLY = 5 + 2 * C;   // copies of one step
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    issue_first();
    issue_rest();
  }
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(FLY));
  interval_barrier();
  if (wt == 1) interval_barrier();   // the second group runs one interval behind

  int unit = 0, slot = 0;
  for (; tile < tile_end; tile += wg_per_xcd) {
    for (int k = 0; k < nk; ++k) {
      i32x8 af[4], bx[4];
      const bool tail = rem < kDepth && k == nk - 1;
      const float* const sc = reinterpret_cast<const float*>(lds + SCALES + slot * SC_SLOT) + (k & 3);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        if (c == 0) {
          const int wu = unit_add(unit, wf >> 1);
#pragma unroll
          for (int fa = 0; fa < 4; ++fa) af[fa] = operand(wu, (wf & 1) * 64 + 16 * fa);
        }
        const int xu = unit_add(unit, 2 + c);
        float f[4];
        const float w = sc[C * 512 + (wf >> 1) * 128];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) {
          bx[tb] = operand(xu, wt * 64 + 16 * tb);
          f[tb] = sc[(wt * 64 * C + c * 64 + 16 * tb + l16) * 4];
        }
        if (c == 0) issue_first();
        if (c == C - 1) issue_rest();
        __builtin_amdgcn_sched_barrier(0);
        if (c == C - 1 && (C == 2 || wt == 1)) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(FLY));
        else __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(63));
#pragma unroll
        for (int tb = 0; tb < 4; ++tb) f[tb] *= w;
        if (__builtin_expect(tail, 0)) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (c == 0) cut_tail(af[i], g4, rem);
            cut_tail(bx[i], g4, rem);
          }
        }
        interval_barrier();
        __builtin_amdgcn_s_setprio(1);
        constexpr int LAG = 3;
        f32x4 part[LAG + 1];
#pragma unroll
        for (int n = 0; n < 16 + LAG; ++n) {
          if (n < 16)
            part[n % (LAG + 1)] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                af[n & 3], bx[n >> 2], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
          if (n >= LAG) {
            const int m = n - LAG;
            f32x4& to = acc[m & 3][4 * c + (m >> 2)];
#pragma unroll
            for (int e = 0; e < 4; ++e) to[e] = fmaf(part[m % (LAG + 1)][e], f[m >> 2], to[e]);
            asm volatile("" : "+v"(to));   // (else the compiler scales all of them later and holds 16 products)
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (C == 1 && wt == 0) __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(FLY));
        interval_barrier();
      }
      unit = unit_add(unit, PER);
      if ((k & 3) == 3 || k == nk - 1) slot = slot == 2 ? 0 : slot + 1;
    }
    int f0, t0;
    tile_origin(a, tile, TF, TT, f0, t0);
    store_results<4, 4 * C>(a, acc, f0 + 64 * wf, t0 + 64 * C * wt, lane);
    clear();
  }
  if (wt == 0) interval_barrier();
  // the copies past the last tile must not outlive the workgroup's LDS
  __builtin_amdgcn_s_waitcnt(waitcnt_vm_lgkm0(0));
}

// The tile shapes, and what a call costs with each: tiles in rounds of one per CU, a round
// fixed + blocks * us (blocks = depth / 128), where us goes from `light` (few CUs busy) to `full`
// (all busy). The shape with the smallest estimate is taken; all give the same bits. The constants
// are fits to calls in captured graphs at 159 sizes (T = 1 .. 16,128, eight pairs of depth and
// features from 256 x 384 to 8,192 x 8,192), all shapes at each (profiles/fp8_linear_shapes.txt): the choice is
// within 8.3 % of the best shape at each and 0.24 % on average; leaving out one shape costs 9 % (32 x 16)
// to 87 % (128 x 128) at its sizes. Examples, us, 6,144 features, depth 4,096, the 128 x 128 tile
// against the chosen one: T = 16: 17.2 / 6.5 (32 x 16); 64: 17.6 / 9.5 (32 x 64); 128: 18.3 / 11.4
// (64 x 64); 256: 18.9; 1,024: 40; 4,096: 127 / 104 (256 x 256); 16,128: 494 / 345 (2.36 PFLOP/s; 334 to 375
// on several cards).
//
// What bounds them: up to 64 tokens the read of W (25 MB in 6.5 us, 3 of them start and end of a
// workgroup, where the last-level cache holds W; 9.7 from HBM); the tiles of 64 to 128 the copies into LDS
// (96 KB in flight a CU, about 60 GB/s each, 11 TB/s over all), so that a step of 128 x 128 takes 1,200
// cycles beside 512 of products; 256 x 256 the vector work beside the products: an interval takes 816
// cycles, 665 without the scaling, 512 of them matrix work (matrix pipe busy 57 %, clock 1.94 GHz).
struct LinearShape {
  int tile_f, tile_t;
  bool persistent;
  double fixed, light, full;   // us
  void (*kernel)(LinearArgs);
};
const LinearShape kShapes[] = {
    {128, 128, false, 4.72, 0.423, 0.512, fp8_linear_block_kernel<128, 128, 1, 4, 2, 2>},
    {64, 64, false, 3.60, 0.244, 0.217, fp8_linear_block_kernel<64, 64, 2, 4, 2, 2>},
    {32, 64, false, 3.32, 0.219, 0.179, fp8_linear_block_kernel<32, 64, 2, 6, 2, 2>},
    {32, 32, false, 3.14, 0.126, 0.105, fp8_linear_block_kernel<32, 32, 4, 4, 2, 2>},
    {32, 16, false, 3.10, 0.113, 0.095, fp8_linear_block_kernel<32, 16, 4, 6, 2, 1>},
    {256, 256, true, 8.47, 1.089, 1.637, fp8_linear_tile_kernel<2>},
    {256, 128, true, 5.89, 1.079, 1.116, fp8_linear_tile_kernel<1>},
};

const LinearShape& pick_shape(int64_t rows, int64_t feats, int64_t blocks) {
  const LinearShape* best = nullptr;
  double best_us = 0;
  for (const LinearShape& s : kShapes) {
    const int64_t tiles = ((feats + s.tile_f - 1) / s.tile_f) * ((rows + s.tile_t - 1) / s.tile_t);
    const int64_t rounds = tiles / cw::kNumCu, rest = tiles % cw::kNumCu;
    double us = double(rounds) * (s.fixed + double(blocks) * s.full);
    if (rest > 0) us += s.fixed + double(blocks) * (s.light + (s.full - s.light) * double(rest) / cw::kNumCu);
    if (!best || us < best_us) {
      best = &s;
      best_us = us;
    }
  }
  return *best;
}

}  // namespace

extern "C" cw_status cw_fp8_linear(const void* x8, const float* x_scale, const void* w8, const float* w_scale,
                                   const void* bias, int64_t rows, int32_t features, int32_t hidden, void* out,
                                   void* stream) {
  if (rows < 0) return cw::fail(CW_EINVAL, "fp8_linear: rows must be >= 0");
  if (!w8 || !w_scale || (rows > 0 && (!x8 || !x_scale || !out)))
    return cw::fail(CW_EINVAL, "fp8_linear: a required pointer is NULL");
  if (hidden < 16 || hidden % 16 != 0 || hidden > (1 << 20))
    return cw::fail(CW_EUNSUPPORTED, "fp8_linear: hidden must be a multiple of 16 in [16, 2^20]");
  if (features < 16 || features % 16 != 0 || features > (1 << 20))
    return cw::fail(CW_EUNSUPPORTED, "fp8_linear: features must be a multiple of 16 in [16, 2^20]");
  if (rows > (1 << 22)) return cw::fail(CW_EUNSUPPORTED, "fp8_linear: more than 2^22 rows");
  if (((reinterpret_cast<uintptr_t>(x8) | reinterpret_cast<uintptr_t>(w8) | reinterpret_cast<uintptr_t>(bias) |
        reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return cw::fail(CW_EINVAL, "fp8_linear: pointers must be 16-byte aligned");
  if (rows == 0) return cw::ok();
  LinearArgs a;
  a.x = static_cast<const uint8_t*>(x8);
  a.xs = x_scale;
  a.w = static_cast<const uint8_t*>(w8);
  a.ws = w_scale;
  a.bias = static_cast<const uint16_t*>(bias);
  a.out = static_cast<uint16_t*>(out);
  a.rows = int(rows);
  a.feats = features;
  a.depth = hidden;
  a.blocks = (hidden + kDepth - 1) / kDepth;
  const LinearShape& sh = pick_shape(rows, features, a.blocks);
  a.n_ftiles = (features + sh.tile_f - 1) / sh.tile_f;
  a.n_ttiles = int((rows + sh.tile_t - 1) / sh.tile_t);
  const int64_t per_xcd = (int64_t(a.n_ftiles) * a.n_ttiles + cw::kNumXcd - 1) / cw::kNumXcd;
  const int64_t grid = (sh.persistent ? std::min<int64_t>(per_xcd, cw::kNumCu / cw::kNumXcd) : per_xcd) * cw::kNumXcd;
  // (a launch has fewer than 2^32 threads; the kernels count tiles in 32 bits)
  if (grid > UINT32_MAX / 512 || per_xcd * cw::kNumXcd > INT32_MAX)
    return cw::fail(CW_EUNSUPPORTED, "fp8_linear: too many tiles");
  a.per_xcd = int(per_xcd);
  hipLaunchKernelGGL(sh.kernel, dim3(unsigned(grid)), dim3(512), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, std::string("fp8_linear launch: ") + hipGetErrorString(e));
  return cw::ok();
}
