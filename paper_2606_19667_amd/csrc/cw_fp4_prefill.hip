// Causal attention of suffix rows over a 4-bit paged KV cache (gfx950).
//
// Paper Sec. 1 and 2.1: with a reused prefix only the suffix tokens are prefilled; they attend
// fully over the prefix and causally over themselves. Here keys and values are e2m1 codes with
// a power-of-two scale per token and 32 columns (cw_fp4.hip has the layout), which holds 3.76
// times the prefix of a bf16 cache. A value is a bfloat16 value: the codes are converted without
// rounding, and what follows is attention over bf16 keys and values.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <string>

#include "cw_fp4.h"
#include "cw_internal.h"

namespace {

using namespace cw4;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef const __attribute__((address_space(4))) int32_t cint32_t;

constexpr int kStep = cw::kKvTile;            // keys of a step (four blocks)
constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kBlocks = kStep / kBs;
static_assert(kWaves * 32 == cw::kTileRows, "one 32-column MFMA block per wave");
static_assert(kWaves == 2 * kBlocks, "a wave stages one block of one tensor");
constexpr int kMergeParts = 8;                // parts of a row that are merged in turn; more: side by side, for
constexpr int64_t kJoinRows = 16384;          // this many rows at most (a workgroup each)
constexpr float kMaxSum = 0x1p30f;            // a row's base moves when its sum exceeds this

// (Maxima that a NaN passes through: with NaN honoured fmaxf would quiet each operand first.)
__device__ __forceinline__ float max_pair32(float x) {   // of this lane and lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_pair32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

struct PrefillArgs {
  const uint16_t* q;
  const uint8_t* pages;
  const int32_t* bt;
  const int32_t* plan;   // device copy of the whole plan (header, then entries)
  uint16_t* out;
  float* part_o;         // split plans: fp32 [splits][part_rows][D], normalised
  float* part_lse;       // and base-2 log-sum-exp [splits][part_rows]
  int64_t part_rows;     // total suffix rows * hq
  int32_t bt_stride, hq, hkv, group, per_tile, num_blocks, num_entries;
  float c_log2;
  uint32_t fp_lo, fp_hi; // the batch fingerprint the host validated
};

template <int D>
struct Geom {
  static constexpr int KP = 2 * D + 16;           // LDS bytes from one K row to the next (bf16, padded:
                                                  // the 16-byte reads of 8 rows lie on distinct banks)
  static constexpr int VP = 2 * D + 64;           // the same of V: the 4 rows x 64 bytes that half a wave
                                                  // reads at once (transposing) lie on distinct banks
  static constexpr int KTILE = kStep * KP;
  static constexpr int STAGE = KTILE + kStep * VP;
  static constexpr int PARTS = 4;                 // of a lane's codes of a block: D / 16 codes, one LDS write
  static constexpr int UNITS = D / 16;            // of 4 codes
  static constexpr int KS = D / 16;               // MFMA k-steps over D
  static constexpr int DT = D / 32;               // 32-row output tiles over D
  static constexpr int OUT = 32 * (64 * 2 + 16);  // per-wave output staging: 32 rows of 64 columns
};

// Work as in the plan: an entry is (request, KV head g, a run of T suffix rows); 256 packed
// rows of an entry are the G query heads of g over T = 256 / G positions, 32 a wave. Workgroup
// w runs entries w, w + grid, ...; keys come in steps of 64, and the steps of all entries of a
// queue form one stream.
//  * A step's four blocks go through registers into LDS: wave w takes K (w even) or V (w odd)
//    of block w / 2, D / 8 bytes a lane in one load, converts the codes to bf16 (exact) and writes
//    rows. So each code is converted once per workgroup, not once per wave. Rows past the prompt
//    and blocks outside the pool are zeros.
//  * S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16; K row pi(i), pi swapping bits
//    2 and 3, is read into A row i, so that the score registers of a lane are its P^T operand:
//    register e of half h holds key 32 h + 16 (e / 8) + 8 (lane / 32) + e % 8. V^T comes from
//    token-major rows by transposing LDS reads.
//  * softmax_scale costs one multiply-add per score, with the row's base. P is rounded to bf16 for the
//    product, and the row's sum takes the rounded values. Q is not rounded again.
//
// The two waves of a SIMD alternate. A step j of a wave takes two intervals, each ended by a
// workgroup barrier:
//   softmax(j):   2^x packed to bf16, row sums (vector work)
//   products(j):  O^T += V(j)^T P(j)^T, then S(j + 1) = K(j + 1) Q^T (matrix work); beside the last
//                 products four codes each of step j + 2 are converted and written to LDS, then the loads
//                 of step j + 3 go out
// Waves 4-7 (group 1) run one interval behind waves 0-3. After an entry's last step S(j + 1) is the
// next entry's first, so only the output and the change of queries come between two entries.
//
// Ring of three stages. Let softmax(s) of group 0 be interval 2 s, of group 1 2 s + 1; products(s) reads
// V(s) and K(s + 1) in 2 s + 1 and 2 s + 2, the first V operands an interval earlier. Step x
// is written in products(x - 2), 2 x - 3 and 2 x - 2, and first read (K) in 2 x - 1; the stage that it
// replaces (step x - 3) was last read in 2 x - 4.
//
// 8 requests of 2,112 rows behind 3,136 keys, 32 / 8 heads of 128: 960 to 1,005 us by card, 1.15 to 1.21 PFLOP/s, where a
// library product of 8,192^3 in bf16 reaches 1.18 to 1.40: the matrix pipe is busy 58 % of the cycles at 2.0 GHz, and a fourth
// less matrix work takes 13 % off, 32 multiply-adds less of the softmax nothing. A step of lightly loaded units is 1.2 to
// 1.4 us. 6 x ~411 rows behind ~700 keys, 28 / 4 heads, 42 to 46 us by card (one card: 41.5 in a loop and 42.2 in a captured
// graph on the same data, 44.1 and 43.2 on three inputs in turn): the longest entry's 24 steps, behind a start in which
// every workgroup reads its queries and three steps' pages (29 MB).
//
// SPLIT: the entries are runs of a tile's keys (a plan of several runs), and each writes its part, zeros and
// -inf for rows that see none of the run's keys. A run of no steps goes through one that no row sees.
template <int D, bool SPLIT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void suffix_prefill_fp4_kernel(const PrefillArgs a) {
  using G = Geom<D>;
  constexpr int KS = G::KS, DT = G::DT, RING = 3;
  using Lane = typename Piece<D>::Lane;
  __shared__ __attribute__((aligned(16))) uint8_t lds[RING * G::STAGE + kWaves * G::OUT];
  static_assert(RING * G::STAGE + kWaves * G::OUT <= 160 * 1024, "LDS of one CU");

  cint32_t* const plan = reinterpret_cast<cint32_t*>(reinterpret_cast<uintptr_t>(a.plan));
  if (uint32_t(plan[cw::kHdrFpLo]) != a.fp_lo || uint32_t(plan[cw::kHdrFpHi]) != a.fp_hi) return;
  const int grid = int(gridDim.x);
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const bool group1 = wave >= 4;

  // ---- plan entries, word l % 16 in lane l; one that is not this batch's ends the queue. (Vector
  // loads, here and below: a scalar load in flight would have to land before any LDS result.)
  const int32_t* const ents = a.plan + cw::kPlanHeaderWords + (lane & 15);
  auto fetch = [&](int e) __attribute__((always_inline)) -> int32_t {
    return ents[int64_t(min(e, a.num_entries - 1)) * cw::kPlanEntryWords];
  };
  auto word = [](int32_t d, int i) __attribute__((always_inline)) -> int { return __builtin_amdgcn_readlane(d, i); };
  auto valid = [&](int32_t d, int e) __attribute__((always_inline)) -> bool {
    return e < a.num_entries && word(d, cw::kEntR) >= 0 &&
           uint32_t(word(d, cw::kEntCheck)) == cw::entry_tag(a.fp_lo, a.fp_hi, uint32_t(e));
  };
  // ---- staging: this wave's tensor and block slot, and the cursor of its loads
  const bool is_v = (wave & 1) != 0;
  const int bs = wave >> 1;
  const int u16 = lane >> 4, c16 = lane & 15;
  // Keys: lane l holds the columns D / 4 (l % 4) .. of row l / 4, part n their n-th sixteenth of the row.
  // Values: the columns D / 16 (l % 16) .. of rows 4 (l / 16) .. + 3, part n of row n of them.
  const int sinc = is_v ? G::VP : D / 8;   // LDS bytes from one part to the next
  const int sdst = is_v ? G::KTILE + (bs * kBs + 4 * u16) * G::VP + c16 * (D / 8)
                        : (bs * kBs + lane / 4) * G::KP + lane % 4 * (D / 2);
  // The word with the lane's scales: a token's (D = 128; two tokens', 64), of which a key lane takes one for
  // all its parts, or the column group's of the four rows.
  const int soff = is_v ? kValueScales<D> + c16 / (512 / D) * kBs + 4 * u16
                        : kKeyScales<D> + (D == 128 ? lane / 4 : lane / 8) * 4;
  const uint32_t ssel = is_v ? 0x03020100u : uint32_t(D == 128 ? lane % 4 : lane % 8 / 2) * 0x01010101u;
  const int coff = (is_v ? kValues<D> : 0) + lane * (D / 8);
  // Table words come up to 64 steps (a chunk: of one entry) at a time, step i's in lane i: what a step loads
  // by itself is its codes and scales, at a scalar base. While a chunk is loaded the words of the next one
  // are on their way.
  int ce = blockIdx.x;          // index of the entry in e_next, which the cursor takes next
  int32_t e_next = fetch(ce);
  int e_left = 0;               // steps of the newest entry behind the next chunk
  int n_left = 0, n_keys = 0;   // the next chunk: steps; keys of the prompt from the first of this wave's block on
  uint32_t n_off = 0, n_max = 0;             // table word of the block, and of the prompt's last one (bytes)
  const int32_t* n_row = a.bt;
  const uint8_t* n_pages = a.pages;          // of the entry's KV head
  int32_t n_ids = 0;
  int c_left = 0, c_keys = 0, c_at = 0;      // the same of the current chunk, and its next step
  const uint8_t* c_pages = a.pages;
  int32_t c_ids = 0;
  const uint32_t blk_bytes = uint32_t(a.hkv) * kPage<D>;   // (2^16 heads at most: below 2^28)
  // Past the queue's last entry the cursor stays behind that prompt's end: what it loads is staged as zeros.
  auto next_chunk = [&]() __attribute__((always_inline)) {
    if (e_left > 0) {
      n_keys -= 64 * kStep;
      n_off += 64 * 4 * kBlocks;
    } else if (valid(e_next, ce)) {
      const int kbeg = word(e_next, cw::kEntKbeg), L = word(e_next, cw::kEntL), g = word(e_next, cw::kEntG);
      e_left = word(e_next, cw::kEntKend) - kbeg;
      n_keys = L - (kbeg * kBlocks + bs) * kBs;
      if (SPLIT && e_left == 0) {   // a run of no steps: one of zeros
        e_left = 1;
        n_keys = 0;
      }
      n_off = uint32_t(kbeg * kBlocks + bs) * 4;
      n_max = uint32_t((L + kBs - 1) / kBs - 1) * 4;
      n_row = a.bt + int64_t(word(e_next, cw::kEntR)) * a.bt_stride;
      n_pages = a.pages + int64_t(g) * kPage<D>;
      ce += grid;
      e_next = fetch(ce);
    } else {
      e_left = INT32_MAX;
      n_keys = 0;
    }
    n_left = min(e_left, 64);
    e_left -= n_left;
    n_ids = *reinterpret_cast<const int32_t*>(reinterpret_cast<const uint8_t*>(n_row) +
                                              min(n_off + uint32_t(lane) * (4 * kBlocks), n_max));
  };
  auto take_chunk = [&]() __attribute__((always_inline)) {
    c_left = n_left;
    c_keys = n_keys;
    c_pages = n_pages;
    c_ids = n_ids;
    c_at = 0;
    next_chunk();
  };
  Lane raw{};
  uint32_t raw_exp = 0;
  int raw_keys = 0;   // rows of the loaded block inside the prompt; 0 or less: none
  auto load = [&]() __attribute__((always_inline)) {
    // (a block outside the pool loads block 0 and is staged as zeros)
    const uint32_t word_id = uint32_t(__builtin_amdgcn_readlane(c_ids, c_at & 63));
    const bool ok = word_id < uint32_t(a.num_blocks);
    raw_keys = __builtin_amdgcn_readfirstlane(ok ? c_keys : 0);
    const uint8_t* page = c_pages + uint64_t(ok ? word_id : 0) * blk_bytes;
    raw = *reinterpret_cast<const Lane*>(page + uint32_t(coff));
    raw_exp = *reinterpret_cast<const uint32_t*>(page + uint32_t(soff));
    c_keys -= kStep;
    ++c_at;
    if (__builtin_expect(--c_left == 0, 0)) take_chunk();
  };
  // The loaded block to LDS, 4 codes at a time; with a part's last ones it is written.
  u32x4 wide{0, 0, 0, 0};
  auto widen4 = [&](int n) __attribute__((always_inline)) {   // codes 4 n .. + 3
    constexpr int PER = G::UNITS / G::PARTS;   // units of a part
    if (n == 0) {
      raw_exp = __builtin_amdgcn_perm(0u, raw_exp, ssel);
      if (__builtin_expect(raw_keys < kBs, 0)) {   // (zeros and a finite scale: a stale one may be NaN)
#pragma unroll
        for (int i = 0; i < G::PARTS; ++i)
          if ((is_v ? 4 * u16 + i : lane / 4) >= raw_keys) {
            if constexpr (D == 128) raw[i] = 0;
            else raw[i / 2] &= i % 2 ? 0xFFFFu : 0xFFFF0000u;
            raw_exp &= ~(0xFFu << (8 * i));
          }
      }
    }
    const int part = n / PER;
    const float s = __uint_as_float((raw_exp >> (8 * part) & 0xFFu) << 23);
    wide[n % PER * 2] = widen_at(raw[n / 2], n % 2 * 2, s);
    wide[n % PER * 2 + 1] = widen_at(raw[n / 2], n % 2 * 2 + 1, s);
  };
  auto stage = [&](int at_stage, int n) __attribute__((always_inline)) {   // behind unit n, the last of a part
    constexpr int PER = G::UNITS / G::PARTS;
    if (n % PER != PER - 1) return;
    uint8_t* const dst = lds + at_stage + sdst + n / PER * sinc;
    if constexpr (D == 128) *reinterpret_cast<u32x4*>(dst) = wide;
    else *reinterpret_cast<u32x2*>(dst) = u32x2{wide[0], wide[1]};
  };
  auto barrier = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // ---- operands
  int k_off = ((l32 & ~12) | ((l32 & 4) << 1) | ((l32 & 8) >> 1)) * G::KP + half * 16;
  const int vj = lane & 15, vg = (lane >> 4) & 1;
  int v_off = G::KTILE + (8 * half + (vj >> 2)) * G::VP + (16 * vg + 4 * (vj & 3)) * 2;
  // (hidden bases: else the compiler keeps a register per offset instead of an immediate)
  asm volatile("" : "+v"(k_off));
  asm volatile("" : "+v"(v_off));
  auto rdk = [&](int kb, int i) __attribute__((always_inline)) -> bf16x8 {   // k-step i / 2, keys 32 (i % 2) ..
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(lds + kb + (i & 1) * 32 * G::KP + (i >> 1) * 32));
  };
  auto rdv = [&](int vb, int i) __attribute__((always_inline)) -> bf16x8 {   // block i / DT, columns 32 (i % DT) ..
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    auto* lp = (__attribute__((address_space(3))) uint8_t*)lds + vb + (i / DT) * kBs * G::VP + (i % DT) * 64;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lp));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lp + 4 * G::VP)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  };

  const int m_col = wave * 32 + l32;   // this lane's query column: head hh of the group, position pos
  const int hh = m_col / a.per_tile, pos = m_col - hh * a.per_tile;
  auto has_row = [&](int32_t x) __attribute__((always_inline)) -> bool {
    return hh < a.group && pos < word(x, cw::kEntNvalid);
  };
  bf16x8 qf[KS];
  // The queries of an entry. A lane without a row takes the entry's first: its column is not stored.
  auto load_q = [&](int32_t x) __attribute__((always_inline)) {
    const bool ok = has_row(x);
    const int64_t row = int64_t(word(x, cw::kEntQrow)) + (ok ? pos : 0);
    const int head = word(x, cw::kEntG) * a.group + (ok ? hh : 0);
    const u32x4* src = reinterpret_cast<const u32x4*>(a.q + (row * a.hq + head) * D) + half;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, src[2 * s]);
  };

  int e_cur = blockIdx.x;
  int32_t cur = fetch(e_cur), next = fetch(e_cur + grid);
  if (!valid(cur, e_cur)) return;   // (the same for every wave)
  next_chunk();
  take_chunk();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    load();
#pragma unroll
    for (int n = 0; n < G::UNITS; ++n) {
      widen4(n);
      stage(i * G::STAGE, n);
    }
  }
  load();
  load_q(cur);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  barrier();

  f32x16 sc[2];      // scores of the step whose softmax comes next
  f32x16 oacc[DT];
  uint32_t w[16];    // packed probabilities
  float m = 0.f, l = 0.f;
#pragma unroll
  for (int t = 0; t < DT; ++t) oacc[t] = f32x16{};
  const bf16x2 ones{(__bf16)1.0f, (__bf16)1.0f};

  constexpr int RA = 4;   // operands in flight ahead of their MFMA
  constexpr int NPV = kBlocks * DT, NQK = 2 * KS, N = NPV + NQK;
  // The loaded codes are converted beside the last products and the next loads go out beside the last of these: the
  // later, the more time a load has. us (of each pair on one card) with both from the first QK product on, 6 operands
  // ahead / so: 8 x 2,112 rows behind 3,136 keys 988 / 976, 6 x ~411 behind ~700 47.6 / 46.5, 1 x 2,000 54.8 / 53.5;
  // twice the conversions beside each of half as many products 980, 46.9, 53.5; a further step of loads in flight,
  // copied into place 991, 47.4, 54.9.
  constexpr int WIDEN_AT = N - G::UNITS;
  bf16x8 op[RA];
  int st0 = 0, st1 = G::STAGE, st2 = 2 * G::STAGE;   // LDS places of the current step and the two after it
  auto row_max = [&]() __attribute__((always_inline)) -> float {   // of the current step's scaled scores
    asm volatile("" : "+v"(sc[0]), "+v"(sc[1]));   // (else it is computed in every step, ahead of its branches)
    float mx = sc[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) mx = __builtin_elementwise_maximum(mx, sc[i >> 4][i & 15]);
    return max_pair32(mx * a.c_log2);
  };
  if (group1) barrier();   // group 1 runs one interval behind
#pragma unroll
  for (int i = 0; i < NQK; ++i)
    sc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rdk(k_off, i), qf[i >> 1], i < 2 ? f32x16{} : sc[i & 1], 0, 0, 0);
  barrier();

  for (;;) {
    const int kbeg = word(cur, cw::kEntKbeg), keysteps = word(cur, cw::kEntKend) - kbeg;
    const int nsteps = SPLIT ? max(keysteps, 1) : keysteps;
    const int n_full = word(cur, cw::kEntNfull), nvalid = word(cur, cw::kEntNvalid);
    const int g = word(cur, cw::kEntG), qrow0 = word(cur, cw::kEntQrow);
    // keys 0 .. qpos are visible (none in a run of no steps, which goes through one)
    const int qpos = SPLIT && keysteps == 0 ? -1 : word(cur, cw::kEntP) + word(cur, cw::kEntRow0) + pos;
    const bool more = valid(next, e_cur + grid);
    for (int j = 0; j < nsteps; ++j) {
      // ---- softmax interval
      if (__builtin_expect(j == nsteps - 1, 0)) load_q(more ? next : cur);   // (first used after the PV products)
      __builtin_amdgcn_sched_barrier(0);
      if (__builtin_expect(j >= n_full, 0)) {
        const int lim = qpos - (kbeg + j) * kStep - half * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) {   // (pinned: else 32 compare results stay live in scalar registers)
            if (h * 32 + (i >> 3) * 16 + (i & 7) > lim) sc[h][i] = -INFINITY;
            asm volatile("" : "+v"(sc[h][i]));
          }
      }
      // An entry's base is the exact row maximum of its first step, and moves only when the row's sum
      // passes 2^30: bf16 and fp32 have the range for it, so later steps need no maximum (27 fewer
      // vector instructions of 180 in the interval that bounds the kernel).
      if (__builtin_expect(j == 0, 0)) {
        const float mx = row_max();
        m = mx == -INFINITY ? 0.f : mx;
      }
      float l_new;
      for (bool moved = false;; moved = true) {
        l_new = l;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          w[i] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(sc[i >> 3][2 * i & 15], a.c_log2, -m)),
                             __builtin_amdgcn_exp2f(fmaf(sc[i >> 3][(2 * i & 15) + 1], a.c_log2, -m)));
          l_new = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[i]), ones, l_new, false);
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(l_new > kMaxSum) == 0, 1)) break;
        // Two passes at most: the second has every row that moved at its own maximum, with l at 1 or below and
        // probabilities up to 1, so its sum is in range again. What is not by then (NaN, value scales near
        // fp32's end) stays as it is. (The exit stands behind `to`: ahead of it the registers spill.)
        const float before = max_pair32(l), top = max_pair32(l_new);   // (both halves hold the same row)
        const float to = top > kMaxSum ? fmaxf(row_max(), before > 1.f ? m + __builtin_amdgcn_logf(before) : m) : m;
        if (moved) break;
        const float alpha = __builtin_amdgcn_exp2f(m - to);
        l *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) oacc[t] *= alpha;
        m = to;
      }
      l = l_new;
      const int vb = v_off + st0, kb = k_off + st1;
#pragma unroll
      for (int i = 0; i < RA; ++i) op[i] = rdv(vb, i);
      barrier();

      // ---- product interval: MFMA and operand read alternate, fenced so that the compiler keeps
      // the read-ahead.
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (i < NPV) {
          const int b = i / DT;
          const bf16x8 pk = __builtin_bit_cast(bf16x8, u32x4{w[4 * b], w[4 * b + 1], w[4 * b + 2], w[4 * b + 3]});
          oacc[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % RA], pk, oacc[i % DT], 0, 0, 0);
        } else {
          const int q = i - NPV;
          sc[q & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[i % RA], qf[q >> 1], q < 2 ? f32x16{} : sc[q & 1], 0, 0, 0);
        }
        if (i + RA < N) op[i % RA] = i + RA < NPV ? rdv(vb, i + RA) : rdk(kb, i + RA - NPV);
        if (i >= WIDEN_AT) {
          widen4(i - WIDEN_AT);
          stage(st2, i - WIDEN_AT);
        }
        if (i == N - 1) load();
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
      const int st = st0;
      st0 = st1;
      st1 = st2;
      st2 = st;
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      barrier();
    }

    // ---- the entry's end (part of the next softmax interval): 64 columns at a time (32 of a part) through the
    // wave's own area, so that whole lines are stored
    const float total = sum_pair32(l);
    if constexpr (SPLIT) {
      // (a row that sees none of the run's keys has the sum +0. Tests of the bits: a NaN has to pass, and its part
      // has to count in the merge, which takes a NaN log-sum-exp for an empty part: a large number stands there.)
      const bool any = __float_as_uint(total) != 0, bad = (__float_as_uint(total) & 0x7FFFFFFFu) > 0x7F800000u;
      const float inv = any ? 1.f / total : 0.f;
      const int64_t at0 = int64_t(word(cur, cw::kEntSplit)) * a.part_rows + int64_t(qrow0) * a.hq + g * a.group;
      if (half == 0 && has_row(cur))
        a.part_lse[at0 + int64_t(pos) * a.hq + hh] = bad ? 1e30f : any ? m + __builtin_amdgcn_logf(total) : -INFINITY;
      uint8_t* const stg = lds + RING * G::STAGE + wave * G::OUT;
      constexpr int OP = 32 * 4 + 16;
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int gq = 0; gq < 4; ++gq)
          *reinterpret_cast<f32x4*>(stg + l32 * OP + gq * 32 + half * 16) =   // (0 times a masked NaN value is one)
              any ? f32x4{oacc[t][4 * gq] * inv, oacc[t][4 * gq + 1] * inv, oacc[t][4 * gq + 2] * inv, oacc[t][4 * gq + 3] * inv}
                  : f32x4{};
        asm volatile("" ::: "memory");   // (as below: lanes read what other lanes of the wave wrote, in order)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int rr = i * 8 + lane / 8, mr = wave * 32 + rr;
          const int hr = mr / a.per_tile, pr = mr - hr * a.per_tile;
          const f32x4 x = *reinterpret_cast<const f32x4*>(stg + rr * OP + (lane & 7) * 16);
          if (hr < a.group && pr < nvalid)
            *reinterpret_cast<f32x4*>(a.part_o + (at0 + int64_t(pr) * a.hq + hr) * D + 32 * t + (lane & 7) * 4) = x;
        }
      }
    } else {
      const float inv = has_row(cur) ? 1.f / total : 0.f;
      uint8_t* const stg = lds + RING * G::STAGE + wave * G::OUT;
      constexpr int OP = 64 * 2 + 16;
#pragma unroll
      for (int rd = 0; rd < D / 64; ++rd) {
        asm volatile("" ::: "memory");
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int gq = 0; gq < 4; ++gq) {
            const f32x16& o = oacc[2 * rd + t];   // rows 8 gq + 4 half .. + 3: columns of the output
            *reinterpret_cast<u32x2*>(stg + l32 * OP + t * 64 + gq * 16 + half * 8) =
                u32x2{pack_bf16x2(o[4 * gq] * inv, o[4 * gq + 1] * inv),
                      pack_bf16x2(o[4 * gq + 2] * inv, o[4 * gq + 3] * inv)};
          }
        asm volatile("" ::: "memory");   // (lanes read what other lanes of the wave wrote, in order)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int rr = i * 8 + lane / 8, mr = wave * 32 + rr;
          const int hr = mr / a.per_tile, pr = mr - hr * a.per_tile;
          const u32x4 x = *reinterpret_cast<const u32x4*>(stg + rr * OP + (lane & 7) * 16);
          if (hr < a.group && pr < nvalid)
            *reinterpret_cast<u32x4*>(a.out + ((int64_t(qrow0) + pr) * a.hq + g * a.group + hr) * D + rd * 64 +
                                      (lane & 7) * 8) = x;
        }
      }
    }
    if (!more) break;
#pragma unroll
    for (int t = 0; t < DT; ++t) oacc[t] = f32x16{};
    l = 0.f;
    e_cur += grid;
    cur = next;
    next = fetch(e_cur + grid);
  }
  if (!group1) barrier();
}

// Checks and launch of both entry points; workspace NULL: of a plan without splits.
cw_status prefill_fp4(const char* what, const void* q, const void* pages, const int32_t* block_table,
                      int32_t bt_stride, const int32_t* cu_suffix_host, const int32_t* prefix_len_host, int32_t batch,
                      int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                      int32_t num_blocks, float softmax_scale, const int32_t* plan_host, const int32_t* plan_dev,
                      bool split, void* workspace, int64_t workspace_bytes, void* out, void* stream) {
  const std::string w(what);
  cw_status st = cw::check_cache_fp4(what, pages, block_table, num_kv_heads, head_dim, block_size, num_blocks);
  if (st != CW_OK) return st;
  if (num_q_heads < 1 || num_q_heads % num_kv_heads != 0)
    return cw::fail(CW_EINVAL, w + ": num_q_heads must be a positive multiple of num_kv_heads");
  const int group = num_q_heads / num_kv_heads;
  if (group > cw::kMaxGroup) return cw::fail(CW_EUNSUPPORTED, w + ": more than 128 query heads per KV head");
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return cw::fail(CW_EINVAL, w + ": softmax_scale must be finite and positive");
  int64_t rows = 0;
  st = cw::check_batch(cu_suffix_host, prefix_len_host, batch, block_size, bt_stride, &rows, true);
  if (st != CW_OK) return st;
  PrefillArgs a;
  int32_t grid = 0, splits = 1;
  st = cw::check_plan_header(what, plan_host, cu_suffix_host, prefix_len_host, batch, num_q_heads, num_kv_heads,
                             head_dim, &grid, &splits, &a.fp_lo, &a.fp_hi, &a.num_entries);
  if (st != CW_OK) return st;
  if (!split && splits != 1) return cw::fail(CW_EINVAL, w + ": the plan has splits");
  a.part_rows = rows * num_q_heads;
  if (split) {
    const int64_t need = cw_suffix_prefill_split_workspace_bytes(rows, num_q_heads, head_dim, splits);
    if (need < 0) return cw_status(need);
    if (rows > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15) != 0))
      return cw::fail(CW_EINVAL, w + ": workspace must hold " + std::to_string(need) + " bytes, 16-byte aligned");
  }
  if (rows == 0 || grid == 0) return cw::ok();
  if (!q || !out || !plan_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  a.q = static_cast<const uint16_t*>(q);
  a.pages = static_cast<const uint8_t*>(pages);
  a.bt = block_table;
  a.plan = plan_dev;
  a.out = static_cast<uint16_t*>(out);
  a.part_o = static_cast<float*>(workspace);
  // (the layout that cw_suffix_prefill_split_workspace_bytes counts: parts, then sums at a multiple of 256)
  a.part_lse = split ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) +
                                                (int64_t(splits) * a.part_rows * head_dim * 4 + 255) / 256 * 256)
                     : nullptr;
  a.bt_stride = bt_stride;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.group = group;
  a.per_tile = cw::tile_positions(group);
  a.num_blocks = num_blocks;
  a.c_log2 = softmax_scale * 1.4426950408889634f;
  auto* const s = static_cast<hipStream_t>(stream);
  auto* const kernel = head_dim == 128 ? (split ? suffix_prefill_fp4_kernel<128, true> : suffix_prefill_fp4_kernel<128, false>)
                                       : (split ? suffix_prefill_fp4_kernel<64, true> : suffix_prefill_fp4_kernel<64, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, w + " launch: " + hipGetErrorString(e));
  if (!split) return cw::ok();
  // The join takes a row's parts side by side, the merge in turn: 64 rows of 32 heads, 64 rows of 3 and of 4 times
  // 32 heads (us of the call over 6,000 keys, captured, merge / join): 8 parts 33.6 / 33.4, 36.4 / 38.4, 39.7 / 42.2;
  // 12 parts 32.1 / 30.6, 47.9 / 47.9, 49.6 / 50.0; 16 parts 32.4 / 29.7, 44.7 / 44.4, 50.3 / 49.2. 8 times 64 rows,
  // 2,000 keys: 12 parts 55.5 / 57.2, 16 parts 67.5 / 65.6.
  const bool join = splits > kMergeParts && a.part_rows <= kJoinRows;
  return join ? cw::decode_join(what, head_dim, a.part_o, a.part_lse, splits, a.part_rows, out, stream)
              : cw_lse_merge(a.part_o, a.part_lse, splits, a.part_rows, head_dim, out, stream);
}

}  // namespace

extern "C" cw_status cw_suffix_prefill_attn_fp4(const void* q, const void* pages, const int32_t* block_table,
                                                int32_t bt_stride, const int32_t* cu_suffix_host,
                                                const int32_t* prefix_len_host, int32_t batch, int32_t num_q_heads,
                                                int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                                                int32_t num_blocks, float softmax_scale, const int32_t* plan_host,
                                                const int32_t* plan_dev, void* out, void* stream) {
  return prefill_fp4("suffix_prefill_attn_fp4", q, pages, block_table, bt_stride, cu_suffix_host, prefix_len_host,
                     batch, num_q_heads, num_kv_heads, head_dim, block_size, num_blocks, softmax_scale, plan_host,
                     plan_dev, false, nullptr, 0, out, stream);
}

extern "C" cw_status cw_suffix_prefill_attn_split_fp4(const void* q, const void* pages, const int32_t* block_table,
                                                      int32_t bt_stride, const int32_t* cu_suffix_host,
                                                      const int32_t* prefix_len_host, int32_t batch,
                                                      int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                                      int32_t block_size, int32_t num_blocks, float softmax_scale,
                                                      const int32_t* plan_host, const int32_t* plan_dev,
                                                      void* workspace, int64_t workspace_bytes, void* out,
                                                      void* stream) {
  return prefill_fp4("suffix_prefill_attn_split_fp4", q, pages, block_table, bt_stride, cu_suffix_host,
                     prefix_len_host, batch, num_q_heads, num_kv_heads, head_dim, block_size, num_blocks,
                     softmax_scale, plan_host, plan_dev, true, workspace, workspace_bytes, out, stream);
}
