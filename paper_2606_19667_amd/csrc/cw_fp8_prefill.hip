// Causal attention of suffix rows over an 8-bit paged KV cache (gfx950).
//
// Paper Sec. 1 and 2.1: with a reused prefix only the suffix tokens are prefilled; they attend
// fully over the prefix and causally over themselves. Here keys and values are e4m3 codes with
// one fp32 scale per (block of 16 tokens, KV head), which doubles the prefix a cache holds.

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <string>

#include "cw_internal.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kBs = cw::kBlockSize;
constexpr int kStep = cw::kKvTile;            // keys of a step (four blocks)
constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kBlocks = kStep / kBs;
static_assert(kWaves * 32 == cw::kTileRows, "one 32-column MFMA block per wave");
static_assert(kWaves == 2 * kBlocks, "a wave stages one block of one tensor");
constexpr float kLazy = 8.0f;                 // the exponent base moves when a score exceeds it by 2^8

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
// Four e4m3 codes to four bfloat16 (every e4m3 value is one).
__device__ __forceinline__ u32x2 widen_fp8x4(uint32_t w) {
  return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false)),
               __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true))};
}
__device__ __forceinline__ float max_pair32(float x) {   // of this lane and lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_pair32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

struct PrefillArgs {
  const uint16_t* q;
  const uint8_t* k8;
  const uint8_t* v8;
  const float* k_scale;
  const float* v_scale;
  const int32_t* bt;
  const int32_t* plan;   // device copy of the whole plan (header, then entries)
  uint16_t* out;
  int32_t bt_stride, hq, hkv, group, per_tile, num_blocks, num_entries;
  float c_log2;
  uint32_t fp_lo, fp_hi; // the batch fingerprint the host validated
};

template <int D>
struct Geom {
  static constexpr int KP = 2 * D + 16;           // LDS bytes from one K row to the next (bf16, padded:
                                                  // the 16-byte reads of 8 rows lie on distinct banks)
  static constexpr int VP = 2 * D + 32;           // the same of V (4 rows of a transposing read)
  static constexpr int KTILE = kStep * KP;
  static constexpr int STAGE = KTILE + kStep * VP;
  static constexpr int PIECES = kBs * D / 1024;   // 16-byte pieces of a block that a lane stages
  static constexpr int KS = D / 16;               // MFMA k-steps over D
  static constexpr int DT = D / 32;               // 32-row output tiles over D
  static constexpr int OUT = 32 * (64 * 2 + 16);  // per-wave output staging: 32 rows of 64 columns
};

// Work as in the plan: an entry is (request, KV head g, a run of T suffix rows); 256 packed
// rows of an entry are the G query heads of g over T = 256 / G positions, 32 a wave. Workgroup
// w runs entries w, w + grid, ...; keys come in steps of 64.
//  * A step's four blocks go through registers into LDS: wave w takes K (w even) or V (w odd)
//    of block w / 2, converts the codes to bf16 (exact) and writes rows. So each code is
//    converted once per workgroup, not once per wave. Rows past the prompt are zeros; a block
//    outside the pool is zeros with scale 1.
//  * S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16_bf16; K row pi(i), pi swapping bits
//    2 and 3, is read into A row i, so that the score registers of a lane are its P^T operand:
//    register e of half h holds key 32 h + 16 (e / 8) + 8 (lane / 32) + e % 8. V^T comes from
//    token-major rows by transposing LDS reads.
//  * The scales cost one multiply-add per score, which softmax_scale needs anyway: with s the
//    raw score, p v_scale = 2^(s (c k_scale) + (log2 v_scale - m)) is rounded to bf16 for the
//    product, and the row's sum takes each block's rounded values divided by its v_scale. Q is
//    not rounded again.
template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void suffix_prefill_fp8_kernel(const PrefillArgs a) {
  using G = Geom<D>;
  constexpr int KS = G::KS, DT = G::DT, P16 = G::PIECES;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * G::STAGE + kWaves * G::OUT];
  // per stage: c_log2 * k_scale, log2(v_scale), 1 / v_scale of the step's blocks
  __shared__ __attribute__((aligned(16))) float s_scale[2][3][kBlocks];

  if (uint32_t(a.plan[cw::kHdrFpLo]) != a.fp_lo || uint32_t(a.plan[cw::kHdrFpHi]) != a.fp_hi) return;
  const int32_t* const ents = a.plan + cw::kPlanHeaderWords;
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // ---- staging role
  const bool is_v = (wave & 1) != 0;
  const int bs = wave >> 1;
  const uint8_t* const codes = is_v ? a.v8 : a.k8;
  const float* const scales = is_v ? a.v_scale : a.k_scale;
  constexpr int LPR = D / 16;   // lanes a row
  const int skey = lane / LPR;  // row of the block, of piece 0
  const int sdst = (is_v ? G::KTILE + bs * kBs * G::VP : bs * kBs * G::KP) + (lane % LPR) * 32;
  const int spitch = is_v ? G::VP : G::KP;

  // ---- operand offsets
  const int k_row = (l32 & ~12) | ((l32 & 4) << 1) | ((l32 & 8) >> 1);
  const int k_off = k_row * G::KP + half * 16;
  const int vj = lane & 15, vg = (lane >> 4) & 1;
  const int v_off = G::KTILE + (8 * half + (vj >> 2)) * G::VP + (16 * vg + 4 * (vj & 3)) * 2;
  auto rdk = [&](int base, int i) __attribute__((always_inline)) -> bf16x8 {   // k-step i / 2, keys 32 (i % 2) ..
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(lds + base + k_off + (i & 1) * 32 * G::KP +
                                                                      (i >> 1) * 32));
  };
  auto rdv = [&](int base, int kk, int t) __attribute__((always_inline)) -> bf16x8 {   // block kk, columns 32 t ..
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    auto* lp = (__attribute__((address_space(3))) uint8_t*)lds + base + v_off + kk * kBs * G::VP + t * 64;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lp));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lp + 4 * G::VP)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  };

  const int m_col = wave * 32 + l32;   // this lane's query column: head hh of the group, position pos
  const int hh = m_col / a.per_tile, pos = m_col - hh * a.per_tile;

  for (int e = blockIdx.x; e < a.num_entries; e += gridDim.x) {
    const int32_t* const d = ents + int64_t(e) * cw::kPlanEntryWords;
    const int r = d[cw::kEntR];
    if (r < 0 || uint32_t(d[cw::kEntCheck]) != cw::entry_tag(a.fp_lo, a.fp_hi, uint32_t(e))) return;
    const int g = d[cw::kEntG], row0 = d[cw::kEntRow0], nvalid = d[cw::kEntNvalid], P = d[cw::kEntP],
              L = d[cw::kEntL], kbeg = d[cw::kEntKbeg], nsteps = d[cw::kEntKend] - kbeg, n_full = d[cw::kEntNfull],
              qrow0 = d[cw::kEntQrow];
    const int32_t* const bt = a.bt + int64_t(r) * a.bt_stride;
    const int last = (L + kBs - 1) / kBs - 1;

    u32x4 raw[P16];
    float scale = 1.f;
    int keys = 0;   // rows of the staged block inside the prompt
    auto load = [&](int j) __attribute__((always_inline)) {
      const int lb = (kbeg + j) * kBlocks + bs;
      const int id = bt[min(lb, last)];
      const bool ok = lb <= last && id >= 0 && id < a.num_blocks;
      const uint8_t* src = codes + (int64_t(ok ? id : 0) * a.hkv + g) * (kBs * D) + lane * 16;
      keys = ok ? L - lb * kBs : 0;
      scale = ok ? scales[int64_t(id) * a.hkv + g] : 1.f;
#pragma unroll
      for (int i = 0; i < P16; ++i) raw[i] = *reinterpret_cast<const u32x4*>(src + 1024 * i);
    };
    auto stage = [&](int slot) __attribute__((always_inline)) {
      uint8_t* const dst = lds + slot * G::STAGE + sdst;
#pragma unroll
      for (int i = 0; i < P16; ++i) {
        const int key = i * (64 / LPR) + skey;
        u32x4 x = raw[i];
        if (key >= keys) x = u32x4{0, 0, 0, 0};
        const u32x2 a0 = widen_fp8x4(x[0]), a1 = widen_fp8x4(x[1]), a2 = widen_fp8x4(x[2]), a3 = widen_fp8x4(x[3]);
        u32x4* at = reinterpret_cast<u32x4*>(dst + key * spitch);
        at[0] = u32x4{a0[0], a0[1], a1[0], a1[1]};
        at[1] = u32x4{a2[0], a2[1], a3[0], a3[1]};
      }
      if (lane == 0) {
        if (is_v) {
          s_scale[slot][1][bs] = __log2f(scale);
          s_scale[slot][2][bs] = 1.f / scale;
        } else {
          s_scale[slot][0][bs] = a.c_log2 * scale;
        }
      }
    };

    const bool row_ok = hh < a.group && pos < nvalid;
    bf16x8 qf[KS];
    {
      const int64_t row = int64_t(qrow0) + (row_ok ? pos : 0);
      const u32x4* src = reinterpret_cast<const u32x4*>(
                             a.q + (row * a.hq + g * a.group + (row_ok ? hh : 0)) * D) + half;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        u32x4 x = src[2 * s];
        if (!row_ok) x = u32x4{0, 0, 0, 0};
        qf[s] = __builtin_bit_cast(bf16x8, x);
      }
    }
    const int qpos = P + row0 + pos;   // keys 0 .. qpos are visible

    f32x16 oacc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) oacc[t] = f32x16{};
    float m = 0.f, l = 0.f;
    load(0);
    __syncthreads();   // the entry before is done with the stages
    stage(0);
    if (nsteps > 1) load(1);
    __syncthreads();
    for (int j = 0; j < nsteps; ++j) {
      if (j + 1 < nsteps) stage((j + 1) & 1);
      if (j + 2 < nsteps) load(j + 2);
      const int base = (j & 1) * G::STAGE;
      f32x16 sc[2] = {f32x16{}, f32x16{}};
#pragma unroll
      for (int i = 0; i < 2 * KS; ++i)
        sc[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rdk(base, i), qf[i >> 1], sc[i & 1], 0, 0, 0);
      float kc[kBlocks], vlog[kBlocks], vinv[kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        kc[b] = s_scale[j & 1][0][b];
        vlog[b] = s_scale[j & 1][1][b];
        vinv[b] = s_scale[j & 1][2][b];
      }
      if (j >= n_full) {
        const int lim = qpos - (kbeg + j) * kStep - half * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (h * 32 + (i >> 3) * 16 + (i & 7) > lim) sc[h][i] = -INFINITY;
            asm volatile("" : "+v"(sc[h][i]));
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        float x = sc[b >> 1][(b & 1) * 8];
#pragma unroll
        for (int i = 1; i < 8; ++i) x = fmaxf(x, sc[b >> 1][(b & 1) * 8 + i]);
        mx = fmaxf(mx, x * kc[b]);
      }
      mx = max_pair32(mx);
      if (j == 0) {
        m = mx == -INFINITY ? 0.f : mx;
      } else if (__builtin_amdgcn_ballot_w64(mx > m + kLazy) != 0) {
        const float to = mx > m + kLazy ? mx : m;
        const float alpha = __builtin_amdgcn_exp2f(m - to);
        m = to;
        l *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t) oacc[t] *= alpha;
      }
      uint32_t w[16];
      const bf16x2 ones{(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const float add = vlog[b] - m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = (b & 1) * 8 + 2 * i;
          w[4 * b + i] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(sc[b >> 1][at], kc[b], add)),
                                     __builtin_amdgcn_exp2f(fmaf(sc[b >> 1][at + 1], kc[b], add)));
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w[4 * b + i]), ones, sum, false);
        }
        l = fmaf(sum, vinv[b], l);
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const bf16x8 pk = __builtin_bit_cast(bf16x8, u32x4{w[4 * b], w[4 * b + 1], w[4 * b + 2], w[4 * b + 3]});
#pragma unroll
        for (int t = 0; t < DT; ++t)
          oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rdv(base, b, t), pk, oacc[t], 0, 0, 0);
      }
      __syncthreads();
    }

    // ---- output: 64 columns at a time through the wave's own area, so that whole lines are stored
    const float total = sum_pair32(l);
    const float inv = row_ok ? 1.f / total : 0.f;
    uint8_t* const stg = lds + 2 * G::STAGE + wave * G::OUT;
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
}

}  // namespace

extern "C" cw_status cw_suffix_prefill_attn_fp8(const void* q, const void* k8, const void* v8, const float* k_scale,
                                                const float* v_scale, const int32_t* block_table, int32_t bt_stride,
                                                const int32_t* cu_suffix_host, const int32_t* prefix_len_host,
                                                int32_t batch, int32_t num_q_heads, int32_t num_kv_heads,
                                                int32_t head_dim, int32_t block_size, int32_t num_blocks,
                                                float softmax_scale, const int32_t* plan_host,
                                                const int32_t* plan_dev, void* out, void* stream) {
  const std::string w("suffix_prefill_attn_fp8");
  cw_status st = cw::check_cache_fp8(w.c_str(), k8, v8, k_scale, v_scale, block_table, num_kv_heads, head_dim,
                                     block_size, num_blocks);
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
  st = cw::check_plan_header("suffix_prefill_attn_fp8", plan_host, cu_suffix_host, prefix_len_host, batch, num_q_heads,
                             num_kv_heads, head_dim, &grid, &splits, &a.fp_lo, &a.fp_hi, &a.num_entries);
  if (st != CW_OK) return st;
  if (splits != 1) return cw::fail(CW_EINVAL, w + ": the plan has splits");
  if (rows == 0 || grid == 0) return cw::ok();
  if (!q || !out || !plan_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15) != 0)
    return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  a.q = static_cast<const uint16_t*>(q);
  a.k8 = static_cast<const uint8_t*>(k8);
  a.v8 = static_cast<const uint8_t*>(v8);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.bt = block_table;
  a.plan = plan_dev;
  a.out = static_cast<uint16_t*>(out);
  a.bt_stride = bt_stride;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.group = group;
  a.per_tile = cw::tile_positions(group);
  a.num_blocks = num_blocks;
  a.c_log2 = softmax_scale * 1.4426950408889634f;
  auto* const s = static_cast<hipStream_t>(stream);
  if (head_dim == 128)
    hipLaunchKernelGGL(suffix_prefill_fp8_kernel<128>, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(suffix_prefill_fp8_kernel<64>, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, w + " launch: " + hipGetErrorString(e));
  return cw::ok();
}
