// The 8-bit layer path for gfx950 (MI355X), except its matrix product: the norm that writes
// 8-bit rows, the append into an 8-bit paged KV cache, and attention over that cache for
// suffix rows and for single tokens.
//
// 8 bits are e4m3 (OCP: 4 exponent and 3 mantissa bits, largest value 448, one NaN pattern
// per sign and no infinity), rounded to nearest even. An e4m3 value is a bfloat16 value, so
// the attention kernels convert keys and values without rounding and multiply in bf16 MFMA.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "cw_internal.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBs = cw::kBlockSize;
constexpr float kFp8Max = 448.f;
constexpr int kGroupCols = 128;   // columns of an 8-bit row that share a scale
constexpr int64_t kMaxGrid = UINT32_MAX / kThreads;   // a launch has fewer than 2^32 threads along an axis

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
// Four floats to four e4m3 codes (low byte first). Beyond 448 (after rounding) and for
// infinities the instruction gives NaN.
__device__ __forceinline__ uint32_t pack_fp8x4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}
// |x|, or 0 where x is infinite or NaN: a scale comes from the finite values alone.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off);
  return x;
}

// ---------------------------------------------------------------------------
// Residual addition, root-mean-square norm and 8-bit rows:
//   h = bf16(x + r),  y = h (mean(h^2) + eps)^(-1/2) w,
//   scale = max|y| / 448 over 128 columns,  code = e4m3(y / scale).
// A row is read once and stays in registers between the sum of squares and the output.
// TPR threads work on a row (64: a wave, four rows a workgroup; 256: the workgroup), each on
// CH pieces of 8 columns TPR apart, so that 16 neighbouring lanes hold a group of 128 columns
// and its maximum takes four exchanges. Sums are fp32.
// HBM-bound: 7 bytes a column with a residual. 16,128 rows of 4,096: 80.5 us, 5.8 TB/s, from the same rows each
// time or from four sets in turn (1.9 GB; a copy, which writes as much as it reads, makes 4.7 to 5.3); 64 rows 3.8 us in a captured graph, one chain of load, sum, maximum and store.
// ---------------------------------------------------------------------------
struct NormArgs {
  const uint16_t* x;
  const uint16_t* residual;   // NULL: none
  const uint16_t* weight;
  uint16_t* residual_out;     // NULL: not written
  uint8_t* out8;
  float* scales;
  int64_t x_stride, residual_stride;   // elements from one row to the next
  int64_t rows;
  int hidden, groups;
  float eps;
};

template <int TPR, int CH>
__global__ __launch_bounds__(kThreads) void add_rms_norm_fp8_kernel(const NormArgs a) {
  constexpr int RPW = kThreads / TPR;
  const int tid = threadIdx.x % TPR;
  const int64_t row = int64_t(blockIdx.x) * RPW + threadIdx.x / TPR;
  const int pieces = a.hidden / 8;
  const bool row_ok = row < a.rows;   // (only where a wave has a row of its own: no barrier below)
  if (TPR == 64 && !row_ok) return;
  u32x4 xr[CH], rr[CH], wr[CH];
  const u32x4 zero{0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int c = i * TPR + tid;
    const bool ok = c < pieces;
    xr[i] = ok ? *reinterpret_cast<const u32x4*>(a.x + row * a.x_stride + 8 * c) : zero;
    rr[i] = ok && a.residual ? *reinterpret_cast<const u32x4*>(a.residual + row * a.residual_stride + 8 * c) : zero;
    wr[i] = ok ? *reinterpret_cast<const u32x4*>(a.weight + 8 * c) : zero;
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (a.residual) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xr[i][j] = pack_bf16x2(bf16_lo(xr[i][j]) + bf16_lo(rr[i][j]), bf16_hi(xr[i][j]) + bf16_hi(rr[i][j]));
    }
    const int c = i * TPR + tid;
    if (a.residual_out && c < pieces)
      *reinterpret_cast<u32x4*>(a.residual_out + row * int64_t(a.hidden) + 8 * c) = xr[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lo = bf16_lo(xr[i][j]), hi = bf16_hi(xr[i][j]);
      ss = fmaf(lo, lo, ss);
      ss = fmaf(hi, hi, ss);
    }
  }
  __shared__ float part[2][kWaves];
  auto row_sum = [&](float v, int slot) __attribute__((always_inline)) -> float {
    v = wave_sum(v);
    if constexpr (TPR > 64) {
      if ((threadIdx.x & 63) == 0) part[slot][threadIdx.x >> 6] = v;
      __syncthreads();
      v = (part[slot][0] + part[slot][1]) + (part[slot][2] + part[slot][3]);
    }
    return v;
  };
  ss = row_sum(ss, 0);
  float inv, down = 1.f;
  bool bad = false;
  if (__builtin_expect(ss < INFINITY, 1)) {
    inv = 1.f / sqrtf(ss / float(a.hidden) + a.eps);
  } else {
    // The squares of values above 2^63 leave fp32 (a row with an infinity or a NaN gets here
    // too): the sum again of values times 2^-96, and the products below times 2^-32. eps is
    // nothing beside it. (The branch is the same for all threads of the row.)
    down = 0x1p-32f;
    float s2 = 0.f;
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float lo = bf16_lo(xr[i][j]) * 0x1p-96f, hi = bf16_hi(xr[i][j]) * 0x1p-96f;
        s2 = fmaf(lo, lo, s2);
        s2 = fmaf(hi, hi, s2);
      }
    s2 = row_sum(s2, 1);
    bad = !(s2 < INFINITY);
    inv = 0x1p-64f / sqrtf(s2 / float(a.hidden));
  }
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    // y / scale = 448 (h w) / max|h w|: the products of two bf16 values are exact in fp32, and
    // the quotient is corrected by its remainder, so that a quotient halfway between two codes
    // (small integers: they are common) is rounded as the tie that it is.
    float y[8];
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      y[2 * j] = bf16_lo(xr[i][j]) * down * bf16_lo(wr[i][j]);
      y[2 * j + 1] = bf16_hi(xr[i][j]) * down * bf16_hi(wr[i][j]);
      top = fmaxf(top, fmaxf(finite_abs(y[2 * j]), finite_abs(y[2 * j + 1])));
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off));
    const bool some = top >= 0x1p-100f;
    const float rcp = __builtin_amdgcn_rcpf(some ? top : 1.f);
    const int c = i * TPR + tid;
    if (c < pieces) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = y[j] * kFp8Max, q = n * rcp;
        y[j] = some ? fmaf(fmaf(-q, top, n), rcp, q) : y[j] * 0.f;
        if (bad) y[j] = __uint_as_float(0x7FC00000u);
      }
      const u32x2 o{pack_fp8x4(y[0], y[1], y[2], y[3]), pack_fp8x4(y[4], y[5], y[6], y[7])};
      *reinterpret_cast<u32x2*>(a.out8 + row * int64_t(a.hidden) + 8 * c) = o;
      if ((c & 15) == 0) a.scales[row * a.groups + c / 16] = some && !bad ? top * inv / kFp8Max : 1.f;
    }
  }
}

// ---------------------------------------------------------------------------
// Append into the 8-bit cache, with the rotary embedding.
//
// The unit of work is one cache block that gets rows: request r touches the logical blocks
// P_r / 16 .. (P_r + S_r - 1) / 16, at most (S_r + 14) / 16 + 1 of them whatever P_r is, so a
// launch depends on the suffix lengths alone (a captured launch goes on with other prefix
// lengths in device memory). One wave handles one (block, head): lane l holds the columns
// 16 (l % 4) .. + 15 of each half of row l / 4 (8 columns at head_dim 64), so a rotary pair
// lies in one lane, and a block's maximum is a wave reduction. Heads are queries, keys, then
// values; a wave keeps the cosines and sines of its rows over all its heads.
// HBM-bound: reads 2 (Hq + 2 Hkv) D bytes a row, writes 2 Hq D + 2 Hkv D. 16,128 rows of 48 heads of 128:
// 84 us, 4.6 TB/s with the rotation table (a copy 4.7 to 5.3; what is missing are the ends of the
// workgroups, each a chain of offsets, table word, rows, maximum, store); 64 requests of one row: 6.7 us in a
// captured graph, 13.9 called one by one, which is the host's time.
// ---------------------------------------------------------------------------
struct AppendArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;   // elements from one row to the next
  const f32x2* rope;                      // NULL: no rotation
  uint16_t* q_out;
  uint8_t* k8;
  uint8_t* v8;
  float* k_scale;
  float* v_scale;
  const int32_t* bt;
  const int32_t* cu;
  const int32_t* plen;
  int bt_stride, batch, hq, hkv, num_blocks, rope_len;   // hq 0: no queries
};

// 2^e of the smallest e with top <= 448 * 2^e, e in [-100, 120] (top 0 or tiny: 2^-100).
// 448 = 1.75 * 2^8: a mantissa above 1.75 carries into the exponent.
__device__ __forceinline__ float block_scale(float top) {
  const int e = int((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 127 - 8;
  return __uint_as_float(uint32_t(min(max(e, -100), 120) + 127) << 23);
}

// Rotates a pair by (cos, sin). Each product is rounded by itself: the bits that elementary
// operations give.
__device__ __forceinline__ void rotate(float& x, float& y, f32x2 turn) {
#pragma clang fp contract(off)
  const float u = x, w = y;
  x = u * turn[0] - w * turn[1];
  y = w * turn[0] + u * turn[1];
}

// A result v that lies `rest` (or a positive multiple of it) off the exact one, with its last bit set to one where
// they differ: rounded on to fewer bits it goes where the exact result goes, as it is never halfway by rounding alone.
__device__ __forceinline__ float to_odd(float v, float rest) {
  const uint32_t b = __float_as_uint(v);
  if (rest == 0.f || (b & 1) != 0 || !(fabsf(v) > 0x1p-60f)) return v;   // (a code of so small a value is zero)
  return __uint_as_float((rest > 0.f) == (v > 0.f) ? b + 1 : b - 1);
}
// x / s by its inverse (inv = 1 / s rounded).
__device__ __forceinline__ float quotient(float x, float s, float inv) {
  const float q = x * inv, r = fmaf(-q, s, x);
  if (r == 0.f) return q;
  const float p = fmaf(r, inv, q);
  return to_odd(p, fmaf(-p, s, x));
}

__device__ __forceinline__ uint32_t rescale_fp8x4(uint32_t w, float f) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(w), true);
  auto times = [f](float c) __attribute__((always_inline)) { return to_odd(c * f, fmaf(c, f, -(c * f))); };
  return pack_fp8x4(times(lo[0]), times(lo[1]), times(hi[0]), times(hi[1]));
}

template <int D>
__global__ __launch_bounds__(kThreads) void rope_append_fp8_kernel(const AppendArgs a) {
  constexpr int W = D / 8;     // columns of a half that a lane holds
  constexpr int N16 = W / 8;   // 16-byte pieces of a half
  __shared__ int s_unit[2];
  const int tid = threadIdx.x;
  if (tid < 64) {   // the unit's request, and which of its touched blocks this is
    const int b = blockIdx.x;
    int base = 0, rr = -1, jb = 0;
    for (int r0 = 0; r0 < a.batch; r0 += 64) {
      const int r = r0 + tid;
      const int rows = r < a.batch ? a.cu[r + 1] - a.cu[r] : 0;
      const int n = rows > 0 ? (rows + kBs - 2) / kBs + 1 : 0;
      int x = n;   // inclusive prefix sum over the lanes
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        if (tid >= off) x += y;
      }
      const uint64_t hit = __ballot(base + x - n <= b && b < base + x);
      if (hit) {
        const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
        rr = r0 + l;
        jb = b - base - __shfl(x - n, l);
        break;
      }
      base += __shfl(x, 63);
    }
    if (tid == 0) {
      s_unit[0] = rr;
      s_unit[1] = jb;
    }
  }
  __syncthreads();
  const int r = s_unit[0];
  if (r < 0) return;
  const int cu0 = a.cu[r], rows = a.cu[r + 1] - cu0, P = a.plen[r];
  if (P < 0 || P > INT32_MAX - rows - 2 * kBs) return;   // (the end of the block behind the last row is counted too)
  const int lb = P / kBs + s_unit[1];
  const int t_begin = max(P, lb * kBs), t_end = min(P + rows, lb * kBs + kBs);
  if (t_begin >= t_end) return;
  const int blk = lb < a.bt_stride ? a.bt[int64_t(r) * a.bt_stride + lb] : -1;
  const bool in_pool = blk >= 0 && blk < a.num_blocks;

  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slot = lane >> 2, c = lane & 3;
  const int t = lb * kBs + slot;
  const bool live = t >= t_begin && t < t_end;
  const int64_t row = cu0 + (live ? t - P : 0);

  f32x2 turn[W];
  if (a.rope) {
    const f32x2* src = a.rope + int64_t(min(live ? t : t_begin, a.rope_len - 1)) * (D / 2) + c * W;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      const f32x4 two = reinterpret_cast<const f32x4*>(src)[i];
      turn[2 * i] = f32x2{two[0], two[1]};
      turn[2 * i + 1] = f32x2{two[2], two[3]};
    }
  }
  const int heads = a.hq + 2 * a.hkv;
  const int step = int(gridDim.y) * kWaves;
  u32x4 lo[N16], hi[N16];   // the head's raw row pieces, of both halves
  auto load = [&](int h) __attribute__((always_inline)) {
    const uint16_t* p = h < a.hq ? a.q + row * a.q_stride + int64_t(h) * D
                        : h < a.hq + a.hkv ? a.k + row * a.k_stride + int64_t(h - a.hq) * D
                                           : a.v + row * a.v_stride + int64_t(h - a.hq - a.hkv) * D;
    p += c * W;
#pragma unroll
    for (int i = 0; i < N16; ++i) {
      lo[i] = live ? reinterpret_cast<const u32x4*>(p)[i] : u32x4{0, 0, 0, 0};
      hi[i] = live ? reinterpret_cast<const u32x4*>(p + D / 2)[i] : u32x4{0, 0, 0, 0};
    }
  };
  int h = int(blockIdx.y) * kWaves + wave;
  if (h < heads) load(h);
  for (; h < heads; h += step) {
    float x[W], y[W];
#pragma unroll
    for (int i = 0; i < N16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[8 * i + 2 * j] = bf16_lo(lo[i][j]);
        x[8 * i + 2 * j + 1] = bf16_hi(lo[i][j]);
        y[8 * i + 2 * j] = bf16_lo(hi[i][j]);
        y[8 * i + 2 * j + 1] = bf16_hi(hi[i][j]);
      }
    if (h + step < heads) load(h + step);
    if (a.rope && h < a.hq + a.hkv) {
#pragma unroll
      for (int i = 0; i < W; ++i) {
        rotate(x[i], y[i], turn[i]);
      }
    }
    if (h < a.hq) {
      if (live) {
        uint16_t* dst = a.q_out + (row * a.hq + h) * D + c * W;
#pragma unroll
        for (int i = 0; i < N16; ++i) {
          u32x4 o0, o1;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o0[j] = pack_bf16x2(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
            o1[j] = pack_bf16x2(y[8 * i + 2 * j], y[8 * i + 2 * j + 1]);
          }
          reinterpret_cast<u32x4*>(dst)[i] = o0;
          reinterpret_cast<u32x4*>(dst + D / 2)[i] = o1;
        }
      }
      continue;
    }
    if (!in_pool) continue;
    const bool is_v = h >= a.hq + a.hkv;
    const int g = h - a.hq - (is_v ? a.hkv : 0);
    float top = 0.f;   // (rows outside the call were loaded as zeros)
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, fmaxf(finite_abs(x[i]), finite_abs(y[i])));
    float scale = block_scale(wave_max(top));
    float* const scale_at = (is_v ? a.v_scale : a.k_scale) + int64_t(blk) * a.hkv + g;
    uint8_t* const dst = (is_v ? a.v8 : a.k8) + ((int64_t(blk) * a.hkv + g) * kBs + slot) * D + c * W;
    if (t_begin > lb * kBs) {   // the block holds earlier rows: its scale never shrinks
      const float had = *scale_at;
      if (had >= scale) {
        scale = had;
      } else if (t < t_begin) {
        // The same values at the larger scale: where both scales are powers of two (this call's are),
        // exact but for values that fall below the smallest normal code.
        const float f = had / scale;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t* const at = reinterpret_cast<uint32_t*>(dst + half * (D / 2));
#pragma unroll
          for (int i = 0; i < W / 4; ++i) at[i] = rescale_fp8x4(at[i], f);
        }
      }
    }
    const float inv = 1.f / scale;
    auto put = [&](auto code) __attribute__((always_inline)) {
      uint32_t o0[W / 4], o1[W / 4];
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        o0[i] = pack_fp8x4(code(x[4 * i]), code(x[4 * i + 1]), code(x[4 * i + 2]), code(x[4 * i + 3]));
        o1[i] = pack_fp8x4(code(y[4 * i]), code(y[4 * i + 1]), code(y[4 * i + 2]), code(y[4 * i + 3]));
      }
      if constexpr (W == 16) {
        *reinterpret_cast<u32x4*>(dst) = u32x4{o0[0], o0[1], o0[2], o0[3]};
        *reinterpret_cast<u32x4*>(dst + D / 2) = u32x4{o1[0], o1[1], o1[2], o1[3]};
      } else {
        *reinterpret_cast<u32x2*>(dst) = u32x2{o0[0], o0[1]};
        *reinterpret_cast<u32x2*>(dst + D / 2) = u32x2{o1[0], o1[1]};
      }
    };
    if (live) {
      if (__builtin_expect((__float_as_uint(scale) & 0x7FFFFFu) == 0, 1))
        put([&](float v) __attribute__((always_inline)) { return v * inv; });
      else   // (a scale of the caller's, no power of two)
        put([&](float v) __attribute__((always_inline)) { return quotient(v, scale, inv); });
    }
    if (lane == 0) *scale_at = scale;
  }
}

// ---------------------------------------------------------------------------
// Attention of one query row per request over the 8-bit cache (a generated token).
//
// A workgroup takes (request, KV head, up to 16 query heads of its group, run of 32-key
// chunks); its four waves take the run's chunks in turn, each with a softmax state of its
// own, and join their states at the end. Reading the cache once bounds it, so a wave keeps
// the next chunk's keys and values (8 KB at head_dim 128) in flight in registers while it
// works on one.
//  * S^T = K Q^T with v_mfma_f32_16x16x32_bf16. Of a key row, lane group u = l / 16 holds the
//    columns u D/4 .. (whole 16-byte pieces; the order of the columns is the same for Q).
//    Rows of the two 16-key tiles are dealt so that the accumulators of lane group u hold the
//    keys 8 u .. 8 u + 7 of the chunk: with them O^T += V^T P^T needs no exchange of P.
//  * V^T comes from bf16 rows in LDS by transposing reads (ds_read_b64_tr_b16). The rows of
//    a wave are its own: no barrier in the loop.
//  * K's scale multiplies the scores and V's the probabilities before they are rounded to
//    bf16 for the product, which reads bf16; sums are fp32. The row's sum takes the probabilities
//    unrounded (they are at hand, and V's scale is not in them): the outputs' relative rms error
//    against 64 bits is 0.0017 to 0.0018, of which the outputs' own rounding is 0.0017.
// HBM-bound when sequences are long: 64 requests of about 10,367 tokens, 8 KV heads of 128 (1.37 GB) 283 us,
// 4.85 TB/s (a copy 4.7 to 5.3). 16 of about 1,407 (46 MB) 16.0 us, 2.9 TB/s, from the last-level cache (from
// 12 caches in turn, which it does not hold, 18.1): there the chain of length,
// table word, codes, softmax and the join of the runs bounds it, with two launches. The launch bounds name two
// waves a SIMD: left to itself the compiler takes fewer registers and the kernel is 25 % slower.
// ---------------------------------------------------------------------------
struct DecodeArgs {
  const uint16_t* q;
  const uint8_t* k8;
  const uint8_t* v8;
  const float* k_scale;
  const float* v_scale;
  const int32_t* bt;
  const int32_t* seq_lens;
  uint16_t* out;      // splits == 1
  float* part_o;      // else fp32 [splits][batch * hq][D], normalised
  float* part_lse;    // and base-2 log-sum-exp [splits][batch * hq]
  int bt_stride, batch, hq, hkv, group, num_blocks, splits, head_tiles;
  float c_log2;
};

constexpr float kLazy = 8.0f;   // the exponent base moves when a score exceeds it by 2^8
constexpr int kChunk = 32;      // keys of a wave's step
constexpr int kTileHeads = 16;

template <int D>
__global__ __launch_bounds__(kThreads, 2) void decode_attn_fp8_kernel(const DecodeArgs a) {
  constexpr int KS = D / 32;          // MFMA k-steps over D
  constexpr int DT = D / 16;          // output tiles over D
  constexpr int KP = D / 64;          // 16-byte pieces of a key row a lane holds
  constexpr int VP = D / 32;          // 1 KB pieces of a chunk's values (16 bytes a lane)
  constexpr int PITCH = 2 * D + 32;   // LDS bytes per V row: 4 rows of a read on distinct banks
  constexpr int WAVE_LDS = kChunk * PITCH;
  static_assert(WAVE_LDS >= kTileHeads * D * 4, "the waves' outputs are joined in the same memory");
  __shared__ __attribute__((aligned(16))) uint8_t lds[kWaves * WAVE_LDS];
  __shared__ float s_m[kWaves][kTileHeads], s_l[kWaves][kTileHeads];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, u = lane >> 4;
  int w = blockIdx.x;
  const int split = w % a.splits;
  w /= a.splits;
  const int ht = w % a.head_tiles;
  w /= a.head_tiles;
  const int g = w % a.hkv, b = w / a.hkv;
  const int head0 = g * a.group + ht * kTileHeads;
  const int nheads = min(kTileHeads, a.group - ht * kTileHeads);
  const int len = int(min(int64_t(max(a.seq_lens[b], 0)), int64_t(a.bt_stride) * kBs));
  const int chunks = (len + kChunk - 1) / kChunk;
  const int c_begin = int(int64_t(chunks) * split / a.splits), c_end = int(int64_t(chunks) * (split + 1) / a.splits);
  const int32_t* const bt = a.bt + int64_t(b) * a.bt_stride;
  const int last_block = (len + kBs - 1) / kBs - 1;   // (-1 for an empty request, which has no chunk)

  // Queries: lane's column `col`, its D / 4 values from u D / 4 on; zeros without a head.
  bf16x8 qf[KS];
  {
    const u32x4* src = reinterpret_cast<const u32x4*>(
        a.q + (int64_t(b) * a.hq + head0 + (col < nheads ? col : 0)) * D + u * (D / 4));
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 x = src[s];
      if (col >= nheads) x = u32x4{0, 0, 0, 0};
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }

  // A chunk's two cache blocks: -1 for one past the sequence or outside the pool, whose rows
  // read as zeros with scale 1.
  auto block_of = [&](int chunk, int i) __attribute__((always_inline)) -> int {
    const int lb = chunk * 2 + i;
    const int id = bt[min(lb, last_block)];
    return lb <= last_block && id >= 0 && id < a.num_blocks ? id : -1;
  };
  struct Chunk {
    u32x4 k[2][KP], v[VP];
    float ks, vs;   // scales of the block that holds the lane's scores (keys 8 u .. + 7)
  };
  const int key_a = 8 * (col >> 2) + (col & 3);   // key of tile A row `col`; tile B: + 4
  auto load = [&](Chunk& x, int b0, int b1) __attribute__((always_inline)) {
    const u32x4 zero{0, 0, 0, 0};
    const int kb = key_a < kBs ? b0 : b1;
    const uint8_t* kp = a.k8 + ((int64_t(max(kb, 0)) * a.hkv + g) * kBs + (key_a & (kBs - 1))) * D + u * (D / 4);
#pragma unroll
    for (int i = 0; i < KP; ++i) {
      x.k[0][i] = kb >= 0 ? reinterpret_cast<const u32x4*>(kp)[i] : zero;
      x.k[1][i] = kb >= 0 ? reinterpret_cast<const u32x4*>(kp + 4 * D)[i] : zero;
    }
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      const int vb = i < VP / 2 ? b0 : b1;
      const uint8_t* vp = a.v8 + (int64_t(max(vb, 0)) * a.hkv + g) * (kBs * D) + (i % (VP / 2)) * 1024 + lane * 16;
      x.v[i] = vb >= 0 ? *reinterpret_cast<const u32x4*>(vp) : zero;
    }
    const int sb = u < 2 ? b0 : b1;
    x.ks = sb >= 0 ? a.k_scale[int64_t(sb) * a.hkv + g] : 1.f;
    x.vs = sb >= 0 ? a.v_scale[int64_t(sb) * a.hkv + g] : 1.f;
  };

  uint8_t* const own = lds + wave * WAVE_LDS;
  auto widen = [&](uint32_t word, bool high) __attribute__((always_inline)) -> uint32_t {
    // (one instruction; an e4m3 value is a bfloat16 value)
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, 1.f, false));
  };
  auto read_tr = [&](int addr) __attribute__((always_inline)) -> u32x2 {
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    auto* lp = (__attribute__((address_space(3))) uint8_t*)own + addr;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)lp));
  };

  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;   // base of the column's exponents; this lane's part of its sum

  int chunk = c_begin + wave;
  Chunk cur, nxt;
  int n0 = -1, n1 = -1;
  if (chunk < c_end) {
    load(cur, block_of(chunk, 0), block_of(chunk, 1));
    if (chunk + kWaves < c_end) {
      n0 = block_of(chunk + kWaves, 0);
      n1 = block_of(chunk + kWaves, 1);
    }
  }
  for (; chunk < c_end; chunk += kWaves) {
    const bool more = chunk + kWaves < c_end;
    if (more) {
      load(nxt, n0, n1);
      if (chunk + 2 * kWaves < c_end) {
        n0 = block_of(chunk + 2 * kWaves, 0);
        n1 = block_of(chunk + 2 * kWaves, 1);
      }
    }
    const int key0 = chunk * kChunk, left = len - key0;   // keys of the chunk that exist
    // V rows to LDS as bf16, zeros past the sequence (stale codes may be NaN)
#pragma unroll
    for (int i = 0; i < VP; ++i) {
      constexpr int LPR = D / 16;   // lanes a row
      const int key = i * (64 / LPR) + lane / LPR;
      u32x4 x = cur.v[i];
      if (key >= left) x = u32x4{0, 0, 0, 0};
      u32x4* dst = reinterpret_cast<u32x4*>(own + key * PITCH + (lane % LPR) * 32);
      dst[0] = u32x4{widen(x[0], false), widen(x[0], true), widen(x[1], false), widen(x[1], true)};
      dst[1] = u32x4{widen(x[2], false), widen(x[2], true), widen(x[3], false), widen(x[3], true)};
    }
    asm volatile("" ::: "memory");
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int st = 0; st < KS; ++st)
#pragma unroll
      for (int tile = 0; tile < 2; ++tile) {
        const uint32_t w0 = cur.k[tile][st / 2][(st & 1) * 2], w1 = cur.k[tile][st / 2][(st & 1) * 2 + 1];
        const u32x4 kf{widen(w0, false), widen(w0, true), widen(w1, false), widen(w1, true)};
        s[tile] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), qf[st], s[tile], 0, 0, 0);
      }
    float x[8], mx = -INFINITY;
    const float c = a.c_log2 * cur.ks;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = 8 * u + i < left ? s[i >> 2][i & 3] * c : -INFINITY;
      mx = fmaxf(mx, x[i]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__builtin_amdgcn_ballot_w64(mx > m + kLazy || m == -INFINITY) != 0) {
      const float base = fmaxf(m, mx);
      const float alpha = base == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - base);
      m = base;
      l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
    }
    const float base = m == -INFINITY ? 0.f : m;
    uint32_t p[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = __builtin_amdgcn_exp2f(x[2 * i] - base), p1 = __builtin_amdgcn_exp2f(x[2 * i + 1] - base);
      l += p0 + p1;
      p[i] = pack_bf16x2(p0 * cur.vs, p1 * cur.vs);
    }
    const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{p[0], p[1], p[2], p[3]});
    const int v0 = (8 * u + (col >> 2)) * PITCH + (col & 3) * 8;
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      const u32x2 lo = read_tr(v0 + t * 32), hi = read_tr(v0 + 4 * PITCH + t * 32);
      const u32x4 vf{lo[0], lo[1], hi[0], hi[1]};
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vf), pf, o[t], 0, 0, 0);
    }
    asm volatile("" ::: "memory");
    if (more) cur = nxt;
  }

  // ---- the waves' states join: out = sum_w 2^(m_w - M) o_w / sum_w 2^(m_w - M) l_w
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  float* const ow = reinterpret_cast<float*>(own);   // [col][D]
#pragma unroll
  for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(ow + col * D + 16 * t + 4 * u) = o[t];
  if (u == 0) {
    s_m[wave][col] = m;
    s_l[wave][col] = l;
  }
  __syncthreads();
  for (int e = tid; e < nheads * (D / 4); e += kThreads) {
    const int hc = e / (D / 4), d = (e % (D / 4)) * 4;
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) M = fmaxf(M, s_m[i][hc]);
    float sum = 0.f;
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      const float f = s_m[i][hc] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[i][hc] - M);
      const f32x4 part = *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(lds + i * WAVE_LDS) + hc * D + d);
      sum += f * s_l[i][hc];
      acc += f * part;
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;   // (a NaN stays one)
    const int64_t row = int64_t(b) * a.hq + head0 + hc;
    acc *= inv;
    if (a.splits == 1) {
      *reinterpret_cast<u32x2*>(a.out + row * D + d) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
    } else {
      const int64_t at = int64_t(split) * a.batch * a.hq + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = acc;
      if (d == 0) a.part_lse[at] = c_begin < c_end ? M + __log2f(sum) : -INFINITY;
    }
  }
}

// Joins the runs of a row: M = max_p lse_p, out = sum_p 2^(lse_p - M) o_p / sum_p 2^(lse_p - M). One
// workgroup per row, D / 4 columns of 4 values x 1024 / D groups of runs. Rows are few and runs up to 64
// (one lane each), so it is bound by latency: the runs' values are loaded with their sums, all of a
// thread's at once. (A run without keys is written as zeros with -inf.) 32 rows of 128, 24 runs, with
// the attention before it: 11.4 us, 19.1 with lse_merge_kernel, which takes the runs in turn; 4,096 rows, 2 to
// 8 runs: 7 us.
template <int D>
__global__ __launch_bounds__(kThreads) void decode_join_kernel(const float* part_o, const float* part_lse, int parts,
                                                               int64_t rows, uint16_t* out) {
  constexpr int COLS = D / 4, NG = kThreads / COLS;
  constexpr int MOST = cw::kMaxSplits / NG;
  __shared__ __attribute__((aligned(16))) f32x4 s_acc[NG][COLS];
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 63, c = threadIdx.x % COLS, g = threadIdx.x / COLS;
  const float lse = lane < parts ? part_lse[lane * rows + row] : -INFINITY;
  f32x4 v[MOST];
#pragma unroll
  for (int i = 0; i < MOST; ++i) {
    const int p = g + i * NG;
    v[i] = p < parts ? *reinterpret_cast<const f32x4*>(part_o + (p * rows + row) * D + 4 * c) : f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float M = wave_max(lse);
  const float w = lse != -INFINITY ? __builtin_amdgcn_exp2f(lse - M) : 0.f;   // (NaN stays one)
  const float sum = wave_sum(w);
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < MOST; ++i) acc += __shfl(w, min(g + i * NG, 63)) * v[i];
  s_acc[g][c] = acc;
  __syncthreads();
  if (g > 0) return;
#pragma unroll
  for (int i = 1; i < NG; ++i) acc += s_acc[i][c];
  acc *= sum > 0.f || sum != sum ? 1.f / sum : 0.f;
  *reinterpret_cast<u32x2*>(out + row * D + 4 * c) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
}

cw_status check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, std::string(what) + ": " + hipGetErrorString(e));
  return cw::ok();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <int TPR, int CH>
void launch_norm(const NormArgs& a, hipStream_t s) {
  constexpr int RPW = kThreads / TPR;
  hipLaunchKernelGGL((add_rms_norm_fp8_kernel<TPR, CH>), dim3(unsigned((a.rows + RPW - 1) / RPW)), dim3(kThreads), 0,
                     s, a);
}

}  // namespace

extern "C" cw_status cw_add_rms_norm_fp8(const void* x, int64_t x_stride, const void* residual,
                                         int64_t residual_stride, const void* weight, float eps, int64_t rows,
                                         int32_t hidden, void* residual_out, void* out8, float* scales,
                                         void* stream) {
  if (rows < 0) return cw::fail(CW_EINVAL, "add_rms_norm_fp8: rows must be >= 0");
  if (!weight || (rows > 0 && (!x || !out8 || !scales)))
    return cw::fail(CW_EINVAL, "add_rms_norm_fp8: a required pointer is NULL");
  if (!(eps >= 1e-20f && eps <= 1.f)) return cw::fail(CW_EINVAL, "add_rms_norm_fp8: eps must be in [1e-20, 1]");
  if (hidden < 16 || hidden % 16 != 0 || hidden > 16384)
    return cw::fail(CW_EUNSUPPORTED, "add_rms_norm_fp8: hidden must be a multiple of 16 in [16, 16384]");
  if (rows > (1 << 22)) return cw::fail(CW_EUNSUPPORTED, "add_rms_norm_fp8: more than 2^22 rows");
  if (x_stride < hidden || x_stride % 8 != 0 || (residual && (residual_stride < hidden || residual_stride % 8 != 0)))
    return cw::fail(CW_EINVAL, "add_rms_norm_fp8: row strides must be multiples of 8, at least hidden");
  if (rows > 1 && residual_out && ((residual_out == x && x_stride != hidden) ||
                                   (residual_out == residual && residual_stride != hidden)))
    return cw::fail(CW_EINVAL, "add_rms_norm_fp8: residual_out is contiguous: it cannot be rows that lie apart");
  if (!aligned16(x) || !aligned16(residual) || !aligned16(weight) || !aligned16(residual_out) || !aligned16(out8))
    return cw::fail(CW_EINVAL, "add_rms_norm_fp8: pointers must be 16-byte aligned");
  if (rows == 0) return cw::ok();
  NormArgs a;
  a.x = static_cast<const uint16_t*>(x);
  a.residual = static_cast<const uint16_t*>(residual);
  a.weight = static_cast<const uint16_t*>(weight);
  a.residual_out = static_cast<uint16_t*>(residual_out);
  a.out8 = static_cast<uint8_t*>(out8);
  a.scales = scales;
  a.x_stride = x_stride;
  a.residual_stride = residual_stride;
  a.rows = rows;
  a.hidden = hidden;
  a.groups = (hidden + kGroupCols - 1) / kGroupCols;
  a.eps = eps;
  auto* const s = static_cast<hipStream_t>(stream);
  // A wave per row needs no barrier, a workgroup per row spreads few rows over more waves. us in a captured
  // graph, 1, 64, 1,000 and 16,000 rows, wave / workgroup: 512 columns 2.76 / 2.79, 3.20 / 3.06, 3.41 / 3.58,
  // 12.1 / 20.2; 1,024: 3.28 / 2.80, 3.72 / 3.11, 4.26 / 4.04, 19.6 / 24.7 (equal at about 1,600); 2,048:
  // 4.62 / 3.00, 5.19 / 3.32, 6.06 / 4.84, 37.2 / 36.0; 4,096: 7.27 / 3.53, 8.08 / 3.84, 9.78 / 7.16, 89 / 81.
  if (hidden <= 512) launch_norm<64, 1>(a, s);
  else if (hidden <= 1024 && rows > 6 * cw::kNumCu) launch_norm<64, 2>(a, s);
  else if (hidden <= 2048) launch_norm<256, 1>(a, s);
  else if (hidden <= 4096) launch_norm<256, 2>(a, s);
  else if (hidden <= 8192) launch_norm<256, 4>(a, s);
  else launch_norm<256, 8>(a, s);
  return check_launch("add_rms_norm_fp8 launch");
}

extern "C" cw_status cw_rope_append_fp8(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                        const void* v, int64_t v_stride, const float* rope, int32_t rope_len,
                                        void* q_out, void* k8, void* v8, float* k_scale, float* v_scale,
                                        const int32_t* block_table, int32_t bt_stride,
                                        const int32_t* cu_suffix_dev, const int32_t* prefix_len_dev,
                                        const int32_t* cu_suffix_host, const int32_t* prefix_len_host,
                                        int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                        int32_t block_size, int32_t num_blocks, void* stream) {
  const std::string w("rope_append_fp8");
  cw_status st = cw::check_cache_fp8(w.c_str(), k8, v8, k_scale, v_scale, block_table, num_kv_heads, head_dim, block_size, num_blocks);
  if (st != CW_OK) return st;
  if (!cu_suffix_dev || !prefix_len_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (num_q_heads < 0 || num_q_heads > (1 << 20)) return cw::fail(CW_EINVAL, w + ": num_q_heads out of range");
  int64_t rows = 0;
  st = cw::check_batch(cu_suffix_host, prefix_len_host, batch, block_size, bt_stride, &rows, true);
  if (st != CW_OK) return st;
  const bool has_q = q != nullptr || q_out != nullptr;
  if (rows > 0 && (!k || !v || (has_q && (!q || !q_out)))) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (has_q && !rope) return cw::fail(CW_EINVAL, w + ": queries are only rotated: rope is required with them");
  if (has_q && num_q_heads < 1) return cw::fail(CW_EINVAL, w + ": num_q_heads must be >= 1 with queries");
  const int64_t kv_row = int64_t(num_kv_heads) * head_dim, q_row = int64_t(num_q_heads) * head_dim;
  if (k_stride < kv_row || k_stride % 8 != 0 || v_stride < kv_row || v_stride % 8 != 0 ||
      (has_q && (q_stride < q_row || q_stride % 8 != 0)))
    return cw::fail(CW_EINVAL, w + ": row strides must be multiples of 8, at least the heads' columns");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(rope))
    return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  int64_t units = 0, longest = 0;
  for (int32_t r = 0; r < batch; ++r) {
    const int64_t n = cu_suffix_host[r + 1] - cu_suffix_host[r];
    if (n > 0) {
      units += (n + kBs - 2) / kBs + 1;
      longest = std::max(longest, prefix_len_host[r] + n);
    }
  }
  if (rope && longest > rope_len)
    return cw::fail(CW_EINVAL, w + ": rope_len " + std::to_string(rope_len) + " is below the longest prompt (" +
                                   std::to_string(longest) + ")");
  if (longest > INT32_MAX - 2 * kBs) return cw::fail(CW_EUNSUPPORTED, w + ": a prompt of 2^31 - 32 tokens or more");
  if (rows == 0) return cw::ok();
  if (units > kMaxGrid) return cw::fail(CW_EUNSUPPORTED, w + ": batch too large");
  AppendArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.rope = reinterpret_cast<const f32x2*>(rope);
  a.q_out = static_cast<uint16_t*>(q_out);
  a.k8 = static_cast<uint8_t*>(k8);
  a.v8 = static_cast<uint8_t*>(v8);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.bt = block_table;
  a.cu = cu_suffix_dev;
  a.plen = prefix_len_dev;
  a.bt_stride = bt_stride;
  a.batch = batch;
  a.hq = has_q ? num_q_heads : 0;
  a.hkv = num_kv_heads;
  a.num_blocks = num_blocks;
  a.rope_len = rope_len;
  // Heads over grid y: a workgroup per CU at least, and two per unit, so that the last round of a
  // large batch is short; more share the rows' cosines and sines less. us for 1, 2, 3, 4, 6, 12 per unit:
  // 1,030 units of 48 heads 94.3, 84.0, 84.6, 96.4, 85.2, 102.3; 64 units 14.8, 9.4, 8.2, 6.7, 7.0, 7.5;
  // 160 units of 36 heads 13.8, 12.0, 11.0, 12.3, 13.0, 13.6.
  const int64_t heads = a.hq + 2 * int64_t(num_kv_heads), full = (heads + kWaves - 1) / kWaves;
  const int64_t gy = std::min({full, int64_t(65535), std::max<int64_t>(2, (cw::kNumCu + units - 1) / units)});
  auto* const s = static_cast<hipStream_t>(stream);
  if (head_dim == 128)
    hipLaunchKernelGGL(rope_append_fp8_kernel<128>, dim3(unsigned(units), unsigned(gy)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(rope_append_fp8_kernel<64>, dim3(unsigned(units), unsigned(gy)), dim3(kThreads), 0, s, a);
  return check_launch("rope_append_fp8 launch");
}

namespace {
int64_t decode_lse_offset(int64_t rows, int head_dim, int num_splits) {
  return (int64_t(num_splits) * rows * head_dim * 4 + 255) / 256 * 256;
}
}  // namespace

extern "C" int64_t cw_decode_attn_fp8_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t head_dim,
                                                      int32_t num_splits) {
  if (batch < 1 || num_q_heads < 1 || (head_dim != 64 && head_dim != 128) || num_splits < 1 ||
      num_splits > cw::kMaxSplits)
    return cw::fail(CW_EINVAL, "decode_attn_fp8_workspace_bytes: invalid argument");
  if (num_splits == 1) return 0;
  const int64_t rows = int64_t(batch) * num_q_heads;
  return decode_lse_offset(rows, head_dim, num_splits) + int64_t(num_splits) * rows * 4;
}

extern "C" cw_status cw_decode_attn_fp8(const void* q, const void* k8, const void* v8, const float* k_scale,
                                        const float* v_scale, const int32_t* block_table, int32_t bt_stride,
                                        const int32_t* seq_lens_dev, int32_t batch, int32_t num_q_heads,
                                        int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                                        int32_t num_blocks, float softmax_scale, int32_t num_splits,
                                        void* workspace, int64_t workspace_bytes, void* out, void* stream) {
  const std::string w("decode_attn_fp8");
  cw_status st = cw::check_cache_fp8(w.c_str(), k8, v8, k_scale, v_scale, block_table, num_kv_heads, head_dim, block_size, num_blocks);
  if (st != CW_OK) return st;
  if (!q || !out || !seq_lens_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (batch < 1) return cw::fail(CW_EINVAL, w + ": batch must be >= 1");
  if (bt_stride < 1) return cw::fail(CW_EINVAL, w + ": bt_stride must be >= 1");
  if (bt_stride > INT32_MAX / kBs - 1) return cw::fail(CW_EUNSUPPORTED, w + ": sequences of 2^31 tokens or more");
  if (num_q_heads < 1 || num_q_heads % num_kv_heads != 0)
    return cw::fail(CW_EINVAL, w + ": num_q_heads must be a positive multiple of num_kv_heads");
  if (num_q_heads / num_kv_heads > cw::kMaxGroup)
    return cw::fail(CW_EUNSUPPORTED, w + ": more than 128 query heads per KV head");
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return cw::fail(CW_EINVAL, w + ": softmax_scale must be finite and positive");
  if (num_splits < 1 || num_splits > cw::kMaxSplits) return cw::fail(CW_EINVAL, w + ": num_splits must be in [1, 64]");
  if (!aligned16(q) || !aligned16(out)) return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  const int64_t need = cw_decode_attn_fp8_workspace_bytes(batch, num_q_heads, head_dim, num_splits);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return cw::fail(CW_EINVAL, w + ": workspace must hold " + std::to_string(need) + " bytes, 16-byte aligned");
  DecodeArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.k8 = static_cast<const uint8_t*>(k8);
  a.v8 = static_cast<const uint8_t*>(v8);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.bt = block_table;
  a.seq_lens = seq_lens_dev;
  a.out = static_cast<uint16_t*>(out);
  const int64_t rows = int64_t(batch) * num_q_heads;
  a.part_o = num_splits > 1 ? static_cast<float*>(workspace) : nullptr;
  a.part_lse = num_splits > 1 ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) +
                                                         decode_lse_offset(rows, head_dim, num_splits))
                              : nullptr;
  a.bt_stride = bt_stride;
  a.batch = batch;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.group = num_q_heads / num_kv_heads;
  a.num_blocks = num_blocks;
  a.splits = num_splits;
  a.head_tiles = (a.group + kTileHeads - 1) / kTileHeads;
  a.c_log2 = softmax_scale * 1.4426950408889634f;
  const int64_t grid = int64_t(batch) * num_kv_heads * a.head_tiles * num_splits;
  if (grid > kMaxGrid || rows > kMaxGrid) return cw::fail(CW_EUNSUPPORTED, w + ": batch too large");
  auto* const s = static_cast<hipStream_t>(stream);
  if (head_dim == 128)
    hipLaunchKernelGGL(decode_attn_fp8_kernel<128>, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL(decode_attn_fp8_kernel<64>, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  st = check_launch("decode_attn_fp8 launch");
  if (st != CW_OK || num_splits == 1) return st;
  if (head_dim == 128)
    hipLaunchKernelGGL(decode_join_kernel<128>, dim3(unsigned(rows)), dim3(kThreads), 0, s, a.part_o, a.part_lse,
                       num_splits, rows, a.out);
  else
    hipLaunchKernelGGL(decode_join_kernel<64>, dim3(unsigned(rows)), dim3(kThreads), 0, s, a.part_o, a.part_lse,
                       num_splits, rows, a.out);
  return check_launch("decode_attn_fp8 join launch");
}
