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

#include <cstdint>
#include <string>

#include "cw_internal.h"

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
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
  int rows, feats, depth, blocks;   // blocks: of 128 along depth
};

// 128 features x 128 tokens a workgroup, four waves of 64 x 64. Rows of a block are staged as
// 128-byte lines, 16-byte chunk c of row r at c ^ (r / 2 % 8), so that an operand read's 16 rows
// lie on distinct banks.
template <int BF, int BT>
__global__ __launch_bounds__(256) void fp8_linear_kernel(const LinearArgs a) {
  constexpr int WF = BF / 2, WT = BT / 2;   // a wave's share
  constexpr int FB = WF / 32, TT = WT / 16;
  constexpr int CW = BF * 8 / 256, CX = BT * 8 / 256;   // 16-byte chunks a thread stages
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][(BF + BT) * kDepth];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int l16 = lane & 15, u = lane >> 4;
  const int f0 = blockIdx.x * BF, t0 = blockIdx.y * BT;
  const int wf = (wave & 1) * WF, wt = (wave >> 1) * WT;

  u32x4 rw[CW], rx[CX];
  auto load = [&](int kb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      const int c = i * 256 + tid, row = min(f0 + c / 8, a.feats - 1), col = kb * kDepth + (c & 7) * 16;
      rw[i] = col < a.depth ? *reinterpret_cast<const u32x4*>(a.w + int64_t(row) * a.depth + col) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < CX; ++i) {
      const int c = i * 256 + tid, row = min(t0 + c / 8, a.rows - 1), col = kb * kDepth + (c & 7) * 16;
      rx[i] = col < a.depth ? *reinterpret_cast<const u32x4*>(a.x + int64_t(row) * a.depth + col) : u32x4{0, 0, 0, 0};
    }
  };
  auto store = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CW; ++i) {
      const int c = i * 256 + tid, r = c / 8;
      *reinterpret_cast<u32x4*>(&lds[buf][r * kDepth + (((c & 7) ^ ((r >> 1) & 7)) << 4)]) = rw[i];
    }
#pragma unroll
    for (int i = 0; i < CX; ++i) {
      const int c = i * 256 + tid, r = c / 8;
      *reinterpret_cast<u32x4*>(&lds[buf][(BF + r) * kDepth + (((c & 7) ^ ((r >> 1) & 7)) << 4)]) = rx[i];
    }
  };
  auto operand = [&](int buf, int r) __attribute__((always_inline)) -> i32x8 {   // 32 bytes of staged row r
    const int sw = (r >> 1) & 7;
    const u32x4 lo = *reinterpret_cast<const u32x4*>(&lds[buf][r * kDepth + (((2 * u) ^ sw) << 4)]);
    const u32x4 hi = *reinterpret_cast<const u32x4*>(&lds[buf][r * kDepth + (((2 * u + 1) ^ sw) << 4)]);
    return i32x8{int(lo[0]), int(lo[1]), int(lo[2]), int(lo[3]), int(hi[0]), int(hi[1]), int(hi[2]), int(hi[3])};
  };

  f32x4 acc[FB][2][TT];
#pragma unroll
  for (int f = 0; f < FB; ++f)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[f][0][t] = acc[f][1][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  int trow[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) trow[t] = min(t0 + wt + 16 * t + l16, a.rows - 1);

  load(0);
  store(0);
  __syncthreads();
  for (int kb = 0; kb < a.blocks; ++kb) {
    const int buf = kb & 1;
    if (kb + 1 < a.blocks) load(kb + 1);
    float xs[TT], ws[FB];
#pragma unroll
    for (int t = 0; t < TT; ++t) xs[t] = a.xs[int64_t(trow[t]) * a.blocks + kb];
#pragma unroll
    for (int f = 0; f < FB; ++f) ws[f] = a.ws[int64_t(min(f0 + wf + 32 * f, a.feats - 1) / 128) * a.blocks + kb];
    i32x8 xb[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) xb[t] = operand(buf, BF + wt + 16 * t + l16);
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // A row i of half h is feature 8 (i / 4) + 4 h + i % 4 of 32: a lane then holds 8 in a row
        const i32x8 wb = operand(buf, wf + 32 * f + 8 * (l16 >> 2) + 4 * h + (l16 & 3));
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          const f32x4 part =
              __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wb, xb[t], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0, 0, 0, 0);
          const float s = xs[t] * ws[f];
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[f][h][t][i] = fmaf(part[i], s, acc[f][h][t][i]);
        }
      }
    if (kb + 1 < a.blocks) store(buf ^ 1);
    __syncthreads();
  }
#pragma unroll
  for (int f = 0; f < FB; ++f) {
    const int n = f0 + wf + 32 * f + 8 * u;
    if (n >= a.feats) continue;   // (a multiple of 8)
    u32x4 b{0, 0, 0, 0};
    if (a.bias) b = *reinterpret_cast<const u32x4*>(a.bias + n);
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int row = t0 + wt + 16 * t + l16;
      if (row >= a.rows) continue;
      const f32x4 lo = acc[f][0][t], hi = acc[f][1][t];
      *reinterpret_cast<u32x4*>(a.out + int64_t(row) * a.feats + n) =
          u32x4{pack_bf16x2(lo[0] + bf16_lo(b[0]), lo[1] + bf16_hi(b[0])),
                pack_bf16x2(lo[2] + bf16_lo(b[1]), lo[3] + bf16_hi(b[1])),
                pack_bf16x2(hi[0] + bf16_lo(b[2]), hi[1] + bf16_hi(b[2])),
                pack_bf16x2(hi[2] + bf16_lo(b[3]), hi[3] + bf16_hi(b[3]))};
    }
  }
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
  hipLaunchKernelGGL((fp8_linear_kernel<128, 128>), dim3(unsigned((features + 127) / 128), unsigned((rows + 127) / 128)),
                     dim3(256), 0, static_cast<hipStream_t>(stream), a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, std::string("fp8_linear launch: ") + hipGetErrorString(e));
  return cw::ok();
}
