// A paged KV cache in 4 bits for gfx950 (MI355X): the append that rotates and quantises, the
// rows read back, and attention of single tokens over it.
//
// 4 bits are e2m1 (sign, 2 exponent bits, 1 mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6) with one
// power-of-two scale per token, KV head and 32 columns, held as its exponent plus 127 in a byte
// (255: NaN), as the OCP microscaling formats have it. A value is a bfloat16 value, so the
// attention kernels convert without rounding and multiply in bf16 MFMA.
//
// A page is one (block of 16 tokens, KV head): 17 D bytes in one piece,
//   key codes      8 D   token by token, two columns a byte (the lower column in the lower half)
//   value codes    8 D   [token / 4][16 pieces of D / 16 columns][token % 4][columns]
//   key scales     D / 2 [token][D / 32]
//   value scales   D / 2 [D / 32][token]
// so that a lane finds what the matrix instructions want of it in consecutive bytes (the decode kernel
// says why), and a wave reads a page's codes in two instructions.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "cw_fp4.h"
#include "cw_internal.h"

namespace {

using namespace cw4;

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int64_t kMaxGrid = UINT32_MAX / kThreads;   // a launch has fewer than 2^32 threads along an axis

typedef const __attribute__((address_space(4))) int32_t cint32_t;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// ---------------------------------------------------------------------------
// Units of the append and of the read: one cache block that holds rows of the call. Request r
// touches the logical blocks P_r / 16 .. (P_r + S_r - 1) / 16, at most (S_r + 14) / 16 + 1 of them
// whatever P_r is, so a launch depends on the row counts alone.
struct Unit {
  int r, first;        // request (-1: none); first token of the block
  int begin, end;      // the block's tokens that are rows of the call (begin >= end: none)
  int P;               // position of the request's first row
  int64_t row0;        // its place in the rows
};

__device__ __forceinline__ Unit find_unit(const int32_t* cu, const int32_t* plen, int batch, int* s_unit) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    const int b = blockIdx.x;
    int base = 0, rr = -1, jb = 0;
    for (int r0 = 0; r0 < batch; r0 += 64) {
      const int r = r0 + tid;
      const int rows = r < batch ? cu[r + 1] - cu[r] : 0;
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
  Unit u;
  u.r = __builtin_amdgcn_readfirstlane(s_unit[0]);
  u.begin = u.end = u.first = u.P = 0;
  u.row0 = 0;
  if (u.r < 0) return u;
  u.row0 = cu[u.r];
  const int rows = cu[u.r + 1] - int(u.row0);
  u.P = plen[u.r];
  if (u.P < 0 || u.P > INT32_MAX - rows - 2 * kBs) return u;   // (the end of the block behind the last row is counted too)
  u.first = (u.P / kBs + __builtin_amdgcn_readfirstlane(s_unit[1])) * kBs;
  u.begin = max(u.P, u.first);
  u.end = min(u.P + rows, u.first + kBs);
  return u;
}

// ---------------------------------------------------------------------------
// Append: rotary embedding, then 4-bit codes and scales.
//
// A wave takes one (four tokens of a block, head) at a time: lane l holds the columns D / 16 (l % 16) ..
// of token l / 16 of the four, so loads and stores are whole rows, of value pages too. A rotation's other
// column is in the same lane (neighbours) or in another of the 16 (halves). Each group of 32 columns lies
// in 512 / D neighbouring lanes. The wave keeps its tokens' cosines and sines over all its heads, and has the
// rows of four heads in flight at once.
//
// A value next to a border of two codes has to fall on its side of it, so keys are rotated by the
// difference of two products without cancellation error (t = w s; d = x c - t; d - (w s - t), at
// most 1.5 units off in the last place), and a wave that holds a value within 4 such units of a
// border (they all have a mantissa of 2 bits) rotates again, exactly: few waves do.
// HBM-bound: reads 2 (Hq + 2 Hkv) D bytes a row, writes 2 Hq D + 17/16 Hkv D. 16,128 rows of 32 / 8 heads of 128:
// 72 us, 4.8 TB/s (a copy 4.8 to 5.3); 64 requests of one row 4.7 us in a captured graph, 18 called one by one
// with a split of the projection's rows and the read, which is the host's time. A wave with 16 tokens of a head at a
// time, whose 64-bit form took 250 registers: 89 and 9.6; one row in flight 130; a wait for stores before each head 103.
struct AppendArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  int64_t q_stride, k_stride, v_stride;   // elements from one row to the next
  const f32x2* rope;                      // NULL: no rotation
  uint16_t* q_out;
  uint8_t* pages;
  const int32_t* bt;
  const int32_t* cu;
  const int32_t* plen;
  int bt_stride, batch, hq, hkv, num_blocks, rope_len, pairs;   // hq 0: no queries; pairs: rotated columns / 2
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
  return uint32_t(__builtin_amdgcn_mov_dpp(int(x), CTRL, 0xF, 0xF, true));
}
// Largest of 4 (D = 128) or 8 (D = 64) neighbouring lanes.
template <int D>
__device__ __forceinline__ uint32_t group_max(uint32_t x) {
  x = max(x, dpp<0xB1>(x));              // lane ^ 1
  x = max(x, dpp<0x4E>(x));              // lane ^ 2
  if (D == 64) x = max(x, dpp<0x141>(x));   // 7 - lane of 8
  return x;
}

// x c - w s, at most 1.5 units off in the last place.
__device__ __forceinline__ float turned(float x, float w, float c, float s) {
  const float t = w * s;
  return fmaf(x, c, -t) - fmaf(w, s, -t);
}
// The same with its last bit set where it is not exact: rounded on to fewer bits it goes where the
// exact value goes, as it is never halfway by rounding alone. Both products are exact in 64 bits, their sum is not
// where they lie more than 53 bits apart (a tiny partner beside a border): what the sum lost decides where the rest of
// its 53 bits is zero, and is less than that rest otherwise. (Few waves look at it: computed for all values it took 9
// registers more, a wave a SIMD, and 16,128 rows 2 % more time; so, with six waves a SIMD named, none. Not marked
// as the unlikely way it spills 110 registers.)
__device__ __forceinline__ float turned_to_odd(float x, float w, float c, float s) {
  asm volatile("" : "+v"(c), "+v"(s));   // (else the table is converted ahead of the loop over heads, in 32 registers)
  const double a = double(x) * double(c), b = -(double(w) * double(s)), y = a + b;
  const float v = float(y);
  double rest = y - double(v);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(rest == 0.) != 0, 0)) {
    const double lost = fabs(a) >= fabs(b) ? b - (y - a) : a - (y - b);   // a + b - y
    if (rest == 0.) rest = lost;
  }
  const uint32_t bits = __float_as_uint(v);
  if (rest == 0. || (bits & 1) != 0 || !(fabsf(v) > 0x1p-110f) || !(fabsf(v) < INFINITY)) return v;   // (a code of so small a value is zero)
  return __uint_as_float((rest > 0.) == (v > 0.f) ? bits + 1 : bits - 1);
}

// HALVES: column j is paired with j + pairs; else 2 j with 2 j + 1. ONCE: rows in and queries out pass the caches'
// order of use.
template <int D, bool HALVES, bool ONCE>
__global__ __launch_bounds__(kThreads, 6) void rope_append_fp4_kernel(const AppendArgs a) {
  constexpr int PC = D / 16;    // columns a lane holds
  constexpr int NT = HALVES ? PC : PC / 2;   // (cos, sin) pairs a lane needs
  using Words = typename Piece<D>::Bf16;     // PC bfloat16 values
  __shared__ int s_unit[2];
  const Unit un = find_unit(a.cu, a.plen, a.batch, s_unit);
  if (un.begin >= un.end) return;
  const int lb = un.first / kBs;
  const int blk = lb < a.bt_stride ? a.bt[int64_t(un.r) * a.bt_stride + lb] : -1;
  const bool in_pool = blk >= 0 && blk < a.num_blocks;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int p = lane & 15, u = lane >> 4, col = p * PC;
  const bool turns = a.rope != nullptr && col < 2 * a.pairs;   // this lane's columns are rotated
  const bool upper = HALVES && col >= a.pairs;
  const int partner = (lane & 48) | (turns && HALVES ? (upper ? col - a.pairs : col + a.pairs) / PC : p);
  const bool far8 = a.pairs == D / 2;   // halves of the whole head: the partner is lane ^ 8 of the 16
  const int j0 = !turns ? 0 : HALVES ? (upper ? col - a.pairs : col) : col / 2;
  const bool first_of_group = (p & (512 / D - 1)) == 0;
  const int grp = p / (512 / D);

  // The four waves share the fours of tokens that have rows, and where these are fewer than three the heads.
  const int i_begin = (un.begin - un.first) / 4, fours = (un.end - un.first + 3) / 4 - i_begin;
  const int share = fours >= 3 ? 1 : fours == 2 ? 2 : 4;   // waves of a four
  const int i = i_begin + wave / share;
  if (i >= i_begin + fours) return;
  const int heads = a.hq + 2 * a.hkv, step = int(gridDim.y) * share, h0 = int(blockIdx.y) * share + wave % share;
  const int t = un.first + 4 * i + u, slot = 4 * i + u;
  const bool live = t >= un.begin && t < un.end;
  const int64_t row = un.row0 + ((live ? t : un.begin) - un.P);
  auto load = [&](int h) __attribute__((always_inline)) -> Words {
    const uint16_t* base = h < a.hq ? a.q + int64_t(h) * D
                           : h < a.hq + a.hkv ? a.k + int64_t(h - a.hq) * D
                                              : a.v + int64_t(h - a.hq - a.hkv) * D;
    const int64_t stride = h < a.hq ? a.q_stride : h < a.hq + a.hkv ? a.k_stride : a.v_stride;
    Words x{};
    if (live) {
      const auto* const at = reinterpret_cast<const Words*>(base + row * stride + col);
      x = ONCE ? __builtin_nontemporal_load(at) : *at;
    }
    return x;
  };
  float cs[NT], sn[NT];
  if (a.rope) {
    const f32x4* src = reinterpret_cast<const f32x4*>(a.rope + int64_t(min(live ? t : un.begin, a.rope_len - 1)) * a.pairs + j0);
#pragma unroll
    for (int n = 0; n < NT / 2; ++n) {
      const f32x4 two = src[n];
      cs[2 * n] = two[0];
      sn[2 * n] = upper ? -two[1] : two[1];
      cs[2 * n + 1] = two[2];
      sn[2 * n + 1] = upper ? -two[3] : two[3];
    }
  }
  auto work = [&](const Words in, int h) __attribute__((always_inline)) {
    const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
    if (!is_q && !in_pool) return;
    float x[PC];
#pragma unroll
    for (int j = 0; j < PC / 2; ++j) {
      x[2 * j] = bf16_lo(in[j]);
      x[2 * j + 1] = bf16_hi(in[j]);
    }
    if (a.rope && !is_v) {
      Words other{};
      if constexpr (HALVES) {
        if (far8) {
#pragma unroll
          for (int j = 0; j < PC / 2; ++j) other[j] = dpp<0x128>(in[j]);
        } else {
#pragma unroll
          for (int j = 0; j < PC / 2; ++j) other[j] = uint32_t(__shfl(int(in[j]), partner));
        }
      }
      auto turn_all = [&](auto turn) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < PC / 2; ++j) {
          const float lo = bf16_lo(in[j]), hi = bf16_hi(in[j]);
          float y0, y1;
          if (HALVES) {
            y0 = turn(lo, bf16_lo(other[j]), cs[2 * j % NT], sn[2 * j % NT]);
            y1 = turn(hi, bf16_hi(other[j]), cs[(2 * j + 1) % NT], sn[(2 * j + 1) % NT]);
          } else {
            y0 = turn(lo, hi, cs[j % NT], sn[j % NT]);
            y1 = turn(hi, lo, cs[j % NT], -sn[j % NT]);
          }
          x[2 * j] = turns ? y0 : lo;
          x[2 * j + 1] = turns ? y1 : hi;
        }
      };
      if (is_q) {   // (an infinite value stays one: turned would subtract it from itself)
        turn_all([](float x, float w, float c, float s) __attribute__((always_inline)) { return fmaf(x, c, -(w * s)); });
      } else {
        turn_all(turned);
        bool near = false;
#pragma unroll
        for (int j = 0; j < PC; ++j) near |= ((__float_as_uint(x[j]) + 4) & 0x1FFFFFu) <= 8 && x[j] != 0.f;
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(near && turns) != 0, 0)) turn_all(turned_to_odd);
      }
    }
    if (is_q) {
      Words o;
#pragma unroll
      for (int j = 0; j < PC / 2; ++j) o[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
      if (live) {
        auto* const at = reinterpret_cast<Words*>(a.q_out + (row * a.hq + h) * D + col);
        if constexpr (ONCE) __builtin_nontemporal_store(o, at);
        else *at = o;
      }
      return;
    }
    const int g = h - a.hq - (is_v ? a.hkv : 0);
    uint8_t* const page = a.pages + (int64_t(blk) * a.hkv + g) * kPage<D>;
    uint32_t top = 0;   // as an integer: an infinity or a NaN is above every finite value
#pragma unroll
    for (int j = 0; j < PC; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    top = group_max<D>(top);
    // the smallest e with top <= 7 * 2^e: 7 = 1.75 * 2^2, and a mantissa above 1.75 carries
    const int e = min(max(int((top + 0x1FFFFFu) >> 23) - 127 - 2, kMinExp), kMaxExp);
    const bool bad = top >= 0x7F800000u;
    const uint32_t exp = bad ? 255u : uint32_t(e + 127);
    const uint32_t code = bad ? 0u : encode<PC>(x, __uint_as_float(uint32_t(e + 127) << 23));
    if (live) {
      const int at = is_v ? kValues<D> + ((i * 16 + p) * 4 + u) * (D / 32) : slot * (D / 2) + p * (D / 32);
      *reinterpret_cast<typename Piece<D>::Code*>(page + at) = typename Piece<D>::Code(code);
      if (first_of_group)
        page[is_v ? kValueScales<D> + grp * kBs + slot : kKeyScales<D> + slot * (D / 32) + grp] = uint8_t(exp);
    }
  };
  constexpr int ROWS = 4;
  constexpr int kAllLoaded = 0x0F70;   // vmcnt(0), no other counter
  for (int h = h0; h < heads; h += ROWS * step) {
    Words in[ROWS];
#pragma unroll
    for (int n = 0; n < ROWS; ++n)
      if (h + n * step < heads) in[n] = load(h + n * step);
    __builtin_amdgcn_s_waitcnt(kAllLoaded);   // (else every head's work begins with a wait for the stores before it)
#pragma unroll
    for (int n = 0; n < ROWS; ++n)
      if (h + n * step < heads) work(in[n], h + n * step);
  }
}

// ---------------------------------------------------------------------------
// Rows of the cache as bf16. A wave takes one (block, head, keys or values): lane l converts the
// columns D / 16 (l % 16) .. of four tokens, so that a store writes whole rows of four tokens.
// HBM-bound by what it writes, past the caches' order of use: 4 D bytes a token and head for 17 D / 16 read. 133,700
// tokens of 8 heads of 128 (693 MB) 133 us, 5.2 TB/s, with ordinary stores 142; 832 tokens 3.7 us in a captured graph.
struct RowsArgs {
  const uint8_t* pages;
  const int32_t* bt;
  const int32_t* cu;
  const int32_t* plen;
  uint16_t* k_rows;   // NULL: no keys
  uint16_t* v_rows;   // NULL: no values
  int bt_stride, batch, hkv, num_blocks;
};

template <int D>
__global__ __launch_bounds__(kThreads) void cache_rows_fp4_kernel(const RowsArgs a) {
  constexpr int PC = D / 16;
  using Words = typename Piece<D>::Bf16;
  using Code = typename Piece<D>::Code;
  __shared__ int s_unit[2];
  const Unit un = find_unit(a.cu, a.plen, a.batch, s_unit);
  if (un.begin >= un.end) return;
  const int lb = un.first / kBs;
  const int blk = lb < a.bt_stride ? a.bt[int64_t(un.r) * a.bt_stride + lb] : -1;
  const bool in_pool = blk >= 0 && blk < a.num_blocks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int p = lane & 15, u = lane >> 4, grp = p / (512 / D);
  for (int w = int(blockIdx.y) * kWaves + wave; w < 2 * a.hkv; w += int(gridDim.y) * kWaves) {
    const bool is_v = w >= a.hkv;
    uint16_t* const rows = is_v ? a.v_rows : a.k_rows;
    if (!rows) continue;
    const int g = w - (is_v ? a.hkv : 0);
    const uint8_t* const page = a.pages + (int64_t(in_pool ? blk : 0) * a.hkv + g) * kPage<D>;
    uint32_t code[4], exp[4];   // of the tokens 4 u + i (values), 4 i + u (keys)
    if (is_v) {
      const auto c = *reinterpret_cast<const typename Piece<D>::Lane*>(page + kValues<D> + lane * (D / 8));
      const uint32_t e = *reinterpret_cast<const uint32_t*>(page + kValueScales<D> + grp * kBs + 4 * u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        code[i] = D == 128 ? c[i % (D / 32)] : c[i / 2] >> (16 * (i & 1));
        exp[i] = e >> (8 * i) & 0xFFu;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        code[i] = *reinterpret_cast<const Code*>(page + (4 * i + u) * (D / 2) + p * (D / 32));
        exp[i] = page[kKeyScales<D> + (4 * i + u) * (D / 32) + grp];
      }
    }
    if (!in_pool)
#pragma unroll
      for (int i = 0; i < 4; ++i) code[i] = exp[i] = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = un.first + (is_v ? 4 * u + i : 4 * i + u);
      Words o;
      const float s = __uint_as_float(exp[i] << 23);
      o[0] = widen<0>(code[i], s);
      o[1] = widen<1>(code[i], s);
      if constexpr (PC == 8) {
        o[2] = widen<2>(code[i], s);
        o[3] = widen<3>(code[i], s);
      }
      if (t >= un.begin && t < un.end)
        __builtin_nontemporal_store(o, reinterpret_cast<Words*>(rows + ((un.row0 + (t - un.P)) * a.hkv + g) * D + p * PC));
    }
  }
}

// ---------------------------------------------------------------------------
// Attention of one query row per request (a generated token).
//
// A workgroup takes (request, KV head, up to 16 query heads of its group, run of 32-key chunks);
// each of its waves takes a part of the run, with a softmax state of its own, and they join their
// states at the end. Reading the cache once bounds it. A wave reads pages straight into registers
// in the operand layout of v_mfma_f32_16x16x32_bf16, a page in four instructions, a chunk ahead;
// nothing passes through LDS:
//  * S^T = K Q^T. Lane (c, u) = (l % 16, l / 16) holds of key c the columns u D / 4 .. + D / 4 - 1,
//    consecutive bytes with one scale (the order of the columns is the same for Q). Its
//    accumulators are the scores of the keys 4 u .. 4 u + 3 of a block for query column c.
//  * O^T += V^T P^T with the keys in the order of those scores (4 u .. of block 0, 4 u .. of block 1),
//    so P needs no exchange. Lane (c, u) holds the columns D / 16 c .. of those four tokens of a
//    block, consecutive bytes; output tile j takes column j of each piece: row c is column
//    D / 16 c + j. A conversion gives two columns of a token, and a byte permute two tokens of a
//    column.
// The base of a column's exponents is the row maximum of the wave's first chunk and moves only when
// a lane's sum passes 2^26 (bf16 and fp32 have the range), so later chunks need no maximum. Four lanes hold parts of
// a column's sum and four waves join unnormalised: weights of 2^30 in all, so values up to 2^96 stay in fp32's range.
// The row's sum takes the probabilities as they are rounded for the product.
// HBM-bound when sequences are long: 64 requests of about 10,367 tokens, 64 / 8 heads of 128 (720 MB) 136 us, 5.3 TB/s
// (a copy 4.8 to 5.3). Of few chunks it is bound by the chain of length, table word, codes, scores, softmax, product
// and join (4.2 us for 300 tokens of 4 heads of 64), and by a wave's instructions: a chunk is 146 vector ones, 64 of
// them conversions and 32 permutes, and takes a lone wave 0.7 us whether one, two or three chunks are in flight ahead.
// More waves a workgroup (8, 12, 16) in place of runs: 16 x 1,407 tokens 12.6, 12.2, 12.0 against 12.0, 1 x 9,000 34 to
// 37 against 8.7.
// n / d for n < 2^31 by a multiplication: a division in software is 25 instructions, and a workgroup with few
// chunks has several ahead of its first load.
struct FastDiv {
  uint32_t mul, shift, d;
  explicit FastDiv(uint32_t by = 1) : shift(0), d(by) {
    while ((uint64_t(1) << shift) < by) ++shift;
    mul = uint32_t(((uint64_t(1) << (31 + shift)) + by - 1) / by);
    shift += 31;
  }
  __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return uint32_t((uint64_t(n) * mul) >> shift); }
};

struct DecodeArgs {
  const uint16_t* q;
  const uint8_t* pages;
  const int32_t* bt;
  const int32_t* seq_lens;
  uint16_t* out;      // splits == 1
  float* part_o;      // else fp32 [splits][batch * hq][D], normalised
  float* part_lse;    // and base-2 log-sum-exp [splits][batch * hq]
  int bt_stride, batch, hq, hkv, group, num_blocks, splits;
  FastDiv by_splits, by_tiles, by_heads;   // division by splits, by the head tiles of a group, by hkv
  float c_log2;
};

constexpr int kChunk = 32;      // keys of a wave's step: two blocks
constexpr int kTileHeads = 16;
constexpr float kMaxSum = 0x1p26f;   // of a lane's part of a column's sum

constexpr int kAhead = 1;       // chunks in flight ahead of the one that a wave works on
constexpr int kRawBuffer = 0x00027000;   // a buffer's last word: bytes at offsets, checked against its size

template <int D, bool ONCE>
__device__ __forceinline__ typename Piece<D>::Lane load_lane(__amdgpu_buffer_rsrc_t page, int offset) {
  constexpr int AUX = ONCE ? 2 : 0;   // non-temporal
  if constexpr (D == 128) return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(page, offset, 0, AUX));
  else return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(page, offset, 0, AUX));
}

// ONCE: the codes are read past the caches' order of use.
template <int D, bool ONCE>
__global__ __launch_bounds__(kThreads, 3) void decode_attn_fp4_kernel(const DecodeArgs a) {
  constexpr int KS = D / 32;          // MFMA k-steps over D
  constexpr int DT = D / 16;          // output tiles over D, and columns of a lane's piece
  using Lane = typename Piece<D>::Lane;
  __shared__ __attribute__((aligned(16))) float s_o[kWaves][kTileHeads][D];
  __shared__ float s_m[kWaves][kTileHeads], s_l[kWaves][kTileHeads];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, u = lane >> 4;
  uint32_t w = a.by_splits.quotient(blockIdx.x);
  const int split = int(blockIdx.x - w * a.by_splits.d);
  uint32_t x = a.by_tiles.quotient(w);
  const int ht = int(w - x * a.by_tiles.d);
  const int b = int(a.by_heads.quotient(x));
  const int g = int(x - uint32_t(b) * a.by_heads.d);
  const int seq = reinterpret_cast<cint32_t*>(reinterpret_cast<uintptr_t>(a.seq_lens))[b];
  const int head0 = g * a.group + ht * kTileHeads;
  const int nheads = min(kTileHeads, a.group - ht * kTileHeads);
  const int len = min(max(seq, 0), a.bt_stride * kBs);   // (the host keeps bt_stride below 2^27 - 256)
  const int chunks = (len + kChunk - 1) / kChunk;
  // runs and parts of runs differ by one chunk at most
  const int per = int(a.by_splits.quotient(uint32_t(chunks))), over = chunks - per * a.splits;
  const int c_begin = per * split + min(split, over), c_len = per + (split < over ? 1 : 0);
  const int w_begin = c_begin + c_len * wave / kWaves, w_end = c_begin + c_len * (wave + 1) / kWaves;
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

  struct Chunk {
    Lane k[2], v[2];
    uint32_t ks[2], vs[2];   // scale of the key's columns; of the four tokens' columns
  };
  const uint8_t* const pages = a.pages + int64_t(g) * kPage<D>;
  const int64_t block_bytes = int64_t(a.hkv) * kPage<D>;
  // Table words, 64 blocks (32 chunks) at a time, block i's in lane i.
  auto words = [&](int chunk) __attribute__((always_inline)) -> int {
    return bt[min(chunk * 2 + lane, max(last_block, 0))];
  };
  int ids = -1, ids_next = -1, ids_at = w_begin;   // of the chunks ids_at .. + 31, and of the 32 after them
  if (w_begin < w_end) {
    ids = words(w_begin);
    if (w_end - w_begin > 32) ids_next = words(w_begin + 32);
  }
  const int ko = col * (D / 2) + u * (D / 8), vo = kValues<D> + lane * (D / 8);
  const int kso = kKeyScales<D> + col * (D / 32) + u * (D / 4) / 32;
  const int vso = kValueScales<D> + col * DT / 32 * kBs + 4 * u;
  auto load = [&](Chunk& x, int chunk) __attribute__((always_inline)) {
    if (chunk - ids_at >= 32) {
      ids = ids_next;
      ids_at += 32;
      ids_next = words(ids_at + 32);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (past the sequence, or outside the pool: a buffer of no bytes, whose loads give zeros)
      const int id = __builtin_amdgcn_readlane(ids, __builtin_amdgcn_readfirstlane((chunk - ids_at) * 2 + i));
      const bool ok = chunk * 2 + i <= last_block && uint32_t(id) < uint32_t(a.num_blocks);
      const auto page = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(pages + int64_t(ok ? id : 0) * block_bytes), 0,
                                                          ok ? kPage<D> : 0, kRawBuffer);
      x.k[i] = load_lane<D, ONCE>(page, ko);
      x.v[i] = load_lane<D, ONCE>(page, vo);
      x.ks[i] = __builtin_amdgcn_raw_buffer_load_b8(page, kso, 0, 0);
      x.vs[i] = __builtin_amdgcn_raw_buffer_load_b32(page, vso, 0, 0);
    }
  };

  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;   // base of the column's exponents; this lane's part of its sum
  const bf16x2 ones{(__bf16)1.0f, (__bf16)1.0f};

  auto work = [&](const Chunk& x, int chunk) __attribute__((always_inline)) {
    const int left = len - chunk * kChunk;   // keys of the chunk that exist
    f32x4 s[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float ks = __uint_as_float(x.ks[i] << 23);
      s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int st = 0; st < KS; ++st) {
        const uint32_t c = x.k[i][st];
        const u32x4 kf{widen<0>(c, ks), widen<1>(c, ks), widen<2>(c, ks), widen<3>(c, ks)};
        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), qf[st], s[i], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);   // (here and below: else conversions far ahead hold registers)
    }
    uint32_t vs[2] = {x.vs[0], x.vs[1]};
    if (__builtin_expect(left < kChunk, 0)) {
      // keys past the sequence: no score, and a finite scale (a stale one may be NaN)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * i + 4 * u + r >= left) {
            s[i][r] = -INFINITY;
            vs[i] &= ~(0xFFu << (8 * r));
          }
    }
    auto top = [&]() __attribute__((always_inline)) -> float {   // the column's maximum, scaled
      float mx = s[0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[i >> 2][i & 3]);
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      return mx * a.c_log2;
    };
    if (__builtin_expect(m == -INFINITY, 0)) {   // (no column has a base but after a chunk of the wave)
      const float mx = top();
      m = mx > -INFINITY && mx < INFINITY ? mx : 0.f;
    }
    uint32_t pk[4];
    float l_new;
    for (bool moved = false;; moved = true) {
      l_new = l;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = (i & 1) * 2;
        pk[i] = pack_bf16x2(__builtin_amdgcn_exp2f(fmaf(s[i >> 1][at], a.c_log2, -m)),
                            __builtin_amdgcn_exp2f(fmaf(s[i >> 1][at + 1], a.c_log2, -m)));
        l_new = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pk[i]), ones, l_new, false);
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(l_new > kMaxSum) == 0 || moved, 1)) break;
      // The base moves, by all lanes of a column alike, to the larger of this chunk's maximum and what
      // the earlier chunks' sum stands for: sums and products are then at most 1 and 32. Once is enough;
      // what is out of range by then (NaN, infinities) stays as it is.
      float most = fmaxf(l_new, __shfl_xor(l_new, 16));
      most = fmaxf(most, __shfl_xor(most, 32));
      float had = fmaxf(l, __shfl_xor(l, 16));
      had = fmaxf(had, __shfl_xor(had, 32));
      const float mx = top();
      const float to = most > kMaxSum ? fmaxf(mx < INFINITY ? mx : m, had > 1.f ? m + __builtin_amdgcn_logf(had) : m) : m;
      const float alpha = __builtin_amdgcn_exp2f(m - to);
      l *= alpha;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] *= alpha;
      m = to;
    }
    l = l_new;
    const bf16x8 pf = __builtin_bit_cast(bf16x8, u32x4{pk[0], pk[1], pk[2], pk[3]});
    float sc[2][4];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[i][t] = __uint_as_float((vs[i] >> (8 * t) & 0xFFu) << 23);
#pragma unroll
    for (int j = 0; j < DT; j += 2) {
      uint32_t wd[2][4];   // columns j, j + 1 of token t of block i
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if constexpr (D == 128) wd[i][t] = widen_at(x.v[i][t], j / 2, sc[i][t]);
          else wd[i][t] = widen_at(x.v[i][t / 2], (t & 1) * 2 + j / 2, sc[i][t]);
        }
      u32x4 lo, hi;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          lo[2 * i + t] = __builtin_amdgcn_perm(wd[i][2 * t + 1], wd[i][2 * t], 0x05040100u);
          hi[2 * i + t] = __builtin_amdgcn_perm(wd[i][2 * t + 1], wd[i][2 * t], 0x07060302u);
        }
      o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, lo), pf, o[j], 0, 0, 0);
      o[j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hi), pf, o[j + 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // Chunks in flight, each in registers of its own: the loop is unrolled over them.
  Chunk ring[kAhead + 1];
#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (w_begin + i < w_end) load(ring[i], w_begin + i);
  for (int chunk = w_begin; chunk < w_end;) {
#pragma unroll
    for (int i = 0; i <= kAhead; ++i) {
      if (chunk + kAhead < w_end) load(ring[(i + kAhead) % (kAhead + 1)], chunk + kAhead);
      work(ring[i], chunk);
      if (++chunk >= w_end) break;
    }
  }

  // ---- the waves' states join: out = sum_w 2^(m_w - M) o_w / sum_w 2^(m_w - M) l_w
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // Row c' of tile j is column D / 16 c' + j: the lane's accumulators 4 u + r of all tiles are the
  // columns u D / 4 + r D / 16 + j of its query.
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < DT; j += 4)
      *reinterpret_cast<f32x4*>(&s_o[wave][col][u * (D / 4) + r * DT + j]) = f32x4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
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
      sum += f * s_l[i][hc];
      acc += f * *reinterpret_cast<const f32x4*>(&s_o[i][hc][d]);
    }
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;   // (a NaN stays one)
    const int64_t row = int64_t(b) * a.hq + head0 + hc;
    acc *= inv;
    if (a.splits == 1) {
      *reinterpret_cast<u32x2*>(a.out + row * D + d) = u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
    } else {
      const int64_t at = int64_t(split) * a.batch * a.hq + row;
      *reinterpret_cast<f32x4*>(a.part_o + at * D + d) = acc;
      if (d == 0) a.part_lse[at] = c_len > 0 ? M + __log2f(sum) : -INFINITY;
    }
  }
}

cw_status check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return cw::fail(CW_EHIP, std::string(what) + ": " + hipGetErrorString(e));
  return cw::ok();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Units of a batch and its longest prompt among requests with rows.
void count_units(const int32_t* cu, const int32_t* plen, int batch, int64_t* units, int64_t* longest) {
  *units = *longest = 0;
  for (int32_t r = 0; r < batch; ++r) {
    const int64_t n = cu[r + 1] - cu[r];
    if (n > 0) {
      *units += (n + kBs - 2) / kBs + 1;
      *longest = std::max(*longest, plen[r] + n);
    }
  }
}

}  // namespace

extern "C" cw_status cw_rope_append_fp4(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                        const void* v, int64_t v_stride, const float* rope, int32_t rope_len,
                                        int32_t rotary_dim, int32_t interleaved, void* q_out, void* pages,
                                        const int32_t* block_table, int32_t bt_stride, const int32_t* cu_suffix_dev,
                                        const int32_t* prefix_len_dev, const int32_t* cu_suffix_host,
                                        const int32_t* prefix_len_host, int32_t batch, int32_t num_q_heads,
                                        int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                                        int32_t num_blocks, void* stream) {
  const std::string w("rope_append_fp4");
  cw_status st = cw::check_cache_fp4(w.c_str(), pages, block_table, num_kv_heads, head_dim, block_size, num_blocks);
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
  if (rope && (rotary_dim < 16 || rotary_dim > head_dim || rotary_dim % 16 != 0))
    return cw::fail(CW_EINVAL, w + ": rotary_dim must be a multiple of 16 in [16, head_dim]");
  if (interleaved != 0 && interleaved != 1) return cw::fail(CW_EINVAL, w + ": interleaved must be 0 or 1");
  const int64_t kv_row = int64_t(num_kv_heads) * head_dim, q_row = int64_t(num_q_heads) * head_dim;
  if (k_stride < kv_row || k_stride % 8 != 0 || v_stride < kv_row || v_stride % 8 != 0 ||
      (has_q && (q_stride < q_row || q_stride % 8 != 0)))
    return cw::fail(CW_EINVAL, w + ": row strides must be multiples of 8, at least the heads' columns");
  if (has_q && rows > 1 && q_out == q && q_stride != q_row)
    return cw::fail(CW_EINVAL, w + ": q_out is contiguous: it cannot be rows that lie apart");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(rope))
    return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  int64_t units, longest;
  count_units(cu_suffix_host, prefix_len_host, batch, &units, &longest);
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
  a.pages = static_cast<uint8_t*>(pages);
  a.bt = block_table;
  a.cu = cu_suffix_dev;
  a.plen = prefix_len_dev;
  a.bt_stride = bt_stride;
  a.batch = batch;
  a.hq = has_q ? num_q_heads : 0;
  a.hkv = num_kv_heads;
  a.num_blocks = num_blocks;
  a.rope_len = rope_len;
  a.pairs = rope ? rotary_dim / 2 : 0;
  // Heads over grid y: a workgroup per CU at least; four per unit, eight where units hold many rows. us for 1, 2, 4,
  // 8, 12 per unit: 1,030 units of about 15.7 rows, 48 heads of 128, 92, 88, 82, 79, 85; 160 units of 12.5, 36 heads,
  // 15.2, 15.6, 12.4, 11.6, 11.4; 256 units of one row, 48 heads, 10.1, 8.3, 7.5, 9.7, 11.1.
  const int64_t heads = a.hq + 2 * int64_t(num_kv_heads), full = (heads + kWaves - 1) / kWaves;
  const int64_t gy = std::min({full, int64_t(65535), std::max<int64_t>(rows >= 8 * units ? 8 : 4, (cw::kNumCu + units - 1) / units)});
  // More rows than the last-level cache (256 MiB) holds pass it: 16,128 rows of 48 heads of 128 (330 MB) 72 us against
  // 79; 2,000 of 36 (32 MB) 12.0 against 11.6.
  const bool once = rows * (2 * (a.hq + int64_t(num_kv_heads))) * head_dim * 2 > (int64_t(256) << 20);
  auto pick = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return interleaved ? (once ? rope_append_fp4_kernel<D, false, true> : rope_append_fp4_kernel<D, false, false>)
                       : (once ? rope_append_fp4_kernel<D, true, true> : rope_append_fp4_kernel<D, true, false>);
  };
  auto* const kernel = head_dim == 128 ? pick(std::integral_constant<int, 128>()) : pick(std::integral_constant<int, 64>());
  hipLaunchKernelGGL(kernel, dim3(unsigned(units), unsigned(gy)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return check_launch("rope_append_fp4 launch");
}

extern "C" cw_status cw_cache_rows_fp4(const void* pages, const int32_t* block_table, int32_t bt_stride,
                                       const int32_t* cu_rows_dev, const int32_t* first_dev,
                                       const int32_t* cu_rows_host, const int32_t* first_host, int32_t batch,
                                       int32_t num_kv_heads, int32_t head_dim, int32_t block_size,
                                       int32_t num_blocks, void* k_rows, void* v_rows, void* stream) {
  const std::string w("cache_rows_fp4");
  cw_status st = cw::check_cache_fp4(w.c_str(), pages, block_table, num_kv_heads, head_dim, block_size, num_blocks);
  if (st != CW_OK) return st;
  if (!cu_rows_dev || !first_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  int64_t rows = 0;
  st = cw::check_batch(cu_rows_host, first_host, batch, block_size, bt_stride, &rows, true);
  if (st != CW_OK) return st;
  if (!aligned16(k_rows) || !aligned16(v_rows)) return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  int64_t units, longest;
  count_units(cu_rows_host, first_host, batch, &units, &longest);
  if (longest > INT32_MAX - 2 * kBs) return cw::fail(CW_EUNSUPPORTED, w + ": a prompt of 2^31 - 32 tokens or more");
  if (rows == 0 || (!k_rows && !v_rows)) return cw::ok();
  if (units > kMaxGrid) return cw::fail(CW_EUNSUPPORTED, w + ": batch too large");
  RowsArgs a;
  a.pages = static_cast<const uint8_t*>(pages);
  a.bt = block_table;
  a.cu = cu_rows_dev;
  a.plen = first_dev;
  a.k_rows = static_cast<uint16_t*>(k_rows);
  a.v_rows = static_cast<uint16_t*>(v_rows);
  a.bt_stride = bt_stride;
  a.batch = batch;
  a.hkv = num_kv_heads;
  a.num_blocks = num_blocks;
  const int64_t full = (2 * int64_t(num_kv_heads) + kWaves - 1) / kWaves;
  const int64_t gy = std::min({full, int64_t(65535), std::max<int64_t>(1, (2 * cw::kNumCu + units - 1) / units)});
  auto* const kernel = head_dim == 128 ? cache_rows_fp4_kernel<128> : cache_rows_fp4_kernel<64>;
  hipLaunchKernelGGL(kernel, dim3(unsigned(units), unsigned(gy)), dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  return check_launch("cache_rows_fp4 launch");
}

namespace {
int64_t lse_offset(int64_t rows, int head_dim, int num_splits) {
  return (int64_t(num_splits) * rows * head_dim * 4 + 255) / 256 * 256;
}
}  // namespace

extern "C" int64_t cw_decode_attn_fp4_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t head_dim,
                                                      int32_t num_splits) {
  if (batch < 1 || num_q_heads < 1 || (head_dim != 64 && head_dim != 128) || num_splits < 1 ||
      num_splits > cw::kMaxSplits)
    return cw::fail(CW_EINVAL, "decode_attn_fp4_workspace_bytes: invalid argument");
  const int64_t rows = int64_t(batch) * num_q_heads;
  if (rows > kMaxGrid) return cw::fail(CW_EUNSUPPORTED, "decode_attn_fp4_workspace_bytes: batch too large");
  if (num_splits == 1) return 0;
  return lse_offset(rows, head_dim, num_splits) + int64_t(num_splits) * rows * 4;
}

extern "C" cw_status cw_decode_attn_fp4(const void* q, const void* pages, const int32_t* block_table,
                                        int32_t bt_stride, const int32_t* seq_lens_dev, int32_t batch,
                                        int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                        int32_t block_size, int32_t num_blocks, float softmax_scale,
                                        int32_t num_splits, void* workspace, int64_t workspace_bytes, void* out,
                                        void* stream) {
  const std::string w("decode_attn_fp4");
  cw_status st = cw::check_cache_fp4(w.c_str(), pages, block_table, num_kv_heads, head_dim, block_size, num_blocks);
  if (st != CW_OK) return st;
  if (!q || !out || !seq_lens_dev) return cw::fail(CW_EINVAL, w + ": a required pointer is NULL");
  if (batch < 1) return cw::fail(CW_EINVAL, w + ": batch must be >= 1");
  if (bt_stride < 1) return cw::fail(CW_EINVAL, w + ": bt_stride must be >= 1");
  if (bt_stride > INT32_MAX / kBs - 256) return cw::fail(CW_EUNSUPPORTED, w + ": sequences of 2^31 - 4096 tokens or more");
  if (num_q_heads < 1 || num_q_heads % num_kv_heads != 0)
    return cw::fail(CW_EINVAL, w + ": num_q_heads must be a positive multiple of num_kv_heads");
  if (num_q_heads / num_kv_heads > cw::kMaxGroup)
    return cw::fail(CW_EUNSUPPORTED, w + ": more than 128 query heads per KV head");
  if (!(softmax_scale > 0.f) || !std::isfinite(softmax_scale))
    return cw::fail(CW_EINVAL, w + ": softmax_scale must be finite and positive");
  if (num_splits < 1 || num_splits > cw::kMaxSplits) return cw::fail(CW_EINVAL, w + ": num_splits must be in [1, 64]");
  if (!aligned16(q) || !aligned16(out)) return cw::fail(CW_EINVAL, w + ": pointers must be 16-byte aligned");
  const int64_t need = cw_decode_attn_fp4_workspace_bytes(batch, num_q_heads, head_dim, num_splits);
  if (need < 0) return cw_status(need);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return cw::fail(CW_EINVAL, w + ": workspace must hold " + std::to_string(need) + " bytes, 16-byte aligned");
  DecodeArgs a;
  a.q = static_cast<const uint16_t*>(q);
  a.pages = static_cast<const uint8_t*>(pages);
  a.bt = block_table;
  a.seq_lens = seq_lens_dev;
  a.out = static_cast<uint16_t*>(out);
  const int64_t rows = int64_t(batch) * num_q_heads;
  a.part_o = num_splits > 1 ? static_cast<float*>(workspace) : nullptr;
  a.part_lse = num_splits > 1 ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) +
                                                         lse_offset(rows, head_dim, num_splits))
                              : nullptr;
  a.bt_stride = bt_stride;
  a.batch = batch;
  a.hq = num_q_heads;
  a.hkv = num_kv_heads;
  a.group = num_q_heads / num_kv_heads;
  a.num_blocks = num_blocks;
  a.splits = num_splits;
  const int head_tiles = (a.group + kTileHeads - 1) / kTileHeads;
  a.by_splits = FastDiv(num_splits);
  a.by_tiles = FastDiv(head_tiles);
  a.by_heads = FastDiv(num_kv_heads);
  a.c_log2 = softmax_scale * 1.4426950408889634f;
  const int64_t grid = int64_t(batch) * num_kv_heads * head_tiles * num_splits;
  if (grid > kMaxGrid) return cw::fail(CW_EUNSUPPORTED, w + ": batch too large");
  auto* const s = static_cast<hipStream_t>(stream);
  // What the last-level cache (256 MiB) cannot hold is read past it. us, 64 requests of about 10,367 tokens,
  // 720 MB: 138 against 153; 8 heads of 9,000 tokens, 10 MB, read again and again: 60 against 55. The host knows the
  // table's width alone: short sequences behind a table for long ones are read past the cache, too.
  const bool once = int64_t(batch) * bt_stride * num_kv_heads * 17 * head_dim > (int64_t(256) << 20);
  auto* const kernel = head_dim == 128 ? (once ? decode_attn_fp4_kernel<128, true> : decode_attn_fp4_kernel<128, false>)
                                       : (once ? decode_attn_fp4_kernel<64, true> : decode_attn_fp4_kernel<64, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(kThreads), 0, s, a);
  st = check_launch("decode_attn_fp4 launch");
  if (st != CW_OK || num_splits == 1) return st;
  return cw::decode_join("decode_attn_fp4", head_dim, a.part_o, a.part_lse, num_splits, rows, out, stream);
}
