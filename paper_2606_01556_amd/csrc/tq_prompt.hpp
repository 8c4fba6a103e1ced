// Attention of many new tokens over the paged cache (prompts, chunks of prompts, tokens to
// verify), and of a batch's tokens over a prefix that they share:
//
//   o_r = sum_j softmax_j(s_rj) v_j,  s_rj = cap tanh(scale q_r . k_j / cap) - slope |p_r - j|,
//   j in [lo_r, hi_r)
//
// (cap and slope or neither).  Every mask that a call can ask for (causal, window, prefix,
// documents) leaves a row one interval, so the kernel knows two numbers a row and no mask.
//
// A row r is a new token and one of the query heads of a key-value head's group: a work-group
// holds 128 rows of one key-value head, 32 to a wavefront, and runs over the keys in tiles of
// 64, which it stages in LDS for its four wavefronts.
//
//  * S^T = K Q^T in 32x32x16 products with the rows as columns: a lane holds scores of one
//    row (lane % 32) for keys 8 i + 4 (lane / 32) + (0 .. 3).  What a row needs (its interval,
//    reference, sum) is one register, and a tile's largest weight is a maximum within lanes.
//  * Two such runs of four keys, exponentiated and rounded, are the second operand of
//    O^T = V^T P^T as they stand: which keys make up a product is free as long as V^T's operand
//    takes the same, and LDS reads it transposed, four keys of a channel at a time.
//  * The reference of the softmax moves only when a weight passes 65504 (bf16 rows: 1 over the
//    number of keys), as in the attention of one token: most tiles neither exchange
//    anything between lanes nor scale what has been summed.
//  * A weight is rounded once to the second product's type (fp16: 2^-11 of itself at most, and
//    2^-37 of the largest one; bf16 rows, whose values may pass fp16's range: 2^-8).  The
//    products are what bounds the kernel, and more terms of a weight are more products; the
//    roundings of different keys are independent and come out below the result's own.  The
//    sum that divides, and the log-sum-exp, take the weights unrounded, in fp32.  FINE: what the
//    rounding leaves enters as a second term, for callers whose next step magnifies last bits.
//  * Rows of 16 bits go from memory to LDS directly, 16 bytes a lane, swizzled by the address
//    that a lane reads, so that rows a few apart lie in different banks; codes are widened on
//    their way, exactly, and their scales apply to scores and weights in fp32.
//  * Tiles of which all rows see all keys come first, in a loop without a mask; a tile's loads
//    are in flight while the one before it is computed on, and keys are half a tile ahead: while
//    32 keys' scores become weights the next 32 keys' are formed, a matrix product at a time.
//
// Keys that a row does not see have no part in it, whatever they hold: a tile in which any
// row's interval ends is searched for infinities and NaN, and where there is one the values
// enter the products without it, and the rows that do see it get a NaN by a product of ones.
//
// Measured, where the products are the bound (PyTorch's bf16 product of two 8192 x 8192 matrices
// reaches 1.22 to 1.27 PFLOP/s on the same card):
//   1 prompt of 8192 tokens, 32 / 8 heads of 128, fp16          561 us, 980 TFLOP/s (exact: 764, 719)
//   2048 tokens behind 30720, 64 / 8 heads of 128, 8 bits      2500 us, 852 TFLOP/s (exact: 3336, 639)
//   2 prompts of 4096, 16 / 8 heads of 256, window 1024, capped 192 us, 518 TFLOP/s (exact: 217, 456)
// (another card of the kind: 624, 2796 and 194 us)
// The matrix cores are busy half of the first's cycles, without bank conflicts, and the clock is
// at 1.9 GHz of 2.4: as steps took cycles away (1.38 million at first, 1.07 now) it went down
// from 2.05.  Left out one at a time (in a copy), the loads give 75 us back, the exponentials 45,
// the maxima 40, half of the second products 58: no single one holds the others up.  With keys a
// whole tile ahead the first takes 548 us, but codes spill registers (8 bits 4100 to 7100 us) and
// 32 prompts up to 700 take 134 us for 121; with none ahead 569, and 215 for the 191.
//
// Registers that the kernels spill as they are: head_dim 128 at 8 bits 8 (exact 19, capped or biased
// 34 to 37), at 4 bits none (exact 5, capped or biased 14 to 23), at 16 bits none (capped or biased 5
// to 8); head_dim 64 at 16 bits, capped or biased, 8 to 15, where three wavefronts a SIMD leave 168.
#pragma once

#include <cfloat>

#include "tq_attention.hpp"
#include "tq_kernels.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

constexpr int kPromptWaves = 4, kPromptThreads = 64 * kPromptWaves;
constexpr int kTileKeys = 64;
constexpr int kLeastTiles = 4;             // of a split
constexpr float kTopBinades = 15.99f;      // 2^15.99 < 65504

// wavefronts of a SIMD that the registers are cut for
constexpr int prompt_occupancy(int d, int bits) { return d == 256 ? 1 : d == 128 || bits < 16 ? 2 : 3; }

// Bytes of LDS: two tiles of keys, two of values, and (codes) what goes with them: the keys'
// scales; the values' as binades and inverse, and which of them are not finite.  Then four bounds a
// wavefront and a flag.
constexpr int kKeyScales = kTileKeys * 4, kValueScales = kTileKeys * 8 + 16;
constexpr int prompt_tiles(int d, int bits) { return kTileKeys * d * 8 + (bits < 16 ? 2 * (kKeyScales + kValueScales) : 0); }
constexpr int prompt_lds_bytes(int d, int bits) { return prompt_tiles(d, bits) + 64 * kPromptWaves; }

template <bool BF16>
__device__ __forceinline__ v16f mfma32(u32x4 a, u32x4 b, v16f c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// a wave-uniform pointer, in scalar registers
__device__ __forceinline__ const uint8_t *uniform_at(const uint8_t *p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const uint8_t *>((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}
// this wavefront's loads and LDS accesses done, then all wavefronts'
__device__ __forceinline__ void wait_all() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
// Four 16-bit values of one column: of 16 lanes, lanes 4 r .. 4 r + 3 address row r's 16 values,
// and lane i gets column i of the four rows.
__device__ __forceinline__ u32x2 read_columns(const uint8_t *p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p));
}

// the halves of w whose exponent is all ones, as their top bits
template <bool BF16>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return BF16 ? ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u : ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u;
}

// the two values of a word
template <bool BF16>
__device__ __forceinline__ float lower_half(uint32_t w) {
  return BF16 ? __builtin_bit_cast(float, w << 16) : half_bits_to_float((uint16_t)w);
}
template <bool BF16>
__device__ __forceinline__ float upper_half(uint32_t w) {
  return BF16 ? __builtin_bit_cast(float, w & 0xffff0000u) : half_bits_to_float((uint16_t)(w >> 16));
}

struct Interval {
  int lo, hi;
};

// How a score is made of its product: by a factor alone; capped or biased; with a cap past 64, whose
// two ways would cost the others registers (16 / 4 heads of 64: 97 us for 86).
enum Scored { kPlain, kCapped, kCappedWide };

template <int D, int BITS, bool BF16, Scored HOW, bool FINE>
__global__ __launch_bounds__(kPromptThreads, prompt_occupancy(D, BITS)) void prompt_kernel(const PromptArgs a) {
  constexpr int KT = kTileKeys, W = kPromptWaves, T = kPromptThreads;
  constexpr int RB = D * BITS / 8;              // bytes of a cache row
  constexpr int LB = D * 2, LC = LB / 16;       // bytes and 16-byte pieces of a row in LDS
  constexpr int KS = D / 16, DT = D / 32;
  constexpr bool VBF = BITS == 16 && BF16;      // type of the second product
  constexpr bool EXT = HOW != kPlain;
  constexpr int TB = KT * LB;                   // bytes of a tile in LDS
  constexpr auto key_tile = [](int odd) { return odd * TB; };
  constexpr auto value_tile = [](int odd) { return (2 + odd) * TB; };
  constexpr auto key_scales = [](int odd) { return 4 * TB + odd * kKeyScales; };
  constexpr auto value_scales = [](int odd) { return 4 * TB + 2 * kKeyScales + odd * kValueScales; };
  constexpr uint32_t kOne = VBF ? 0x3f80u : 0x3c00u;

  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  int *const bounds = reinterpret_cast<int *>(smem + prompt_tiles(D, BITS)), *const flag = bounds + 4 * W;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;

  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int r32 = lane & 31, half = lane >> 5;
  const int hkv = a.c.heads, lps = a.c.lps;
  // tiles of the longest intervals first (a causal prompt's last ones)
  const int kvh = blockIdx.x % hkv, unit = blockIdx.x / hkv, split = unit % a.splits;
  const int tile = a.tiles - 1 - unit / a.splits;

  auto start_of = [&](int i) -> int { return min(max(a.starts[i], 0), a.tokens); };

  // rows of no stream, cleared at the end (in shared mode the join leaves them to the tokens' own keys)
  const int stream_rows = a.shared ? 0 : start_of(0), stream_end = a.shared ? a.tokens : start_of(a.batch);
  auto clear = [&]() {
    if (threadIdx.x >= 64) return;
    for (int i = blockIdx.x; i < stream_rows + a.tokens - stream_end; i += gridDim.x) {
      const int64_t row = (int64_t)(i < stream_rows ? i : i - stream_rows + stream_end) * a.hq;
      for (int e = lane; e < a.hq * (D / 2); e += 64) reinterpret_cast<uint32_t *>(a.out + row * D)[e] = 0;
      if (a.lse != nullptr)
        for (int e = lane; e < a.hq; e += 64) a.lse[row + e] = -INFINITY;
    }
  };

  // The stream whose tile this is.  Stream i's tiles are numbered from floor(rows before it / 128) +
  // i: numbers enough for each, in order, without a sum over the streams; so it is the last whose
  // first number is not past this tile, found 64 candidates at a time, which bring its start, its
  // end and its length along.
  int s = 0, start, after, length;
  for (int n = a.batch;;) {
    const int step = (n + 63) / 64, i = s + lane * step;
    const int first = start_of(min(i, a.batch)), long_ = a.lengths[min(i, a.batch - 1)];
    const bool before = lane * step < n && (int)((int64_t)first * a.group / kPromptRows) + i <= tile;
    const int count = max(__builtin_popcountll(__ballot(before)), 1) - 1;
    s = uniform(s + count * step);
    if (step == 1) {
      start = uniform(__shfl(first, count));
      length = uniform(__shfl(long_, count));
      after = uniform(count < 63 ? __shfl(first, count + 1) : start_of(s + 1));
      break;
    }
    n = uniform(min(step, n - count * step));
  }
  const int tokens = after - start;
  const int at = tile - ((int)((int64_t)start * a.group / kPromptRows) + s);
  const int row0 = at * kPromptRows, rows = tokens * a.group;     // < 2^31 (host)
  if (at < 0 || row0 >= rows) {
    clear();
    return;
  }

  // tiles of keys that are a work-group's share
  int share = 0;
  if (a.splits > 1) {
    int64_t all = 0;
    for (int i = lane; i < a.batch; i += 64) {
      const int rows_i = (start_of(i + 1) - start_of(i)) * a.group, keys_i = min(max(a.lengths[i], 0), a.longest);
      all += (int64_t)((rows_i + kPromptRows - 1) / kPromptRows) * ((keys_i + KT - 1) / KT);
    }
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) all += __shfl_xor(all, x);
    share = uniform((int)max((all * hkv + a.room - 1) / a.room, (int64_t)kLeastTiles));
  }

  // this lane's row and its interval
  const int cap = a.max_pages << lps;                             // <= 2^30 (host)
  const int len = min(max(length, 0), cap);
  const bool live = row0 + 32 * w < rows;                         // the wavefront holds rows
  const int row = min(row0 + 32 * w + r32, rows - 1);
  const int token = (int)((uint32_t)row / (uint32_t)a.group), head = kvh * a.group + (row - token * a.group);
  int pos;
  Interval seen;
  if (a.shared) {
    const int own = min(max(a.own[start + token], 0), a.own_most);
    pos = len + own - 1;
    seen = {0, len};
  } else {
    pos = len - tokens + token;
    seen = {0, max(pos + 1, 0)};
    if (a.prefix != nullptr) seen.hi = max(seen.hi, min(a.prefix[s], len));
    if (a.window > 0 && pos >= a.window) seen.lo = pos - a.window + 1;
    if (a.first != nullptr) seen.lo = max(seen.lo, a.first[start + token]);
  }
  // (a row that sees nothing takes part in no bound; what it sums up is dropped at the end)
  const bool sees = seen.lo < seen.hi;

  // bounds of the wavefront's rows, and of all rows
  int lo_min = sees ? seen.lo : INT32_MAX, lo_max = sees ? seen.lo : 0, hi_min = sees ? seen.hi : INT32_MAX, hi_max = sees ? seen.hi : 0;
#pragma unroll
  for (int m = 1; m < 32; m <<= 1) {
    lo_min = min(lo_min, __shfl_xor(lo_min, m)); lo_max = max(lo_max, __shfl_xor(lo_max, m));
    hi_min = min(hi_min, __shfl_xor(hi_min, m)); hi_max = max(hi_max, __shfl_xor(hi_max, m));
  }
  lo_min = uniform(lo_min); lo_max = uniform(lo_max); hi_min = uniform(hi_min); hi_max = uniform(hi_max);
  if (lane == 0) {
    bounds[4 * w] = lo_min; bounds[4 * w + 1] = lo_max; bounds[4 * w + 2] = hi_min; bounds[4 * w + 3] = hi_max;
    if (w == 0) *flag = 0;
  }

  // Q^T: column r32, values 16 k + 8 half ...  (the scale's sign goes to Q)
  u32x4 q[KS];
  {
    const uint16_t *qp = a.q + (int64_t)(start + token) * a.q_ts + (int64_t)head * a.q_hs + 8 * half;
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int k = 0; k < KS; k++) {
      q[k] = *reinterpret_cast<const u32x4 *>(qp + 16 * k);
#pragma unroll
      for (int i = 0; i < 4; i++) q[k][i] ^= flip;
    }
  }
  __syncthreads();
  int all_lo = INT32_MAX, all_lo_max = 0, all_hi_min = INT32_MAX, all_hi = 0;
#pragma unroll
  for (int i = 0; i < W; i++) {
    all_lo = min(all_lo, bounds[4 * i]); all_lo_max = max(all_lo_max, bounds[4 * i + 1]);
    all_hi_min = min(all_hi_min, bounds[4 * i + 2]); all_hi = max(all_hi, bounds[4 * i + 3]);
  }
  all_lo = uniform(all_lo); all_lo_max = uniform(all_lo_max); all_hi_min = uniform(all_hi_min); all_hi = uniform(all_hi);

  // This split's keys [k0, k1), from a multiple of 64.  Where there are splits, a work-group is to
  // have about its share of all streams' tiles (as their lengths leave them), so that a long
  // stream has many parts and a short one few.
  int k0 = 0, k1 = 0;
  if (all_lo < all_hi) {
    const int base = all_lo & ~(KT - 1), n = (all_hi - base + KT - 1) / KT;
    int parts = 1;
    if (a.splits > 1) parts = min(a.splits, max((n + share - 1) / share, 1));
    if (split < parts) {
      k0 = base + (int)((int64_t)n * split / parts) * KT;
      k1 = min(base + (int)((int64_t)n * (split + 1) / parts) * KT, all_hi);
    }
  }

  // what a score's product with the key's scale is multiplied by, in binades
  const float c1 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-149f);     // (-infinity times it has to stay so)
  const Shape shape = EXT ? shape_of(a.scale, a.cap, c1, 1.0f) : Shape{};
  const float slope = EXT && a.slopes != nullptr ? a.slopes[head] * kLog2e : 0.0f;
  // binades above the reference at which it has to move, and where it puts the largest weight
  float most = kTopBinades, headroom = kHeadroom;
  if constexpr (VBF) {
    // (a shared prefix: its sums are added to those of a stream's own keys, half the range each)
    most = (float)(__builtin_clz(max(len, 1)) - 32 - (a.shared ? 1 : 0));
    headroom = most - kBelow;
  }

  v16f o[DT];
#pragma unroll
  for (int i = 0; i < DT; i++) o[i] = v16f{0};
  float m = -FLT_MAX, l = 0.0f;      // (finite: keys whose score is -infinity have the weight 0 also before the first other one)

  // ---- loads.  A wavefront takes 16 rows of a tile, which lie in one page; keys outside the
  // rows' intervals take the nearest one's row.
  const_i32 *const pages = (const_i32 *)(a.table + s * a.table_stride);
  auto held = [&](int key) -> int { return min(max(key, all_lo), all_hi - 1); };
  constexpr int PIECE = BITS == 16 ? 16 : KT * RB / T < 16 ? KT * RB / T : 16;    // bytes of a lane's load
  constexpr int PR = RB / PIECE, LR = 64 / PR, NL = 16 / LR;                      // lanes of a row, rows of a load, loads
  static_assert(LR <= 16 && NL * LR == 16 && 16 * W == KT);
  const int lrow = lane / PR, lpiece = lane % PR;
  const uint32_t in_page = (1u << lps) - 1;
  auto page_of = [&](int k) -> int { return uniform(pages[held(k + 16 * w) >> lps]); };
  const uint32_t page_rows = (uint32_t)hkv << lps;                // <= 2^25 (host)
  const int64_t first_row = (int64_t)kvh << lps;
  auto swizzle = [](int r, bool value) -> int { return value ? 4 * (LC > 8 ? r & 3 : r >> 1 & 1) : (LC > 8 ? r & 15 : r >> 1 & 7); };
  constexpr int NR = BITS < 16 ? NL : 1;
  u32x4 kraw[NR], vraw[NR];                                       // codes on their way
  uint16_t kscale = 0, vscale = 0;
  // The keys or values from k on (in that page) to LDS, or codes to registers.  inside: all of
  // them lie between the intervals' ends.
  auto load = [&](auto value, u32x4 (&raw)[NR], uint16_t &scale, int k, int page, uint32_t to, auto inside) __attribute__((always_inline)) {
    constexpr bool INSIDE = decltype(inside)::value;
    constexpr bool VALUE = decltype(value)::value;
    const int k16 = k + 16 * w;
    int64_t rows = (int64_t)((uint64_t)(uint32_t)min(max(page, 0), a.c.pages - 1) * page_rows) + first_row;
    if constexpr (INSIDE) rows += (uint32_t)k16 & in_page;
    const uint8_t *const p = uniform_at((VALUE ? a.c.v : a.c.k) + rows * RB);
    auto go = [&](auto row_of) {
#pragma unroll
      for (int i = 0; i < NL; i++) {
        const int r = i * LR + lrow;
        const uint32_t off = row_of(r) * RB;
        if constexpr (BITS == 16) {
          load_to_lds(off + 16 * (lpiece ^ swizzle(r, VALUE)), p, lds0 + to + w * 16 * LB + i * 1024);
        } else if constexpr (PIECE == 16) {
          raw[i] = *reinterpret_cast<const u32x4 *>(p + off + 16 * lpiece);
        } else {
          const u32x2 x = *reinterpret_cast<const u32x2 *>(p + off + 8 * lpiece);
          raw[i] = u32x4{x.x, x.y, 0, 0};
        }
      }
      // (16 lanes each: 0 to 15 the keys' scales, 16 to 31 the values')
      if constexpr (BITS < 16)
        if (lane >> 4 == (VALUE ? 1 : 0)) scale = (VALUE ? a.c.vs : a.c.ks)[rows + row_of(lane & 15)];
    };
    if constexpr (INSIDE) go([](int r) -> uint32_t { return r; });
    else go([&](int r) -> uint32_t { return (uint32_t)held(k16 + r) & in_page; });
  };
  // codes as 16-bit values in LDS: keys in Q's type, values in fp16
  auto widen = [&](auto value, const u32x4 (&raw)[NR], uint16_t scale, uint32_t tile_at, uint32_t scales) __attribute__((always_inline)) {
    if constexpr (BITS < 16) {
      constexpr bool VALUE = decltype(value)::value, TO = BF16 && !VALUE;
      constexpr int WORDS = PIECE / 4, PER = BITS == 8 ? 2 : 1;   // words of a piece, words of 8 codes
#pragma unroll
      for (int i = 0; i < NL; i++) {
        const int r = 16 * w + i * LR + lrow;
#pragma unroll
        for (int e = 0; e < WORDS / PER; e++) {
          uint32_t w0, w1, y0, y1, y2, y3;
          if constexpr (BITS == 8) { w0 = raw[i][2 * e]; w1 = raw[i][2 * e + 1]; }
          else tq4_to_fp8(raw[i][e], w0, w1);
          widen4<TO>(w0, BITS == 4 ? 512.0f : 1.0f, y0, y1);
          widen4<TO>(w1, BITS == 4 ? 512.0f : 1.0f, y2, y3);
          *reinterpret_cast<u32x4 *>(smem + tile_at + r * LB + 16 * ((lpiece * (WORDS / PER) + e) ^ swizzle(r, VALUE))) = u32x4{y0, y1, y2, y3};
        }
      }
      // The keys' scales; the values' as binades and their inverse.  (A value scale of zero, whose
      // codes are zero, counts as fp16's smallest, and so do infinity and NaN, whose rows are
      // marked: binades of infinity would be added to the scores of rows that do not see it, too.)
      float *const to = reinterpret_cast<float *>(smem + scales) + 16 * w + (lane & 15);
      const float x = half_bits_to_float(scale);
      const bool none = VALUE && (scale & 0x7c00u) == 0x7c00u;
      if (lane >> 4 == (VALUE ? 1 : 0)) {
        if constexpr (!VALUE) {
          to[0] = x;
        } else {
          const float y = none ? kLeastScale : fmaxf(x, kLeastScale);
          to[0] = __builtin_amdgcn_logf(y);
          to[KT] = 1.0f / y;
        }
      }
      if constexpr (VALUE) {
        const uint64_t nan = __ballot(none);
        if (lane == 0) reinterpret_cast<uint16_t *>(smem + scales + 8 * KT)[w] = (uint16_t)(nan >> 16);
      }
    }
  };

  // ---- addresses of the two kinds of LDS reads
  const uint32_t kx = swizzle(r32, false);
  const uint32_t krow = r32 * LB;
  const int tq = lane >> 4, ti = lane & 15;
  const int vr = 4 * (tq >> 1) + (ti >> 2);
  const uint32_t vx = swizzle(vr, true);
  const uint32_t vrow = vr * LB + (ti & 1) * 8, vc = 2 * (tq & 1) + ((ti & 3) >> 1);

  // A tile is taken in halves of 32 keys, i = 0, 1.
  auto key_of = [&](int i, int v) -> int { return 32 * i + 8 * (v >> 2) + 4 * half + (v & 3); };
  auto scale4 = [&](uint32_t scales, int i, int g) -> v4f { return *reinterpret_cast<const v4f *>(smem + scales + 4 * key_of(i, 4 * g)); };
  const uint32_t count = sees ? (uint32_t)(seen.hi - seen.lo) : 0u;
  auto masked = [&](int k, int i, int v) -> bool { return (uint32_t)(k + key_of(i, v) - seen.lo) >= count; };
  // products of Q and half a tile's keys, times the keys' scales
  auto times_scales = [&](v16f &sc, uint32_t kscales, int i) __attribute__((always_inline)) {
    if constexpr (BITS < 16) {
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const v4f x = scale4(kscales, i, g);
#pragma unroll
        for (int j = 0; j < 4; j++) sc[4 * g + j] *= x[j];
      }
    }
  };
  constexpr bool BINADES = EXT || BITS < 16;
  // Scores of half a tile from its products: in binades (16-bit rows without cap and bias: before
  // their factor), values' scales among them; the reference moved where it has to be.
  // edge: some row does not see all keys.
  auto refer = [&](v16f &sc, int k, int i, uint32_t vscales, auto edge) __attribute__((always_inline)) {
    if constexpr (EXT) {
      if (a.cap > 0.0f) {
        cap_scores<16, HOW == kCappedWide>([&](int v) -> float { return sc[v]; }, [&](int v, float y) { sc[v] = y; }, shape);
      } else {
#pragma unroll
        for (int v = 0; v < 16; v++) sc[v] *= c1;
      }
      if (a.slopes != nullptr) {
        const float far = (float)(k + 4 * half - pos);
#pragma unroll
        for (int v = 0; v < 16; v++) sc[v] = fmaf(-slope, fabsf(far + (float)(32 * i + 8 * (v >> 2) + (v & 3))), sc[v]);
      }
    }
    if constexpr (decltype(edge)::value) {
#pragma unroll
      for (int v = 0; v < 16; v++) sc[v] = masked(k, i, v) ? -INFINITY : sc[v];
    }
    if constexpr (BITS < 16) {
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const v4f x = scale4(vscales, i, g);
#pragma unroll
        for (int j = 0; j < 4; j++) sc[4 * g + j] = EXT ? sc[4 * g + j] + x[j] : fmaf(sc[4 * g + j], c1, x[j]);
      }
    }
    float y = -INFINITY;
#pragma unroll
    for (int v = 0; v < 16; v++) y = fmaxf(y, sc[v]);
    if constexpr (!BINADES) y *= c1;
    if (__any(y - m > most)) {   // (also the first finite score)
      // (only that row's: what a row gives does not depend on the rows beside it)
      y = fmaxf(y, __shfl_xor(y, 32));
      const float m1 = y - m > most ? y - headroom : m;
      const float f = __builtin_amdgcn_exp2f(m - m1);
      m = m1;
      l *= f;
#pragma unroll
      for (int c = 0; c < DT; c++)
#pragma unroll
        for (int v = 0; v < 16; v++) o[c][v] *= f;
    }
  };
  // keys 16 t .. 16 t + 15 of half a tile, channels 32 c .. 32 c + 31
  auto values_of = [&](uint32_t at_lds, int t, int c) -> u32x4 {
    const uint8_t *p = smem + at_lds + 16 * t * LB + vrow + 16 * ((4 * c + vc) ^ vx);
    const u32x2 x = read_columns(p), y = read_columns(p + 8 * LB);
    return u32x4{x.x, x.y, y.x, y.y};
  };
  // ---- the tiles: first those that all rows see whole, [p0, p1), then the others
  int p0 = k0, p1 = k0;
  if (all_lo_max < all_hi_min) {
    p0 = min(k0 + max(all_lo_max - k0 + KT - 1, 0) / KT * KT, k1);
    p1 = max(min(k0 + max(all_hi_min - k0, 0) / KT * KT, k1), p0);
  }
  const int skip = p1 - p0;
  // the t-th of all tiles in that order, t counted in keys (past the last one: any)
  auto tile_at = [&](int t) -> int { return t < skip ? p0 + t : t - skip < p0 - k0 ? k0 + t - skip : k0 + t; };
  const int end = k1 - k0;

  // Keys are half a tile ahead: while half a tile's scores become weights and enter the products
  // with the values, the products of Q and the next half's keys are formed, so that the matrix
  // cores and the vector ALU both have work all the time.  A step's loads are therefore the
  // values of the next tile, the second half of its keys (wavefronts 2, 3), and the first half
  // of the keys of the tile behind it (0, 1): each into a place that the step before was the
  // last to read.
  typedef std::true_type Value;
  typedef std::false_type Key;
  const int lead = w < 2 ? 2 * KT : KT;
  v16f sa = {0}, sb = {0};
  int kpage = 0, vpage = 0;
  if (end > 0) {
    vpage = page_of(tile_at(0));
    kpage = page_of(tile_at(KT));
    load(Key(), kraw, kscale, tile_at(0), vpage, key_tile(0), std::false_type());
    load(Value(), vraw, vscale, tile_at(0), vpage, value_tile(0), std::false_type());
    widen(Key(), kraw, kscale, key_tile(0), key_scales(0));
    widen(Value(), vraw, vscale, value_tile(0), value_scales(0));
    vpage = kpage;
    if (KT < end && w < 2) {
      load(Key(), kraw, kscale, tile_at(KT), kpage, key_tile(1), std::false_type());
      widen(Key(), kraw, kscale, key_tile(1), key_scales(1));
      kpage = page_of(tile_at(2 * KT));
    }
    wait_all();
    if (live) {
#pragma unroll
      for (int e = 0; e < KS; e++)
        sa = mfma32<BF16>(*reinterpret_cast<const u32x4 *>(smem + key_tile(0) + krow + 16 * ((2 * e + half) ^ kx)), q[e], sa);
      times_scales(sa, key_scales(0), 0);
    }
  }
  int t = 0;
  // The data of step t is there; that of the next one on its way.  odd: t / 64 mod 2.  fast: four
  // more tiles that all rows see whole follow the first of two steps.
  auto next = [&](int odd, auto fast) __attribute__((always_inline)) {
    wait_all();
    const uint32_t keys = w < 2 ? key_tile(odd) : key_tile(1 - odd);
    if constexpr (decltype(fast)::value) {
      load(Key(), kraw, kscale, p0 + t + lead, kpage, keys, std::true_type());
      load(Value(), vraw, vscale, p0 + t + KT, vpage, value_tile(1 - odd), std::true_type());
      kpage = page_of(p0 + t + KT + lead);
      vpage = page_of(p0 + t + 2 * KT);
    } else {
      if (t + lead < end) load(Key(), kraw, kscale, tile_at(t + lead), kpage, keys, std::false_type());
      if (t + KT < end) load(Value(), vraw, vscale, tile_at(t + KT), vpage, value_tile(1 - odd), std::false_type());
      kpage = page_of(tile_at(t + KT + lead));
      vpage = page_of(tile_at(t + 2 * KT));
    }
    if constexpr (BITS < 16) {
      // rows whose value scale is not finite read as NaN
      const uint64_t nan = *reinterpret_cast<const uint64_t *>(smem + value_scales(odd) + 8 * KT);
      if (uniform((int)(nan | nan >> 32)) != 0) {
        for (int i = threadIdx.x; i < KT * LC; i += T)
          if (nan >> (i / LC) & 1) *reinterpret_cast<u32x4 *>(smem + value_tile(odd) + 16 * i) = u32x4{0x7e007e00u, 0x7e007e00u, 0x7e007e00u, 0x7e007e00u};
        wait_lds();
      }
    }
  };
  auto done = [&](int odd, auto fast) __attribute__((always_inline)) {
    constexpr bool ON = decltype(fast)::value;
    if (ON || t + lead < end) widen(Key(), kraw, kscale, w < 2 ? key_tile(odd) : key_tile(1 - odd), w < 2 ? key_scales(odd) : key_scales(1 - odd));
    if (ON || t + KT < end) widen(Value(), vraw, vscale, value_tile(1 - odd), value_scales(1 - odd));
    t += KT;
  };
  // Half i of step t: one matrix product at a time with its share of the vector work behind it,
  // in this order.  A product occupies the matrix core for 32 cycles, in which its wavefront
  // issues five or six other instructions; operands are read some products before their use.
  auto half_step = [&](v16f &now, v16f &then, int i, int odd, int k, auto edge) __attribute__((always_inline)) {
    constexpr int NQ = KS, NV = 2 * DT, ALL = NQ + (FINE ? 2 : 1) * NV, AHEAD = BITS < 16 ? 4 : 8;
    u32x4 ring[AHEAD], pt[2];
    // (past the last tile: keys of what is there, for nothing)
    const uint32_t keys = i == 0 ? key_tile(odd) + 32 * LB : key_tile(1 - odd), values = value_tile(odd) + 32 * i * LB;
    auto operand = [&](int n) -> u32x4 {
      if (n < NQ) return *reinterpret_cast<const u32x4 *>(smem + keys + krow + 16 * ((2 * n + half) ^ kx));
      const int e = (n - NQ) % NV;
      return values_of(values, e / DT, e % DT);
    };
#pragma unroll
    for (int n = 0; n < AHEAD - 1; n++) ring[n] = operand(n);
    __builtin_amdgcn_sched_barrier(0);
    refer(now, k, i, value_scales(odd), edge);
    float sum = 0.0f;
    then = v16f{0};
    // (products go first: 8 bits 2595 -> 2530 us, 16 bits 1 % or less)
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int n = 0; n < ALL; n++) {
      __builtin_amdgcn_sched_barrier(0);
      if (n + AHEAD - 1 < ALL) ring[(n + AHEAD - 1) % AHEAD] = operand(n + AHEAD - 1);
      const u32x4 op = ring[n % AHEAD];
      if (n < NQ) {
        then = mfma32<BF16>(op, q[n], then);
#pragma unroll
        for (int x = 16 * n / NQ; x < 16 * (n + 1) / NQ; x++) {
          const float z = now[x], y = __builtin_amdgcn_exp2f(BINADES ? z - m : fmaf(z, c1, -m));
          now[x] = y;
          if (x & 1) pt[x / 8][x / 2 % 4] = pack2<VBF>(now[x - 1], y);
        }
      } else {
        const int e = (n - NQ) % NV;
        if (n == NQ + NV) {      // what the rounding left
#pragma unroll
          for (int x = 0; x < 16; x += 2) {
            const uint32_t z = pt[x / 8][x / 2 % 4];
            pt[x / 8][x / 2 % 4] = pack2<VBF>(now[x] - lower_half<VBF>(z), now[x + 1] - upper_half<VBF>(z));
          }
        }
        o[e % DT] = mfma32<VBF>(op, pt[e / DT], o[e % DT]);
        if (n < NQ + NV) {
#pragma unroll
          for (int x = 16 * e / NV; x < 16 * (e + 1) / NV; x++) {
            if constexpr (BITS < 16) sum = fmaf(now[x], reinterpret_cast<const float *>(smem + value_scales(odd))[KT + key_of(i, x)], sum);
            else sum += now[x];
          }
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    // (now: the step's end is free to overwrite these scales' place, as that of their keys)
    times_scales(then, key_scales(i == 0 ? odd : 1 - odd), 1 - i);
    l += sum;
  };
  auto step = [&](int odd, auto fast, auto edge, int k) __attribute__((always_inline)) {
    if constexpr (!decltype(edge)::value) next(odd, fast);
    if (live) {
      half_step(sa, sb, 0, odd, k, edge);
      half_step(sb, sa, 1, odd, k, edge);
    }
    done(odd, fast);
  };
  typedef std::true_type Yes;
  typedef std::false_type No;
  // (the second step of a pair looks up the page of the first one's t + 4 tiles)
  while (t + 5 * KT <= skip) {
    step(0, Yes(), No(), p0 + t);
    step(1, Yes(), No(), p0 + t);
  }
  while (t < skip) step(t / KT & 1, No(), No(), p0 + t);
  while (t < end) {
    const int odd = t / KT & 1, k = tile_at(t);
    next(odd, No());
    // is a value not finite?
    auto value_at = [&](int i) -> u32x4 & { return *reinterpret_cast<u32x4 *>(smem + value_tile(odd) + 16 * (i * T + (int)threadIdx.x)); };
    constexpr int NV = TB / (16 * T);
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const u32x4 x = value_at(i);
#pragma unroll
      for (int j = 0; j < 4; j++) bad |= not_finite<VBF>(x[j]);
    }
    if (__any(bad != 0) && lane == 0) *flag = t + 1;
    wait_lds();
    if (uniform(*flag) == t + 1) {
      // ones where a value is not finite, times ones where a row sees it, leave NaN; then zeros there
      auto mask_of = [&](uint32_t x) -> uint32_t { return (not_finite<VBF>(x) >> 15) * 0xffffu; };
      for (int c = 0; c < DT; c++) {
        // (32 channels at a time, read as ones from where the values lie)
        v16f n = {0};
#pragma unroll
        for (int h = 0; h < 4; h++) {
          u32x4 op = values_of(value_tile(odd) + 32 * (h / 2) * LB, h % 2, c), ones;
#pragma unroll
          for (int j = 0; j < 4; j++) {
            op[j] = mask_of(op[j]) & (kOne << 16 | kOne);
            ones[j] = (masked(k, h / 2, 8 * (h % 2) + 2 * j) ? 0u : kOne) | (masked(k, h / 2, 8 * (h % 2) + 2 * j + 1) ? 0u : kOne << 16);
          }
          n = mfma32<VBF>(op, ones, n);
        }
#pragma unroll
        for (int d = 0; d < DT; d++)
#pragma unroll
          for (int v = 0; v < 16; v++) o[d][v] = d == c && n[v] > 0.0f ? NAN : o[d][v];
      }
      wait_lds();
#pragma unroll
      for (int i = 0; i < NV; i++) {
        u32x4 x = value_at(i);
#pragma unroll
        for (int j = 0; j < 4; j++) x[j] &= ~mask_of(x[j]);
        value_at(i) = x;
      }
      wait_lds();
    }
    step(odd, No(), Yes(), k);
  }

  // ---- results
  clear();
  l += __shfl_xor(l, 32);
  if (!sees) l = 0.0f;
  if (!live || row0 + 32 * w + r32 >= rows) return;
  const int64_t to = (int64_t)(start + token) * a.hq + head;
  if (a.splits == 1 && !a.shared) {
    const float inv = 1.0f / l;
    const bool none = l == 0.0f;
#pragma unroll
    for (int c = 0; c < DT; c++)
#pragma unroll
      for (int g = 0; g < 4; g++) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; j++) y[j] = none ? 0.0f : o[c][4 * g + j] * inv;
        *reinterpret_cast<u32x2 *>(a.out + to * D + 32 * c + 8 * g + 4 * half) = u32x2{pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3])};
      }
    if (a.lse != nullptr && half == 0) a.lse[to] = none ? -INFINITY : log_sum(m, l);
  } else {
    const int64_t heads = (int64_t)a.tokens * a.hq, part = split * heads + to;
    float *const op = a.scratch + parts_head(a.splits, heads) + part * D;
    // (a part without keys is told by its sum, and not read)
    if (k0 < k1)
#pragma unroll
    for (int c = 0; c < DT; c++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        *reinterpret_cast<v4f *>(op + 32 * c + 8 * g + 4 * half) = v4f{o[c][4 * g], o[c][4 * g + 1], o[c][4 * g + 2], o[c][4 * g + 3]};
    if (half == 0) *reinterpret_cast<f2 *>(a.scratch + 2 * part) = f2{m, l};
  }
}

template <int D, int BITS, bool BF16, Scored HOW, bool FINE>
hipError_t go_prompt(const PromptArgs &a, hipStream_t s) {
  const int bytes = prompt_lds_bytes(D, BITS);
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(prompt_kernel<D, BITS, BF16, HOW, FINE>), bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((prompt_kernel<D, BITS, BF16, HOW, FINE>), dim3((uint32_t)a.blocks), dim3(kPromptThreads), bytes, s, a);
  return hipGetLastError();
}

}  // namespace

// one head size's kernels (a file each)
template <int D>
hipError_t launch_prompt_d(const PromptArgs &a, bool bf16, hipStream_t s) {
  typedef std::true_type Yes;
  typedef std::false_type No;
  auto go = [&](auto bits, auto b, auto how) -> hipError_t {
    constexpr int BITS = decltype(bits)::value;
    constexpr bool BF16 = decltype(b)::value;
    constexpr Scored HOW = decltype(how)::value;
    return a.fine ? go_prompt<D, BITS, BF16, HOW, true>(a, s) : go_prompt<D, BITS, BF16, HOW, false>(a, s);
  };
  auto go_ext = [&](auto bits, auto b) -> hipError_t {
    if (a.cap > kWide) return go(bits, b, std::integral_constant<Scored, kCappedWide>());
    if (a.cap > 0.0f || a.slopes != nullptr) return go(bits, b, std::integral_constant<Scored, kCapped>());
    return go(bits, b, std::integral_constant<Scored, kPlain>());
  };
  auto go_type = [&](auto bits) -> hipError_t { return bf16 ? go_ext(bits, Yes()) : go_ext(bits, No()); };
  if (a.c.bits == 16) return go_type(std::integral_constant<int, 16>());
  if (a.c.bits == 8) return go_type(std::integral_constant<int, 8>());
  return go_type(std::integral_constant<int, 4>());
}

}  // namespace tq
