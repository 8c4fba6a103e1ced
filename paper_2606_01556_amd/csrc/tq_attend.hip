// Attention of one new token per stream over the paged cache:
//
//   o_h = sum_t softmax_t(scale q_h . k_t) v_t,  t in [max(0, len - window), len)
//
// Bound by the cache's bytes (at most 4 flops per value and query head of the
// group), so the kernel is built around one pass over them with nothing but
// registers between memory and the matrix cores:
//
//  * S^T = K Q^T in 16x16x32 products, with the group's query heads (up to 16) as
//    columns.  A lane of the first operand holds values of one token's key, a run of
//    the cache row as it lies in memory: which of a row's values make up one product
//    is free as long as Q is laid out alike, so each format loads the widest run a lane
//    can.  Codes become values of Q's type (exactly) on their way.
//  * The result has column lane % 16 and rows 4 (lane / 16) + i: a lane holds the
//    scores of one head for tokens 4 g + i.  Two such tiles, exponentiated, are
//    the second operand of O^T = V^T P^T as they stand (the order of the tokens
//    is free too), so no score crosses lanes.
//  * V^T's operand takes eight tokens' values of one channel per lane.  A lane
//    loads rows 4 g + i of the tile, channels DV r .. DV r + DV - 1 (r = lane %
//    16, DV = d / 16), and pairs the rows up with byte permutes.  The scale of a
//    quantized row is part of its weight.
//  * The softmax's reference (and with it the scaling of the weights) only moves
//    when some weight passes 65504 (bf16 rows: 1 over the number of tokens): most
//    steps have no exchange between lanes and no rescaling.
//  * A weight enters the products as several 16-bit terms, as the matrix cores have
//    the time: for codes and fp16 rows two fp16 ones, its rounded value and what that
//    leaves (22 bits); for bf16 rows three bf16 ones, which hold all 24 (two of them
//    left 2^-18 of every weight; the third costs up to 1 %: 95 us for 32 streams up to
//    8192 either way, 65.4 after 64.9 for 16 of 4096 at d = 256).
//  * With fp16 terms the reference moves so that the largest weight becomes 2^12:
//    fp16's smallest step, 2^-24, is 2^-36 of that or less, and 2^17 small weights
//    beside a large one lose 2^-20 in all.  (With the largest weight at 1 they all but
//    vanish from 17 e-folds below it, where a first token that takes most of the weight
//    leaves them.)  With bf16 ones, which have fp32's exponents, it becomes 2^-8 over the
//    number of tokens, or less: a sum of values near bf16's largest must not pass fp32's.
//
// The work is cut evenly whatever the lengths: all (stream, head) ranges of steps
// laid end to end are split into equal runs, two to four work-groups a CU, and a
// work-group's four wavefronts take its steps in turn.  A range that one run holds
// whole is written at once; a second launch joins the parts of the others, in their
// order, so that a result does not depend on timing.  Short ranges get a work-group
// each and need no second launch.
//
// Measured (d = 128 but for the last, both launches, back-to-back calls; reading alone
// streams 512 MB at 6.9 TB/s):
//   1 stream of 131072 tokens, 8 kv heads, fp16              88 us, 6.1 TB/s
//   32 streams up to 8192, bf16                              95 us, 6.1 TB/s
//   64 streams up to 8192, 8 bits, pages of 64              101 us, 5.8 TB/s
//   48 streams up to 16384, 4 bits, pages of 16              85 us, 5.2 TB/s
//   16 streams up to 4096, 8 kv heads of 256, fp16           64 us, 4.5 TB/s
// In a kernel trace the first launch takes 84, 92, 98, 81 and 60 us (6.0 to 6.5 TB/s of what
// it reads in the first four, at 4 bits 9 % more than it has to: the scales of 16 tokens
// are 32 bytes) and the join 4 to 5.5, together up to 2 % more than a call takes.  At 4 bits the vector ALU is 54 % busy, at 16 bits 10 %.  Without effect or worse: e4m3 products of the keys with Q split into e4m3
// terms (and scores off by 2^-15 of sum |q k|), eight wavefronts in one work-group, a
// join by whichever work-group comes last (its fences drop the L2s under the others).
#include <cfloat>

#include "tq_device.hpp"
#include "tq_kernels.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef uint16_t s2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const int32_t __attribute__((address_space(4))) const_i32;

constexpr int kHeads = 16;                 // query heads of a product (its columns)
constexpr int kRunWaves = 4;               // wavefronts of a work-group that holds a run of steps
// Work-groups of runs that fit a CU by their registers.  (Four instead of three at d = 64, 16
// streams of 16384: 16 bits 89.0 us and 89.6, 8 bits 52 and 54, 4 bits 43.7 and 45.)
constexpr int runs_per_cu(int d) { return d == 256 ? 2 : d == 128 ? 3 : 4; }
constexpr int kDirectWaves = 8;            // wavefronts of a work-group that holds one short range
constexpr int kJoinThreads = 256;
constexpr int kCus = 256;

// Tokens of one step of a wavefront.  (64 for codes: 98 us instead of 94 for 48
// streams up to 16384 in 4 bits, with registers for two wavefronts per SIMD only.)
constexpr int kStep = 32;

// A kv head's group of query heads is one range of one or two blocks of up to 16 heads,
// or, past 32 heads, several ranges.
__host__ __device__ constexpr int head_blocks(int group) { return group > kHeads ? 2 : 1; }
constexpr int ranges_of(int group) { return (group + kHeads * head_blocks(group) - 1) / (kHeads * head_blocks(group)); }
constexpr int range_heads(int group) { return group < kHeads * head_blocks(group) ? group : kHeads * head_blocks(group); }

constexpr float kLog2e = 1.4426950408889634f;

// The largest weight that a step may have (fp16's largest value), and the power of two at
// which the largest one is put when the reference moves.
constexpr float kTopWeight = 65504.0f, kHeadroom = 12.0f;
// With bf16 rows, whose values fp32 itself just holds, the weights of a range of fewer than
// 2^e tokens stay at 2^-e or below, so that no sum passes the largest value; the largest
// weight is put kBelow binades lower.
constexpr int kBelow = 8;
constexpr float kLeastScale = 0x1p-24f;    // fp16's smallest number

template <bool BF16>
__device__ __forceinline__ v4f mfma16(u32x4 a, u32x4 b, v4f c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// four e4m3 bytes times `scale` (a power of two) as two words of 16-bit values
template <bool BF16>
__device__ __forceinline__ void widen4(uint32_t w, float scale, uint32_t &lo, uint32_t &hi) {
  if constexpr (BF16) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, true));
  }
}

// Bytes I of w0 and J of w1, codes as tq4_to_fp8 gives them (sign, four zeros, three bits),
// as the high bytes of two fp16 values: the three bits end below the second exponent
// bit, where fp16's subnormals and the next binade have the same steps, so the value is
// the code times 2^-16, exactly, for one instruction.
constexpr float kSmall = 65536.0f;
template <int I, int J>
__device__ __forceinline__ uint32_t small_halves(uint32_t w0, uint32_t w1) {
  return __builtin_amdgcn_perm(w1, w0, (uint32_t)(4 + J) << 24 | 0x0c0000u | I << 8 | 0x0cu);
}

// two fp32 values rounded to a word of 16-bit ones
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const f2 v = {x, y};
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
}
// the two values of a word of fp16 ones
__device__ __forceinline__ f2 unpack2(uint32_t w) { return __builtin_convertvector(__builtin_bit_cast(h2, w), f2); }

// NB bytes from p (p aligned to min(NB, 16)).  The cache is read once per call:
// non-temporal loads stream it at 6.9 TB/s instead of 6.2 (512 MB).
template <bool ONCE, typename T>
__device__ __forceinline__ T stream_load(const uint8_t *p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const T *>(p));
  else return *reinterpret_cast<const T *>(p);
}
template <bool ONCE, int NB>
__device__ __forceinline__ void load_bytes(const uint8_t *p, uint32_t *out) {
  if constexpr (NB >= 16) {
#pragma unroll
    for (int i = 0; i < NB / 16; i++) {
      const u32x4 v = stream_load<ONCE, u32x4>(p + 16 * i);
      out[4 * i] = v.x; out[4 * i + 1] = v.y; out[4 * i + 2] = v.z; out[4 * i + 3] = v.w;
    }
  } else if constexpr (NB == 8) {
    const u32x2 v = stream_load<ONCE, u32x2>(p);
    out[0] = v.x; out[1] = v.y;
  } else {
    static_assert(NB == 4);
    out[0] = stream_load<ONCE, uint32_t>(p);
  }
}

// fp16 scale j of four
__device__ __forceinline__ float scale_of(u32x2 four, int j) {
  const uint32_t two = j < 2 ? four.x : four.y;
  return (float)__builtin_bit_cast(h2, two)[j & 1];
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The tokens [first, len) of a stream in steps from first rounded down to 16.
struct Range {
  int first, len, base, steps;
};
template <int ST>
__device__ __forceinline__ Range range_of(int len, int cap, int window) {
  Range r;
  r.len = min(max(len, 0), cap);
  r.first = window > 0 && r.len > window ? r.len - window : 0;
  r.base = r.first & ~15;
  r.steps = (r.len - r.base + ST - 1) / ST;
  return r;
}

// v summed over the lanes up to this one
__device__ __forceinline__ int scan64(int v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int o = __shfl_up(v, m);
    if (lane >= m) v += o;
  }
  return v;
}
__device__ __forceinline__ int lane_of(int v, int lane) { return uniform(__shfl(v, lane)); }

// floats of one part of a range: the group's references and sums, then its products
__host__ __device__ constexpr int part_head(int cols) { return (2 * cols + 3) & ~3; }
__host__ __device__ constexpr int part_floats(int d, int cols) { return part_head(cols) + cols * d; }

// Q in LDS instead of registers, which 16-bit rows of 256 values leave none for
constexpr bool q_in_lds(int d, int bits) { return d == 256 && bits == 16; }

// floats of LDS: [W][kHeads] references and sums, Q where it is there, then [W][cols up
// to kHeads][d + 4] products (rows staggered over the banks)
constexpr int lds_floats(int waves, int hb, int d, int bits, int cols) {
  return 2 * waves * kHeads + (q_in_lds(d, bits) ? hb * (d / 32) * 64 * 4 : 0) + waves * cols * (d + 4);
}

// a head's four output values from d0, and its log-sum-exp
template <bool BF16>
__device__ __forceinline__ void store4(const AttendArgs &a, int d, int64_t row, int d0, float m, float l, v4f o) {
  const float inv = 1.0f / l;
  *reinterpret_cast<u32x2 *>(a.out + row * d + d0) = u32x2{pack2<BF16>(o[0] * inv, o[1] * inv), pack2<BF16>(o[2] * inv, o[3] * inv)};
  // (m and l's binade all but cancel: they go together first)
  if (a.lse != nullptr && d0 == 0)
    a.lse[row] = (m + (float)__builtin_amdgcn_frexp_expf(l) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(l))) * (1.0f / kLog2e);
}

// What the first launch tells the join about a range, [batch][vheads]: the number
// of its first part and of its parts (0: nothing to join).  Part 2 w is the first
// that run w holds, 2 w + 1 the last one if that is another; so the parts of a range
// are its first, and the first ones of the runs behind it.
struct Join {
  int first, parts;
};

// ---------------------------------------------------------------------------
// HB: blocks of up to 16 query heads per range.  With two, half of the wavefronts take
// each, step by step alongside, so that the cache is read from memory once.
template <int W, int HB, int D, int BITS, bool BF16>
__global__ __launch_bounds__(64 * W, W == kDirectWaves ? 2 : runs_per_cu(D)) void attend_kernel(const AttendArgs a) {
  constexpr bool DIRECT = W == kDirectWaves;   // one range per work-group
  constexpr int SW = W / HB, HR = kHeads * HB; // wavefronts that share a block's steps; heads of a range
  constexpr int ST = kStep, NT = ST / 16;
  constexpr uint32_t RB = D * BITS / 8;       // bytes of a row
  constexpr int CE = BITS == 16 ? 8 : BITS == 8 ? 16 : (D / 4 < 32 ? D / 4 : 32);  // a lane's run of a key row
  constexpr uint32_t CB = CE * BITS / 8;      // its bytes
  constexpr int KL = D / (4 * CE);            // runs per lane
  constexpr int KW = KL * (int)CB / 4;        // words
  constexpr int KS = D / 32;                  // products per tile of keys
  constexpr int DV = D / 16;                  // channels per lane of a value row
  constexpr uint32_t VBr = DV * BITS / 8;     // their bytes; two lanes share a word of 4-bit codes at d = 64
  constexpr uint32_t VB = VBr < 4 ? 4 : VBr;
  constexpr int VW = (int)VB / 4;
  constexpr bool VBF = BITS == 16 && BF16;    // type of the second product: bf16, else fp16
  constexpr int TERMS = VBF ? 3 : 2;          // of a weight
  constexpr int LD = D + 4;
  constexpr bool QL = q_in_lds(D, BITS);
  constexpr bool SK = BITS == 4 && !BF16;     // keys as small_halves

  extern __shared__ __attribute__((aligned(16))) float lds[];
  float *const lds_m = lds, *const lds_l = lds + W * kHeads, *const lds_q = lds + 2 * W * kHeads,
               *const lds_o = lds_q + (QL ? HB * KS * 64 * 4 : 0);

  // a wavefront that is behind goes first: wavefronts that progress alike end together
  // (oldest first, the younger ones are left to themselves at the end)
  __builtin_amdgcn_s_setprio(3);
  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int lps = a.c.lps, hkv = a.c.heads;
  const int cap = a.max_pages << lps;
  const int hblocks = (a.group + HR - 1) / HR, vheads = hkv * hblocks;
  const int cols = min(a.group, HR), wcols = min(a.group, kHeads);
  const int wb = w / SW, ws = w % SW;          // the wavefront's block of heads and its turn

  // this work-group's run of steps
  int b, vh, t, x0, x1, chunk;
  Range rg = {};
  if constexpr (DIRECT) {
    b = blockIdx.x / vheads;
    vh = blockIdx.x % vheads;
    rg = range_of<ST>(uniform(a.lengths[b]), cap, a.window);
    t = x0 = 0;
    x1 = chunk = rg.steps;
  } else {
    // Run w holds steps [w chunk, (w + 1) chunk) of all ranges laid end to end, those of
    // every stream's vheads ranges in turn.  A lane adds up `each` streams.
    auto steps_of = [&](int i, int end) -> int { return i < end ? range_of<ST>(a.lengths[i], cap, a.window).steps : 0; };
    const int each = (a.batch + 63) / 64;
    int mine = 0;
#pragma unroll 4
    for (int i = 0; i < each; i++) mine += steps_of(lane * each + i, a.batch);
    int upto = scan64(mine);
    const int total = lane_of(upto, 63) * vheads;        // < 2^31 (host)
    chunk = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kRunWaves);
    x0 = blockIdx.x * chunk;
    x1 = min(total, x0 + chunk);
    b = 0;
    vh = t = 0;
    if (x0 < x1) {
      // the stream that holds step x0: the first whose steps end past it
      const int y = x0 / vheads;
      int before = 0, at = __builtin_ctzll(__ballot(upto > y));
      if (at > 0) before = lane_of(upto, at - 1);
      b = at * each;
      if (each > 1) {
        const int end = min(a.batch, b + each);
        uint64_t past;
        while ((past = __ballot(before + (upto = scan64(steps_of(b + lane, end))) > y)) == 0) {
          before += lane_of(upto, 63);
          b += 64;
        }
        at = __builtin_ctzll(past);
        if (at > 0) before += lane_of(upto, at - 1);
        b += at;
      }
      b = uniform(b);
      rg = range_of<ST>(uniform(a.lengths[b]), cap, a.window);
      vh = (x0 - before * vheads) / rg.steps;
      t = (x0 - before * vheads) % rg.steps;
    }
  }
  float *const parts = a.scratch;
  Join *const joins = reinterpret_cast<Join *>(a.scratch + (int64_t)gridDim.x * 2 * part_floats(D, cols));
  // streams that hold nothing
  auto clear = [&](int64_t row0, int rows) {
    for (int e = threadIdx.x; e < rows * (D / 2); e += 64 * W) reinterpret_cast<uint32_t *>(a.out + row0 * D)[e] = 0;
    if (a.lse != nullptr)
      for (int e = threadIdx.x; e < rows; e += 64 * W) a.lse[row0 + e] = -INFINITY;
  };
  if constexpr (DIRECT) {
    const int h0 = vh % hblocks * HR;
    if (x1 == 0) clear((int64_t)b * a.hq + vh / hblocks * a.group + h0, min(HR, a.group - h0));
  } else {
    for (int i = blockIdx.x; i < a.batch; i += gridDim.x)
      if (range_of<ST>(uniform(a.lengths[i]), cap, a.window).steps == 0) {
        clear((int64_t)i * a.hq, a.hq);
        for (int e = threadIdx.x; e < vheads; e += 64 * W) joins[(int64_t)i * vheads + e] = Join{0, 0};
      }
  }
  if (x0 >= x1) return;
  const int quarter = max((x1 - x0) / 4, 1);

  for (int x = x0; x < x1;) {
    const int n = min(rg.steps - t, x1 - x);
    const int kvh = vh / hblocks, h0 = vh % hblocks * HR;
    const int heads = max(0, min(kHeads, a.group - h0 - wb * kHeads));   // live columns

    const_i32 *pages = (const_i32 *)(a.table + b * a.table_stride);
    const int last_page = (rg.len - 1) >> lps;
    uint32_t kraw[NT][KW], vraw[NT][4][VW];
    u32x2 ksr[NT], vsr[NT];
    // the page of the tile at token tt (a tile past the end takes the last page and is masked)
    auto page_of = [&](int tt) -> int { return pages[min(tt >> lps, last_page)]; };
    // row of the cache sections at which the tile starts
    auto row_of = [&](int page, int tt) -> int64_t {
      page = min(max(page, 0), a.c.pages - 1);
      return (((int64_t)page * hkv + kvh) << lps) + (tt & ((1 << lps) - 1));
    };
    const uint32_t kofs = r * RB + g * CB, vofs = 4 * g * RB + (VBr < 4 ? (r >> 1) * 4 : r * VB), sofs = 8 * g;
    auto load_k = [&](const int64_t (&row)[NT]) {
#pragma unroll
      for (int i = 0; i < NT; i++) {
        const uint8_t *kp = a.c.k + row[i] * RB;
#pragma unroll
        for (int j = 0; j < KL; j++) load_bytes<HB == 1, CB>(kp + j * 4 * CB + kofs, &kraw[i][j * (int)CB / 4]);
        if constexpr (BITS < 16)
          ksr[i] = *reinterpret_cast<const u32x2 *>(reinterpret_cast<const uint8_t *>(a.c.ks + row[i]) + sofs);
      }
    };
    auto load_v = [&](const int64_t (&row)[NT]) {
#pragma unroll
      for (int i = 0; i < NT; i++)
        if constexpr (BITS < 16)
          vsr[i] = *reinterpret_cast<const u32x2 *>(reinterpret_cast<const uint8_t *>(a.c.vs + row[i]) + sofs);
#pragma unroll
      for (int i = 0; i < NT; i++) {
        const uint8_t *vp = a.c.v + row[i] * RB;
#pragma unroll
        for (int j = 0; j < 4; j++) load_bytes<HB == 1, VB>(vp + j * RB + vofs, vraw[i][j]);
      }
    };

    // the wavefront's steps t + ws, t + ws + SW, ... of the range
    int t0 = uniform(rg.base + (t + ws) * ST);
    const int steps = (n - ws + SW - 1) / SW;
    int64_t row[NT];
    if (steps > 0) {
#pragma unroll
      for (int i = 0; i < NT; i++) row[i] = row_of(page_of(t0 + 16 * i), t0 + 16 * i);
      load_k(row);
      load_v(row);
    }

    // Q^T: column r, the values of the runs a key lane loads; c1: what a score's
    // product with the key's scale is multiplied by, log2(e) |scale| (its sign goes to Q)
    u32x4 q[KS];
    const float c1 = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-149f) * (SK ? kSmall : 1.0f);  // (-infinity times it has to stay so)
    {
      const uint16_t *qp = a.q + b * a.q_ts + (int64_t)(kvh * a.group + h0 + min(wb * kHeads + r, a.group - h0 - 1)) * a.q_hs;
      const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u, live = r < heads ? 0xffffffffu : 0u;
#pragma unroll
      for (int k = 0; k < KS; k++) {
        if (QL && k % SW != ws) continue;
        q[k] = *reinterpret_cast<const u32x4 *>(qp + (8 * k / CE) * 4 * CE + g * CE + 8 * k % CE);
#pragma unroll
        for (int i = 0; i < 4; i++) q[k][i] = (q[k][i] ^ flip) & live;
        if constexpr (QL) *reinterpret_cast<u32x4 *>(lds_q + ((wb * KS + k) * 64 + lane) * 4) = q[k];
      }
      if constexpr (QL) __syncthreads();
    }
    v4f o[DV];
#pragma unroll
    for (int i = 0; i < DV; i++) o[i] = v4f{0, 0, 0, 0};
    // (finite, so that keys whose score is -infinity have the weight 0 also before the
    // first finite one)
    float m = -FLT_MAX, l = 0.0f;
    float most = kTopWeight, headroom = kHeadroom;
    if constexpr (VBF) {
      const int e = 32 - __builtin_clz(rg.len);
      most = __builtin_bit_cast(float, (127 - e) << 23);
      headroom = (float)(-e - kBelow);
    }
    float s[NT][4];
    // scores, times the keys' scales: row 4 g + j of tile i, head r
    auto scores = [&]() {
      v4f acc[NT] = {};
#pragma unroll
      for (int e = 0; e < KS * NT; e++) {
        // (tile by tile at 16 bits; codes, which take longer to prepare, in turn)
        const int i = BITS == 16 ? e / KS : e % NT, k = BITS == 16 ? e % KS : e / NT;
        u32x4 op;
        if constexpr (BITS == 16) {
          op = u32x4{kraw[i][4 * k], kraw[i][4 * k + 1], kraw[i][4 * k + 2], kraw[i][4 * k + 3]};
        } else {
          uint32_t w0, w1, y0, y1, y2, y3;
          if constexpr (BITS == 8) {
            w0 = kraw[i][2 * k];
            w1 = kraw[i][2 * k + 1];
          } else {
            tq4_to_fp8(kraw[i][k], w0, w1);
          }
          if constexpr (SK) {
            op = u32x4{small_halves<0, 1>(w0, w0), small_halves<2, 3>(w0, w0), small_halves<0, 1>(w1, w1), small_halves<2, 3>(w1, w1)};
          } else {
            widen4<BF16>(w0, BITS == 4 ? 512.0f : 1.0f, y0, y1);
            widen4<BF16>(w1, BITS == 4 ? 512.0f : 1.0f, y2, y3);
            op = u32x4{y0, y1, y2, y3};
          }
        }
        acc[i] = mfma16<BF16>(op, QL ? *reinterpret_cast<const u32x4 *>(lds_q + ((wb * KS + k) * 64 + lane) * 4) : q[k], acc[i]);
      }
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) s[i][j] = BITS < 16 ? fmaf(acc[i][j], scale_of(ksr[i], j), 0.0f) : acc[i][j];
    };
    // tokens outside the range: no score, and nothing of what their rows hold
    auto masked = [&](int i, int j) -> bool {
      const int tok = t0 + 16 * i + 4 * g + j;
      return tok < rg.first || tok >= rg.len;
    };
    auto mask_scores = [&]() {
      asm volatile("");          // (a branch: selects in every step would cost a fifth of it)
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          s[i][j] = masked(i, j) ? -INFINITY : s[i][j];
          if constexpr (BITS < 16) vsr[i][j / 2] &= masked(i, j) ? (j & 1 ? 0x0000ffffu : 0xffff0000u) : 0xffffffffu;
        }
    };
    auto mask_values = [&]() {
      asm volatile("");
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
          for (int k = 0; k < VW; k++) vraw[i][j][k] = masked(i, j) ? 0u : vraw[i][j][k];
    };
    // weights p in s, times the values' scales
    auto softmax = [&]() {
      float p[NT][4], wt[NT][4], top = 0.0f, ptop = 0.0f;
      u32x2 vs[NT];
      if constexpr (BITS < 16) {
        // (a scale of zero, whose codes are zero, counts as fp16's smallest: p stays bounded.
        // The larger one by its bits, so that NaN stays.)
        const s2 least = {1, 1};
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int k = 0; k < 2; k++) {
            const uint32_t two = k == 0 ? vsr[i].x : vsr[i].y;
            vs[i][k] = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s2, two), least));
          }
      }
      auto weights = [&]() {
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            p[i][j] = __builtin_amdgcn_exp2f(fmaf(s[i][j], c1, -m));
            wt[i][j] = BITS < 16 ? fmaf(p[i][j], scale_of(vs[i], j), 0.0f) : p[i][j];
            top = fmaxf(top, wt[i][j]);
            if constexpr (BITS < 16) ptop = fmaxf(ptop, p[i][j]);
          }
        // (a scale that is NaN counts as fp16's smallest, so that the sum of p stays one; the
        // others leave top as it is)
        if constexpr (BITS < 16) top = fmaxf(top, ptop * kLeastScale);
      };
      weights();
      if (__any(top > most)) {                // (also the first finite score: top is infinite)
        float y = -INFINITY;
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int j = 0; j < 4; j++)
            y = fmaxf(y, s[i][j] * c1 + (BITS < 16 ? fmaxf(__builtin_amdgcn_logf(scale_of(vs[i], j)), -24.0f) : 0.0f));
        y = fmaxf(y, __shfl_xor(y, 16));
        y = fmaxf(y, __shfl_xor(y, 32));
        const float m1 = fmaxf(m, y - headroom);
        const float f = __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= f;
#pragma unroll
        for (int i = 0; i < DV; i++) o[i] *= f;
        weights();
      }
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          l += p[i][j];
          s[i][j] = wt[i][j];
        }
    };
    // O^T += V^T P^T, 32 tokens (two tiles) at a time
    auto products = [&]() {
#pragma unroll
      for (int i = 0; i < NT; i += 2) {
        u32x4 pt[TERMS];
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const int h = i + j / 2, k = 2 * (j & 1);
          if constexpr (VBF) {
            // the upper halves, three times over: all 24 bits
            float x = s[h][k], y = s[h][k + 1];
#pragma unroll
            for (int t = 0; t < TERMS; t++) {
              const uint32_t xb = __builtin_bit_cast(uint32_t, x), yb = __builtin_bit_cast(uint32_t, y);
              pt[t][j] = __builtin_amdgcn_perm(yb, xb, 0x07060302u);
              x -= __builtin_bit_cast(float, xb & 0xffff0000u);
              y -= __builtin_bit_cast(float, yb & 0xffff0000u);
            }
          } else {
            pt[0][j] = pack2<false>(s[h][k], s[h][k + 1]);
            const f2 u = unpack2(pt[0][j]);
            pt[1][j] = pack2<false>(fmaf(u.x, -1.0f, s[h][k]), fmaf(u.y, -1.0f, s[h][k + 1]));
          }
        }
        if constexpr (BITS == 16) {
          // two channels a word: rows 2 j and 2 j + 1 paired up
#pragma unroll
          for (int c = 0; c < DV; c++) {
            const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
            u32x4 op;
#pragma unroll
            for (int j = 0; j < 4; j++)
              op[j] = __builtin_amdgcn_perm(vraw[i + j / 2][2 * (j & 1) + 1][c / 2], vraw[i + j / 2][2 * (j & 1)][c / 2], sel);
#pragma unroll
            for (int t = 0; t < TERMS; t++) o[c] = mfma16<VBF>(op, pt[t], o[c]);
          }
        } else {
          // four channels a word of bytes: the bytes paired up, then widened
#pragma unroll
          for (int c = 0; c < DV; c += 4) {
            u32x4 op[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
              uint32_t pair[2];
#pragma unroll
              for (int k = 0; k < 2; k++) {
                const uint32_t *raw = vraw[i + j / 2][2 * (j & 1) + k];
                if constexpr (BITS == 8) {
                  pair[k] = raw[c / 4];
                } else {
                  // a word's codes 0..3, then 4..7; of a word that two lanes share, theirs
                  uint32_t lo, hi;
                  tq4_to_fp8(raw[c / 8], lo, hi);
                  pair[k] = (VBr < 4 ? r & 1 : (c >> 2) & 1) ? hi : lo;
                }
              }
              if constexpr (BITS == 4) {
                op[0][j] = small_halves<0, 0>(pair[0], pair[1]);
                op[1][j] = small_halves<1, 1>(pair[0], pair[1]);
                op[2][j] = small_halves<2, 2>(pair[0], pair[1]);
                op[3][j] = small_halves<3, 3>(pair[0], pair[1]);
              } else {
                const uint32_t p01 = __builtin_amdgcn_perm(pair[1], pair[0], 0x05010400u);
                const uint32_t p23 = __builtin_amdgcn_perm(pair[1], pair[0], 0x07030602u);
                uint32_t w0, w1, w2, w3;
                widen4<VBF>(p01, 1.0f, w0, w1);
                widen4<VBF>(p23, 1.0f, w2, w3);
                op[0][j] = w0; op[1][j] = w1; op[2][j] = w2; op[3][j] = w3;
              }
            }
#pragma unroll
            for (int k = 0; k < 4; k++)
#pragma unroll
              for (int t = 0; t < TERMS; t++) o[c + k] = mfma16<VBF>(op[k], pt[t], o[c + k]);
          }
        }
      }
    };

    // The keys of the next step are loaded as soon as this one's scores are formed, its
    // values after the products, so that either is in flight while the other is computed
    // on; page numbers a step earlier still.
    if (steps > 0) {
      int ahead[NT];
#pragma unroll
      for (int i = 0; i < NT; i++) ahead[i] = page_of(t0 + SW * ST + 16 * i);
      for (int u = 0; u < steps - 1; u++) {
#pragma unroll
        for (int i = 0; i < NT; i++) {
          row[i] = row_of(ahead[i], t0 + SW * ST + 16 * i);
          ahead[i] = page_of(t0 + 2 * SW * ST + 16 * i);
        }
        scores();
        load_k(row);
        if (t0 < rg.first) mask_scores();
        softmax();
        if (t0 < rg.first) mask_values();
        products();
        load_v(row);
        t0 += SW * ST;
        const int done = x - x0 + SW * u;
        if (done >= quarter) {
          if (done < 2 * quarter) __builtin_amdgcn_s_setprio(2);
          else if (done < 3 * quarter) __builtin_amdgcn_s_setprio(1);
          else __builtin_amdgcn_s_setprio(0);
        }
      }
      const bool edge = t0 < rg.first || t0 + ST > rg.len;
      scores();
      if (edge) mask_scores();
      softmax();
      if (edge) mask_values();
      products();
    }

    // the wavefronts' parts, joined: lane (r, g) holds channels DV (4 g + i) + c of head r
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      lds_m[w * kHeads + r] = m;
      lds_l[w * kHeads + r] = l;
    }
    if (r < heads) {
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int c = 0; c < DV; c += 4)
          *reinterpret_cast<v4f *>(&lds_o[(w * wcols + r) * LD + DV * (4 * g + i) + c]) =
              v4f{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]} * (BITS == 4 ? kSmall : 1.0f);
    }
    __syncthreads();
    const bool whole = n == rg.steps;
    const int64_t row0 = (int64_t)b * a.hq + kvh * a.group + h0;
    const int slot = 2 * blockIdx.x + (x == x0 ? 0 : 1);
    float *part = parts + (int64_t)slot * part_floats(D, cols);
    if (!DIRECT && t == 0 && threadIdx.x == 0) {
      const int end = x + rg.steps - 1;      // the range's last step
      joins[(int64_t)b * vheads + vh] = Join{slot, whole ? 0 : end / chunk - (int)blockIdx.x + 1};
    }
    for (int e = threadIdx.x; e < min(cols, a.group - h0) * (D / 4); e += 64 * W) {
      const int h = e / (D / 4), d0 = 4 * (e % (D / 4));
      const int first = h / kHeads * SW, c = h % kHeads;    // its wavefronts, its column
      float mm = lds_m[first * kHeads + c];
#pragma unroll
      for (int i = 1; i < SW; i++) mm = fmaxf(mm, lds_m[(first + i) * kHeads + c]);
      float ll = 0.0f;
      v4f y = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < SW; i++) {
        const float f = __builtin_amdgcn_exp2f(lds_m[(first + i) * kHeads + c] - mm);
        const v4f z = *reinterpret_cast<const v4f *>(&lds_o[((first + i) * wcols + c) * LD + d0]);
        ll = fmaf(f, lds_l[(first + i) * kHeads + c], ll);
#pragma unroll
        for (int k = 0; k < 4; k++) y[k] = fmaf(f, z[k], y[k]);
      }
      if (whole) {
        store4<BF16>(a, D, row0 + h, d0, mm, ll, y);
      } else {
        *reinterpret_cast<v4f *>(part + part_head(cols) + h * D + d0) = y;
        if (d0 == 0) *reinterpret_cast<f2 *>(part + 2 * h) = f2{mm, ll};
      }
    }
    x += n;
    t = 0;
    if (x < x1) {
      __syncthreads();           // the LDS is free again
      if (++vh == vheads) {
        vh = 0;
        do {
          b++;
          rg = range_of<ST>(uniform(a.lengths[b]), cap, a.window);
        } while (rg.steps == 0);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The join, for ranges of more than one part: gridDim.z work-groups per range share
// its heads, a work-group's threads its parts; every sum in an order of its own.
// ---------------------------------------------------------------------------
template <int D, bool BF16>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const AttendArgs a) {
  constexpr int Q = D / 4, GROUPS = kJoinThreads / Q;
  __shared__ __attribute__((aligned(16))) float lds_o[GROUPS][D], lds_ml[GROUPS][2];
  const int b = blockIdx.y, vh = blockIdx.x, vheads = gridDim.x;
  const int hr = kHeads * head_blocks(a.group), hblocks = (a.group + hr - 1) / hr, cols = min(a.group, hr);
  const Join *joins = reinterpret_cast<const Join *>(a.scratch + (int64_t)a.blocks * 2 * part_floats(D, cols));
  const Join j = joins[(int64_t)b * vheads + vh];
  if (j.parts == 0) return;                      // written by its work-group
  const int kvh = vh / hblocks, h0 = vh % hblocks * hr;
  const int heads = min(hr, a.group - h0);
  const int pg = threadIdx.x / Q, d0 = 4 * (threadIdx.x % Q);
  for (int h = blockIdx.z; h < heads; h += gridDim.z) {
    float m = -INFINITY, l = 0.0f;
    v4f o = {0, 0, 0, 0};
    auto add = [&](f2 ml, v4f y) {
      const float m1 = fmaxf(m, ml.x);          // (of a part: finite)
      const float f0 = __builtin_amdgcn_exp2f(m - m1), f1 = __builtin_amdgcn_exp2f(ml.x - m1);
      m = m1;
      l = l * f0 + ml.y * f1;
#pragma unroll
      for (int i = 0; i < 4; i++) o[i] = o[i] * f0 + y[i] * f1;
    };
#pragma unroll 4
    for (int k = pg; k < j.parts; k += GROUPS) {
      const int slot = k == 0 ? j.first : (j.first & ~1) + 2 * k;
      const float *part = a.scratch + (int64_t)slot * part_floats(D, cols);
      add(*reinterpret_cast<const f2 *>(part + 2 * h), *reinterpret_cast<const v4f *>(part + part_head(cols) + h * D + d0));
    }
    if (pg > 0) {
      *reinterpret_cast<v4f *>(&lds_o[pg][d0]) = o;
      if (d0 == 0) *reinterpret_cast<f2 *>(lds_ml[pg]) = f2{m, l};
    }
    __syncthreads();
    if (pg == 0) {
#pragma unroll
      for (int k = 1; k < GROUPS; k++) add(*reinterpret_cast<const f2 *>(lds_ml[k]), *reinterpret_cast<const v4f *>(&lds_o[k][d0]));
      store4<BF16>(a, D, (int64_t)b * a.hq + kvh * a.group + h0 + h, d0, m, l, o);
    }
    __syncthreads();
  }
}

template <int W, int HB, int D, int BITS, bool BF16>
hipError_t go_attend(const AttendArgs &a, hipStream_t s) {
  const int bytes = lds_floats(W, HB, D, BITS, a.group < kHeads ? a.group : kHeads) * 4;
  const hipError_t e = allow_lds(reinterpret_cast<const void *>(attend_kernel<W, HB, D, BITS, BF16>), bytes);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attend_kernel<W, HB, D, BITS, BF16>), dim3(a.blocks), dim3(64 * W), bytes, s, a);
  return hipGetLastError();
}
template <int D, int BITS, bool BF16>
hipError_t go(const AttendArgs &a, hipStream_t s) {
  const bool two = head_blocks(a.group) == 2;
  if (a.direct) return two ? go_attend<kDirectWaves, 2, D, BITS, BF16>(a, s) : go_attend<kDirectWaves, 1, D, BITS, BF16>(a, s);
  const hipError_t e = two ? go_attend<kRunWaves, 2, D, BITS, BF16>(a, s) : go_attend<kRunWaves, 1, D, BITS, BF16>(a, s);
  if (e != hipSuccess) return e;
  // (a head each while that is a few thousand work-groups: those of whole ranges end at once)
  const int vheads = a.c.heads * ranges_of(a.group), cols = range_heads(a.group), share = 4096 / (vheads * a.batch);
  hipLaunchKernelGGL((join_kernel<D, BF16>), dim3(vheads, a.batch, share < 1 ? 1 : share < cols ? share : cols),
                     dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}
template <int D>
hipError_t go_bits(const AttendArgs &a, bool bf16, hipStream_t s) {
  if (a.c.bits == 16) return bf16 ? go<D, 16, true>(a, s) : go<D, 16, false>(a, s);
  if (a.c.bits == 8) return bf16 ? go<D, 8, true>(a, s) : go<D, 8, false>(a, s);
  return bf16 ? go<D, 4, true>(a, s) : go<D, 4, false>(a, s);
}

}  // namespace

AttendPlan attend_plan(const KvCache &c, int batch, int hq, int64_t max_len, int window) {
  AttendPlan p;
  const int group = hq / c.heads, st = kStep;
  const int64_t ranges = (int64_t)batch * c.heads * ranges_of(group);
  // (15 tokens more: a window may start within a tile)
  const int64_t longest = window > 0 && window < max_len ? window + 15 : max_len;
  const int64_t steps = (longest + st - 1) / st;
  // One work-group per range where a range is short: up to two rounds of steps of its
  // wavefronts at 16 bits and 128 channels, up to four of lighter ones, and twice that
  // where the ranges alone fill half the CUs.  Graph replays, us, direct against runs
  // and their join (8 kv heads of 128, all streams alike; tokens):
  //            1 stream                          16 streams
  //   16 bits  512: 8.0, 8.0   768: 10.0, 8.4    1024: 17.9, 21.2   1536: 28.0, 23.9
  //    8 bits  768: 8.3, 8.3  1024:  9.7, 8.3    2048: 20.3, 22.4
  //    4 bits 1024: 8.1, 8.0  1536: 10.2, 8.3    2048: 13.1, 18.6
  // (So at 8 bits the rule keeps a few streams of 769 to 1024 tokens in one launch, up to 1.4 us
  // longer than runs would take.  Only d = 128 was compared.)
  const int rounds2 = 32768 / (c.d * c.bits), most_steps = (rounds2 < 32 ? rounds2 : 32) * (ranges >= kCus / 2 ? 2 : 1);
  // (and a launch numbers its lanes in 32 bits)
  p.direct = steps <= most_steps && ranges * 64 * kDirectWaves < ((int64_t)1 << 32);
  p.steps = ranges * steps;
  if (p.direct) {
    p.blocks = (int)ranges;
    p.scratch = 0;
    return p;
  }
  const int64_t runs = (p.steps + kRunWaves - 1) / kRunWaves;
  const int most = kCus * runs_per_cu(c.d);
  p.blocks = (int)(runs < most ? runs : most);
  p.scratch = (size_t)p.blocks * 2 * part_floats(c.d, range_heads(group)) * 4 + (size_t)ranges * sizeof(Join);
  return p;
}

hipError_t launch_attend(const AttendArgs &a, bool bf16, hipStream_t s) {
  if (a.c.d == 64) return go_bits<64>(a, bf16, s);
  if (a.c.d == 128) return go_bits<128>(a, bf16, s);
  return go_bits<256>(a, bf16, s);
}

}  // namespace tq
