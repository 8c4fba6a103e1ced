// Norm and position rotation of queries and keys, and the paged key-value
// cache: rows quantized as they are written, and read back.
//
// All three are one pass over head rows of d = 64, 128 or 256 16-bit values and
// bound by memory.  d / 16 lanes own a row, each two runs of eight values (16
// bytes), half of the rotated channels apart, so that both values of every rotated
// pair are in one lane whichever way they are paired; the row's sum of squares and
// largest value come from DPP lane swaps among its lanes.  Nothing passes through
// LDS, and a row is read and written once.
//
// Measured (d = 128; a copy kernel reaches 6.5 TB/s):
//   rotation of 8192 tokens of 64 + 8 heads, fp16         55 us, 5.6 TB/s
//   the same with norms, bf16                             59 us, 5.2 TB/s
//   rotation of 2048 tokens of 32 + 8 heads into the 16-bit cache and read back, bf16   15 us
//   8192 tokens of 8 + 8 heads written in 8 bits (bf16) 11 us, in 4 (fp16) 14, read back 10
//   norm, rotation and 4-bit write of 8192 tokens of 32 + 8 heads, bf16   43 us
// One row per lane: with two to four, whose loads would be in flight together, the
// first takes 61 us and 8192 tokens written and read in 8 bits 32 instead of 21.
// Non-temporal stores of q and k save 2 us here and cost the kernel that reads them next
// 2.5.
#include "tq_device.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

template <bool BF16>
__device__ __forceinline__ float value_of(uint16_t b) {
  return BF16 ? bf16_bits_to_float(b) : half_bits_to_float(b);
}
// (the compiler's conversions: also NaN stays NaN)
template <bool BF16>
__device__ __forceinline__ uint16_t bits_of(float f) {
  return BF16 ? __builtin_bit_cast(uint16_t, (__bf16)f) : float_to_half_bits(f);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float a) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, a), CTRL, 0xF, 0xF, false));
}

// Sum / max over the L = 4, 8 or 16 lanes of a row: neighbours, pairs, then the
// mirrors of eight and of sixteen lanes.
template <int L>
__device__ __forceinline__ float row_sum(float a) {
  a += dpp<0xB1>(a);
  a += dpp<0x4E>(a);
  if constexpr (L >= 8) a += dpp<0x141>(a);
  if constexpr (L >= 16) a += dpp<0x140>(a);
  return a;
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t a) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, CTRL, 0xF, 0xF, false);
}
template <int L>
__device__ __forceinline__ uint32_t row_max(uint32_t a) {
  a = max(a, dpp<0xB1>(a));
  a = max(a, dpp<0x4E>(a));
  if constexpr (L >= 8) a = max(a, dpp<0x141>(a));
  if constexpr (L >= 16) a = max(a, dpp<0x140>(a));
  return a;
}

template <bool BF16>
__device__ __forceinline__ void widen(u32x4 r, float *v) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[2 * i] = value_of<BF16>((uint16_t)(r[i] & 0xffffu));
    v[2 * i + 1] = value_of<BF16>((uint16_t)(r[i] >> 16));
  }
}
template <bool BF16>
__device__ __forceinline__ u32x4 narrow(const float *v) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; i++)
    r[i] = (uint32_t)bits_of<BF16>(v[2 * i]) | (uint32_t)bits_of<BF16>(v[2 * i + 1]) << 16;
  return r;
}

// a b + c d to within about an ulp also where the products cancel: the rounding of
// the second is found by an fma and added back (Kahan's difference of products).
__device__ __forceinline__ float two_products(float a, float b, float c, float d) {
  const float w = c * d;
  return fmaf(a, b, w) + fmaf(c, d, -w);
}

// e4m3 codes of eight values over their scale: clamp(v / s), rounded half to
// even.  y = 1 / s to within an ulp or two; t = v y is put right by its exact
// remainder, so that a quotient on a rounding boundary of e4m3 (at most five
// significant bits) comes out exactly, and any other is 2^-17 or further, by its
// size, from the nearest one.
__device__ __forceinline__ uint2 quant8_e4m3(const float *v, float s, float y) {
  float f[8];
#pragma unroll
  for (int e = 0; e < 8; e++) {
    const float t = v[e] * y;
    const float q = fmaf(fmaf(-t, s, v[e]), y, t);
    f[e] = fminf(fmaxf(q, -448.0f), 448.0f);
  }
  uint32_t lo, hi;
  lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
  lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], (int)lo, true);
  hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
  hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], (int)hi, true);
  return make_uint2(lo, hi);
}

// The row of a slot in a cache section, or -1 for a slot outside the cache.
__device__ __forceinline__ int64_t cache_row(const KvCache &c, int64_t slot, int head) {
  if (slot < 0 || slot >= (int64_t)c.pages << c.lps) return -1;
  return ((((slot >> c.lps) * c.heads + head) << c.lps) + (slot & ((1 << c.lps) - 1)));
}

// ---------------------------------------------------------------------------
// Rows of one call: per token hq query rows, hkv key rows and (with a cache) hkv
// value rows.  Query and key rows are normed and rotated in fp32 and rounded
// once to 16 bits; key (rounded) and value rows go to the token's cache slot.
// BITS 0: no cache.
// ---------------------------------------------------------------------------
template <int D, int BITS, bool BF16>
__global__ __launch_bounds__(256) void tokens_kernel(const TokenArgs a) {
  constexpr int L = D / 16;               // lanes per row
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int e = lane & (L - 1);
  const uint32_t row = wave * (64 / L) + lane / L;
  const uint32_t rows = (uint32_t)a.tokens * (uint32_t)a.rows_per_token;   // < 2^31 (host)
  if (row >= rows) return;                // whole rows of lanes leave together
  const uint32_t token = __umulhi(row, a.magic) >> a.shift;
  const int r = (int)(row - token * (uint32_t)a.rows_per_token);
  const int kind = r < a.hq ? 0 : r < a.hq + a.hkv ? 1 : 2;
  const int head = kind == 0 ? r : kind == 1 ? r - a.hq : r - a.hq - a.hkv;
  const HeadRows &src = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
  // the lane's two runs of eight values, in the two halves of the rotated channels or
  // of the others: either is a stretch that neighbouring lanes continue (two runs side
  // by side: 24 us instead of 21 for 8192 tokens in 8 bits, written and read back)
  const bool turned = e < a.rot / 16;
  const int i0 = 8 * e + (turned ? 0 : a.rot / 2);
  const int i1 = 8 * e + (turned ? a.rot / 2 : D / 2);
  const uint16_t *p = src.p + (int64_t)token * src.ts + head * src.hs;
  const u32x4 r0 = *reinterpret_cast<const u32x4 *>(p + i0);
  const u32x4 r1 = *reinterpret_cast<const u32x4 *>(p + i1);
  int64_t slot = -1;
  if constexpr (BITS != 0) {
    if (kind != 0) slot = a.slots[token];
  }
  float v[16];
  u32x4 o0 = r0, o1 = r1;
  widen<BF16>(r0, v);
  widen<BF16>(r1, v + 8);
  const uint16_t *w = kind == 0 ? a.qw : a.kw;
  const bool normed = kind != 2 && w != nullptr;
  float cs[16];
  const bool turn = turned && kind != 2;
  if (turn) {
    int pos = a.positions[token];
    pos = min(max(pos, 0), a.max_pos - 1);
    // angles of pairs 8 e .. 8 e + 7, or of those in the two runs
    const float *t = a.table + (int64_t)pos * a.rot;
    const int at[2] = {a.interleaved ? 4 * e : 8 * e, a.interleaved ? a.rot / 4 + 4 * e : 8 * e + 4};
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const v4f c = *reinterpret_cast<const v4f *>(t + at[i]);
      const v4f s = *reinterpret_cast<const v4f *>(t + a.rot / 2 + at[i]);
#pragma unroll
      for (int j = 0; j < 4; j++) {
        cs[4 * i + j] = c[j];
        cs[8 + 4 * i + j] = s[j];
      }
    }
  }
  if (normed) {
    float wv[16];
    widen<BF16>(*reinterpret_cast<const u32x4 *>(w + i0), wv);
    widen<BF16>(*reinterpret_cast<const u32x4 *>(w + i1), wv + 8);
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) ss = fmaf(v[i], v[i], ss);
    ss = row_sum<L>(ss);
    const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
    for (int i = 0; i < 16; i++) v[i] = v[i] * inv * wv[i];
  }
  if (turn) {
    if (a.interleaved) {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float x = v[2 * i], y = v[2 * i + 1];
        v[2 * i] = two_products(x, cs[i], -y, cs[8 + i]);
        v[2 * i + 1] = two_products(y, cs[i], x, cs[8 + i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float x = v[i], y = v[8 + i];
        v[i] = two_products(x, cs[i], -y, cs[8 + i]);
        v[8 + i] = two_products(y, cs[i], x, cs[8 + i]);
      }
    }
  }
  if (normed || turn) {
    o0 = narrow<BF16>(v);
    o1 = narrow<BF16>(v + 8);
  }
  if (kind != 2) {
    uint16_t *out = kind == 0 ? a.q_out : a.k_out;
    if (out != nullptr) {
      out += ((int64_t)token * (kind == 0 ? a.hq : a.hkv) + head) * D;
      *reinterpret_cast<u32x4 *>(out + i0) = o0;
      *reinterpret_cast<u32x4 *>(out + i1) = o1;
    }
  }
  if constexpr (BITS != 0) {
    if (kind == 0) return;
    uint8_t *base = kind == 1 ? a.c.k : a.c.v;
    const int64_t at = cache_row(a.c, slot, head);
    if constexpr (BITS == 16) {
      if (at < 0) return;
      uint16_t *dst = reinterpret_cast<uint16_t *>(base) + at * D;
      *reinterpret_cast<u32x4 *>(dst + i0) = o0;
      *reinterpret_cast<u32x4 *>(dst + i1) = o1;
    } else {
      // the codes of the rounded values
      widen<BF16>(o0, v);
      widen<BF16>(o1, v + 8);
      // the largest value by its bits, in which NaN comes after infinity
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 16; i++) top = max(top, __builtin_bit_cast(uint32_t, v[i]) & 0x7fffffffu);
      top = row_max<L>(top);
      const float amax = __builtin_bit_cast(float, top);
      // (a row that is not finite, or a bf16 one whose scale no fp16 number holds, gets the
      // scale NaN, since its codes could not tell)
      const uint16_t h = float_to_half_bits(amax / (BITS == 4 ? 7.0f : 448.0f)), s16 = h >= 0x7c00 ? 0x7e00 : h;
      const float s = half_bits_to_float(s16);
      const float y = s == 0.0f ? 0.0f : 1.0f / s;
      if (at < 0) return;
      if constexpr (BITS == 8) {
        uint8_t *dst = base + at * D;
        *reinterpret_cast<uint2 *>(dst + i0) = quant8_e4m3(v, s, y);
        *reinterpret_cast<uint2 *>(dst + i1) = quant8_e4m3(v + 8, s, y);
      } else {
        uint8_t *dst = base + at * (D / 2);
        uint32_t lo, hi;
        quant8_fp8(*reinterpret_cast<const float(*)[8]>(v), s, y, lo, hi);
        *reinterpret_cast<uint32_t *>(dst + i0 / 2) = lo | __builtin_amdgcn_alignbit(hi, hi, 28);
        quant8_fp8(*reinterpret_cast<const float(*)[8]>(v + 8), s, y, lo, hi);
        *reinterpret_cast<uint32_t *>(dst + i1 / 2) = lo | __builtin_amdgcn_alignbit(hi, hi, 28);
      }
      if (e == 0) (kind == 1 ? a.c.ks : a.c.vs)[at] = s16;
    }
  }
}

// ---------------------------------------------------------------------------
// Cache rows of the given slots as 16-bit values: code times scale in fp32,
// rounded once.  Slots outside the cache give zeros.
// ---------------------------------------------------------------------------
template <bool BF16, int BITS>
__device__ __forceinline__ u32x4 read8(const uint8_t *row, int i, float s) {
  if constexpr (BITS == 16) {
    return *reinterpret_cast<const u32x4 *>(row + 2 * i);
  } else {
    uint32_t w[2];
    if constexpr (BITS == 8) {
      const uint2 u = *reinterpret_cast<const uint2 *>(row + i);
      w[0] = u.x;
      w[1] = u.y;
    } else {
      tq4_to_fp8(*reinterpret_cast<const uint32_t *>(row + i / 2), w[0], w[1]);
    }
    float f[8];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const auto x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false);
      const auto y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
      f[4 * j] = x[0] * s;
      f[4 * j + 1] = x[1] * s;
      f[4 * j + 2] = y[0] * s;
      f[4 * j + 3] = y[1] * s;
    }
    return narrow<BF16>(f);
  }
}

template <int D, int BITS, bool BF16>
__global__ __launch_bounds__(256) void kv_read_kernel(const ReadArgs a) {
  constexpr int L = D / 16;
  const int lane = threadIdx.x & 63;
  const uint32_t wave = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int e = lane & (L - 1);
  const uint32_t row = wave * (64 / L) + lane / L;
  const uint32_t per = 2u * a.c.heads;
  if (row >= (uint32_t)a.tokens * per) return;
  const uint32_t token = __umulhi(row, a.magic) >> a.shift;
  int head = (int)(row - token * per);
  const bool is_v = head >= a.c.heads;
  head -= is_v ? a.c.heads : 0;
  const int i0 = 8 * e, i1 = D / 2 + 8 * e;
  const int64_t at = cache_row(a.c, a.slots[token], head);
  u32x4 o0 = {0, 0, 0, 0}, o1 = {0, 0, 0, 0};
  if (at >= 0) {
    const uint8_t *src = (is_v ? a.c.v : a.c.k) + at * (D * BITS / 8);
    // (4-bit codes come out of the conversion as code * 2^-9)
    const float s = BITS == 16 ? 0.0f : half_bits_to_float((is_v ? a.c.vs : a.c.ks)[at]) * (BITS == 4 ? 512.0f : 1.0f);
    o0 = read8<BF16, BITS>(src, i0, s);
    o1 = read8<BF16, BITS>(src, i1, s);
  }
  uint16_t *out = (is_v ? a.v_out : a.k_out) + ((int64_t)token * a.c.heads + head) * D;
  *reinterpret_cast<u32x4 *>(out + i0) = o0;
  *reinterpret_cast<u32x4 *>(out + i1) = o1;
}

template <int D, int BITS>
void go_tokens(const TokenArgs &a, bool bf16, unsigned blocks, hipStream_t s) {
  if (bf16) hipLaunchKernelGGL((tokens_kernel<D, BITS, true>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((tokens_kernel<D, BITS, false>), dim3(blocks), dim3(256), 0, s, a);
}
template <int D>
void go_tokens_bits(const TokenArgs &a, bool bf16, unsigned blocks, hipStream_t s) {
  if (a.slots == nullptr) go_tokens<D, 0>(a, bf16, blocks, s);
  else if (a.c.bits == 16) go_tokens<D, 16>(a, bf16, blocks, s);
  else if (a.c.bits == 8) go_tokens<D, 8>(a, bf16, blocks, s);
  else go_tokens<D, 4>(a, bf16, blocks, s);
}

template <int D, int BITS>
void go_read(const ReadArgs &a, bool bf16, unsigned blocks, hipStream_t s) {
  if (bf16) hipLaunchKernelGGL((kv_read_kernel<D, BITS, true>), dim3(blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv_read_kernel<D, BITS, false>), dim3(blocks), dim3(256), 0, s, a);
}
template <int D>
void go_read_bits(const ReadArgs &a, bool bf16, unsigned blocks, hipStream_t s) {
  if (a.c.bits == 16) go_read<D, 16>(a, bf16, blocks, s);
  else if (a.c.bits == 8) go_read<D, 8>(a, bf16, blocks, s);
  else go_read<D, 4>(a, bf16, blocks, s);
}

// work-groups of four wavefronts for `rows` rows of d values
unsigned row_blocks(int64_t rows, int d) {
  const int64_t per = 4 * (64 / (d / 16));
  return (unsigned)((rows + per - 1) / per);
}

}  // namespace

hipError_t launch_tokens(const TokenArgs &args, bool bf16, hipStream_t s) {
  TokenArgs a = args;
  divide_by((uint32_t)a.rows_per_token, a.magic, a.shift);
  const unsigned blocks = row_blocks((int64_t)a.tokens * a.rows_per_token, a.c.d);
  if (a.c.d == 64) go_tokens_bits<64>(a, bf16, blocks, s);
  else if (a.c.d == 128) go_tokens_bits<128>(a, bf16, blocks, s);
  else go_tokens_bits<256>(a, bf16, blocks, s);
  return hipGetLastError();
}

hipError_t launch_kv_read(const ReadArgs &args, bool bf16, hipStream_t s) {
  ReadArgs a = args;
  divide_by(2u * (uint32_t)a.c.heads, a.magic, a.shift);
  const unsigned blocks = row_blocks((int64_t)a.tokens * 2 * a.c.heads, a.c.d);
  if (a.c.d == 64) go_read_bits<64>(a, bf16, blocks, s);
  else if (a.c.d == 128) go_read_bits<128>(a, bf16, blocks, s);
  else go_read_bits<256>(a, bf16, blocks, s);
  return hipGetLastError();
}

}  // namespace tq
