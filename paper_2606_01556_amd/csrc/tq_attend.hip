// Attention of one new token per stream over the paged cache:
//
//   o_h = sum_t softmax_t(scale q_h . k_t) v_t,  t in [max(0, len - window), len)
//
// Bound by the cache's bytes (at most 4 flops per value and query head of the
// group), so the kernel is built around one pass over them with nothing but
// registers between memory and the matrix cores:
//
//  * S^T = K Q^T in 16x16x32 products.  A lane of the first operand holds eight
//    values of one token's key, which is a run of the cache row as it lies in
//    memory; the group's query heads (up to 16) are the columns.  Which of a
//    row's values make up one product is free as long as Q is laid out alike, so
//    each format loads the widest run a lane can.
//  * The result has column lane % 16 and rows 4 (lane / 16) + i: a lane holds the
//    scores of one head for tokens 4 g + i.  Two such tiles, exponentiated, are
//    the second operand of O^T = V^T P^T as they stand (the order of the tokens
//    is free too), so no score crosses lanes.
//  * V^T's operand takes eight tokens' values of one channel per lane.  A lane
//    loads rows 4 g + i of the tile, channels DV r .. DV r + DV - 1 (r = lane %
//    16, DV = d / 16), and pairs the rows up with byte permutes.
//  * The running maximum is a reference only: it moves when some score passes it
//    by 2^8, so that most steps have no exchange between lanes and no rescaling.
//
// The work is cut evenly whatever the lengths: all (stream, head) ranges of
// units laid end to end are split into equal runs, one per work-group.  A range
// that one run holds whole is written at once; the ends of the others are joined
// by a second launch, in order, so a result does not depend on timing.
#include "tq_device.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef const int32_t __attribute__((address_space(4))) const_i32;

constexpr int kWaves = 4;
constexpr int kHeads = 16;                 // query heads per work-group (columns of a product)

// tokens a wavefront takes at a time, and a work-group's unit
constexpr int step_tokens(int bits) { return bits == 16 ? 32 : 64; }
constexpr int unit_tokens(int bits) { return kWaves * step_tokens(bits); }

constexpr float kLog2e = 1.4426950408889634f;

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

// two fp32 values rounded to a word of 16-bit ones
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const f2 v = {x, y};
  if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
  else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, h2));
}

// NB bytes from p (p aligned to min(NB, 16))
template <int NB>
__device__ __forceinline__ void load_bytes(const uint8_t *p, uint32_t *out) {
  if constexpr (NB >= 16) {
#pragma unroll
    for (int i = 0; i < NB / 16; i++) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(p + 16 * i);
      out[4 * i] = v.x; out[4 * i + 1] = v.y; out[4 * i + 2] = v.z; out[4 * i + 3] = v.w;
    }
  } else if constexpr (NB == 8) {
    const uint2 v = *reinterpret_cast<const uint2 *>(p);
    out[0] = v.x; out[1] = v.y;
  } else {
    static_assert(NB == 4);
    out[0] = *reinterpret_cast<const uint32_t *>(p);
  }
}

// Units of a stream: [first, len) in units from first rounded down to 16.
struct Range {
  int first, len, base, units;
};
template <int UT>
__device__ __forceinline__ Range range_of(int len, int cap, int window) {
  Range r;
  r.len = min(max(len, 0), cap);
  r.first = window > 0 && r.len > window ? r.len - window : 0;
  r.base = r.first & ~15;
  r.units = (r.len - r.base + UT - 1) / UT;
  return r;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sum of units of streams [0, until) in every lane of the wavefront.
template <int UT>
__device__ int units_before(const AttendArgs &a, int cap, int until) {
  int s = 0;
  for (int b = threadIdx.x & 63; b < until; b += 64) s += range_of<UT>(a.lengths[b], cap, a.window).units;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) s += __shfl_xor(s, m);
  return uniform(s);
}

// The stream that holds unit x of all streams' units laid end to end, and the
// units before it (x below the total).
template <int UT>
__device__ void locate(const AttendArgs &a, int cap, int x, int &stream, int &before) {
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const int b = b0 + lane;
    int incl = b < a.batch ? range_of<UT>(a.lengths[b], cap, a.window).units : 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int o = __shfl_up(incl, m);
      if (lane >= m) incl += o;
    }
    const uint64_t past = __ballot(sum + incl > x);
    if (past != 0) {
      const int at = __builtin_ctzll(past);
      stream = b0 + at;
      before = sum + (at == 0 ? 0 : uniform(__shfl(incl, at - 1)));
      stream = uniform(stream);
      before = uniform(before);
      return;
    }
    sum += uniform(__shfl(incl, 63));
  }
  stream = a.batch;
  before = sum;
}

// floats of one partial result: the group's maxima and sums, then its products
__host__ __device__ constexpr int partial_head(int cols) { return (2 * cols + 3) & ~3; }
__host__ __device__ constexpr int partial_floats(int d, int cols) { return partial_head(cols) + cols * d; }

// ---------------------------------------------------------------------------
template <int D, int BITS, bool BF16>
__global__ __launch_bounds__(64 * kWaves) void attend_kernel(const AttendArgs a) {
  constexpr int ST = step_tokens(BITS), UT = unit_tokens(BITS), NT = ST / 16;
  constexpr int RB = D * BITS / 8;            // bytes of a row
  constexpr int CE = BITS == 16 ? 8 : BITS == 8 ? 16 : (D / 4 < 32 ? D / 4 : 32);  // a lane's run of a key row
  constexpr int CB = CE * BITS / 8;           // its bytes
  constexpr int KL = D / (4 * CE);            // runs per lane
  constexpr int KW = KL * CB / 4;             // words
  constexpr int KS = D / 32;                  // products per tile of keys
  constexpr int DV = D / 16;                  // channels per lane of a value row
  constexpr int VBr = DV * BITS / 8;          // their bytes; two lanes share a word of 4-bit codes at d = 64
  constexpr int VB = VBr < 4 ? 4 : VBr;
  constexpr int VW = VB / 4;
  constexpr bool VBF = BITS == 16 ? BF16 : true;   // type of the second product
  constexpr bool SPLIT = VBF;                 // its weights in two parts (bf16 has 8 bits)
  constexpr int LD = D + 4;                   // LDS row of one head, staggered over the banks

  __shared__ float lds_o[kWaves][kHeads][LD];
  __shared__ float lds_m[kWaves][kHeads], lds_l[kWaves][kHeads];

  const int lane = threadIdx.x & 63, w = uniform(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const int lps = a.c.lps, hkv = a.c.heads;
  const int cap = a.max_pages << lps;
  const int hblocks = (a.group + kHeads - 1) / kHeads, vheads = hkv * hblocks;
  const int cols = min(a.group, kHeads);

  // this work-group's run of units
  const int per_head = units_before<UT>(a, cap, a.batch);
  const int64_t total = (int64_t)per_head * vheads;
  const int64_t chunk = (total + gridDim.x - 1) / gridDim.x;
  const int64_t x0 = blockIdx.x * chunk, x1 = min(total, x0 + chunk);
  if (x0 >= x1) return;
  int b, before;
  locate<UT>(a, cap, (int)(x0 / vheads), b, before);
  Range rg = range_of<UT>(uniform(a.lengths[b]), cap, a.window);
  int vh = (int)((x0 - (int64_t)before * vheads) / rg.units);
  int t = (int)((x0 - (int64_t)before * vheads) % rg.units);
  const float c1 = a.scale * kLog2e;
  float *part = a.scratch + (int64_t)blockIdx.x * 2 * partial_floats(D, cols);

  for (int64_t x = x0; x < x1;) {
    const int n = (int)min((int64_t)(rg.units - t), x1 - x);
    const int kvh = vh / hblocks, hb = vh % hblocks;
    const int heads = min(kHeads, a.group - hb * kHeads);   // live columns

    // Q^T: column r, the values of the runs a key lane loads
    u32x4 q[KS];
    {
      const uint16_t *qp = a.q + b * a.q_ts + (int64_t)(kvh * a.group + hb * kHeads + min(r, heads - 1)) * a.q_hs;
#pragma unroll
      for (int s = 0; s < KS; s++) {
        const int d0 = (8 * s / CE) * 4 * CE + g * CE + 8 * s % CE;
        q[s] = *reinterpret_cast<const u32x4 *>(qp + d0);
        if (r >= heads) q[s] = u32x4{0, 0, 0, 0};
      }
    }
    v4f o[DV];
#pragma unroll
    for (int i = 0; i < DV; i++) o[i] = v4f{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    const_i32 *pages = (const_i32 *)(a.table + b * a.table_stride);
    const int last_page = (rg.len - 1) >> lps;
    for (int u = t; u < t + n; u++) {
      const int t0 = uniform(rg.base + u * UT + w * ST);
      if (t0 >= rg.len) break;
      uint32_t kraw[NT][KW], vraw[NT][4][VW];
      uint2 ksr[NT], vsr[NT];
#pragma unroll
      for (int i = 0; i < NT; i++) {
        const int tt = t0 + 16 * i;
        // (a tile past the end reads the last page and is masked)
        int page = pages[min(tt >> lps, last_page)];
        page = min(max(page, 0), a.c.pages - 1);
        const int64_t row = (((int64_t)page * hkv + kvh) << lps) + (tt & ((1 << lps) - 1));
        const uint8_t *kp = a.c.k + row * RB, *vp = a.c.v + row * RB;
#pragma unroll
        for (int j = 0; j < KL; j++) load_bytes<CB>(kp + r * RB + j * 4 * CB + g * CB, &kraw[i][j * CB / 4]);
#pragma unroll
        for (int j = 0; j < 4; j++)
          load_bytes<VB>(vp + (4 * g + j) * RB + (VBr < 4 ? (r >> 1) * 4 : r * VB), vraw[i][j]);
        if constexpr (BITS < 16) {
          ksr[i] = *reinterpret_cast<const uint2 *>(a.c.ks + row + 4 * g);
          vsr[i] = *reinterpret_cast<const uint2 *>(a.c.vs + row + 4 * g);
        }
      }
      // scores: row 4 g + j of tile i, head r, times log2 e
      float s[NT][4];
#pragma unroll
      for (int i = 0; i < NT; i++) {
        v4f acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; k++) {
          u32x4 op;
          if constexpr (BITS == 16) {
            op = u32x4{kraw[i][4 * k], kraw[i][4 * k + 1], kraw[i][4 * k + 2], kraw[i][4 * k + 3]};
          } else {
            uint32_t w0, w1, x0_, x1_, x2_, x3_;
            if constexpr (BITS == 8) {
              w0 = kraw[i][2 * k];
              w1 = kraw[i][2 * k + 1];
            } else {
              tq4_to_fp8(kraw[i][k], w0, w1);
            }
            const float sc = BITS == 4 ? 512.0f : 1.0f;
            widen4<BF16>(w0, sc, x0_, x1_);
            widen4<BF16>(w1, sc, x2_, x3_);
            op = u32x4{x0_, x1_, x2_, x3_};
          }
          acc = mfma16<BF16>(op, q[k], acc);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
          float c = c1;
          if constexpr (BITS < 16) {
            const uint32_t sw = j < 2 ? ksr[i].x : ksr[i].y;
            c *= half_bits_to_float((uint16_t)(j & 1 ? sw >> 16 : sw & 0xffffu));
          }
          s[i][j] = acc[j] * c;
        }
      }
      float vs[NT][4];
      if constexpr (BITS < 16) {
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const uint32_t sw = j < 2 ? vsr[i].x : vsr[i].y;
            vs[i][j] = half_bits_to_float((uint16_t)(j & 1 ? sw >> 16 : sw & 0xffffu));
          }
      }
      if (t0 < rg.first || t0 + ST > rg.len) {
        // tokens outside the range: no score, and nothing of what their rows hold
#pragma unroll
        for (int i = 0; i < NT; i++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const int tok = t0 + 16 * i + 4 * g + j;
            const bool in = tok >= rg.first && tok < rg.len;
            s[i][j] = in ? s[i][j] : -INFINITY;
            if constexpr (BITS < 16) vs[i][j] = in ? vs[i][j] : 0.0f;
#pragma unroll
            for (int k = 0; k < VW; k++) vraw[i][j][k] = in ? vraw[i][j][k] : 0u;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) top = fmaxf(top, s[i][j]);
      if (__any(top > m + 8.0f)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float m1 = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - m1);
        m = m1;
        l *= f;
#pragma unroll
        for (int i = 0; i < DV; i++) o[i] *= f;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int i = 0; i < NT; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
          s[i][j] = __builtin_amdgcn_exp2f(s[i][j] - ref);
          l += s[i][j];
          if constexpr (BITS < 16) s[i][j] *= vs[i][j];
        }
      // O^T += V^T P^T, 32 tokens (two tiles) at a time
#pragma unroll
      for (int i = 0; i < NT; i += 2) {
        u32x4 ph, pl;
#pragma unroll
        for (int j = 0; j < 4; j++) {
          const float p0 = s[i + j / 2][2 * (j & 1)], p1 = s[i + j / 2][2 * (j & 1) + 1];
          ph[j] = pack2<VBF>(p0, p1);
          if constexpr (SPLIT)
            pl[j] = pack2<true>(p0 - __builtin_bit_cast(float, ph[j] << 16),
                                p1 - __builtin_bit_cast(float, ph[j] & 0xffff0000u));
        }
        // rows as 16-bit values, two channels a word: row[tile][j][channel / 2]
        uint32_t row[2][4][DV / 2];
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
          for (int j = 0; j < 4; j++) {
            const uint32_t *raw = vraw[i + h][j];
            if constexpr (BITS == 16) {
#pragma unroll
              for (int k = 0; k < DV / 2; k++) row[h][j][k] = raw[k];
            } else if constexpr (BITS == 8) {
#pragma unroll
              for (int k = 0; k < DV / 4; k++) widen4<true>(raw[k], 1.0f, row[h][j][2 * k], row[h][j][2 * k + 1]);
            } else if constexpr (VBr < 4) {
              // codes 0..3 of the shared word for even lanes, 4..7 for odd ones
              uint32_t lo, hi;
              tq4_to_fp8(raw[0], lo, hi);
              widen4<true>(r & 1 ? hi : lo, 512.0f, row[h][j][0], row[h][j][1]);
            } else {
#pragma unroll
              for (int k = 0; k < DV / 8; k++) {
                uint32_t lo, hi;
                tq4_to_fp8(raw[k], lo, hi);
                widen4<true>(lo, 512.0f, row[h][j][4 * k], row[h][j][4 * k + 1]);
                widen4<true>(hi, 512.0f, row[h][j][4 * k + 2], row[h][j][4 * k + 3]);
              }
            }
          }
#pragma unroll
        for (int c = 0; c < DV; c++) {
          const uint32_t sel = c & 1 ? 0x07060302u : 0x05040100u;
          u32x4 op;
#pragma unroll
          for (int j = 0; j < 4; j++)
            op[j] = __builtin_amdgcn_perm(row[j / 2][2 * (j & 1) + 1][c / 2], row[j / 2][2 * (j & 1)][c / 2], sel);
          o[c] = mfma16<VBF>(op, ph, o[c]);
          if constexpr (SPLIT) o[c] = mfma16<VBF>(op, pl, o[c]);
        }
      }
    }

    // the wavefronts' parts, joined: lane (r, g) holds channels DV (4 g + i) + c of head r
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
      lds_m[w][r] = m;
      lds_l[w][r] = l;
    }
    if (r < heads) {
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int c = 0; c < DV; c += 4)
          *reinterpret_cast<v4f *>(&lds_o[w][r][DV * (4 * g + i) + c]) = v4f{o[c][i], o[c + 1][i], o[c + 2][i], o[c + 3][i]};
    }
    __syncthreads();
    const bool whole = n == rg.units;
    float *slot = part + (x == x0 ? 0 : partial_floats(D, cols));
    for (int e = threadIdx.x; e < heads * (D / 2); e += 64 * kWaves) {
      const int h = e / (D / 2), d0 = 2 * (e % (D / 2));
      float mm = lds_m[0][h];
#pragma unroll
      for (int i = 1; i < kWaves; i++) mm = fmaxf(mm, lds_m[i][h]);
      const float ref = mm == -INFINITY ? 0.0f : mm;
      float ll = 0.0f, y0 = 0.0f, y1 = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; i++) {
        const float f = __builtin_amdgcn_exp2f(lds_m[i][h] - ref);
        ll = fmaf(f, lds_l[i][h], ll);
        y0 = fmaf(f, lds_o[i][h][d0], y0);
        y1 = fmaf(f, lds_o[i][h][d0 + 1], y1);
      }
      const int qh = kvh * a.group + hb * kHeads + h;
      if (whole) {
        const float inv = 1.0f / ll;
        *reinterpret_cast<uint32_t *>(a.out + ((int64_t)b * a.hq + qh) * D + d0) = pack2<BF16>(y0 * inv, y1 * inv);
        if (a.lse != nullptr && d0 == 0) a.lse[(int64_t)b * a.hq + qh] = (mm + log2f(ll)) * (1.0f / kLog2e);
      } else {
        *reinterpret_cast<f2 *>(slot + partial_head(cols) + h * D + d0) = f2{y0, y1};
        if (d0 == 0) *reinterpret_cast<f2 *>(slot + 2 * h) = f2{mm, ll};
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
          rg = range_of<UT>(uniform(a.lengths[b]), cap, a.window);
        } while (rg.units == 0);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Joins the parts of ranges that several work-groups hold, in their order, and
// fills the rows of streams that hold nothing.  One work-group per stream and
// query head.
// ---------------------------------------------------------------------------
template <int D, int BITS, bool BF16>
__global__ __launch_bounds__(256) void join_kernel(const AttendArgs a) {
  constexpr int UT = unit_tokens(BITS);
  constexpr int LN = D / 4, PG = 256 / LN;     // lanes per part, parts at a time
  __shared__ float lds_o[PG][D];
  __shared__ float lds_m[PG], lds_l[PG];
  const int b = blockIdx.y, qh = blockIdx.x;
  const int cap = a.max_pages << a.c.lps;
  const int hblocks = (a.group + kHeads - 1) / kHeads, vheads = a.c.heads * hblocks;
  const int cols = min(a.group, kHeads);
  const Range rg = range_of<UT>(uniform(a.lengths[b]), cap, a.window);
  uint16_t *out = a.out + ((int64_t)b * a.hq + qh) * D;
  if (rg.units == 0) {
    if (threadIdx.x < D / 2) reinterpret_cast<uint32_t *>(out)[threadIdx.x] = 0;
    if (a.lse != nullptr && threadIdx.x == 0) a.lse[(int64_t)b * a.hq + qh] = -INFINITY;
    return;
  }
  const int64_t total = (int64_t)units_before<UT>(a, cap, a.batch) * vheads;
  const int64_t chunk = (total + a.blocks - 1) / a.blocks;
  const int kvh = qh / a.group, hb = qh % a.group / kHeads, h = qh % a.group % kHeads;
  const int64_t p0 = (int64_t)units_before<UT>(a, cap, b) * vheads + (int64_t)(kvh * hblocks + hb) * rg.units;
  const int64_t w0 = p0 / chunk, w1 = (p0 + rg.units - 1) / chunk;
  if (w0 == w1) return;                        // written by its work-group
  const int pg = threadIdx.x / LN, d0 = 4 * (threadIdx.x % LN);
  float m = -INFINITY, l = 0.0f;
  v4f o = {0, 0, 0, 0};
  for (int64_t w = w0 + pg; w <= w1; w += PG) {
    const float *slot = a.scratch + (2 * w + (w * chunk >= p0 ? 0 : 1)) * partial_floats(D, cols);
    const f2 ml = *reinterpret_cast<const f2 *>(slot + 2 * h);
    const v4f y = *reinterpret_cast<const v4f *>(slot + partial_head(cols) + h * D + d0);
    const float m1 = fmaxf(m, ml.x), ref = m1 == -INFINITY ? 0.0f : m1;
    const float f0 = __builtin_amdgcn_exp2f(m - ref), f1 = __builtin_amdgcn_exp2f(ml.x - ref);
    m = m1;
    l = l * f0 + ml.y * f1;
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = o[i] * f0 + y[i] * f1;
  }
  *reinterpret_cast<v4f *>(&lds_o[pg][d0]) = o;
  if (d0 == 0) {
    lds_m[pg] = m;
    lds_l[pg] = l;
  }
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  const int e = 2 * threadIdx.x;
  float mm = lds_m[0];
#pragma unroll
  for (int i = 1; i < PG; i++) mm = fmaxf(mm, lds_m[i]);
  const float ref = mm == -INFINITY ? 0.0f : mm;
  float ll = 0.0f, y0 = 0.0f, y1 = 0.0f;
#pragma unroll
  for (int i = 0; i < PG; i++) {
    const float f = __builtin_amdgcn_exp2f(lds_m[i] - ref);
    ll = fmaf(f, lds_l[i], ll);
    y0 = fmaf(f, lds_o[i][e], y0);
    y1 = fmaf(f, lds_o[i][e + 1], y1);
  }
  const float inv = 1.0f / ll;
  *reinterpret_cast<uint32_t *>(out + e) = pack2<BF16>(y0 * inv, y1 * inv);
  if (a.lse != nullptr && e == 0) a.lse[(int64_t)b * a.hq + qh] = (mm + log2f(ll)) * (1.0f / kLog2e);
}

template <int D, int BITS, bool BF16>
void go(const AttendArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((attend_kernel<D, BITS, BF16>), dim3(a.blocks), dim3(64 * kWaves), 0, s, a);
  hipLaunchKernelGGL((join_kernel<D, BITS, BF16>), dim3(a.hq, a.batch), dim3(256), 0, s, a);
}
template <int D>
void go_bits(const AttendArgs &a, bool bf16, hipStream_t s) {
  if (a.c.bits == 16) bf16 ? go<D, 16, true>(a, s) : go<D, 16, false>(a, s);
  else if (a.c.bits == 8) bf16 ? go<D, 8, true>(a, s) : go<D, 8, false>(a, s);
  else bf16 ? go<D, 4, true>(a, s) : go<D, 4, false>(a, s);
}

}  // namespace

int attend_blocks(const KvCache &c, int batch, int hq, int64_t max_len) {
  const int group = hq / c.heads, ut = unit_tokens(c.bits);
  // (one unit more: a window may start within a tile)
  const int64_t units = (max_len + 15 + ut - 1) / ut * batch * c.heads * ((group + kHeads - 1) / kHeads);
  const int64_t most = 256 * 3;
  return (int)(units < most ? units : most);
}

size_t attend_scratch_bytes(const KvCache &c, int batch, int hq, int64_t max_len) {
  const int group = hq / c.heads;
  return (size_t)attend_blocks(c, batch, hq, max_len) * 2 * partial_floats(c.d, group < kHeads ? group : kHeads) * 4;
}

hipError_t launch_attend(const AttendArgs &a, bool bf16, hipStream_t s) {
  if (a.c.d == 64) go_bits<64>(a, bf16, s);
  else if (a.c.d == 128) go_bits<128>(a, bf16, s);
  else go_bits<256>(a, bf16, s);
  return hipGetLastError();
}

}  // namespace tq
