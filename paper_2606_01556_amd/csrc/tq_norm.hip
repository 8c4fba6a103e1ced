// Between two blocks of a decoder: the norm after a block, its gate and scale, the residual sum
// and the norm before the next block, for rows x and r of n values:
//
//   z = x / sqrt(mean(x^2) + eps) * w1 * g,   s = r + scale z,   y = s / sqrt(mean(s^2) + eps) * w2
//
// (each of w1, g, r and w2 may be left out).  Bound by the bytes of x, r and the gate in and of s
// and y out, so a row is read once and stays in registers, in fp32, through both of its sums;
// y is made of s before that is rounded.
//
// A row of up to 512 values is a wavefront's, of up to 4096 256 threads', of up to 8192 512
// threads', past that 1024 threads': the more of a row a thread holds, the fewer rows a CU has
// under way (8192 rows of 8192 bf16 values, both norms and a gate of each: 128 us with 256
// threads, 121 with 512 or 1024, 153 with 128; one row of 4096: 5.3 us whichever, the host's time,
// 2.8 of them the kernel).  What is read and written at 6.5 TB/s would take 103 us.  Reading the
// weights before the sums instead of after them: 2 us more.
#include "tq_attention.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

// Sums past these are formed again of scaled values: the largest values' squares pass fp32's
// range, the smallest ones' vanish.  (Down: 32768 values of 2^128 sum up to 2^(2 (128 - 80) + 15)
// = 2^111; a row whose sum passed 2^126 has a mean of 2^(111 - 160) or more.  Up: a sum below
// 2^(15 - 100) ends below 2^115, and fp32's smallest value at 2^(2 (100 - 149)) = 2^-98.)
constexpr float kMost = 0x1p126f, kLeast = 0x1p-100f, kDown = 0x1p-80f, kUp = 0x1p100f;

template <bool BF16>
__device__ __forceinline__ void unpack8(u32x4 w, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    f[2 * i] = BF16 ? __builtin_bit_cast(float, w[i] << 16) : half_bits_to_float((uint16_t)w[i]);
    f[2 * i + 1] = BF16 ? __builtin_bit_cast(float, w[i] & 0xffff0000u) : half_bits_to_float((uint16_t)(w[i] >> 16));
  }
}
template <bool BF16>
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  return u32x4{pack2<BF16>(f[0], f[1]), pack2<BF16>(f[2], f[3]), pack2<BF16>(f[4], f[5]), pack2<BF16>(f[6], f[7])};
}

// Rows are read once: non-temporal (8192 rows of 8192, with a gate of each: 121 -> 117 us).
__device__ __forceinline__ u32x4 read_once(const uint16_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }

// T threads own a row, C pieces of eight values each: T * C * 8 >= n
template <int T, int C, bool BF16>
__global__ __launch_bounds__(T < 256 ? 256 : T) void norm_kernel(const NormArgs a) {
  constexpr int ROWS = T < 256 ? 256 / T : 1, W = T / 64;
  __shared__ float lds[2][ROWS * W + 1];
  const int t = threadIdx.x % T;
  const int64_t row = (int64_t)blockIdx.x * ROWS + threadIdx.x / T;
  const bool live = row < a.tokens;
  const int pieces = a.n / 8;
  int turn = 0;

  // the sum of v over a row's threads, in one order
  auto row_sum = [&](float v) -> float {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m);
    if constexpr (W > 1) {
      const int w = threadIdx.x / 64;
      if ((threadIdx.x & 63) == 0) lds[turn][w] = v;
      __syncthreads();
      v = 0.0f;
#pragma unroll
      for (int i = 0; i < W; i++) v += lds[turn][i];
      turn ^= 1;
    }
    return v;
  };
  auto squares = [&](const float (&f)[C][8], float by) -> float {
    float v = 0.0f;
#pragma unroll
    for (int c = 0; c < C; c++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float x = f[c][i] * by;
        v = fmaf(x, x, v);
      }
    return row_sum(v);
  };
  // 1 / sqrt(mean(f^2) + eps) as up * inv: of a row of small values it may pass fp32's range
  struct Inverse {
    float up, inv;
  };
  const float inv_n = 1.0f / (float)a.n;
  auto inverse = [&](const float (&f)[C][8]) -> Inverse {
    float sum = squares(f, 1.0f), by = 1.0f, up = 1.0f, eps = a.eps;
    const bool again = !(sum <= kMost) || fmaf(sum, inv_n, eps) < kLeast;
    // (the threads of a row agree; where a row is a wavefront's, wavefronts need not)
    if (again) {
      by = sum < 1.0f ? kUp : kDown;
      sum = squares(f, by);
      eps = eps * by * by;       // (by * by may vanish, or pass the range)
      if (by > 1.0f) {
        up = by;
        by = 1.0f;
      }
    }
    return {up, by / sqrtf(fmaf(sum, inv_n, eps))};
  };

  float x[C][8], s[C][8], gate[C][8];
#pragma unroll
  for (int c = 0; c < C; c++) {
    const int p = c * T + t;
    const bool in = live && p < pieces;
    const u32x4 zero = {0, 0, 0, 0};
    unpack8<BF16>(in ? read_once(a.x + row * a.x_stride + 8 * p) : zero, x[c]);
    unpack8<BF16>(in && a.residual != nullptr ? read_once(a.residual + row * a.r_stride + 8 * p) : zero, s[c]);
    if (a.gate != nullptr) {
      const uint16_t *const g = a.gate + row * a.g_stride + 8 * p;
      unpack8<BF16>(!in ? zero : a.g_stride == 0 ? *reinterpret_cast<const u32x4 *>(g) : read_once(g), gate[c]);
    }
  }
  if (a.post != nullptr) {
    const Inverse i1 = inverse(x);
#pragma unroll
    for (int c = 0; c < C; c++) {
      const int p = c * T + t;
      float w[8];
      unpack8<BF16>(*reinterpret_cast<const u32x4 *>(a.post + 8 * min(p, pieces - 1)), w);
#pragma unroll
      for (int i = 0; i < 8; i++) x[c][i] = x[c][i] * i1.up * i1.inv * w[i];
    }
  }
#pragma unroll
  for (int c = 0; c < C; c++)
#pragma unroll
    for (int i = 0; i < 8; i++) s[c][i] = fmaf(a.scale, a.gate != nullptr ? x[c][i] * gate[c][i] : x[c][i], s[c][i]);
  if (a.sum != nullptr) {
#pragma unroll
    for (int c = 0; c < C; c++) {
      const int p = c * T + t;
      if (live && p < pieces) *reinterpret_cast<u32x4 *>(a.sum + row * a.n + 8 * p) = pack8<BF16>(s[c]);
    }
  }
  if (a.normed == nullptr) return;
  // (pieces past the row: x, s and the gate are zero there, but a weight or inverse may be NaN)
#pragma unroll
  for (int c = 0; c < C; c++)
    if (c * T + t >= pieces)
#pragma unroll
      for (int i = 0; i < 8; i++) s[c][i] = 0.0f;
  const Inverse i2 = inverse(s);
#pragma unroll
  for (int c = 0; c < C; c++) {
    const int p = c * T + t;
    if (live && p < pieces) {
      float w[8];
      unpack8<BF16>(*reinterpret_cast<const u32x4 *>(a.weight + 8 * p), w);
#pragma unroll
      for (int i = 0; i < 8; i++) w[i] = s[c][i] * i2.up * i2.inv * w[i];
      *reinterpret_cast<u32x4 *>(a.normed + row * a.n + 8 * p) = pack8<BF16>(w);
    }
  }
}

template <int T, int C>
hipError_t go_norm(const NormArgs &a, bool bf16, hipStream_t s) {
  constexpr int ROWS = T < 256 ? 256 / T : 1;
  const dim3 grid((uint32_t)((a.tokens + ROWS - 1) / ROWS)), block(T < 256 ? 256 : T);
  if (bf16) hipLaunchKernelGGL((norm_kernel<T, C, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_kernel<T, C, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, bool bf16, hipStream_t s) {
  const int pieces = a.n / 8;
  if (pieces <= 64) return go_norm<64, 1>(a, bf16, s);
  if (pieces <= 128) return go_norm<64, 2>(a, bf16, s);
  if (pieces <= 256) return go_norm<256, 1>(a, bf16, s);
  if (pieces <= 512) return go_norm<256, 2>(a, bf16, s);
  if (pieces <= 1024) return go_norm<512, 2>(a, bf16, s);
  if (pieces <= 2048) return go_norm<1024, 2>(a, bf16, s);
  return go_norm<1024, 4>(a, bf16, s);
}

}  // namespace tq
