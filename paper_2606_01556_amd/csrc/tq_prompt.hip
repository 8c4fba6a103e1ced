// Attention of many tokens: how a call is cut, and the join of the parts of rows whose keys
// several work-groups share.
#include "tq_attention.hpp"
#include "tq_kernels.hpp"
#include "tq_kv.hpp"

namespace tq {

namespace {

constexpr int kJoinThreads = 256, kCus = 256;

// A row's parts, joined: D / 4 lanes hold a row's products, `side` groups of them take its
// parts in turn and are joined in their order, so that every sum has one order.
template <int D, bool BF16>
__global__ __launch_bounds__(kJoinThreads) void join_rows_kernel(const PromptArgs a, int side) {
  constexpr int Q = D / 4, GROUPS = kJoinThreads / Q;
  __shared__ __attribute__((aligned(16))) float lds_o[GROUPS][D], lds_ml[GROUPS][2];
  const int g = threadIdx.x / Q, d0 = 4 * (threadIdx.x % Q), mine = g % side;
  const int64_t heads = (int64_t)a.tokens * a.hq, row = (int64_t)blockIdx.x * (GROUPS / side) + g / side;
  const int begin = min(max(a.starts[0], 0), a.tokens), end = min(max(a.starts[a.batch], 0), a.tokens);
  const bool live = row >= (int64_t)begin * a.hq && row < (int64_t)end * a.hq;     // (the others are cleared)
  float m = -INFINITY, l = 0.0f;
  v4f o = {0, 0, 0, 0};
  auto add = [&](f2 ml, v4f y) {
    const float m1 = fmaxf(m, ml.x);            // (of a part: finite)
    const float f0 = __builtin_amdgcn_exp2f(m - m1), f1 = __builtin_amdgcn_exp2f(ml.x - m1);
    m = m1;
    l = l * f0 + ml.y * f1;
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = o[i] * f0 + y[i] * f1;
  };
  if (live) {
    const float *const parts = a.scratch + parts_head(a.splits, heads);
#pragma unroll 4
    for (int k = mine; k < a.splits; k += side) {
      const f2 ml = *reinterpret_cast<const f2 *>(a.scratch + 2 * (k * heads + row));
      if (ml.y != 0.0f) add(ml, *reinterpret_cast<const v4f *>(parts + (k * heads + row) * D + d0));
    }
    *reinterpret_cast<v4f *>(&lds_o[g][d0]) = o;
    if (d0 == 0) *reinterpret_cast<f2 *>(lds_ml[g]) = f2{m, l};
  }
  __syncthreads();
  if (!live || mine != 0) return;
  for (int k = 1; k < side; k++) {
    const f2 ml = *reinterpret_cast<const f2 *>(lds_ml[g + k]);
    if (ml.y != 0.0f) add(ml, *reinterpret_cast<const v4f *>(&lds_o[g + k][d0]));      // (it had parts)
  }
  const bool none = l == 0.0f;
  const float inv = 1.0f / l;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; i++) y[i] = none ? 0.0f : o[i] * inv;
  *reinterpret_cast<u32x2 *>(a.out + row * D + d0) = u32x2{pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3])};
  if (a.lse != nullptr && d0 == 0) a.lse[row] = none ? -INFINITY : log_sum(m, l);
}

template <int D>
hipError_t join_rows(const PromptArgs &a, bool bf16, hipStream_t s) {
  constexpr int GROUPS = kJoinThreads / (D / 4);
  int side = 1;
  while (side < a.splits && side < GROUPS) side *= 2;
  const int64_t heads = (int64_t)a.tokens * a.hq, each = GROUPS / side;
  const dim3 grid((uint32_t)((heads + each - 1) / each));
  if (bf16) hipLaunchKernelGGL((join_rows_kernel<D, true>), grid, dim3(kJoinThreads), 0, s, a, side);
  else hipLaunchKernelGGL((join_rows_kernel<D, false>), grid, dim3(kJoinThreads), 0, s, a, side);
  return hipGetLastError();
}

}  // namespace

PromptPlan prompt_plan(const KvCache &c, int tokens, int batch, int hq, int64_t max_len, int window, bool shared) {
  PromptPlan p;
  const int64_t tiles = (int64_t)tokens * (hq / c.heads) / kPromptRows + batch;
  const int64_t units = tiles * c.heads;
  // Where the row tiles leave half of the CUs without work, a tile's keys are split, down to 256 of
  // them.  How many parts a tile has is for the kernel to say, which knows the lengths: of several
  // streams up to twice as many as would fill the CUs if all were alike.  (16 streams up to 8192
  // with 5 new tokens each: 75 us with as many parts of each, 71.5 with a share of the whole each.
  // One group of 64 streams behind 16384: 80 us with 32 parts, 84.5 with room for 64.)
  p.room = kCus * (c.d == 256 ? 1 : c.d == 128 || c.bits < 16 ? 2 : 3);
  const int64_t longest = window > 0 && (int64_t)window + tokens < max_len ? (int64_t)window + tokens : max_len;
  const int64_t rows = ((int64_t)tokens * (hq / c.heads) + kPromptRows - 1) / kPromptRows, real = (rows > batch ? rows : batch) * c.heads;
  int64_t splits = real > 0 && 2 * real <= p.room ? ((batch > 1 ? 2 : 1) * p.room + real - 1) / real : 1;
  if (splits > (longest + 255) / 256) splits = (longest + 255) / 256;
  if (splits < 1) splits = 1;
  p.longest = (int)longest;
  p.tiles = (int)(tiles < INT32_MAX ? tiles : INT32_MAX);
  p.splits = (int)splits;
  p.blocks = units * splits;
  p.scratch = splits > 1 || shared ? (size_t)(parts_head(p.splits, (int64_t)tokens * hq) + splits * tokens * hq * c.d) * sizeof(float) : 0;
  return p;
}

hipError_t launch_prompt(const PromptArgs &a, bool bf16, hipStream_t s) {
  const hipError_t e = a.c.d == 64 ? launch_prompt_64(a, bf16, s) : a.c.d == 128 ? launch_prompt_128(a, bf16, s) : launch_prompt_256(a, bf16, s);
  if (e != hipSuccess || a.splits == 1 || a.shared) return e;
  return a.c.d == 64 ? join_rows<64>(a, bf16, s) : a.c.d == 128 ? join_rows<128>(a, bf16, s) : join_rows<256>(a, bf16, s);
}

}  // namespace tq
