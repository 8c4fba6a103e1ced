// Attention of one new token of every stream over a prefix that a group of streams shares and
// over the stream's own tokens:
//
//   o = sum over the prefix's and the stream's keys of softmax(s) v
//
// The prefix's keys and values are read once for all of a group's streams (and not once a
// stream): its streams are the rows of the attention of many tokens, which splits the prefix
// over work-groups; a stream's own tokens are read by the attention of one token.  Both leave
// parts (a reference, a sum, unscaled products), and this file's join adds those of a row.
// Three launches, whatever the sizes.
#include "tq_attend.hpp"

namespace tq {

namespace {

// D / 4 lanes hold a row's products, `side` groups of them take its parts in turn (the
// prefix's, then its own) and are joined in their order, so that every sum has one order.
template <int D, bool BF16>
__global__ __launch_bounds__(kJoinThreads) void join_prefix_kernel(const PrefixArgs a, int side) {
  constexpr int Q = D / 4, GROUPS = kJoinThreads / Q;
  __shared__ __attribute__((aligned(16))) float lds_o[GROUPS][D], lds_ml[GROUPS][2];
  const PromptArgs &p = a.prefix;
  const AttendArgs &t = a.own;
  const int g = threadIdx.x / Q, d0 = 4 * (threadIdx.x % Q), mine = g % side;
  const int64_t heads = (int64_t)p.tokens * p.hq, row = (int64_t)blockIdx.x * (GROUPS / side) + g / side;
  const bool live = row < heads;
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
    const int stream = (int)(row / p.hq), h = (int)(row - (int64_t)stream * p.hq);
    const int begin = min(max(p.starts[0], 0), p.tokens), end = min(max(p.starts[p.batch], 0), p.tokens);
    const int shared = stream >= begin && stream < end ? p.splits : 0;
    // the row's own parts: of its kv head's range, its place among the range's heads
    const int hr = kHeads * head_blocks(t.group), cols = min(t.group, hr), ranges = (t.group + hr - 1) / hr;
    const int kvh = h / t.group, in = h - kvh * t.group, place = in % hr;
    const int64_t all = (int64_t)t.batch * p.c.heads * ranges;
    const Join j = reinterpret_cast<const Join *>(t.scratch + (run_slots(t.blocks, t.direct) + all) * part_floats(D, cols))[
        ((int64_t)stream * p.c.heads + kvh) * ranges + in / hr];
    const float *const parts = p.scratch + parts_head(p.splits, heads);
#pragma unroll 4
    for (int k = mine; k < shared; k += side) {
      const f2 ml = *reinterpret_cast<const f2 *>(p.scratch + 2 * (k * heads + row));
      if (ml.y != 0.0f) add(ml, *reinterpret_cast<const v4f *>(parts + (k * heads + row) * D + d0));
    }
#pragma unroll 2
    for (int k = mine; k < j.parts; k += side) {
      const int slot = k == 0 ? j.first : (j.first & ~1) + 2 * k;
      const float *part = t.scratch + (int64_t)slot * part_floats(D, cols);
      add(*reinterpret_cast<const f2 *>(part + 2 * place), *reinterpret_cast<const v4f *>(part + part_head(cols) + place * D + d0));
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
  *reinterpret_cast<u32x2 *>(p.out + row * D + d0) = u32x2{pack2<BF16>(y[0], y[1]), pack2<BF16>(y[2], y[3])};
  if (p.lse != nullptr && d0 == 0) p.lse[row] = none ? -INFINITY : log_sum(m, l);
}

template <int D>
hipError_t join_prefix(const PrefixArgs &a, bool bf16, hipStream_t s) {
  constexpr int GROUPS = kJoinThreads / (D / 4);
  int side = 1;
  while (side < a.prefix.splits && side < GROUPS) side *= 2;
  const int64_t heads = (int64_t)a.prefix.tokens * a.prefix.hq, each = GROUPS / side;
  const dim3 grid((uint32_t)((heads + each - 1) / each));
  if (bf16) hipLaunchKernelGGL((join_prefix_kernel<D, true>), grid, dim3(kJoinThreads), 0, s, a, side);
  else hipLaunchKernelGGL((join_prefix_kernel<D, false>), grid, dim3(kJoinThreads), 0, s, a, side);
  return hipGetLastError();
}

}  // namespace

size_t attend_parts_bytes(const KvCache &c, int batch, int hq, const AttendPlan &p) {
  const int group = hq / c.heads;
  const int64_t ranges = (int64_t)batch * c.heads * ranges_of(group);
  return (size_t)(run_slots(p.blocks, p.direct) + ranges) * part_floats(c.d, range_heads(group)) * sizeof(float) + (size_t)ranges * sizeof(Join);
}

hipError_t launch_prefix(const PrefixArgs &a, bool bf16, hipStream_t s) {
  hipError_t e = launch_prompt(a.prefix, bf16, s);
  if (e != hipSuccess) return e;
  e = launch_attend_scored(a.own, bf16, s);
  if (e != hipSuccess) return e;
  return a.own.c.d == 64 ? join_prefix<64>(a, bf16, s) : a.own.c.d == 128 ? join_prefix<128>(a, bf16, s) : join_prefix<256>(a, bf16, s);
}

}  // namespace tq
