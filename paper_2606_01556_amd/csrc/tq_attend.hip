// Attention of one new token per stream: how a call is cut, and the plain kernels.
#include "tq_attend.hpp"

namespace tq {

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
  return a.cap > 0.0f || a.slopes != nullptr || a.parts ? launch_attend_scored(a, bf16, s) : go_heads<false>(a, bf16, s);
}

}  // namespace tq
