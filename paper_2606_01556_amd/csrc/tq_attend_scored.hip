// Attention of one new token per stream with capped or biased scores, or with its parts as
// the result: the kernels.  (32 streams up to 8192 tokens, 8 bits, pages of 64, a cap: 56.7 us, 53.6
// of them this launch's, for 295 MB.  With 16-bit rows of 128 or 256 they spill 2 to 24 registers, rows of
// codes none or one.)
#include "tq_attend.hpp"

namespace tq {

hipError_t launch_attend_scored(const AttendArgs &a, bool bf16, hipStream_t s) { return go_heads<true>(a, bf16, s); }

}  // namespace tq
