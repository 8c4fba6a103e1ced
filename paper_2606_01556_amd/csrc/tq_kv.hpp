// Arguments and launch interface of the kernels between a block's linear
// layers: norm and rotation of queries and keys, the paged key-value cache, and
// the attention of one new token over it (internal to libtq).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tq {

// A paged cache: rows [pages][heads][2^lps][d] of 16-bit values (bits 16), e4m3
// codes (8) or TQ4 words (4), scales [pages][heads][2^lps] fp16 (8 and 4).
struct KvCache {
  uint8_t *k, *v;
  uint16_t *ks, *vs;
  int pages, lps, heads, d, bits;
};

// [tokens][heads][d] of 16-bit values; strides in values.
struct HeadRows {
  const uint16_t *p;
  int64_t ts, hs;
};

struct TokenArgs {
  HeadRows q, k, v;          // v.p may be null (no v rows)
  int tokens, hq, hkv;       // hq 0: k and v rows only
  uint16_t *q_out, *k_out;   // [tokens][hq][d], [tokens][hkv][d]; k_out may be null
  // norm and rotation of q and k rows
  const uint16_t *qw, *kw;   // [d] or null
  float eps;
  const int32_t *positions;
  const float *table;        // [max_pos][rot]: rot / 2 cosines, then as many sines
  int rot, max_pos, interleaved;
  // the cache that takes k and v rows; slots null: none
  KvCache c;
  const int64_t *slots;
  // rows per token and its division: row / rows_per_token = mulhi(row, magic) >> shift
  int rows_per_token;
  uint32_t magic;
  int shift;
};

struct ReadArgs {
  KvCache c;
  const int64_t *slots;
  int tokens;
  uint16_t *k_out, *v_out;   // [tokens][heads][d]
  uint32_t magic;
  int shift;
};

struct AttendArgs {
  KvCache c;
  const uint16_t *q;         // [batch][hq][d]
  int64_t q_ts, q_hs;
  int batch, hq, group;      // group = hq / c.heads
  const int32_t *table;      // [batch][table_stride] page numbers
  int64_t table_stride;
  int max_pages;
  const int32_t *lengths;
  float scale;
  int window;                // 0: none
  uint16_t *out;             // [batch][hq][d]
  float *lse;                // [batch][hq] or null
  float *scratch;
  int blocks;                // work-groups
  int direct;
};

hipError_t launch_tokens(const TokenArgs &a, bool bf16, hipStream_t s);
hipError_t launch_kv_read(const ReadArgs &a, bool bf16, hipStream_t s);
// How an attention call is cut, by what the host knows of it: direct, one
// work-group per (stream, head) range and no scratch, or runs of all ranges.
struct AttendPlan {
  bool direct;
  int blocks;
  int64_t steps;           // upper bound of all ranges' steps
  size_t scratch;          // bytes
};
AttendPlan attend_plan(const KvCache &c, int batch, int hq, int64_t max_len, int window);
hipError_t launch_attend(const AttendArgs &a, bool bf16, hipStream_t s);

// row / d for 0 <= row < 2^31 and 2 <= d < 2^31: with L = ceil(log2 d) and
// magic = ceil(2^(31 + L) / d) <= 2^32 - 1 (2^31 where d is a power of two), the
// excess magic * d - 2^(31 + L) < d <= 2^L times row stays below 2^(31 + L).
inline void divide_by(uint32_t d, uint32_t &magic, int &shift) {
  int L = 1;
  while ((1ull << L) < d) L++;
  magic = (uint32_t)(((1ull << (31 + L)) + d - 1) / d);
  shift = L - 1;
}

}  // namespace tq
