// Rows on their way from a projection to queries or into a cache: positions
// rotated in (wf_rotary_apply), rows written into pages (wf_paged_append).
#pragma once

#include "wf_div.cuh"
#include "wf_internal.cuh"

namespace wf {

// Pair i of a rotation plan: 2^64 f_i / (2 pi) mod 2^64, the turns of one
// position as a fraction of 2^64, and the axis whose position it takes.
struct RotaryPair {
  unsigned long long turn;
  long long axis;
};

// One call.  Tensor 0 is rotated (queries; new keys), tensor 1 is too where
// `both` (keys), else it goes through as it is (new values).
struct RowsArgs {
  const void* src[2];
  void* dst[2];
  uint8_t* scales[2];
  int64_t ssb[2], ssh[2], sss[2];  // elements
  int64_t dsb[2], dsh[2], dss[2];  // elements, or bytes of codes; dsb: batch entry or page
  int heads[2];
  int both;
  const RotaryPair* plan;          // null: no rotation
  int pairs, adjacent;
  const int32_t* pos;              // [axes][B][rows], or null: the place in the sequence
  int axes, B, rows;
  // Rows that go into pages.
  const int32_t* pages;            // [B][table], or null: row i to row i
  const int32_t* start;
  const int32_t* rows_at;          // [B][m] source rows, or null: the first m
  const int32_t* count;            // [B] of the m rows that go in, or null: all
  int table, pool;
  FastDiv by_ps;
  FastDiv by_m;                    // rows a batch entry
  uint32_t total;                  // B m
  int each, groups;                // heads a thread, groups of so many
  FastDiv by_groups;
};

cudaError_t launch_rotate(RowsArgs a, int dtype, int d, cudaStream_t s);
cudaError_t launch_append(RowsArgs a, int dtype, int cache, int d, cudaStream_t s);

}  // namespace wf
