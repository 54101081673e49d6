// Attention over shared prompts (wf_prefix_attn): what its kernels share.
#pragma once

#include "wf_div.cuh"
#include "wf_internal.cuh"

namespace wf {

// One call.  A prompt unit is one (prompt, key head): its R = each G q query
// rows are those of all its sequences, row r belonging to sequence
// r / (G q) of the prompt, head (r / q) % G of the group and row r % q of the
// block.  An own unit is one (sequence, key head) with its G q rows.  A part is
// what one CTA finds for its rows over a range of their keys: the row's maximum
// m (log2 units) and sum l of 2^(s - m), and the unnormalised O; parts [0, S)
// are ranges of the prompt, the rest of the own rows.
struct PrefixArgs {
  const void* Q;
  int64_t qsb, qsh, qss;
  const void* K;
  const void* V;
  const uint8_t* Ks;
  const uint8_t* Vs;
  int64_t ksb, ksh, kss;  // elements (fp32, bf16) or bytes (codes)
  const void* Kg;
  const void* Vg;
  int64_t gsb, gsh, gss;
  void* O;
  int64_t osb, osh, oss;
  const int32_t* idx;
  const int32_t* plen;
  const int32_t* glen;
  int B, P, H, G, q, d, n, k, ng;
  int each;       // sequences a prompt
  int R, Ro;      // query rows of a prompt unit, of an own unit
  FastDiv by_q, by_Ro, by_H, by_S, by_So, by_mt, by_mto;
  int S, So;      // parts of the prompt, of the own rows
  int mt, mto;    // row tiles of a prompt unit, of an own unit
  int ob;         // query rows a CTA where the own rows are folded in
  int direct;     // the prompt's rows are attended there too (S = 0)
  int whole;      // a part is the whole softmax: O goes out as it is
  int64_t rows;   // B Hq q
  float* part_o;  // [parts][rows][d], rows in [B, Hq, q] order
  float2* part_ml;
  float sl2;      // scale log2(e)
  int* status;
  long long wait_limit;  // bound of the tensor-core kernel's waits (cycles)
  int stall;             // test-only: its first wait is on a barrier that nothing completes
};

// With at least so many units of own rows, and not too many rows for them, they are
// attended where the parts are joined; else they are units of the prompt's kernel, where
// few of them fit beside the prompt's.  Measured in us, joined against units: 16
// tokens' units of 100 rows 14.5, 11.5; 64 of 65 rows 21.0, 22.6, of 300 rows 34, 25;
// 64 of 32 query rows and 32 own rows 14.4, 19.1; 128 of those 32.7, 39.9; 1024
// tokens' units of 100 rows 47, 72, of 500 rows 81, 91, of 1000 rows 123, 120; 512
// units of 32 query rows and 300 own rows 103, 95.
constexpr int kPrefixOwn = 64;
// SMs of the machine that the estimates of plan_prefix and prefix_own_rows are
// of, with their times a tile; a call's split and size follow from its shapes alone.
constexpr int kPrefixSms = 152;
constexpr int kPrefixTcRows = 256;  // query rows a CTA of the tensor-core kernel

// The workspace of a call: the status word, then the parts.
struct PrefixPlan {
  PrefixArgs a;  // shapes and splits; pointers are filled in by the call
  int dtype, fmt;
  int tr, tk;    // query rows a CTA, keys a tile
  int parts;     // 1: the kernel writes O itself
  bool fold;     // the own rows are attended where the parts are joined (So = 0)
  size_t off_ml, off_o, used;  // used: what this call writes
  size_t total;                // what it asks for
};
PrefixPlan plan_prefix(const wf_tensor& q, const wf_tensor& kv, int k, int n_g);
cudaError_t launch_prefix(const PrefixPlan& p, cudaStream_t s);
// Query rows a CTA of that kernel for S parts and so many keys.
int prefix_own_rows(const PrefixArgs& a, int S, int keys);
cudaError_t launch_prefix_own(const PrefixPlan& p, cudaStream_t s);  // own rows and the joining of parts, bf16
cudaError_t launch_prefix_tc(const PrefixPlan& p, cudaStream_t s);  // the parts (or O) of bf16 queries

// Sequence, query head and block row of row r of the unit of prompt p (or of
// sequence b) and key head h.
struct RowAt {
  int b, hq, i;
};
__device__ __forceinline__ RowAt prompt_row(const PrefixArgs& a, int p, int h, int r) {
  const int s = fastdiv(r, a.by_Ro), w = r - s * a.Ro, g = fastdiv(w, a.by_q);
  return {p * a.each + s, h * a.G + g, w - g * a.q};
}
__device__ __forceinline__ RowAt own_row(const PrefixArgs& a, int b, int h, int r) {
  const int g = fastdiv(r, a.by_q);
  return {b, h * a.G + g, r - g * a.q};
}
__device__ __forceinline__ int64_t flat_row(const PrefixArgs& a, const RowAt& r) {
  return ((int64_t)r.b * (a.H * a.G) + r.hq) * a.q + r.i;
}
// Rows that count of prompt p, of sequence b.
__device__ __forceinline__ int prompt_count(const PrefixArgs& a, int p) {
  return a.plen ? min(a.k, max(0, __ldg(a.plen + p))) : a.k;
}
__device__ __forceinline__ int own_count(const PrefixArgs& a, int b) {
  return a.glen ? min(a.ng, max(0, __ldg(a.glen + b))) : a.ng;
}

}  // namespace wf
