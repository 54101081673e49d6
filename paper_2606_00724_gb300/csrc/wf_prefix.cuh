// Attention over shared prompts (wf_prefix_attn) and over pages (wf_tree_attn): what
// their kernels share.
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
  // A cache in pages (wf_tree_attn; else null): row j of a sequence is row j % ps
  // of page pages[b][j / ps], and ksb is the stride between pages.
  const int32_t* pages;
  int table, pool;       // entries a sequence, pages of the pool
  FastDiv by_ps;
  int64_t kx;            // ksb - ps kss: what a page adds to the rows before it
  // The drafted rows that a query row sees (null: all): bit j of mask[b][i].
  const uint32_t* mask;
  int mw;                // words a row
  // bf16 queries over pages: the key tiles (tk keys each) that the sequences really have
  // are spread over C CTAs evenly (see Walk), a unit's rows in mt tiles of tr.  A
  // part is a slot of tr rows; info says where an item's are and how many, flags
  // which of them left drafted values out that are not finite.
  int C, tk, tr, pad;
  int box;               // rows of the pieces of pages that the copy engine brings; 0: not by it
  int2* info;
  int* flags;
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
  bool few;      // wf_tree_attn's kernel for few query rows a unit
  bool join;     // an item may have several parts
  size_t off_info, off_ml, off_o, used;  // used: what this call writes
  size_t total;                // what it asks for
};
PrefixPlan plan_prefix(const wf_tensor& q, const wf_tensor& kv, int k, int n_g);
cudaError_t launch_prefix(const PrefixPlan& p, cudaStream_t s);
// The same for wf_tree_attn: k rows a sequence and n_t drafted ones.
PrefixPlan plan_tree(const wf_tensor& q, const wf_tensor& kv, int k, int n_t);
cudaError_t launch_tree(const PrefixPlan& p, cudaStream_t s);
// Query rows a CTA of that kernel for S parts and so many keys.
int prefix_own_rows(const PrefixArgs& a, int S, int keys);
cudaError_t launch_prefix_own(const PrefixPlan& p, cudaStream_t s);  // own rows and the joining of parts, bf16
cudaError_t launch_prefix_tc(const PrefixPlan& p, cudaStream_t s);  // the parts (or O) of bf16 queries
// The same of wf_tree_attn: of more query rows a unit, of few, and their joining.
cudaError_t launch_tree_tc(const PrefixPlan& p, cudaStream_t s);
cudaError_t launch_tree_few(const PrefixPlan& p, cudaStream_t s);
cudaError_t launch_tree_join(const PrefixPlan& p, cudaStream_t s);
// Empty places before an item (see Walk), in tiles of either kernel.  256 rows of 32 units on 32K: none 132 us,
// two 127, four 125, six 124, eight 125.  Few rows: one token of 8 sequences of 2K none 21.0, one 20.7, two 19.5, four
// 19.1; of one of 8K 17.2, 16.1, 14.6, 14.4; of 32 of 16K in 8 bits 363, 364, 366, 368.
constexpr int kFewPad = 1, kTreePad = 6;
// Query rows of a unit that the kernel for few of them takes.
constexpr int kFewRows = 16;
// Keys of its tiles: four warps' steps, of 16 rows, or of 32 rows of codes, whose
// bytes are fewer while a step's set-up is the same.
constexpr int few_keys(int fmt) { return fmt == WF_BF16 ? 64 : 128; }
// Its CTAs an SM: at head_dim 128 two, whose threads have the registers (three spilled: one token of 32
// sequences of 8K 195 against 186 us), at 64 three (109 against 117).
constexpr int few_per_sm(int d) { return d == 128 ? 2 : 3; }

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

// A row of a cache in pages: its number in the pool, and its page.
struct PagedRow {
  int flat, page;
};
// In two steps, so that what is loaded is not used before it has to be: the table's
// entry of row j, and the row itself.
__device__ __forceinline__ int page_entry(const PrefixArgs& a, int b, int j) {
  return __ldg(a.pages + (int64_t)b * a.table + fastdiv((uint32_t)j, a.by_ps));
}
__device__ __forceinline__ PagedRow paged_row(const PrefixArgs& a, int entry, int j) {
  const int page = min(max(entry, 0), a.pool - 1), in = j - (int)(fastdiv((uint32_t)j, a.by_ps) * a.by_ps.d);
  return {page * (int)a.by_ps.d + in, page};
}
__device__ __forceinline__ int64_t paged_offset(const PrefixArgs& a, const PagedRow& r) {
  return r.flat * a.kss + r.page * a.kx;
}
// Its row among the scales of key head h.
__device__ __forceinline__ int64_t paged_scale(const PrefixArgs& a, const PagedRow& r, int h) {
  return r.flat + ((int64_t)r.page * (a.H - 1) + h) * a.by_ps.d;
}
// Work over pages spread over C CTAs: the key tiles of all items, an item being a
// row tile of tr rows of a unit, lie in one line, items in the order [sequence][key
// head][row tile], an item's cached tiles before its drafted ones and one tile at
// least; CTA c takes tiles [c per, (c + 1) per), which are ranges of one item or of
// several that follow each other.  A range that begins inside a CTA's share costs it
// `pad` tiles' time more (rows in, first products, rows out), so the line has as many
// empty places before each item.  The lengths are known on the device alone, so every
// warp finds its place in the line from them.  A range is a part, and its slot is
// c + item: along the line either grows by one from range to range, so no two
// ranges share a slot and those of an item follow each other.
struct Walk {
  uint32_t per;               // places a CTA; all of them are below 2^31
  uint32_t x, end, first;     // next place, end of the CTA's; first place of sequence b
  int b, count, drafts;       // sequence, its cached and drafted rows
  int cached, tiles;          // tiles of an item of b: cached ones, all
  int item, t0, t1;           // the range: item of b, tiles [t0, t1)
  __device__ __forceinline__ void enter(const PrefixArgs& a, int sequence) {
    b = sequence;
    count = prompt_count(a, b);
    drafts = own_count(a, b);
    cached = (count + a.tk - 1) / a.tk;
    tiles = max(1, cached + (drafts + a.tk - 1) / a.tk);
  }
  // The places of the items of sequence b.
  __device__ __forceinline__ static uint32_t places_of(const PrefixArgs& a, int b) {
    if (b >= a.B) return 0;
    return (a.pad + max(1, (prompt_count(a, b) + a.tk - 1) / a.tk + (own_count(a, b) + a.tk - 1) / a.tk)) * a.H * a.mt;
  }
  // By a whole warp; false if the CTA has nothing to do.
  __device__ __forceinline__ bool start(const PrefixArgs& a) {
    const int lane = threadIdx.x & 31;
    const uint32_t here = places_of(a, lane);  // of the first 32 sequences, often all
    uint32_t mine = here;
    for (int s = lane + 32; s < a.B; s += 32) mine += places_of(a, s);
    const uint32_t total = __reduce_add_sync(0xffffffffu, mine);
    per = (total + a.C - 1) / a.C;
    x = blockIdx.x * per;
    end = min(x + per, total);
    if (x >= end) return false;
    first = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const uint32_t p = b0 ? places_of(a, b0 + lane) : here;
      uint32_t sum = p;
#pragma unroll
      for (int w = 1; w < 32; w *= 2) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, sum, w);
        if (lane >= w) sum += y;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, x < first + sum);
      if (past) {
        const int at = __ffs(past) - 1;
        first += __shfl_sync(0xffffffffu, sum - p, at);
        enter(a, b0 + at);
        return true;
      }
      first += __shfl_sync(0xffffffffu, sum, 31);
    }
    return false;
  }
  // To the next range; false behind the last.
  __device__ __forceinline__ bool next(const PrefixArgs& a) {
    for (;;) {
      if (x >= end) return false;
      const uint32_t places = a.pad + tiles, in = x - first, all = places * a.H * a.mt;
      if (in >= all) {
        if (b + 1 >= a.B) return false;
        first += all;
        enter(a, b + 1);
        continue;
      }
      item = (int)(in / places);
      const int at = (int)(in - item * places), to = (int)min(places, at + (end - x));
      x += to - at;
      t0 = max(0, at - a.pad);
      t1 = to - a.pad;
      if (t1 > t0) return true;  // else empty places alone
    }
  }
  __device__ __forceinline__ int64_t items(const PrefixArgs& a) const { return (int64_t)b * a.H * a.mt + item; }
  __device__ __forceinline__ int64_t slot(const PrefixArgs& a) const { return blockIdx.x + items(a); }
  // The whole item: there are no other parts.
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
  // The parts of the item whose first one this is.
  __device__ __forceinline__ int parts() const { return (int)((x - t1 + tiles - 1) / per - blockIdx.x) + 1; }
};

// Whether one of a pair of bf16 is an infinity or a NaN; the pair with 0 there.  Drafted
// values that some query rows do not see are left out of the products where they are
// not finite, since 0 times them is not 0, and added by the joining kernel.
__device__ __forceinline__ bool not_finite(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0 : w & 0xffffu) | ((w & 0x7f800000u) == 0x7f800000u ? 0 : w & 0xffff0000u);
}
// Whether query row i of sequence b sees drafted row j.
__device__ __forceinline__ bool sees(const PrefixArgs& a, int b, int i, int j) {
  return !a.mask || (__ldg(a.mask + ((int64_t)b * a.q + i) * a.mw + (j >> 5)) >> (j & 31) & 1);
}

}  // namespace wf
