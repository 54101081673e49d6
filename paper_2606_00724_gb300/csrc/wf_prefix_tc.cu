// Attention over shared prompts for bf16 queries on the tensor cores.
//
// A CTA takes up to 256 stacked query rows of a unit and a range of its keys,
// in tiles of 128 keys that arrive in a ring of shared-memory stages:
//   S = Q K^T  (128 rows x 128 keys, TMEM)
//   P = 2^(s - m), bf16, written over S in TMEM
//   O += P V   (A operand from TMEM, V the MN-major B operand)
// The query rows lie on the TMEM lanes, so a thread owns a row, or half of its
// columns: maxima and sums are serial, and two threads exchange a maximum through
// shared memory.  m is raised lazily, when a tile's maximum exceeds it by more
// than 2^8, so P stays below 2^8 and O is rescaled only then.
//
// Two pairs of warpgroups form P in turn, each pair with an S and an O of its own
// in TMEM, each warpgroup with half of the columns.  With more than 128 rows
// (`wide`) the pairs own a row tile each and meet the same key tiles; with at
// most 128 they share the row tile and take every other key tile, so that one
// works while the other's products run, and their O are put together at the
// end.  Copies and products run ahead: the key tile of a pair's next step is
// multiplied as soon as its P is consumed.
//
// Measured (d = 128): 512 rows of 32 heads on 32K keys 245 us, 1.1 PFLOP/s, a
// tile of 256 rows 3100 cycles where its products take 2048 and its softmax 1050
// to 1180 in turn; 128 rows of 48 heads on 32K 131 us, 6.2 TB/s; 32 rows of 8
// heads on 128K in 8 bits 82 us, where widening fills half of the integer pipe.
//
// bf16 prompt rows are copied by cp.async into the 128-byte-swizzled stages,
// gathered through idx where there is one.  Codes are copied as they are by two
// loader warps into a ring of their own, and the producers widen them to bf16
// (exact: at most 4 digits and a power of two) into the stage.  Rows past a
// count are zero-filled and never read.
//
// P is rounded to bf16, one term of it, as the operand of the product; sums,
// maxima and O stay in fp32.  Against 64 bits the outputs are 1.6e-3 to 2.2e-3
// off, where the rounding of O alone leaves 1.6e-3 to 1.7e-3.  What P's rounding
// drops, as a second operand, would bring them to that and cost half of the
// products again: with PV issued twice, 512 rows of 32 heads took 281 us instead
// of 242 and the other cases 1 to 5 % more, before the second term's own
// instructions and registers, of which the softmax has none left.
//
// Every wait is bounded: one that gives up sets the status word and the
// abort word, every role leaves its loops, work in flight is drained and the
// tensor memory freed.
#include <float.h>

#include "wf_mx.cuh"
#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int TM = kPrefixTcRows / 2;  // rows of a row tile, keys of a key tile
constexpr int HALF = TM * 128;         // 64 channels of a tile of bf16 rows
constexpr float kLazy = 8.f;

constexpr int kMaxStages = 9;
struct Bars {
  unsigned long long full[kMaxStages], empty[kMaxStages], raw_full[4], raw_empty[4], qfull, sfull[2], pready[2], odone[2], turn[2], drain[2], stall;
  uint32_t tmem, abort;
  // Between the two warps that share 32 rows of a tile: whether the tile is
  // there, whether a maximum rises, and the rows' maxima.
  int go[2][4], raise[2][2][4];
  float top[2][TM];
  uint32_t row[kPrefixTcRows];  // a row's number among all, for the way out
};

template <int D, int FMT>
struct Cfg {
  static constexpr bool CODES = FMT != WF_BF16;
  static constexpr int NPT = CODES ? 256 : 128;          // producer threads
  // Softmax warps, producers, two MMA warps and, with codes, two loader warps.
  static constexpr int NTH = 512 + NPT + (CODES ? 128 : 64);
  static constexpr int TILE = TM * D * 2;                // a stage
  static constexpr int ROWB = FMT == WF_MXFP4 ? D / 2 : D;  // bytes of a row of codes
  static constexpr int DEPTH = FMT == WF_MXFP8 ? 3 : 4;  // tiles of codes in flight
  // A tile's chunks of codes go to the widening threads so that the 8 lanes of a
  // shared-memory phase hold the PX chunks of one 64-channel half for 8 / PX
  // consecutive rows: the stores into the swizzled stage then take 8 different
  // banks of 16 bytes, and the loads do as well with chunk x of row r at chunk
  // place(x, r) of the slot's row.
  static constexpr int CR = ROWB / 16, PX = D == 128 ? CR / 2 : CR;
  __device__ static int place(int x, int r) { return D == 128 ? x ^ (r * ROWB / 128 % 2 * PX) : x; }
  static constexpr int SLOT = TM * ROWB + TM * 4;        // a tile of codes and its scales
  static constexpr int RAW = CODES ? DEPTH * SLOT : 0;
  static constexpr int ROOM = 232448 - (int)sizeof(Bars) - 2 * TILE - RAW;
  // Stages beside two tiles of query rows; with one tile its place is a stage more.
  static constexpr int STAGES = ROOM / TILE > kMaxStages - 1 ? kMaxStages - 1 : ROOM / TILE;
  static_assert(STAGES * TILE + RAW >= 2 * TM * D * 4, "the rows go out through the stages");
  static constexpr size_t SMEM = 2 * TILE + RAW + (size_t)STAGES * TILE + sizeof(Bars);
};

__device__ __forceinline__ uint32_t bar(const unsigned long long& b) { return smem_u32(&b); }

// A wait that gives up, or follows one that did, returns false.
__device__ __forceinline__ bool wait(uint32_t b, uint32_t parity, Bars& s, const PrefixArgs& a) {
  if (mbar_wait_bounded(b, parity, a.wait_limit, smem_u32(&s.abort))) return true;
  if (!abort_set(smem_u32(&s.abort))) {
    atomicExch(&s.abort, 1u);
    atomicExch(a.status, 1);
  }
  return false;
}

// The same for a whole warp: every lane gets one answer.
__device__ __forceinline__ bool warp_wait(uint32_t b, uint32_t parity, Bars& s, const PrefixArgs& a) {
  return __all_sync(0xffffffffu, wait(b, parity, s, a));
}

// D[tmem] (+)= A[tmem] B[smem]: A's rows on the lanes, two bf16 a column.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// What a CTA works on: from the launch alone, and its keys from the lengths.
struct Item {
  bool own, wide;
  int u, b, h;          // unit: prompt or sequence, key head
  int part, r0, nr;     // part, first row, rows
  int k0, k1, T;        // keys [k0, k1), tiles
};

__device__ __forceinline__ Item item_of(const PrefixArgs& a) {
  Item w;
  const int prompts = a.P * a.H * a.mt * a.S;
  int it = blockIdx.x;
  w.own = it >= prompts;
  if (w.own) it -= prompts;
  const FastDiv by_mt = w.own ? a.by_mto : a.by_mt, by_S = w.own ? a.by_So : a.by_S;
  const int x = fastdiv(it, by_mt), tile = it - x * (int)by_mt.d;
  w.u = fastdiv(x, by_S);
  const int sp = x - w.u * (int)by_S.d;
  w.b = fastdiv(w.u, a.by_H);
  w.h = w.u - w.b * a.H;
  w.part = w.own ? a.S + sp : sp;
  w.r0 = tile * kPrefixTcRows;
  w.nr = min(kPrefixTcRows, (w.own ? a.Ro : a.R) - w.r0);
  w.wide = w.nr > TM;
  return w;
}
__device__ __forceinline__ void keys_of(const PrefixArgs& a, Item& w) {
  const int S = w.own ? a.So : a.S, sp = w.own ? w.part - a.S : w.part;
  const int count = w.own ? own_count(a, w.b) : prompt_count(a, w.b);
  const int tiles = (count + TM - 1) / TM, per = (tiles + S - 1) / S;
  w.k0 = min(count, sp * per * TM);
  w.k1 = min(count, (sp + 1) * per * TM);
  w.T = (w.k1 - w.k0 + TM - 1) / TM;
}

// The ring of stages: position p of the order below is in stage p % n.
struct Ring {
  uint32_t base;
  int n;
  uint32_t inv;  // 2^32 / n rounded up: exact quotients below 2^28
  __device__ __forceinline__ int turn(int p) const { return (int)__umulhi((uint32_t)p, inv); }
  __device__ __forceinline__ int stage(int p) const { return p - turn(p) * n; }
};

// Key tiles meet the MMA warps in the order K_0 .. K_(A-1), then V_j, K_(j+A)
// for j = 0 .., A = 1 (wide) or 2, and the last V_j.  f(tile, is V) for each in
// that order.  So with L = min(A, T), K_t has ring position t (t < L) or
// L + 2 (t - A) + 1, and V_j position L + 2 j (j < T - L) or T + j.
template <typename F>
__device__ __forceinline__ void in_order(int T, int A, F f) {
  const int lead = min(A, T), paired = 2 * T - lead;  // positions [lead, paired) are V_j, K_(j+A) in turn
#pragma unroll 1
  for (int p = 0; p < 2 * T; ++p) {  // one call, so that f's code is there once
    const int o = p - lead;
    const bool v = o >= 0 && (p >= paired || !(o & 1));
    f(o < 0 ? p : p >= paired ? p - T : o / 2 + ((o & 1) ? A : 0), v);
  }
}

// ---------------------------------------------------------------------------
// Producers.
// ---------------------------------------------------------------------------
// Byte offset of 16-byte chunk ch of row r in a swizzled tile.
__device__ __forceinline__ uint32_t swizzled(int r, int ch) {
  return (uint32_t)((ch >> 3) * HALF + r * 128 + (((ch ^ r) & 7) << 4));
}

// One tile of bf16 rows, NPT threads: chunk tid % CH of rows tid / CH + RS i.
// With idx, lane ch of the CH lanes that share a row looks up rows
// tid / CH + RS (ch + CH k) and the lanes pass them on.
template <int D, int NPT>
__device__ __forceinline__ void copy_tile(uint32_t st, const bf16* base, int64_t stride, const int32_t* idx, int n, int t0,
                                          int k1, int tid) {
  constexpr int CH = D / 8, RS = NPT / CH, NI = TM / RS;
  const int ch = tid % CH, rr = tid / CH;
  const bf16* src = base + ch * 8;
  if (idx) {
    constexpr int NL = (NI + CH - 1) / CH;
    int row[NL];
#pragma unroll
    for (int k = 0; k < NL; ++k) {
      const int j = t0 + rr + RS * (ch + CH * k);
      row[k] = ch + CH * k < NI && j < k1 ? min(max(__ldg(idx + j), 0), n - 1) : 0;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = rr + RS * i;
      const int at = __shfl_sync(0xffffffffu, row[i / CH], i % CH, CH);
      const bool ok = t0 + r < k1;
      cp_async16_zfill(st + swizzled(r, ch), src + (ok ? (int64_t)at * stride : 0), ok);
    }
  } else if (t0 + TM <= k1) {
    const bf16* p = src + (t0 + rr) * stride;
    const uint32_t dst = st + swizzled(rr, ch);
    static_assert(RS % 8 == 0, "a thread's rows share their swizzle");
#pragma unroll
    for (int i = 0; i < NI; ++i, p += RS * stride) cp_async16(dst + RS * i * 128, p);
  } else {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = rr + RS * i;
      const bool ok = t0 + r < k1;
      cp_async16_zfill(st + swizzled(r, ch), src + (ok ? (int64_t)(t0 + r) * stride : 0), ok);
    }
  }
}

__device__ __forceinline__ RowAt row_at(const PrefixArgs& a, const Item& w, int r) {
  return w.own ? own_row(a, w.b, w.h, w.r0 + r) : prompt_row(a, w.b, w.h, w.r0 + r);
}
template <int D, int FMT>
__device__ void produce(const PrefixArgs& a, const Item& w, const Ring& ring, uint32_t raw, Bars& s, int tid) {
  typedef Cfg<D, FMT> C;
  constexpr int NPT = C::NPT;
  const int64_t b = w.b, h = w.h;
  const int A = w.wide ? 1 : 2;
  if (!C::CODES || w.own) {
    const int64_t sb = w.own ? a.gsb : a.ksb, sh = w.own ? a.gsh : a.ksh, ss = w.own ? a.gss : a.kss;
    const bf16* K = static_cast<const bf16*>(w.own ? a.Kg : a.K) + b * sb + h * sh;
    const bf16* V = static_cast<const bf16*>(w.own ? a.Vg : a.V) + b * sb + h * sh;
    const int32_t* idx = a.idx && !w.own ? a.idx + (int64_t)w.u * a.k : nullptr;
    int pos = 0;
    bool ok = true;
    in_order(w.T, A, [&](int t, bool v) {
      const int st = ring.stage(pos), n = ring.turn(pos);
      ++pos;
      if (ok && n > 0) ok = warp_wait(bar(s.empty[st]), (n - 1) & 1, s, a);
      if (ok) copy_tile<D, NPT>(ring.base + st * C::TILE, v ? V : K, ss, idx, a.n, w.k0 + t * TM, w.k1, tid);
      cp_async_arrive_noinc(bar(s.full[st]));
    });
    cp_async_wait_all();
    return;
  }
  if constexpr (C::CODES) {
    // Widen the tiles that the loader warps bring.  Two groups of four warps take
    // every other tile, so that one's waits run under the other's work: with all
    // eight on each tile a third of the time went by in waits.  Thread tid of a
    // group takes chunk x of rows rr + RS i.
    constexpr bool FP4 = FMT == WF_MXFP4;
    constexpr int CR = C::CR, PX = C::PX, NG = NPT / 2, CPT = TM * CR / NG, RS = NG / CR;
    constexpr int EL = FP4 ? 32 : 16, OUT = EL / 8;  // channels a chunk, bf16 chunks they make
    static_assert(RS % 8 == 0, "a thread's rows share their swizzle and place");
    const int group = tid / NG, gt = tid % NG;
    const int x = gt % PX + PX * (gt / 8 % (CR / PX)), rr = gt / PX % (8 / PX) + 8 / PX * (gt / (8 * CR / PX));
    const uint32_t chunk = (uint32_t)(rr * CR + C::place(x, rr)) * 16;
    const uint32_t scale = TM * C::ROWB + rr * 4 + x * EL / kMxBlock;
#pragma unroll 1
    for (int p = group; p < 2 * w.T; p += 2) {
      const int slot = p % C::DEPTH, st = ring.stage(p), n = ring.turn(p);
      if (!warp_wait(bar(s.raw_full[slot]), p / C::DEPTH & 1, s, a)) break;
      // All of the thread's codes first, and the slot back to the loaders, so that a
      // copy's latency covers one tile's widening and not two (82 against 85 us for
      // a token from 8 bits, with four chunks at a time).
      const uint32_t src = raw + slot * C::SLOT, dst = ring.base + st * C::TILE;
      uint4 code[CPT];
      uint32_t byte[CPT];
      bool large = false;  // a scale that takes a second factor
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        code[i] = lds_v4(src + chunk + NG * 16 * i);
        byte[i] = lds_u8(src + scale + RS * 4 * i);
      }
#pragma unroll
      for (int i = 0; i < CPT; ++i) large |= byte[i] > kMxOne<FP4>;
      large = __any_sync(0xffffffffu, large);
      __syncwarp();  // every lane has read its chunks
      if ((gt & 31) == 0) mbar_arrive(bar(s.raw_empty[slot]));
      if (n > 0 && !warp_wait(bar(s.empty[st]), (n - 1) & 1, s, a)) break;
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        const uint32_t cw[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
        const uint32_t f = mx_factor<FP4>(byte[i]);
        uint32_t y[OUT * 4];
#pragma unroll
        for (int e = 0; e < 4; ++e) mx_pairs<FP4>(cw[e], y + e * OUT);
#pragma unroll
        for (int e = 0; e < OUT * 4; ++e) y[e] = mul_bf16x2(y[e], f);
        if (large) {
          const uint32_t f2 = mx_second_factor<FP4>(byte[i]);
#pragma unroll
          for (int e = 0; e < OUT * 4; ++e) y[e] = mul_bf16x2(y[e], f2);
        }
#pragma unroll
        for (int o = 0; o < OUT; ++o)
          sts_v4(dst + swizzled(rr, x * OUT + o) + RS * 128 * i, make_uint4(y[4 * o], y[4 * o + 1], y[4 * o + 2], y[4 * o + 3]));
      }
      fence_proxy_async();
      __syncwarp();
      if ((gt & 31) == 0) mbar_arrive(bar(s.full[st]));
    }
  }
}

// The loader warps of a prompt in codes: tiles of codes and their scales, as
// they are, into DEPTH slots.  A warp brings half of a tile's rows: lane l looks
// up two of them (rows q = l, l + 32 of the warp's 64) one tile ahead, copies
// their scales, and the lanes pass the rows on for the chunks.  A row's scale
// bytes have 4 bytes of a slot; where they are 2, they are stored by the thread,
// since the smallest copy is 4 bytes on 4.
template <int D, int FMT>
__device__ void load_codes(const PrefixArgs& a, const Item& w, uint32_t raw, Bars& s, int warp, int lane) {
  typedef Cfg<D, FMT> C;
  constexpr int CR = C::CR, RP = 32 / CR, NI = 64 / RP, SR = D / kMxBlock;  // rows a pass of the warp, passes
  const int64_t b = w.b, h = w.h;
  const int x = lane % CR;
  const int32_t* idx = a.idx ? a.idx + (int64_t)w.u * a.k : nullptr;
  const uint8_t* kbase = static_cast<const uint8_t*>(a.K) + b * a.ksb + h * a.ksh + x * 16;
  const uint8_t* vbase = static_cast<const uint8_t*>(a.V) + b * a.ksb + h * a.ksh + x * 16;
  const int64_t srow = (int64_t)w.u * a.n * SR;
  // Row q of the warp's half is row 64 warp + q of the tile; -1 past the last.
  auto look_up = [&](int t, int* row) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int j = w.k0 + t * TM + 64 * warp + lane + 32 * k;
      row[k] = j >= w.k1 ? -1 : idx ? min(max(__ldg(idx + j), 0), a.n - 1) : j;
    }
  };
  int slot = 0, n = 0;
  bool ok = true;
  const uint32_t first = (uint32_t)((64 * warp + lane / CR) * CR) * 16;  // this lane's first row in a slot
  auto bring = [&](int t, const int* row, bool v) {
    if (ok && n > 0) ok = warp_wait(bar(s.raw_empty[slot]), (n - 1) & 1, s, a);
    if (ok) {
      const uint32_t dst = raw + slot * C::SLOT;
      const uint8_t* base = v ? vbase : kbase;
      const uint8_t* sc = (v ? a.Vs : a.Ks) + srow;
      const bool full = w.k0 + (t + 1) * TM <= w.k1;
      if (!idx && full) {
        const uint8_t* p = base + (w.k0 + t * TM + 64 * warp + lane / CR) * a.kss;
#pragma unroll
        for (int i = 0; i < NI; ++i, p += RP * a.kss)
          cp_async16(dst + first + RP * CR * 16 * i + C::place(x, lane / CR + RP * i) * 16, p);
      } else {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          const int at = __shfl_sync(0xffffffffu, row[RP * i / 32], (RP * i + lane / CR) % 32);
          cp_async16_zfill(dst + first + RP * CR * 16 * i + C::place(x, lane / CR + RP * i) * 16,
                           base + max(at, 0) * a.kss, at >= 0);
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint32_t at = dst + TM * C::ROWB + (uint32_t)(64 * warp + lane + 32 * k) * 4;
        const uint8_t* p = sc + (int64_t)max(row[k], 0) * SR;
        if (SR == 4) cp_async4(at, p, row[k] < 0 ? 0 : 4);  // rows past the last: scale 2^-127 of zeros
        else sts_u32(at, row[k] < 0 ? 0u : __ldg(reinterpret_cast<const uint16_t*>(p)));
      }
    }
    if (SR == 2) mbar_arrive(bar(s.raw_full[slot]));  // releases the plain stores
    cp_async_arrive_noinc(bar(s.raw_full[slot]));
    if (++slot == C::DEPTH) { slot = 0; ++n; }
  };
  int row[2], ahead[2], tile = -1;
  bool kind = false;
  in_order(w.T, w.wide ? 1 : 2, [&](int t, bool v) {
    look_up(t, ahead);
    if (tile >= 0) bring(tile, row, kind);
    row[0] = ahead[0];
    row[1] = ahead[1];
    kind = v;
    tile = t;
  });
  if (tile >= 0) bring(tile, row, kind);
  cp_async_wait_all();
}

// ---------------------------------------------------------------------------
// MMA warps, one a warpgroup: the tensor unit queues about four products (256
// cycles), less than the waits of a step take, so one warp waits for its operands
// while the other's products run.  The steps (PV, then the next QK) go out in
// turn: unordered, the warpgroups fell into step, both waiting for products
// and then both forming P (4030 cycles a tile instead of 2900).  All 32 lanes
// walk the loop, so that addresses and descriptors are uniform over the warp, as
// the instruction takes them; one lane issues.
// ---------------------------------------------------------------------------
__device__ __forceinline__ bool elect() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}

template <int D, int FMT>
__device__ void multiply(const PrefixArgs& a, const Item& w, uint32_t sq, const Ring& ring, Bars& s, int g) {
  typedef Cfg<D, FMT> C;
  if (w.T == 0) return;
  const uint32_t tm = __shfl_sync(0xffffffffu, s.tmem, 0);
  constexpr uint32_t qk = idesc_bf16(TM, TM, 0, 0), pv = idesc_bf16(TM, D, 0, 1);
  constexpr int T4 = C::TILE >> 4, H4 = HALF >> 4;  // in units of a descriptor's address
  const uint64_t q = smem_desc_sw128(sq, 16, 1024) + (w.wide ? g : 0) * T4, k0 = smem_desc_sw128(ring.base, 16, 1024),
                 v0 = smem_desc_sw128(ring.base, HALF, 1024);
  const int A = w.wide ? 1 : 2, first = w.wide ? 0 : g;
  bool ok = warp_wait(bar(a.stall ? s.stall : s.qfull), 0, s, a);
  // Ring position of key tile t and of value tile t: see in_order.
  const int lead = min(A, w.T);
  auto arrived = [&](int pos) {
    if (ok) ok = warp_wait(bar(s.full[ring.stage(pos)]), ring.turn(pos) & 1, s, a);
    fence_proxy_async();
    tc_fence_after();
  };
  auto scores = [&](int stage) {
    if (elect()) {
      const uint64_t k = k0 + stage * T4;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        mma_bf16(tm + TM * g, q + (kk / 4) * H4 + (kk % 4) * 2, k + (kk / 4) * H4 + (kk % 4) * 2, qk, kk != 0);
      mma_commit(bar(s.sfull[g]));
      mma_commit(bar(s.empty[stage]));
    }
    __syncwarp();
  };
  if (first < w.T) {
    arrived(first);
    if (ok) scores(first);
  }
#pragma unroll 1
  for (int j = first, i = 0; j < w.T && ok; j += A, ++i) {
    const bool more = j + A < w.T;
    const int pv_pos = j < w.T - lead ? lead + 2 * j : w.T + j, pk_pos = pv_pos + 1;
    arrived(pv_pos);
    if (more && w.wide) arrived(pk_pos);
    if (ok) ok = warp_wait(bar(s.pready[g]), i & 1, s, a);
    if (ok && (g || i > 0)) ok = warp_wait(bar(s.turn[g]), (g ? i : i - 1) & 1, s, a);
    tc_fence_after();
    if (!ok) break;
    const int sv = ring.stage(pv_pos);
    if (elect()) {
      const uint64_t v = v0 + sv * T4;
#pragma unroll
      for (int kq = 0; kq < TM / 16; ++kq)
        mma_bf16_ts(tm + 2 * TM + D * g, tm + TM * g + (kq / 4) * 64 + (kq % 4) * 8, v + kq * (2048 >> 4), pv, i > 0 || kq > 0);
      mma_commit(bar(s.empty[sv]));
      if (!more) mma_commit(bar(s.odone[g]));
    }
    __syncwarp();
    // With one row tile the products are short and the rows' arrival is what
    // bounds the loop: the value tile's stage goes back before the wait for the
    // next key tile.
    if (more && !w.wide) arrived(pk_pos);
    if (more && ok) scores(ring.stage(pk_pos));
    if (elect()) mbar_arrive(bar(s.turn[g ^ 1]));
    __syncwarp();
  }
  if (!ok) {  // products issued so far end before the tensor memory is freed
    if (elect()) mma_commit(bar(s.drain[g]));
    __syncwarp();
    (void)mbar_wait_bounded(bar(s.drain[g]), 0, kDefaultWaitLimit);
  }
}

// ---------------------------------------------------------------------------
// Softmax warpgroups.
// ---------------------------------------------------------------------------
// 16 columns of a thread's TMEM lane; valid behind got(), through which the
// registers pass, so that no use of them moves before the wait.
__device__ __forceinline__ void get(uint32_t taddr, uint32_t* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void got(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                 "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}

// The larger of the two halves' maxima of row r.
__device__ __forceinline__ float row_top(Bars& s, int g, int half, int r, int pair, float top) {
  if (half) s.top[g][r] = top;
  named_sync(pair, 64);
  if (!half) s.top[g][r] = top = fmaxf(top, s.top[g][r]);
  named_sync(pair, 64);
  return half ? s.top[g][r] : top;
}

// P of half a tile (64 keys) from S: one pass over chunks of CW columns, the next
// chunk on its way while one is worked on, with the maximum of the tiles before
// as m.  P stays in registers until the tile's own maximum is known; where that
// is more than 2^kLazy above m in either half (seldom) m is raised, O and l are
// rescaled and the pass runs again, S being still there.  P takes the first 32
// of its half's columns.
constexpr int CW = 16;
template <int D, bool MASK>
__device__ __forceinline__ void soften_tile(const PrefixArgs& a, Bars& s, uint32_t sc, uint32_t oc, bool have_o, int nk,
                                            int g, int half, int r, int pair, float& m, float& l) {
  constexpr int NC = TM / 2 / CW;
  const f32x2 sl = pk2(a.sl2, a.sl2);
  uint32_t p[TM / 4];
  f32x2 sum[2];
  if (!have_o) {  // the first tile: its maximum first, in a short pass
    float top = -INFINITY;
#pragma unroll 1
    for (int c = 0; c < NC; ++c) {
      uint32_t x[CW];
      get(sc + CW * c, x);
      got(x);
#pragma unroll
      for (int e = 0; e < CW; ++e) top = fmaxf(top, !MASK || CW * c + e < nk ? __uint_as_float(x[e]) : -INFINITY);
    }
    m = fmaxf(m, row_top(s, g, half, r, pair, top) * a.sl2);
  }
#pragma unroll 1
  for (;;) {
    const f32x2 nm = pk2(-m, -m);
    uint32_t v[2][CW];
    float top = -INFINITY;
    sum[0] = sum[1] = pk2(0.f, 0.f);
    get(sc, v[0]);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint32_t* x = v[c & 1];
      got(x);
      if (c + 1 < NC) get(sc + CW * (c + 1), v[(c + 1) & 1]);
      if (MASK) {
#pragma unroll
        for (int e = 0; e < CW; ++e) x[e] = CW * c + e < nk ? x[e] : __float_as_uint(-INFINITY);
      }
#pragma unroll
      for (int e = 0; e < CW; e += 2) {
        const float s0 = __uint_as_float(x[e]), s1 = __uint_as_float(x[e + 1]);
        top = fmax3(top, s0, s1);
        const float2 z = up2(fma2(pk2(s0, s1), sl, nm));
        const float p0 = ex2(z.x), p1 = ex2(z.y);
        sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pk2(p0, p1));
        p[(CW * c + e) / 2] = pack_bf16(p0, p1);
      }
    }
    const bool mine = __any_sync(0xffffffffu, top * a.sl2 > m + kLazy);
    if ((r & 31) == 0) s.raise[g][half][r >> 5] = mine;
    named_sync(pair, 64);
    if (!(mine | s.raise[g][half ^ 1][r >> 5])) break;
    const float mt = row_top(s, g, half, r, pair, top) * a.sl2;
    const bool raise = mt > m + kLazy;
    const float f = raise ? ex2(m - mt) : 1.f;
    m = raise ? mt : m;
    l *= f;
    if (have_o) {  // half of O's columns; the products into it are done: this S was issued behind them
#pragma unroll 1
      for (int c = 0; c < D / 2 / CW; ++c) {
        uint32_t o[CW];
        get(oc + CW * c, o);
        got(o);
#pragma unroll
        for (int e = 0; e < CW; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
        tmem_st16(oc + CW * c, o);
      }
    }
  }
  tmem_st16(sc, p);
  tmem_st16(sc + 16, p + 16);
  const float2 z = up2(add2(sum[0], sum[1]));
  l += z.x + z.y;
}

// Warpgroup wg of four: half wg % 2 of the columns of S and O of row tile (or
// key tile parity) wg / 2.  Thread r has TMEM lane r.
template <int D, int FMT>
__device__ void soften(const PrefixArgs& a, const Item& w, uint8_t* sm, uint8_t* stages, Bars& s, int tid) {
  typedef Cfg<D, FMT> C;
  constexpr int CH = D / 8;
  const int g = tid >> 8, half = (tid >> 7) & 1, r = tid & 127, lane = tid & 31;
  const int pair = 3 + g * 4 + (r >> 5);             // the named barrier of the two warps with these rows
  const uint32_t lanes = (uint32_t)(r & ~31) << 16;  // the warp's quarter of the TMEM lanes
  const uint32_t tm = s.tmem, sc = tm + TM * g + TM / 2 * half + lanes, oc = tm + 2 * TM + D * g + D / 2 * half + lanes;
  const int rt = w.wide ? g * TM : 0;                // first row of the row tile
  const bool active = rt + (r & ~31) < w.nr;         // the warp has a row
  const int step = w.wide ? 1 : 2, first = w.wide ? 0 : g;
  if (w.T > 0) {
    // The query rows, K-major; rows past the last are zero.
    const uint32_t sq = smem_u32(sm);
    const int tiles = w.wide ? 2 : 1;
    for (int i = 0; i < tiles * TM * CH / 512; ++i) {
      const int q = tid / CH + 512 / CH * i, ch = tid % CH;
      const bool ok = q < w.nr;
      const RowAt at = row_at(a, w, ok ? q : 0);
      cp_async16_zfill(sq + (q / TM) * C::TILE + swizzled(q % TM, ch),
                       static_cast<const bf16*>(a.Q) + at.b * a.qsb + at.hq * a.qsh + at.i * a.qss + ch * 8, ok);
    }
    cp_async_arrive_noinc(bar(s.qfull));
  }
  if (tid < w.nr) s.row[tid] = (uint32_t)flat_row(a, row_at(a, w, tid));
  float m = -FLT_MAX, l = 0.f;  // finite, so that logits of -inf add 0 and not 2^(-inf + inf)
  bool ok = true;
  if (active) {
    int i = 0;
#pragma unroll 1
    for (int t = first; t < w.T; t += step, ++i) {
      // One warp of a pair waits and tells the other: a wait that gives up must
      // not leave one of them at the barriers below.
      if (!half) {
        ok = warp_wait(bar(s.sfull[g]), i & 1, s, a);
        if (lane == 0) s.go[g][r >> 5] = ok;
      }
      named_sync(pair, 64);
      ok = s.go[g][r >> 5];
      if (!ok) break;
      tc_fence_after();
      const int nk = w.k1 - (w.k0 + t * TM);  // keys of the tile
      if (nk >= TM) soften_tile<D, false>(a, s, sc, oc, i > 0, TM, g, half, r, pair, m, l);
      else soften_tile<D, true>(a, s, sc, oc, i > 0, nk - TM / 2 * half, g, half, r, pair, m, l);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(s.pready[g]));
    }
  }
  cp_async_wait_all();
  // The last products of both row tiles: the exchange below is in their stages.
  if (ok && w.T > 0) ok = warp_wait(bar(s.odone[0]), 0, s, a);
  if (ok && w.T > step - 1) ok = warp_wait(bar(s.odone[1]), 0, s, a);
  tc_fence_after();
  // The rows go out through the stages, which nothing reads any more: a thread has
  // a row, a store to memory wants a row's bytes from consecutive lanes (32
  // rows' 16 bytes a store took 5 us a CTA).  Two warpgroups on one row tile
  // scale their O to the larger maximum and the sum is formed on the way out.
  const bool have = w.T > first;  // this row tile (parity) had a key tile
  float* buf = reinterpret_cast<float*>(stages);   // [2][128][D], 16-byte chunks swizzled
  float2* ml = reinterpret_cast<float2*>(sm);      // [2][2][128], in Q's place
  ml[tid] = make_float2(m, l);
  named_sync(1, 512);
  l = ml[g * 256 + r].y + ml[g * 256 + 128 + r].y;
  float f = have ? 1.f : 0.f;
  if (!w.wide) {
    const float m0 = ml[r].x, m1 = ml[256 + r].x, M = fmaxf(m0, m1);
    const float l0 = ml[r].y + ml[128 + r].y, l1 = ml[256 + r].y + ml[384 + r].y;
    f *= ex2(m - M);
    l = l0 * ex2(m0 - M) + l1 * ex2(m1 - M);
    m = M;
  }
  if (a.whole) f = l == 0.f ? 0.f : f / l;
  const bool none = !have || l == 0.f;
  const bool gone = abort_set(smem_u32(&s.abort));
  if (active) {
    float* row = buf + (g * TM + r) * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[16];
      if (have) {
        get(oc + 16 * c, o);
        got(o);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = none ? 0u : __float_as_uint(__uint_as_float(o[e]) * f);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<uint4*>(row + (((D / 8 * half + 4 * c + e) ^ (r & 7)) << 2)) =
            make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
    }
  }
  named_sync(1, 512);
  constexpr int LPR = D / 4, RPW = 32 / LPR;  // lanes a row, rows a warp
  const int cc = lane % LPR;
#pragma unroll 4
  for (int q = tid / LPR; q < w.nr && !gone; q += 16 * RPW) {
    const float* row = buf + q * D + ((cc ^ (q & 7)) << 2);
    float4 y = *reinterpret_cast<const float4*>(row);
    if (!w.wide) {
      const float4 z = *reinterpret_cast<const float4*>(row + TM * D);
      y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
    }
    if (a.whole) {
      const RowAt at = row_at(a, w, q);
      *reinterpret_cast<uint2*>(static_cast<bf16*>(a.O) + at.b * a.osb + at.hq * a.osh + at.i * a.oss + 4 * cc) =
          make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    } else {
      *reinterpret_cast<float4*>(a.part_o + ((int64_t)w.part * a.rows + s.row[q]) * D + 4 * cc) = y;
    }
  }
  const int row = rt + r;
  if (!a.whole && !gone && row < w.nr && !half && (w.wide || g == 0))
    a.part_ml[(int64_t)w.part * a.rows + s.row[row]] = make_float2(m, l);
}

template <int D, int FMT>
__global__ void __launch_bounds__(Cfg<D, FMT>::NTH, 1) tc_kernel(const __grid_constant__ PrefixArgs a) {
  typedef Cfg<D, FMT> C;
  extern __shared__ __align__(1024) uint8_t sm[];
  uint8_t* raw = sm + (2 + C::STAGES) * C::TILE;
  Bars& s = *reinterpret_cast<Bars*>(raw + C::RAW);
  const int tid = threadIdx.x, warp = tid >> 5;
  constexpr int MMA_WARP = 16 + C::NPT / 32;
  Item w = item_of(a);
  uint8_t* stages = sm + (w.wide ? 2 : 1) * C::TILE;
  const int ns = C::STAGES + (w.wide ? 0 : 1);
  const Ring ring = {smem_u32(stages), ns, 0xffffffffu / ns + 1};
  if (warp == MMA_WARP) {
    tmem_alloc(smem_u32(&s.tmem), 512);
    tmem_relinquish();
  }
  // A barrier a thread: one after the other they took 0.4 us.
  if (tid < 2 * kMaxStages) {
    const int arrivals = C::CODES && !w.own ? C::NPT / 64 : C::NPT;
    // A stage is free with a commit of every MMA warp that reads it.
    mbar_init(bar(tid < kMaxStages ? s.full[tid] : s.empty[tid - kMaxStages]), tid < kMaxStages ? arrivals : w.wide ? 2 : 1);
  } else if (tid >= 32 && tid < 40) {
    const int i = tid & 3;
    mbar_init(bar(tid < 36 ? s.raw_full[i] : s.raw_empty[i]), tid < 36 ? (D == 128 ? 64 : 128) : C::NPT / 64);
  } else if (tid >= 64 && tid < 66) {
    const int g = tid - 64, rows = w.wide ? w.nr - g * TM : w.nr;
    mbar_init(bar(s.sfull[g]), 1);
    mbar_init(bar(s.pready[g]), (min(rows, TM) + 31) / 32 * 2);
    mbar_init(bar(s.odone[g]), 1);
  } else if (tid >= 96 && tid < 98) {
    mbar_init(bar(s.turn[tid - 96]), 1);
    mbar_init(bar(s.drain[tid - 96]), 1);
  } else if (tid == 128) {
    mbar_init(bar(s.qfull), 512);
    mbar_init(bar(s.stall), 1);
    s.abort = 0;
  }
  fence_mbar_init();
  grid_dep_wait();
  keys_of(a, w);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_launch();  // after the barrier that publishes the tensor memory (see Launch)
  // (Moving registers from the producers to the softmax warps was slower with
  // codes: 93 against 88-90 us for a token at 128K.)
  if (warp < 16) {
    soften<D, FMT>(a, w, sm, stages, s, tid);
  } else if (warp < MMA_WARP) {
    produce<D, FMT>(a, w, ring, smem_u32(raw), s, tid - 512);
  } else {
    if (warp < MMA_WARP + 2) multiply<D, FMT>(a, w, smem_u32(sm), ring, s, warp - MMA_WARP);
    else if (!w.own) load_codes<D, FMT>(a, w, smem_u32(raw), s, warp - MMA_WARP - 2, tid & 31);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(s.tmem, 512);
  }
}

template <int D, int FMT>
cudaError_t launch(const PrefixArgs& a, cudaStream_t s) {
  typedef Cfg<D, FMT> C;
  const int64_t items = (int64_t)a.P * a.H * a.mt * a.S + (int64_t)a.B * a.H * a.mto * a.So;
  if (!items) return cudaSuccess;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(tc_kernel<D, FMT>), C::SMEM);
  if (e != cudaSuccess) return e;
  return Launch(dim3((unsigned)items), C::NTH, C::SMEM, s)(tc_kernel<D, FMT>, a);
}

}  // namespace

cudaError_t launch_prefix_tc(const PrefixPlan& p, cudaStream_t s) {
  const bool wide = p.a.d == 128;
  if (p.fmt == WF_MXFP8) return wide ? launch<128, WF_MXFP8>(p.a, s) : launch<64, WF_MXFP8>(p.a, s);
  if (p.fmt == WF_MXFP4) return wide ? launch<128, WF_MXFP4>(p.a, s) : launch<64, WF_MXFP4>(p.a, s);
  return wide ? launch<128, WF_BF16>(p.a, s) : launch<64, WF_BF16>(p.a, s);
}

}  // namespace wf
