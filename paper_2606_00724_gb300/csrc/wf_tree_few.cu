// Drafted tokens over pages for few query rows: at most 16 a (sequence, key head), as
// one token of a group of heads makes them (wf_tree_attn, bf16 queries).
//
// So few rows use every cached byte once and hardly compute, so the rows' way in is
// all that counts, and a 128-row tensor-memory tile would stand seven eighths empty
// behind barriers and a set-up of 5 us.  Here a warp is on its own: it takes 16 keys a
// step, forms their logits and weights in registers (m16n8k16, fp32 accumulators) and
// adds their share of O, with no barrier but the warp's.  It copies its own rows, QD
// steps ahead, by cp.async into slots of its own.  A contraction may go through its
// channels in any order, so a lane's operands of K are 16 consecutive bytes of a row;
// V's pairs of keys are put together by byte permutes.
//
// The CTAs share all the sequences' keys evenly (Walk), a range's four warps taking every
// fourth step of it; the ranges are joined by tree_join_kernel, and a range that is
// its whole item goes out as it is.  Drafted rows are the last steps of an item, straight
// from memory, since they are few.  m is raised lazily, by more than 2^8, as in the kernel
// for more rows, each row for itself.  P is one bf16 term, as in all of the library's attention on the
// tensor cores but wf_sparse_attn's, and l is summed before the rounding: against 64 bits O is 1.8e-3 to 2.0e-3 off,
// where its own rounding leaves 1.5e-3 to 1.7e-3.  What P's rounding drops, as a second operand, brings it to that
// and costs 1 % from bf16 pages (136.2 against 134.5 us for 32 sequences of up to 8K) and 4 to 5 % from codes, whose own
// rounding is 2^-4 and more (379 against 364 for 32 of 16K in 8 bits).
//
// Measured (d = 128, 4 query rows of 8 key heads): 32 sequences of 8K in bf16 177 to 185 us,
// 6 TB/s, bound by the rows' way in (176 us without the arithmetic); 32 of 16K in 8 bits
// 353 to 364 us, bound by chains of the 850 instructions a 16 keys: 232 registers leave two warps a scheduler, which
// issues in 45 % of its cycles (the integer pipe is 42 % busy, HBM at 2.9 TB/s); against the kernel for
// more rows 145 and 205 us for 32 sequences of up to 8K, 12 and 25 for 32 of 64 rows.
#include <float.h>

#include "wf_mx.cuh"
#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int NTH = 128, NW = NTH / 32;
constexpr float kLazy = 8.f;
static_assert(kFewRows == 16, "one m16n8k16 operand");

__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <int BYTES>
__device__ __forceinline__ void fetch(uint32_t* w, uint32_t a) {
  if constexpr (BYTES == 16) {
    const uint4 v = lds_v4(a);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (BYTES == 8) {
    const uint2 v = lds_v2(a);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = lds_u32(a);
  }
}

// A lane's bytes of a row: as an operand of K, KN chunks of KB bytes of four lanes' share;
// of V, VN of VB of eight lanes'.
template <int D, int FMT>
struct Few {
  static constexpr bool CODES = FMT != WF_BF16, FP4 = FMT == WF_MXFP4;
  static constexpr int ROWB = FMT == WF_BF16 ? 2 * D : FP4 ? D / 2 : D;
  static constexpr int KB = ROWB / 4 < 16 ? ROWB / 4 : 16, KN = ROWB / 4 / KB, KE = KB * D / ROWB;  // KE: elements
  static constexpr int VB = ROWB / 8 < 16 ? ROWB / 8 : 16, VN = ROWB / 8 / VB, VE = VB * D / ROWB;
  // A slot holds the rows of K and of V with their 16-byte chunks permuted by the row, so that the
  // lanes of a phase read from different banks: of K, rows g and g + 1 and chunks c; of V,
  // rows 2 c and chunks g and g + 1.
  static constexpr int CPR = ROWB / 16, RPI = 32 / CPR;  // chunks a row, rows a copying instruction of the warp
  __device__ static int k_place(int r, int ch) { return r * ROWB + (CPR >= 8 ? ch ^ (r & 1) * 4 : ch) * 16; }
  __device__ static int v_place(int r, int ch) {
    return r * ROWB + (CPR >= 8 ? ch ^ (r >> 1 & 3) * 2 : CPR == 4 ? ch ^ (r >> 1 & 3) : ch) * 16;
  }
  static constexpr int TK = few_keys(FMT), SK = TK / NW;  // keys a tile, a step of a warp: one or two times 16
  static constexpr int STEP = 2 * SK * ROWB + (CODES ? 8 * SK : 0);
  static constexpr int QD = 16896 / STEP > 8 ? 8 : 16896 / STEP;
  static constexpr int PO = D + 4;
  static constexpr size_t QUEUE = (size_t)NW * QD * STEP, SMEM = QUEUE + 16 * (PO + 2) * sizeof(float);
};

// N bytes of codes (or of bf16) to pairs of bf16; byte: their scale.
template <int D, int FMT, int BYTES>
__device__ __forceinline__ void pairs_of(const uint32_t* w, uint32_t byte, uint32_t* y) {
  typedef Few<D, FMT> C;
  if constexpr (!C::CODES) {
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) y[i] = w[i];
  } else {
    constexpr int P = C::FP4 ? 4 : 2;  // pairs a word
    const uint32_t f = mx_factor<C::FP4>(byte);
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) mx_pairs<C::FP4>(w[i], y + P * i);
#pragma unroll
    for (int i = 0; i < BYTES / 4 * P; ++i) y[i] = mul_bf16x2(y[i], f);
    if (byte > kMxOne<C::FP4>) {
      const uint32_t f2 = mx_second_factor<C::FP4>(byte);
#pragma unroll
      for (int i = 0; i < BYTES / 4 * P; ++i) y[i] = mul_bf16x2(y[i], f2);
    }
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(NTH, few_per_sm(D)) few_kernel(const __grid_constant__ PrefixArgs a) {
  typedef Few<D, FMT> C;
  constexpr int SK = C::SK, TK = C::TK;
  extern __shared__ __align__(128) uint8_t sm[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  const uint32_t queue = smem_u32(sm) + warp * C::QD * C::STEP;
  float* const so = reinterpret_cast<float*>(sm + C::QUEUE);        // [16][PO]
  float2* const sml = reinterpret_cast<float2*>(so + 16 * C::PO);  // [16]
  grid_dep_wait();
  grid_dep_launch();
  Walk in;  // the range of the next step to be copied
  if (!in.start(a)) return;
  Walk now = in;  // the range at work
  const bool in_page = a.by_ps.d % 16 == 0;  // 16 rows of a step are in one page
  const int SR = D / kMxBlock;

  // The next step: its place is looked up a step before it is copied, since a table's
  // entry takes as long to come as a row.  What a range fixes is found once.
  constexpr int EB = C::CODES ? 1 : 2;  // bytes of a stride's unit
  int t = 0, t_end = 0;
  bool more = true;
  int entry = 0, row_in = 0;  // what this lane looked up
  const uint8_t *K = nullptr, *V = nullptr;
  const int64_t kss = a.kss * EB, kx = a.kx * EB;
  auto enter = [&] {
    do more = in.next(a);
    while (more && in.t0 >= in.cached);  // drafted rows alone
    if (!more) return;
    t = in.t0;
    t_end = min(in.t1, in.cached);
    K = static_cast<const uint8_t*>(a.K) + in.item * a.ksh * EB + lane % C::CPR * 16;
    V = static_cast<const uint8_t*>(a.V) + in.item * a.ksh * EB + lane % C::CPR * 16;
  };
  auto look_up = [&] {
    row_in = t * TK + warp * SK + (in_page ? lane & (SK - 16) : lane % SK);
    entry = more && row_in < in.count ? page_entry(a, in.b, row_in) : 0;
  };
  uint32_t odd = 0;  // D = 64: whether the scales that this lane copied are the second half of their word
  auto bring = [&](uint32_t slot) {
    if (more) {
      const int left = in.count - (t * TK + warp * SK);
      const bool full = left >= SK;
      const PagedRow at = row_in < in.count ? paged_row(a, entry, row_in) : PagedRow{0, 0};
      const int64_t first = at.flat * kss + at.page * kx;  // bytes to the first of its 16 rows, where that finds them all
      auto half = [&](int n) { return SK == 16 ? first : __shfl_sync(0xffffffffu, first, 16 * n); };
      if (in_page && full) {
#pragma unroll
        for (int n = 0; n < SK / 16; ++n) {
          const int64_t o = half(n) + lane / C::CPR * kss;
          const uint8_t *k = K + o, *v = V + o;
#pragma unroll
          for (int x = 0; x < 16 / C::RPI; ++x, k += C::RPI * kss, v += C::RPI * kss) {
            const int r = 16 * n + C::RPI * x + lane / C::CPR;
            cp_async16(slot + C::k_place(r, lane % C::CPR), k);
            cp_async16(slot + SK * C::ROWB + C::v_place(r, lane % C::CPR), v);
          }
        }
      } else {
#pragma unroll
        for (int n = 0; n < SK / C::RPI; ++n) {
          const int r = C::RPI * n + lane / C::CPR;
          const bool ok = r < left;
          int64_t o;
          if (in_page) {
            o = half(C::RPI * n / 16);
            o = ok ? o + r % 16 * kss : 0;
          } else {
            const PagedRow w = {__shfl_sync(0xffffffffu, at.flat, r), __shfl_sync(0xffffffffu, at.page, r)};
            o = w.flat * kss + w.page * kx;
          }
          cp_async16_zfill(slot + C::k_place(r, lane % C::CPR), K + o, ok);
          cp_async16_zfill(slot + SK * C::ROWB + C::v_place(r, lane % C::CPR), V + o, ok);
        }
      }
      if constexpr (C::CODES) {  // a lane copies the scales of row lane of K and of V
        PagedRow w = at;
        if (in_page) w.flat += lane % 16;
        const bool ok = lane < left;
        const int64_t z = ok ? paged_scale(a, w, in.item) : 0;
        const uint32_t to = slot + 2 * SK * C::ROWB + lane * 4;
        // The smallest copy is 4 bytes on 4; at D = 64 the word's other half is another row's, or
        // nobody's.
        const bool second = D == 64 && (z & 1);
        const int size = !ok ? 0 : D == 128 || second ? 4 : 2;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const uint8_t* p = (v ? a.Vs : a.Ks) + z * SR - (second ? 2 : 0);
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 128 * v), "l"(p), "r"(size) : "memory");
        }
        if (D == 64) odd = odd << 1 | (uint32_t)second;
      }
      if (++t == t_end) enter();
      look_up();
    } else if (D == 64) {
      odd <<= 1;
    }
    cp_async_commit();
  };
  enter();
  look_up();
#pragma unroll 1
  for (int i = 0; i < C::QD; ++i) bring(queue + i * C::STEP);

  int stage = 0;
#pragma unroll 1
  while (now.next(a)) {
    // Query rows g and g + 8, the channels in the order in which a lane has those of K.
    uint32_t q[D / 16][4];
    int block_row[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int r = g + 8 * n;
      const RowAt w = own_row(a, now.b, now.item, r < a.Ro ? r : 0);
      block_row[n] = w.i;
      const bf16* p = static_cast<const bf16*>(a.Q) + w.b * a.qsb + w.hq * a.qsh + w.i * a.qss;
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {  // runs of 8 channels
        constexpr int RUNS = C::KE / 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < a.Ro) v = __ldg(reinterpret_cast<const uint4*>(p + (4 * (j / RUNS) + c) * C::KE + 8 * (j % RUNS)));
        q[2 * j][n] = v.x; q[2 * j][2 + n] = v.y;
        q[2 * j + 1][n] = v.z; q[2 * j + 1][2 + n] = v.w;
      }
    }
    int flag = 0;
    float o[D / 8][4], m[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
#pragma unroll 1
    for (int tile = now.t0; tile < now.t1; ++tile) {
      const uint32_t slot = queue + stage * C::STEP;
      const bool draft = tile >= now.cached;
      const int first0 = (draft ? tile - now.cached : tile) * TK + warp * SK;
      if (!draft) {
        cp_async_wait<C::QD - 1>();
        if constexpr (C::CODES) {
          if (D == 64 && (odd >> (C::QD - 1) & 1)) {  // every lane puts the scales that it copied in the word's first half
            const uint32_t w = slot + 2 * SK * C::ROWB + lane * 4;
            sts_u32(w, lds_u32(w) >> 16);
            sts_u32(w + 128, lds_u32(w + 128) >> 16);
          }
        }
        __syncwarp();  // every lane's copies are there
      }
      const int64_t own = now.b * a.gsb + now.item * a.gsh;  // drafted rows come straight from memory
#pragma unroll 1
      for (int part = 0; part < SK / 16; ++part) {  // 16 keys at a time
        const int first = first0 + 16 * part, left = (draft ? now.drafts : now.count) - first;
        if (left <= 0) break;
        float s[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
          const uint32_t scale = C::CODES && !draft ? lds_u32(slot + 2 * SK * C::ROWB + (16 * part + 8 * n + g) * 4) : 0;
          uint32_t k[D / 8];
          if (draft) {
            const bf16* p = static_cast<const bf16*>(a.Kg) + own + (int64_t)(first + min(8 * n + g, left - 1)) * a.gss;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
              constexpr int RUNS = C::KE / 8;
              const uint4 v = __ldg(reinterpret_cast<const uint4*>(p + (4 * (j / RUNS) + c) * C::KE + 8 * (j % RUNS)));
              k[4 * j] = v.x; k[4 * j + 1] = v.y; k[4 * j + 2] = v.z; k[4 * j + 3] = v.w;
            }
          } else {
#pragma unroll
          for (int j = 0; j < C::KN; ++j) {
            uint32_t w[C::KB / 4];
            const int at = (4 * j + c) * C::KB;
            fetch<C::KB>(w, slot + 16 * part * C::ROWB + C::k_place(8 * n + g, at / 16) + at % 16);
            pairs_of<D, FMT, C::KB>(w, scale >> 8 * ((4 * j + c) * C::KE / kMxBlock) & 0xffu, k + j * C::KE / 2);
          }
          }
#pragma unroll
          for (int i = 0; i < D / 16; ++i) mma16816(s[n], q[i], k[2 * i], k[2 * i + 1]);
        }
        if (left < 16) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (8 * n + 2 * c + (e & 1) >= left) s[n][e] = -INFINITY;
        }
        if (draft && a.mask) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const uint32_t w =
                __ldg(a.mask + ((int64_t)now.b * a.q + block_row[i]) * a.mw + (first >> 5)) >> ((first & 31) + 2 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(w >> (8 * (e >> 1) + (e & 1)) & 1)) s[e >> 1][2 * i + (e & 1)] = -INFINITY;
          }
        }
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
          top[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1])) * a.sl2;
        if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            // Of rows that ask for it themselves: a row's bits do not depend on its neighbours.
            const float mn = top[i] > m[i] + kLazy ? top[i] : m[i], f = ex2(m[i] - mn);
            m[i] = mn;
            l[i] *= f;
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
              o[e][2 * i] *= f;
              o[e][2 * i + 1] *= f;
            }
          }
        }
        uint32_t p[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {  // rows g (even x), g + 8; keys 0-7 (x < 2), 8-15
          const float* v = s[x >> 1] + 2 * (x & 1);
          const float p0 = ex2(fmaf(v[0], a.sl2, -m[x & 1])), p1 = ex2(fmaf(v[1], a.sl2, -m[x & 1]));
          l[x & 1] += p0 + p1;
          p[x] = pack_bf16(p0, p1);
        }
#pragma unroll
        for (int j = 0; j < C::VN; ++j) {
          uint32_t v[4][C::VE / 2];
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const int r = 2 * c + (n & 1) + 8 * (n >> 1);
            if (draft) {
              const bf16* p = static_cast<const bf16*>(a.Vg) + own + (int64_t)(first + min(r, left - 1)) * a.gss +
                              (8 * j + g) * C::VE;
#pragma unroll
              for (int i = 0; i < C::VE / 8; ++i) {
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(p) + i);
                v[n][4 * i] = w.x; v[n][4 * i + 1] = w.y; v[n][4 * i + 2] = w.z; v[n][4 * i + 3] = w.w;
              }
#pragma unroll
              for (int i = 0; i < C::VE / 2; ++i) {
                if (r >= left) v[n][i] = 0;
                if (a.mask && not_finite(v[n][i])) {
                  flag = 1;
                  v[n][i] = finite_only(v[n][i]);
                }
              }
              continue;
            }
            uint32_t w[C::VB / 4], byte = 0;
            const int at = (8 * j + g) * C::VB;
            fetch<C::VB>(w, slot + (SK + 16 * part) * C::ROWB + C::v_place(r, at / 16) + at % 16);
            if (C::CODES)
              byte = lds_u32(slot + 2 * SK * C::ROWB + (32 + 16 * part + r) * 4) >> 8 * ((8 * j + g) * C::VE / kMxBlock) & 0xffu;
            pairs_of<D, FMT, C::VB>(w, byte, v[n]);
          }
#pragma unroll
          for (int e = 0; e < C::VE / 2; ++e) {
            mma16816(o[j * C::VE + 2 * e], p, __byte_perm(v[0][e], v[1][e], 0x5410), __byte_perm(v[2][e], v[3][e], 0x5410));
            mma16816(o[j * C::VE + 2 * e + 1], p, __byte_perm(v[0][e], v[1][e], 0x7632),
                     __byte_perm(v[2][e], v[3][e], 0x7632));
          }
        }
      }
      if (!draft) {
        __syncwarp();  // every lane has read the slot
        bring(slot);
        if (++stage == C::QD) stage = 0;
      }
    }

    // The four warps' O, added from the last to the first, which writes the part.
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    auto channel = [&](int e, int x) { return (8 * (e / C::VE) + 2 * c + x) * C::VE + e % C::VE; };
    auto put = [&] {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i;
        if (r >= a.Ro) continue;
        if (c == 0) sml[r] = make_float2(m[i], l[i]);
#pragma unroll
        for (int e = 0; e < D / 8; e += 4)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            *reinterpret_cast<float4*>(so + r * C::PO + channel(e, x)) =
                make_float4(o[e][2 * i + x], o[e + 1][2 * i + x], o[e + 2][2 * i + x], o[e + 3][2 * i + x]);
      }
    };
    auto take = [&] {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i;
        if (r >= a.Ro) continue;
        // Without weight (l = 0) O is 0 x V, which is NaN where V is not finite.
        const float2 y = sml[r];
        const bool have = l[i] != 0.f, add = y.y != 0.f;
        if (!add) continue;
        const float M = have ? fmaxf(m[i], y.x) : y.x, f0 = have ? ex2(m[i] - M) : 0.f, f1 = ex2(y.x - M);
        m[i] = M;
        l[i] = (have ? l[i] * f0 : 0.f) + y.y * f1;
#pragma unroll
        for (int e = 0; e < D / 8; e += 4)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float4 v = *reinterpret_cast<const float4*>(so + r * C::PO + channel(e, x));
            const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int z = 0; z < 4; ++z)
              o[e + z][2 * i + x] = have ? fmaf(o[e + z][2 * i + x], f0, w[z] * f1) : w[z] * f1;
          }
      }
    };
#pragma unroll 1
    for (int w = NW - 1; w > 0; --w) {
      flag = __syncthreads_or(flag);  // the last exchange is over
      if (warp == w) put();
      __syncthreads();
      if (warp == w - 1) take();
    }
    const bool whole = now.whole();
    if (threadIdx.x == 0) {
      if (now.t0 == 0) a.info[now.items(a)] = make_int2((int)now.slot(a), now.parts());
      a.flags[now.slot(a)] = flag;
    }
    if (warp == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = g + 8 * i;
        if (r >= a.Ro) continue;
        const int64_t row = now.slot(a) * a.tr + r;
        const bool none = l[i] == 0.f;
        const float f = whole ? 1.f / l[i] : 1.f;
        if (c == 0) a.part_ml[row] = make_float2(m[i], l[i]);
        const RowAt w = own_row(a, now.b, now.item, r);
        bf16* out = static_cast<bf16*>(a.O) + w.b * a.osb + w.hq * a.osh + w.i * a.oss;
#pragma unroll
        for (int e = 0; e < D / 8; e += 4)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int at = channel(e, x);
            float4 y = make_float4(o[e][2 * i + x], o[e + 1][2 * i + x], o[e + 2][2 * i + x], o[e + 3][2 * i + x]);
            if (none) y = make_float4(0.f, 0.f, 0.f, 0.f);
            if (!whole) *reinterpret_cast<float4*>(a.part_o + row * D + at) = y;
            else *reinterpret_cast<uint2*>(out + at) =
                none ? make_uint2(0, 0) : make_uint2(pack_bf16(y.x * f, y.y * f), pack_bf16(y.z * f, y.w * f));
          }
      }
    }
  }
  cp_async_wait_all();
}

template <int D, int FMT>
cudaError_t launch(const PrefixArgs& a, cudaStream_t s) {
  const auto k = few_kernel<D, FMT>;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(k), Few<D, FMT>::SMEM);
  return e != cudaSuccess ? e : Launch(dim3((unsigned)a.C), NTH, Few<D, FMT>::SMEM, s)(k, a);
}

}  // namespace

cudaError_t launch_tree_few(const PrefixPlan& p, cudaStream_t s) {
  const bool wide = p.a.d == 128;
  if (p.fmt == WF_MXFP8) return wide ? launch<128, WF_MXFP8>(p.a, s) : launch<64, WF_MXFP8>(p.a, s);
  if (p.fmt == WF_MXFP4) return wide ? launch<128, WF_MXFP4>(p.a, s) : launch<64, WF_MXFP4>(p.a, s);
  return wide ? launch<128, WF_BF16>(p.a, s) : launch<64, WF_BF16>(p.a, s);
}

}  // namespace wf
