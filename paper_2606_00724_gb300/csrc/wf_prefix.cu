// Attention of several sequences over one cached prompt (wf_prefix_attn), in
// fp32 arithmetic for fp32 queries, and the joining of parts.
//
// Every query row of a prompt's key head, whatever its sequence, meets the same
// keys, so the rows of all of them are stacked and the prompt is read once a
// tile of rows instead of once a sequence; the own rows of a sequence are a
// second, short unit of the same kernel.  A CTA takes TR rows and a range of
// the keys in tiles of 64 and keeps the running maximum and sum of the softmax
// (base 2, the scale folded in) and O in registers, so no logit leaves the SM.
// A range that is not the whole softmax leaves a part in the workspace, and
// join_kernel puts the parts together.
#include <float.h>

#include <algorithm>

#include "wf_mx.cuh"
#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int TK = 64;      // keys a tile
constexpr int kWaves = 4;   // the parts of a call fill at most so many

// How prompt rows are kept: like the own rows, or in codes.
enum Cache { kPlain, kFp8, kFp4 };

// The threads of a CTA of TR rows, and its shared memory: query rows, one K and
// one V tile, P.
template <int TR> constexpr int kThreads = TR == 128 ? 512 : 256;
constexpr int PP = TK + 4;  // pitch of P
template <int D, int TR>
constexpr size_t simt_smem() {
  return sizeof(float) * (TR * D + 2 * TK * D + TR * PP);
}

// 16-byte chunk c of row r of a [rows][D] fp32 tile, chunks XOR-permuted by the
// row: eight consecutive rows' chunks lie in different banks.
template <int D>
__device__ __forceinline__ int at(int r, int c) { return r * D + ((c ^ (r & 7)) << 2); }

// Thread (ty, tx) = (tid / 16, tid % 16) owns rows ty RT .. + RT of the tile, keys
// tx + 16 j of a key tile and channels 4 tx + 64 c of O.  A key tile's V is copied
// while its logits are formed and the next tile's K while O is, so one buffer
// each is enough; codes come into registers a phase ahead and are widened into
// the buffer when it is free.
//
// 64 x 64 logits of 128 channels and their products with V are 2 x 4096 cycles of
// the fp32 pipe, and the corrections of the logits' sums (below) 2560 more; the
// shared-memory reads stay below that with 4 rows x 4 keys a thread.
template <int CACHE, int D, int TR, bool PAGED>
__global__ void __launch_bounds__(kThreads<TR>, TR == 128 ? 1 : 2) simt_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int NTH = kThreads<TR>, RT = TR * 16 / NTH, C = D / 64;
  constexpr bool FP4 = CACHE == kFp4;
  constexpr int IT = TK * D / 16 / NTH > 0 ? TK * D / 16 / NTH : 1;  // groups of 16 codes a thread
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;            // [TR][D]
  float* sk = sq + TR * D;   // [TK][D]
  float* sv = sk + TK * D;   // [TK][D]
  float* sp = sv + TK * D;   // [TR][PP]
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  // The CTA's unit, row tile and part.
  const int prompts = a.P * a.H * a.mt * a.S;
  int it = blockIdx.x;
  const bool own = it >= prompts;
  if (own) it -= prompts;
  const FastDiv by_mt = own ? a.by_mto : a.by_mt, by_S = own ? a.by_So : a.by_S;
  const int x0 = fastdiv(it, by_mt), tile = it - x0 * (int)by_mt.d, u = fastdiv(x0, by_S), sp_i = x0 - u * (int)by_S.d;
  const int b = fastdiv(u, a.by_H), h = u - b * a.H, S = by_S.d;
  const int r0 = tile * TR, nr = min(TR, (own ? a.Ro : a.R) - r0);
  grid_dep_wait();
  const int count = own ? own_count(a, b) : prompt_count(a, b);
  const int tiles = (count + TK - 1) / TK, per = (tiles + S - 1) / S;
  const int k0 = min(count, sp_i * per * TK), k1 = min(count, (sp_i + 1) * per * TK);
  const bool coded = CACHE != kPlain && !own;
  const int32_t* idx = a.idx && !own ? a.idx + (int64_t)u * a.k : nullptr;
  // Row j of a contiguous prompt; pages are looked up with it.
  auto row_of = [&](int j) { return idx ? min(max(__ldg(idx + j), 0), a.n - 1) : j; };
  auto place = [&](int j) { return paged_row(a, page_entry(a, b, j), j); };

  // Rows t0 .. of K or V as they are, by cp.async.
  auto copy = [&](bool v, int t0) {
    const float* base = static_cast<const float*>(v ? (own ? a.Vg : a.V) : (own ? a.Kg : a.K)) +
                        (PAGED && !own ? 0 : b * (own ? a.gsb : a.ksb)) + h * (own ? a.gsh : a.ksh);
    const int64_t ss = own ? a.gss : a.kss;
    const uint32_t dst = smem_u32(v ? sv : sk);
#pragma unroll 4
    for (int e = tid; e < TK * (D / 4); e += NTH) {
      const int r = e / (D / 4), c = e % (D / 4);
      const bool ok = t0 + r < k1;
      const int64_t o = !ok ? 0 : PAGED && !own ? paged_offset(a, place(t0 + r)) : row_of(t0 + r) * ss;
      cp_async16_zfill(dst + 4 * at<D>(r, c), base + o + 4 * c, ok);
    }
    cp_async_commit();
  };
  // The same of codes: into registers, and from there widened into the buffer.
  uint4 code[IT];
  uint32_t byte[IT];
  auto fetch = [&](bool v, int t0) {
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int e = tid + NTH * i, r = e / (D / 16), c = e % (D / 16);
      code[i] = make_uint4(0, 0, 0, 0);
      byte[i] = 0;
      if (r < TK && t0 + r < k1) {
        int64_t offset, scales;
        if (PAGED) {
          const PagedRow w = place(t0 + r);
          offset = h * a.ksh + paged_offset(a, w);
          scales = paged_scale(a, w, h);
        } else {
          const int64_t row = row_of(t0 + r);
          offset = b * a.ksb + h * a.ksh + row * a.kss;
          scales = (int64_t)u * a.n + row;
        }
        const uint8_t* p = static_cast<const uint8_t*>(v ? a.V : a.K) + offset;
        if (FP4) {
          const uint2 w = __ldg(reinterpret_cast<const uint2*>(p) + c);
          code[i].x = w.x;
          code[i].y = w.y;
        } else {
          code[i] = __ldg(reinterpret_cast<const uint4*>(p) + c);
        }
        byte[i] = __ldg((v ? a.Vs : a.Ks) + scales * (D / kMxBlock) + c / 2);
      }
    }
  };
  auto widen = [&](bool v) {
    float* dst = v ? sv : sk;
#pragma unroll
    for (int i = 0; i < IT; ++i) {
      const int e = tid + NTH * i, r = e / (D / 16), c = e % (D / 16);
      if (r >= TK) break;
      const uint32_t w[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
      const float s = mx_scale(byte[i]);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t q = FP4 ? w[k / 2] >> (16 * (k & 1)) : w[k];
        const float2 lo = mx_decode2<FP4>(FP4 ? q & 0xffu : q & 0xffffu), hi = mx_decode2<FP4>(FP4 ? q >> 8 & 0xffu : q >> 16);
        *reinterpret_cast<float4*>(dst + at<D>(r, 4 * c + k)) = make_float4(lo.x * s, lo.y * s, hi.x * s, hi.y * s);
      }
    }
  };

  for (int e = tid; e < TR * (D / 4); e += NTH) {
    const int r = e / (D / 4), c = e % (D / 4);
    const bool ok = r < nr;
    const RowAt w = own ? own_row(a, b, h, r0 + (ok ? r : 0)) : prompt_row(a, b, h, r0 + (ok ? r : 0));
    cp_async16_zfill(smem_u32(sq) + 4 * at<D>(r, c),
                     static_cast<const float*>(a.Q) + w.b * a.qsb + w.hq * a.qsh + w.i * a.qss + 4 * c, ok);
  }
  if (coded) {
    cp_async_commit();
    fetch(false, k0);
    widen(false);
    fetch(true, k0);
  } else {
    copy(false, k0);
  }

  float m[RT], l[RT];
  f32x2 o[RT][2 * C];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = -FLT_MAX;  // finite, so that logits of -inf add 0 and not 2^(-inf + inf)
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 2 * C; ++c) o[i][c] = 0ull;
  }
#pragma unroll 1
  for (int t0 = k0; t0 < k1; t0 += TK) {
    const int nk = min(TK, k1 - t0);
    const bool more = t0 + TK < k1;
    cp_async_wait_all();
    __syncthreads();  // K has arrived, V is free
    if (coded) {
      widen(true);
      if (more) fetch(false, t0 + TK);
    } else {
      copy(true, t0);
    }
    // Logits: even and odd channels in packed FMAs, chains of four of them, eight
    // channels, added to a sum with a running correction.  A logit of 100 has a
    // unit of 2^-17 in fp32; a plain sum of 128 products would leave an error of
    // several of them, and the softmax turns it into a relative error of the
    // weights.
    float s[RT][4], low[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[i][j] = low[i][j] = 0.f;
#pragma unroll 1
    for (int c = 0; c < D / 4; c += 2) {
      ulonglong2 ka[4], kb[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        ka[j] = *reinterpret_cast<const ulonglong2*>(sk + at<D>(tx + 16 * j, c));
        kb[j] = *reinterpret_cast<const ulonglong2*>(sk + at<D>(tx + 16 * j, c + 1));
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const ulonglong2 qa = *reinterpret_cast<const ulonglong2*>(sq + at<D>(ty * RT + i, c));
        const ulonglong2 qb = *reinterpret_cast<const ulonglong2*>(sq + at<D>(ty * RT + i, c + 1));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 x = up2(fma2(qb.y, kb[j].y, fma2(qb.x, kb[j].x, fma2(qa.y, ka[j].y, mul2(qa.x, ka[j].x)))));
          const float y = __fadd_rn(__fadd_rn(x.x, x.y), low[i][j]), t = __fadd_rn(s[i][j], y);
          low[i][j] = __fsub_rn(y, __fsub_rn(t, s[i][j]));
          s[i][j] = t;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float top = -INFINITY;
      const int block_row = PAGED && own && a.mask ? own_row(a, b, h, min(r0 + ty * RT + i, a.Ro - 1)).i : 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float h2 = s[i][j];
        if (!(fabsf(h2) <= FLT_MAX)) {  // an infinity in the rows makes the correction NaN: the plain sum
          h2 = low[i][j] = 0.f;
#pragma unroll 1
          for (int c = 0; c < D; ++c)
            h2 = fmaf(sq[at<D>(ty * RT + i, c / 4) + c % 4], sk[at<D>(tx + 16 * j, c / 4) + c % 4], h2);
        }
        s[i][j] = tx + 16 * j < nk ? h2 : -INFINITY;
        if (PAGED && own && a.mask && tx + 16 * j < nk && !sees(a, b, block_row, t0 + tx + 16 * j)) {
          s[i][j] = -INFINITY;
          low[i][j] = -1.f;  // hidden: its weight is -0
        }
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int w = 1; w < 16; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float mn = fmaxf(m[i], top * a.sl2), f = exp2f(m[i] - mn);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float none = PAGED && low[i][j] < 0.f ? -0.f : 0.f;
        const float p = s[i][j] == -INFINITY ? none : exp2f(fmaf(low[i][j], a.sl2, fmaf(s[i][j], a.sl2, -mn)));
        sum += p;
        sp[(ty * RT + i) * PP + tx + 16 * j] = p;
      }
      l[i] = l[i] * f + sum;  // this thread's keys; the 16 threads of the row are summed at the end
#pragma unroll
      for (int c = 0; c < 2 * C; ++c) o[i][c] = mul2(o[i][c], pk2(f, f));
    }
    cp_async_wait_all();
    __syncthreads();  // V has arrived, K is free (and a row's P, which one half-warp writes and reads)
    if (more) {
      if (coded) {
        widen(false);
        fetch(true, t0 + TK);
      } else {
        copy(false, t0 + TK);
      }
    }
#pragma unroll 1
    for (int j = 0; j < TK; j += 4) {
      float4 p[RT];
#pragma unroll
      for (int i = 0; i < RT; ++i) p[i] = *reinterpret_cast<const float4*>(sp + (ty * RT + i) * PP + j);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        ulonglong2 vv[C];
#pragma unroll
        for (int c = 0; c < C; ++c) vv[c] = *reinterpret_cast<const ulonglong2*>(sv + at<D>(j + k, tx + 16 * c));
#pragma unroll
        for (int i = 0; i < RT; ++i) {
          const float pi = k == 0 ? p[i].x : k == 1 ? p[i].y : k == 2 ? p[i].z : p[i].w;
          // A hidden row of V may hold anything, and 0 times it is not 0; a weight that is 0 for its
          // smallness (+0) is a seen row's, which counts.
          if (PAGED && own && __float_as_uint(pi) == 0x80000000u) continue;
          const f32x2 pp = pk2(pi, pi);
#pragma unroll
          for (int c = 0; c < C; ++c) {
            o[i][2 * c] = fma2(pp, vv[c].x, o[i][2 * c]);
            o[i][2 * c + 1] = fma2(pp, vv[c].y, o[i][2 * c + 1]);
          }
        }
      }
    }
  }
  grid_dep_launch();
  cp_async_wait_all();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int w = 1; w < 16; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    const int r = ty * RT + i;
    if (r >= nr) continue;
    const RowAt w = own ? own_row(a, b, h, r0 + r) : prompt_row(a, b, h, r0 + r);
    const bool none = l[i] == 0.f;
    const float f = none ? 0.f : a.whole ? 1.f / l[i] : 1.f;
    const int64_t flat = (int64_t)(own ? a.S + sp_i : sp_i) * a.rows + flat_row(a, w);
    float* op = a.whole ? static_cast<float*>(a.O) + w.b * a.osb + w.hq * a.osh + w.i * a.oss : a.part_o + flat * D;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const float2 y0 = up2(o[i][2 * c]), y1 = up2(o[i][2 * c + 1]);
      const float4 y = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y0.x * f, y0.y * f, y1.x * f, y1.y * f);
      *reinterpret_cast<float4*>(op + 4 * tx + 64 * c) = y;
    }
    if (!a.whole && tx == 0) a.part_ml[flat] = make_float2(m[i], l[i]);
  }
}

// O of every query row from its parts: with M the largest m, the sum of
// 2^(m - M) O over that of 2^(m - M) l.  A part without a key (l = 0) adds
// nothing, and a row without any is 0.  D / 4 threads hold a row's channels; GR
// groups of them take every GR-th part (many parts one after the other were 30
// us for one row) and the first puts the groups together, in their order.
constexpr int JTH = 256;
template <typename T, int D, int GR>
__global__ void __launch_bounds__(JTH) join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int LPR = D / 4;
  __shared__ float4 so[GR > 1 ? JTH : 1];
  __shared__ float2 sml[GR > 1 ? JTH / LPR : 1];
  const int c = threadIdx.x % LPR, slot = threadIdx.x / LPR, gr = slot % GR;
  const int64_t row = (int64_t)blockIdx.x * (JTH / LPR / GR) + slot / GR;
  const bool ok = row < a.rows;
  grid_dep_wait();
  grid_dep_launch();
  const int parts = ok ? a.S + a.So : 0;
  const float2* ml = a.part_ml + (ok ? row : 0);
  const float* po = a.part_o + (ok ? row : 0) * D + 4 * c;
  float M = -FLT_MAX, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int j = gr; j < parts; j += GR) {
    const float2 x = ml[j * a.rows];
    M = fmaxf(M, x.y != 0.f ? x.x : -FLT_MAX);
  }
#pragma unroll 4
  for (int j = gr; j < parts; j += GR) {
    const float2 x = ml[j * a.rows];
    const float4 v = *reinterpret_cast<const float4*>(po + j * a.rows * D);
    const float w = x.y != 0.f ? exp2f(x.x - M) : 0.f;
    l = fmaf(w, x.y, l);
    o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
  }
  if (GR > 1) {
    so[threadIdx.x] = o;
    if (c == 0) sml[slot] = make_float2(M, l);
    __syncthreads();
    if (gr == 0) {
      const float2* g = sml + slot;
#pragma unroll
      for (int j = 1; j < GR; ++j) M = fmaxf(M, g[j].y != 0.f ? g[j].x : -FLT_MAX);
      l = 0.f;
      o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        const float w = g[j].y != 0.f ? exp2f(g[j].x - M) : 0.f;
        const float4 v = so[threadIdx.x + j * LPR];
        l = fmaf(w, g[j].y, l);
        o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
      }
    }
  }
  if (!ok || gr) return;
  const int64_t b = row / (a.q * a.H * a.G), hq = row / a.q % (a.H * a.G), i = row % a.q;
  T* op = static_cast<T*>(a.O) + b * a.osb + hq * a.osh + i * a.oss + 4 * c;
  const float inv = l == 0.f ? 0.f : 1.f / l, y[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) from_f32(op[e], l == 0.f ? 0.f : y[e] * inv);
}

// Rows a CTA of the fp32 kernel: enough for the unit's rows, up to 128.
int simt_rows(const PrefixArgs& a) {
  const int r = std::max(a.R, a.Ro);
  return r <= 16 ? 16 : r <= 64 ? 64 : 128;
}

template <int CACHE, int D, int TR, bool PAGED>
cudaError_t launch_rows(const PrefixArgs& a, unsigned items, cudaStream_t s) {
  const auto k = simt_kernel<CACHE, D, TR, PAGED>;
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(k), simt_smem<D, TR>());
  return e != cudaSuccess ? e : Launch(dim3(items), kThreads<TR>, simt_smem<D, TR>(), s)(k, a);
}
template <int CACHE, int D, bool PAGED>
cudaError_t launch_simt(const PrefixArgs& a, cudaStream_t s) {
  const int64_t items = (int64_t)a.P * a.H * a.mt * a.S + (int64_t)a.B * a.H * a.mto * a.So;
  if (!items) return cudaSuccess;
  const int tr = simt_rows(a);
  return tr == 16 ? launch_rows<CACHE, D, 16, PAGED>(a, (unsigned)items, s)
         : tr == 64 ? launch_rows<CACHE, D, 64, PAGED>(a, (unsigned)items, s)
                    : launch_rows<CACHE, D, 128, PAGED>(a, (unsigned)items, s);
}
template <bool PAGED>
cudaError_t launch_cached(const PrefixPlan& p, cudaStream_t s) {
  const bool wide = p.a.d == 128;
  if (p.fmt == WF_MXFP8) return wide ? launch_simt<kFp8, 128, PAGED>(p.a, s) : launch_simt<kFp8, 64, PAGED>(p.a, s);
  if (p.fmt == WF_MXFP4) return wide ? launch_simt<kFp4, 128, PAGED>(p.a, s) : launch_simt<kFp4, 64, PAGED>(p.a, s);
  return wide ? launch_simt<kPlain, 128, PAGED>(p.a, s) : launch_simt<kPlain, 64, PAGED>(p.a, s);
}

template <typename T, int D>
cudaError_t launch_join(const PrefixArgs& a, cudaStream_t s) {
  constexpr int SLOTS = JTH / (D / 4);
  const bool many = a.S + a.So > 4;
  const int per = many ? 1 : SLOTS;
  Launch l(dim3((unsigned)((a.rows + per - 1) / per)), JTH, 0, s);
  return many ? l(join_kernel<T, D, SLOTS>, a) : l(join_kernel<T, D, 1>, a);
}

}  // namespace

PrefixPlan plan_prefix(const wf_tensor& q, const wf_tensor& kv, int k, int n_g) {
  PrefixPlan p = {};
  PrefixArgs& a = p.a;
  a.B = q.batch; a.P = kv.batch; a.H = kv.heads; a.G = q.heads / kv.heads;
  a.q = q.seq; a.d = q.head_dim; a.n = kv.seq; a.k = k; a.ng = n_g;
  a.each = a.B / a.P;
  a.Ro = a.G * a.q;
  a.R = a.each * a.Ro;
  a.by_q = make_fastdiv((uint32_t)a.q);
  a.by_Ro = make_fastdiv((uint32_t)a.Ro);
  a.rows = (int64_t)a.B * q.heads * a.q;
  p.dtype = q.dtype;
  p.fmt = kv.dtype;
  const bool tc = p.dtype == WF_BF16;
  const int tr = p.tr = tc ? kPrefixTcRows : simt_rows(a);
  a.mt = (a.R + tr - 1) / tr;
  a.mto = (a.Ro + tr - 1) / tr;
  // Parts: the count with the least estimated time, in us: waves of CTAs, each a
  // set-up and its key tiles, the parts' way through memory and, without own rows,
  // the joining kernel.  Measured at d = 128: a call of one tile 6 us, a key tile 1.5
  // with a row tile of 256 (products) or of 128 (the rows' bytes), a 64-key tile
  // of the fp32 kernel 13 for 128 rows; parts move at 5 TB/s; joining 2.5.
  const int tk = p.tk = tc ? kPrefixTcRows / 2 : TK, slots = tc || tr == 128 ? kPrefixSms : 2 * kPrefixSms;
  const double wide = a.d / 128.0, tile_us = wide * (tc ? 1.5 : tr == 128 ? 13.0 : tr == 64 ? 10.0 : 4.0);
  const double set_up = tc ? 5.0 : 4.0, part_us = (double)a.rows * a.d * 8 / 5e6;
  auto split = [&](int64_t units, int keys, double* least) {
    *least = 0.0;
    if (!keys) return 0;
    const int tiles = (keys + tk - 1) / tk;
    int best = 1;
    *least = 1e30;
    // The counts that fill one to four waves, and halves of them.
    for (int w = 1; w <= kWaves; ++w)
      for (int64_t most = std::max<int64_t>(1, w * slots / units); most; most /= 2) {
        const int per = (tiles + (int)std::min<int64_t>(most, tiles) - 1) / (int)std::min<int64_t>(most, tiles);
        const int S = (tiles + per - 1) / per;
        const double t = (double)((units * S + slots - 1) / slots) * (set_up + per * tile_us) +
                         (S > 1 || n_g ? S * part_us : 0.0) + (S > 1 && !n_g ? 2.5 : 0.0);
        if (t < *least) { *least = t; best = S; }
      }
    return best;
  };
  double prompt_us, own_us;
  a.S = split((int64_t)a.P * a.H * a.mt, k, &prompt_us);
  const int64_t own = (int64_t)a.B * a.H * a.mto;
  p.fold = tc && n_g > 0 && own >= kPrefixOwn && n_g <= std::min<int64_t>(2 * own, a.Ro <= 16 ? 512 : 256);
  a.So = p.fold ? 0 : split(own, n_g, &own_us);
  // Prompt rows that every sequence attends to for itself, where its own rows are
  // (one launch): a 64-key tile takes 1.25 us, or its bytes for all blocks of
  // query rows at the 2.4 TB/s that they come out of L2 with.  Measured, both ways:
  // 4 heads' tokens, 128 rows and 32 own ones 6.0 against 9.5 us, 400 and 32 10.8
  // against 10.1; blocks of 32 rows of 4 sequences and 16 heads on 128 rows 7.3
  // against 12.8, of 32 sequences on 400 rows 36 against 26.
  if (tc && p.fmt == WF_BF16 && k > 0 && k + n_g <= 1024) {
    auto direct = [&](int keys) {
      const double blocks = (double)a.B * a.H * ((a.Ro + prefix_own_rows(a, 0, keys) - 1) / prefix_own_rows(a, 0, keys));
      return ((keys + 63) / 64) * std::max(1.25, blocks * 256 * a.d / 2.4e6);
    };
    if (2.6 + direct(k + n_g) < prompt_us + (p.fold ? 3.2 + direct(n_g) : n_g ? 3.5 : 0.0)) {
      a.direct = 1;
      a.S = a.So = 0;
      p.fold = true;
    }
  }
  p.parts = a.S + a.So;
  a.by_H = make_fastdiv(a.H);
  a.by_S = make_fastdiv(std::max(1, a.S));
  a.by_So = make_fastdiv(std::max(1, a.So));
  a.by_mt = make_fastdiv(a.mt);
  a.by_mto = make_fastdiv(a.mto);
  a.whole = p.parts == 1 && !p.fold;
  const int64_t kept = a.whole ? 0 : a.rows * p.parts;  // rows of parts
  p.off_ml = 256;
  p.off_o = align_up(p.off_ml + sizeof(float2) * (size_t)kept, 256);
  p.used = p.off_o + sizeof(float) * (size_t)kept * a.d;
  // The size is the most that a call with as many keys and query rows, or fewer of
  // any, can take, so that one workspace serves them all: S itself is not monotone.
  // S units is at most kWaves slots where S > 1, and a unit has at most tr rows.
  const int64_t most = (int64_t)kWaves * (tc ? kPrefixSms * kPrefixTcRows : 2 * kPrefixSms * 64);
  auto room = [&](int keys, bool alone) {
    const int64_t tiles = (keys + tk - 1) / tk;
    return std::min(tiles * a.rows, alone ? most : std::max(a.rows, most));
  };
  const int64_t reserved = room(k, n_g == 0) + room(n_g, false);
  p.total = align_up(p.off_ml + sizeof(float2) * (size_t)reserved, 256) + sizeof(float) * (size_t)reserved * a.d;
  return p;
}

namespace {
cudaError_t join(const PrefixPlan& p, cudaStream_t s) {
  if (p.dtype == WF_BF16) return p.a.d == 128 ? launch_join<bf16, 128>(p.a, s) : launch_join<bf16, 64>(p.a, s);
  return p.a.d == 128 ? launch_join<float, 128>(p.a, s) : launch_join<float, 64>(p.a, s);
}
}  // namespace

cudaError_t launch_prefix(const PrefixPlan& p, cudaStream_t s) {
  const cudaError_t e = p.dtype == WF_BF16 ? launch_prefix_tc(p, s) : launch_cached<false>(p, s);
  if (e != cudaSuccess || p.a.whole) return e;
  return p.fold ? launch_prefix_own(p, s) : join(p, s);
}

PrefixPlan plan_tree(const wf_tensor& q, const wf_tensor& kv, int k, int n_t) {
  // fp32 queries: ranges and own units as wf_prefix_attn's.
  PrefixPlan p = plan_prefix(q, kv, k, n_t);
  if (p.dtype != WF_BF16) return p;
  PrefixArgs& a = p.a;
  a.S = a.So = a.direct = a.whole = 0;
  p.few = a.Ro <= kFewRows;
  a.tk = p.few ? few_keys(p.fmt) : kPrefixTcRows / 2;
  a.pad = p.few ? kFewPad : kTreePad;
  a.mt = (a.Ro + kPrefixTcRows - 1) / kPrefixTcRows;
  // Row tiles of equal height, whole warps of them.
  a.tr = a.mt == 1 ? a.Ro : ((a.Ro + a.mt - 1) / a.mt + 31) / 32 * 32;
  const int64_t U = (int64_t)a.B * a.H, items = U * a.mt;
  const int64_t tiles = std::max<int64_t>(1, ((int64_t)k + a.tk - 1) / a.tk + ((int64_t)n_t + a.tk - 1) / a.tk);
  a.C = (int)std::min<int64_t>(kPrefixSms * (p.few ? few_per_sm(a.d) : 1), items * tiles);
  p.join = tiles > 1;
  const size_t slots = (size_t)(a.C + items) * a.tr;
  p.off_info = 256;
  p.off_ml = align_up(p.off_info + (size_t)items * sizeof(int2) + (size_t)(a.C + items) * sizeof(int), 256);
  p.off_o = align_up(p.off_ml + sizeof(float2) * slots, 256);
  p.used = p.off_o + sizeof(float) * slots * a.d;
  // The size is the most that a call with as many rows and keys, or fewer of any, can take:
  // tr is R at most, or, with several row tiles, 256, and R + 32 mt in all.
  const int64_t most = kPrefixSms * few_per_sm(a.d);
  const int64_t reserved = most * std::min(a.Ro, kFewRows) +
                           kPrefixSms * (int64_t)std::min(a.Ro, kPrefixTcRows) + U * (a.Ro + (a.mt > 1 ? 32 * (int64_t)a.mt : 0));
  const size_t heads = align_up(p.off_info + (size_t)items * (sizeof(int2) + sizeof(int)) + (size_t)most * sizeof(int), 256);
  p.total = align_up(heads + sizeof(float2) * (size_t)reserved, 256) + sizeof(float) * (size_t)reserved * a.d;
  return p;
}

cudaError_t launch_tree(const PrefixPlan& p, cudaStream_t s) {
  if (p.dtype == WF_BF16) {
    const cudaError_t e = p.few ? launch_tree_few(p, s) : launch_tree_tc(p, s);
    return e != cudaSuccess || !(p.join || p.a.mask) ? e : launch_tree_join(p, s);
  }
  const cudaError_t e = launch_cached<true>(p, s);
  return e != cudaSuccess || p.a.whole ? e : join(p, s);
}

}  // namespace wf
