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

constexpr int NTH = 256;
constexpr int TK = 64;  // keys a tile

// How prompt rows are kept: like the own rows, or in codes.
enum Cache { kPlain, kFp8, kFp4 };

// 4 consecutive channels (4 c ..) of a row, in fp32.
__device__ __forceinline__ float4 row4(const float* p, int c) { return __ldg(reinterpret_cast<const float4*>(p) + c); }
template <bool FP4>
__device__ __forceinline__ float4 code4(const uint8_t* p, const uint8_t* scales, int c) {
  const uint32_t w = FP4 ? __ldg(reinterpret_cast<const uint16_t*>(p) + c) : __ldg(reinterpret_cast<const uint32_t*>(p) + c);
  const float s = mx_scale(__ldg(scales + c / 8));
  const float2 x = mx_decode2<FP4>(FP4 ? w & 0xffu : w & 0xffffu), y = mx_decode2<FP4>(FP4 ? w >> 8 : w >> 16);
  return make_float4(x.x * s, x.y * s, y.x * s, y.y * s);
}

template <int D, int TR>
constexpr size_t simt_smem() {
  return sizeof(float) * (TR * (D + 4) + TK * (D + 4) + TK * D + TR * (TK + 4));
}

// Thread (ty, tx) = (tid / 16, tid % 16) owns rows ty RT .. + RT of the tile,
// keys tx + 16 j of a key tile and channels 4 tx + 64 j of O.
template <typename T, int CACHE, int D, int TR>
__global__ void __launch_bounds__(NTH, 2) simt_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int RT = TR / 16, PITCH = D + 4, PP = TK + 4, C = D / 64;
  extern __shared__ __align__(16) float sm[];
  float* sq = sm;                // [TR][PITCH]
  float* sk = sq + TR * PITCH;   // [TK][PITCH]
  float* sv = sk + TK * PITCH;   // [TK][D]
  float* sp = sv + TK * D;       // [TR][PP]
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  // The CTA's unit, row tile and part.
  const int prompts = a.P * a.H * a.mt * a.S;
  int it = blockIdx.x;
  const bool own = it >= prompts;
  if (own) it -= prompts;
  const int mt = own ? a.mto : a.mt, S = own ? a.So : a.S;
  const int tile = it % mt, sp_i = (it / mt) % S, u = it / mt / S;
  const int r0 = tile * TR, nr = min(TR, (own ? a.Ro : a.R) - r0);
  grid_dep_wait();
  const int count = own ? own_count(a, u / a.H) : prompt_count(a, u / a.H);
  const int tiles = (count + TK - 1) / TK, per = (tiles + S - 1) / S;
  const int k0 = min(count, sp_i * per * TK), k1 = min(count, (sp_i + 1) * per * TK);

  for (int e = tid; e < TR * (D / 4); e += NTH) {
    const int r = e / (D / 4), c = e % (D / 4);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < nr) {
      const RowAt w = own ? own_row(a, u / a.H, u % a.H, r0 + r) : prompt_row(a, u / a.H, u % a.H, r0 + r);
      v = row4(static_cast<const T*>(a.Q) + w.b * a.qsb + w.hq * a.qsh + w.i * a.qss, c);
    }
    *reinterpret_cast<float4*>(sq + r * PITCH + 4 * c) = v;
  }

  float m[RT], l[RT], o[RT][4 * C];
#pragma unroll
  for (int i = 0; i < RT; ++i) {
    m[i] = -FLT_MAX;  // finite, so that logits of -inf add 0 and not 2^(-inf + inf)
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * C; ++c) o[i][c] = 0.f;
  }
#pragma unroll 1
  for (int t0 = k0; t0 < k1; t0 += TK) {
    const int nk = min(TK, k1 - t0);
    __syncthreads();  // the last tile's readers
    for (int e = tid; e < TK * (D / 4); e += NTH) {
      const int r = e / (D / 4), c = e % (D / 4);
      float4 kv = make_float4(0.f, 0.f, 0.f, 0.f), vv = kv;
      if (r < nk) {
        if (own) {
          const int64_t at = (int64_t)(u / a.H) * a.gsb + (int64_t)(u % a.H) * a.gsh + (int64_t)(t0 + r) * a.gss;
          kv = row4(static_cast<const T*>(a.Kg) + at, c);
          vv = row4(static_cast<const T*>(a.Vg) + at, c);
        } else {
          int row = t0 + r;
          if (a.idx) row = min(max(__ldg(a.idx + (int64_t)u * a.k + row), 0), a.n - 1);
          const int64_t at = (int64_t)(u / a.H) * a.ksb + (int64_t)(u % a.H) * a.ksh + (int64_t)row * a.kss;
          if (CACHE == kPlain) {
            kv = row4(static_cast<const T*>(a.K) + at, c);
            vv = row4(static_cast<const T*>(a.V) + at, c);
          } else {
            const int64_t sa = ((int64_t)u * a.n + row) * (D / kMxBlock);
            kv = code4<CACHE == kFp4>(static_cast<const uint8_t*>(a.K) + at, a.Ks + sa, c);
            vv = code4<CACHE == kFp4>(static_cast<const uint8_t*>(a.V) + at, a.Vs + sa, c);
          }
        }
      }
      *reinterpret_cast<float4*>(sk + r * PITCH + 4 * c) = kv;
      *reinterpret_cast<float4*>(sv + r * D + 4 * c) = vv;
    }
    __syncthreads();
    // Logits: even and odd channels in packed FMAs, chains of four of them
    // summed with a running correction.  A logit of 100 has a unit of 2^-17 in
    // fp32; a plain sum of 128 products would leave an error of several of them,
    // and the softmax turns it into a relative error of the weights.
    f32x2 s2[RT][4], e2[RT][4];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s2[i][j] = e2[i][j] = 0ull;
#pragma unroll 1
    for (int c = 0; c < D; c += 8) {
      ulonglong2 ka[4], kb[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float* kr = sk + (tx + 16 * j) * PITCH + c;
        ka[j] = *reinterpret_cast<const ulonglong2*>(kr);
        kb[j] = *reinterpret_cast<const ulonglong2*>(kr + 4);
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float* qr = sq + (ty * RT + i) * PITCH + c;
        const ulonglong2 qa = *reinterpret_cast<const ulonglong2*>(qr), qb = *reinterpret_cast<const ulonglong2*>(qr + 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x2 x = fma2(qb.y, kb[j].y, fma2(qb.x, kb[j].x, fma2(qa.y, ka[j].y, mul2(qa.x, ka[j].x))));
          const f32x2 y = add2(x, e2[i][j]), t = add2(s2[i][j], y);
          e2[i][j] = sub2(y, sub2(t, s2[i][j]));
          s2[i][j] = t;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float s[4], low[4], top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = up2(s2[i][j]), e = up2(e2[i][j]);
        float h = v.x + v.y;
        const float z = h - v.x;
        low[j] = ((v.x - (h - z)) + (v.y - z)) + (e.x + e.y);  // what h has not got
        if (!(fabsf(h) <= FLT_MAX)) {  // an infinity in the rows makes the correction NaN: the plain sum
          h = low[j] = 0.f;
          for (int c = 0; c < D; ++c) h = fmaf(sq[(ty * RT + i) * PITCH + c], sk[(tx + 16 * j) * PITCH + c], h);
        }
        s[j] = tx + 16 * j < nk ? h : -INFINITY;
        top = fmaxf(top, s[j]);
      }
#pragma unroll
      for (int w = 1; w < 16; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
      const float mn = fmaxf(m[i], top * a.sl2), f = exp2f(m[i] - mn);
      m[i] = mn;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = s[j] == -INFINITY ? 0.f : exp2f(fmaf(low[j], a.sl2, fmaf(s[j], a.sl2, -mn)));
        sum += p;
        sp[(ty * RT + i) * PP + tx + 16 * j] = p;
      }
      l[i] = l[i] * f + sum;  // this thread's keys; the 16 threads of the row are summed at the end
#pragma unroll
      for (int c = 0; c < 4 * C; ++c) o[i][c] *= f;
    }
    __syncwarp();  // a row's P is written and read by one half-warp
#pragma unroll 2
    for (int j = 0; j < TK; ++j) {
      float4 vv[C];
#pragma unroll
      for (int c = 0; c < C; ++c) vv[c] = *reinterpret_cast<const float4*>(sv + j * D + 4 * tx + 64 * c);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float p = sp[(ty * RT + i) * PP + j];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          o[i][4 * c] = fmaf(p, vv[c].x, o[i][4 * c]);
          o[i][4 * c + 1] = fmaf(p, vv[c].y, o[i][4 * c + 1]);
          o[i][4 * c + 2] = fmaf(p, vv[c].z, o[i][4 * c + 2]);
          o[i][4 * c + 3] = fmaf(p, vv[c].w, o[i][4 * c + 3]);
        }
      }
    }
  }
  grid_dep_launch();
#pragma unroll
  for (int i = 0; i < RT; ++i) {
#pragma unroll
    for (int w = 1; w < 16; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
    const int r = ty * RT + i;
    if (r >= nr) continue;
    const RowAt w = own ? own_row(a, u / a.H, u % a.H, r0 + r) : prompt_row(a, u / a.H, u % a.H, r0 + r);
    if (a.whole) {
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
      T* op = static_cast<T*>(a.O) + w.b * a.osb + w.hq * a.osh + w.i * a.oss;
#pragma unroll
      for (int c = 0; c < 4 * C; ++c) from_f32(op[4 * tx + 64 * (c / 4) + c % 4], l[i] == 0.f ? 0.f : o[i][c] * inv);
    } else {
      const int64_t at = (int64_t)(own ? a.S + sp_i : sp_i) * a.rows + flat_row(a, w);
#pragma unroll
      for (int c = 0; c < C; ++c)
        *reinterpret_cast<float4*>(a.part_o + at * D + 4 * tx + 64 * c) =
            make_float4(o[i][4 * c], o[i][4 * c + 1], o[i][4 * c + 2], o[i][4 * c + 3]);
      if (tx == 0) a.part_ml[at] = make_float2(m[i], l[i]);
    }
  }
}

// O of every query row from its parts: with M the largest m, the sum of
// 2^(m - M) O over that of 2^(m - M) l.  A part without a key (l = 0) adds
// nothing, and a row without any is 0.  D / 4 threads a row.
template <typename T, int D>
__global__ void __launch_bounds__(NTH) join_kernel(const __grid_constant__ PrefixArgs a) {
  const int c = threadIdx.x % (D / 4);
  const int64_t row = (int64_t)blockIdx.x * (NTH / (D / 4)) + threadIdx.x / (D / 4);
  grid_dep_wait();
  grid_dep_launch();
  if (row >= a.rows) return;
  const int parts = a.S + a.So;
  float M = -FLT_MAX;
  for (int j = 0; j < parts; ++j) {
    const float2 ml = a.part_ml[j * a.rows + row];
    if (ml.y != 0.f) M = fmaxf(M, ml.x);
  }
  float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j = 0; j < parts; ++j) {
    const float2 ml = a.part_ml[j * a.rows + row];
    if (ml.y == 0.f) continue;
    const float w = exp2f(ml.x - M);
    const float4 v = *reinterpret_cast<const float4*>(a.part_o + (j * a.rows + row) * D + 4 * c);
    l = fmaf(w, ml.y, l);
    o[0] = fmaf(w, v.x, o[0]); o[1] = fmaf(w, v.y, o[1]); o[2] = fmaf(w, v.z, o[2]); o[3] = fmaf(w, v.w, o[3]);
  }
  const int64_t b = row / (a.q * a.H * a.G), hq = row / a.q % (a.H * a.G), i = row % a.q;
  T* op = static_cast<T*>(a.O) + b * a.osb + hq * a.osh + i * a.oss + 4 * c;
  const float inv = 1.f / l;
#pragma unroll
  for (int e = 0; e < 4; ++e) from_f32(op[e], l == 0.f ? 0.f : o[e] * inv);
}

template <int CACHE, int D>
cudaError_t launch_simt(const PrefixArgs& a, cudaStream_t s) {
  const int64_t items = (int64_t)a.P * a.H * a.mt * a.S + (int64_t)a.B * a.H * a.mto * a.So;
  if (!items) return cudaSuccess;
  const bool few = (a.R > a.Ro ? a.R : a.Ro) <= 16;
  const auto k = few ? simt_kernel<float, CACHE, D, 16> : simt_kernel<float, CACHE, D, 64>;
  const size_t smem = few ? simt_smem<D, 16>() : simt_smem<D, 64>();
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(k), smem);
  return e != cudaSuccess ? e : Launch(dim3((unsigned)items), NTH, smem, s)(k, a);
}

cudaError_t launch_parts(const PrefixPlan& p, cudaStream_t s) {
  const bool wide = p.a.d == 128;
  if (p.dtype == WF_BF16) return launch_prefix_tc(p, s);
  if (p.fmt == WF_MXFP8) return wide ? launch_simt<kFp8, 128>(p.a, s) : launch_simt<kFp8, 64>(p.a, s);
  if (p.fmt == WF_MXFP4) return wide ? launch_simt<kFp4, 128>(p.a, s) : launch_simt<kFp4, 64>(p.a, s);
  return wide ? launch_simt<kPlain, 128>(p.a, s) : launch_simt<kPlain, 64>(p.a, s);
}

template <typename T, int D>
cudaError_t launch_join(const PrefixArgs& a, cudaStream_t s) {
  const int per = NTH / (D / 4);
  return Launch(dim3((unsigned)((a.rows + per - 1) / per)), NTH, 0, s)(join_kernel<T, D>, a);
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
  const int tr = tc ? kPrefixTcRows : (a.R > a.Ro ? a.R : a.Ro) <= 16 ? 16 : 64;
  a.mt = (a.R + tr - 1) / tr;
  a.mto = (a.Ro + tr - 1) / tr;
  // Splits: as many parts as fill the SMs once (one CTA an SM, two of the fp32
  // kernel), of at least two tiles of 128 keys each.
  const int slots = tc ? 152 : 304;
  auto split = [&](int64_t units, int keys) {
    if (!keys) return 0;
    const int64_t most = std::max(1, (keys + 255) / 256);
    return (int)std::min(most, std::max<int64_t>(1, slots / units));
  };
  a.S = split((int64_t)a.P * a.H * a.mt, k);
  p.fold = tc && n_g > 0 && n_g <= kPrefixFold;
  a.So = p.fold ? 0 : split((int64_t)a.B * a.H * a.mto, n_g);
  p.parts = a.S + a.So;
  a.by_H = make_fastdiv(a.H);
  a.by_S = make_fastdiv(std::max(1, a.S));
  a.by_So = make_fastdiv(std::max(1, a.So));
  a.by_mt = make_fastdiv(a.mt);
  a.by_mto = make_fastdiv(a.mto);
  a.whole = p.parts == 1 && !p.fold;
  p.off_ml = 256;
  const int kept = a.whole ? 0 : p.parts;
  p.off_o = align_up(p.off_ml + sizeof(float2) * (size_t)a.rows * kept, 256);
  p.total = p.off_o + sizeof(float) * (size_t)a.rows * a.d * kept;
  return p;
}

cudaError_t launch_prefix(const PrefixPlan& p, cudaStream_t s) {
  const cudaError_t e = launch_parts(p, s);
  if (e != cudaSuccess || p.a.whole) return e;
  if (p.fold) return launch_prefix_own(p, s);
  if (p.dtype == WF_BF16) return p.a.d == 128 ? launch_join<bf16, 128>(p.a, s) : launch_join<bf16, 64>(p.a, s);
  return p.a.d == 128 ? launch_join<float, 128>(p.a, s) : launch_join<float, 64>(p.a, s);
}

}  // namespace wf
