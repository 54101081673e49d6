// The parts of wf_tree_attn's bf16 queries put together.
//
// With M the largest m of a row's parts, O is the sum of 2^(m - M) O over that of
// 2^(m - M) l; a part without weight (l = 0) adds nothing, and a row without any is 0.
// A row that is one part was written by the kernel before, which is all that its warp
// finds here.  D / 4 lanes hold a row; where a row may have many parts, GR groups
// of them take every GR-th part and the first adds them up, in their order: from eight parts
// on that a row has where all sequences are equally long.  One group against eight, the whole call: a token of one
// sequence of 8K (38 parts) 20.7 and 16.1 us, of 128K 95 and 89; 182 rows of 8 sequences (4.75) 63 and 74; 64-wide
// heads of 32 sequences (1.8) 96 and 135.  One long sequence among many short ones counts as equal lengths do: a
// token of one of 128K and 63 of 64 rows, one key head, 74 and 29.
//
// Bound by two loads one after the other, the item's place and its parts: 2 to 5 us behind the
// kernel before, where attending the drafted rows here as well had taken 12 to 16.
//
// Drafted values that are not finite were left out of the products (see not_finite), so
// where a part says so they are added here, to the rows that see them.
#include <float.h>

#include <algorithm>

#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int NTH = 256;

// The sum of the values of channel ch that are not finite, of the drafted rows that
// row i of sequence b sees; 0 if there are none.
__device__ __noinline__ float left_out(const PrefixArgs& a, int b, int h, int i, int ch) {
  const bf16* v = static_cast<const bf16*>(a.Vg) + b * a.gsb + h * a.gsh + ch;
  float sum = 0.f;
  for (int j = 0; j < own_count(a, b); ++j) {
    const float x = to_f32(v[j * a.gss]);
    if (!(fabsf(x) <= FLT_MAX) && sees(a, b, i, j)) sum += x;
  }
  return sum;
}

template <int D, int GR>
__global__ void __launch_bounds__(NTH) tree_join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int LPR = D / 4, ROWS = NTH / LPR / GR;
  __shared__ float4 so[GR > 1 ? NTH : 1];
  __shared__ float2 sml[GR > 1 ? NTH / LPR : 1];
  const int c = threadIdx.x % LPR, group = threadIdx.x / LPR, gr = group % GR;
  const int64_t row = (int64_t)blockIdx.x * ROWS + group / GR;
  const bool ok = row < a.rows;
  const uint32_t flat = ok ? (uint32_t)row : 0;
  const uint32_t unit = fastdiv(flat, a.by_Ro), r = flat - unit * a.Ro;  // rows of a unit follow each other: [B][H][G][q]
  const uint32_t b = fastdiv(unit, a.by_H), h = unit - b * a.H, hg = fastdiv(r, a.by_q), i = r - hg * a.q;
  const uint32_t tile = a.mt > 1 ? r / a.tr : 0;
  grid_dep_wait();
  grid_dep_launch();
  const int2 info = __ldcg(a.info + (int64_t)unit * a.mt + tile);
  // A kernel whose wait gave up may have left its info unwritten.
  const bool known = info.x >= 0 && info.y > 0 && (int64_t)info.x + info.y <= a.C + (int64_t)a.B * a.H * a.mt;
  const int parts = known ? info.y : 0;
  int flag = 0;
  if (a.mask)
    for (int j = c; j < parts; j += LPR) flag |= __ldcg(a.flags + info.x + j);
  const int64_t first = (known ? (int64_t)info.x * a.tr : 0) + (r - tile * a.tr);
  const float2* ml = a.part_ml + first;
  const float* po = a.part_o + first * D + 4 * c;
  bf16* op = static_cast<bf16*>(a.O) + b * a.osb + (h * a.G + hg) * (int64_t)a.osh + i * a.oss + 4 * c;
  const uint32_t lanes = LPR == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);
  flag = __any_sync(lanes, flag);
  if (parts == 1 && !flag && GR == 1) return;
  float M = -FLT_MAX, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (parts > 1) {
    for (int j = gr + GR * c; j < parts; j += GR * LPR) {
      const float2 x = __ldcg(ml + (int64_t)j * a.tr);
      if (x.y != 0.f) M = fmaxf(M, x.x);
    }
#pragma unroll
    for (int w = 1; w < LPR; w *= 2) M = fmaxf(M, __shfl_xor_sync(lanes, M, w));
#pragma unroll 8
    for (int j = gr; j < parts; j += GR) {
      const float2 x = __ldcg(ml + (int64_t)j * a.tr);
      const float4 v = __ldcg(reinterpret_cast<const float4*>(po + (int64_t)j * a.tr * D));
      const float w = x.y != 0.f ? ex2(x.x - M) : 0.f;
      l = fmaf(w, x.y, l);
      o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
    }
  }
  if (GR > 1) {
    so[threadIdx.x] = o;
    if (c == 0) sml[group] = make_float2(M, l);
    __syncthreads();
    if (gr == 0 && parts > 1) {
#pragma unroll
      for (int j = 1; j < GR; ++j) M = fmaxf(M, sml[group + j].y != 0.f ? sml[group + j].x : -FLT_MAX);
      l = 0.f;
      o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int j = 0; j < GR; ++j) {
        const float2 x = sml[group + j];
        const float4 v = so[threadIdx.x + j * LPR];
        const float w = x.y != 0.f ? ex2(x.x - M) : 0.f;
        l = fmaf(w, x.y, l);
        o.x = fmaf(w, v.x, o.x); o.y = fmaf(w, v.y, o.y); o.z = fmaf(w, v.z, o.z); o.w = fmaf(w, v.w, o.w);
      }
    }
  }
  if (!ok || gr || (parts == 1 && !flag)) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  float y[4] = {o.x * inv, o.y * inv, o.z * inv, o.w * inv};
  if (parts == 1) {
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to_f32(op[e]);
  }
  if (flag && (parts == 1 ? __ldcg(ml).y : l) != 0.f) {
    for (int e = 0; e < 4; ++e) y[e] += left_out(a, b, h, i, 4 * c + e);
  }
  *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
}

template <int D>
cudaError_t launch(const PrefixArgs& a, cudaStream_t s) {
  // Parts of a row where all sequences are equally long.
  const bool many = a.C / std::max<int64_t>(1, (int64_t)a.B * a.H * a.mt) >= 8;
  const int per = NTH / (D / 4) / (many ? 8 : 1);
  Launch l(dim3((unsigned)((a.rows + per - 1) / per)), NTH, 0, s);
  return many ? l(tree_join_kernel<D, 8>, a) : l(tree_join_kernel<D, 1>, a);
}

}  // namespace

cudaError_t launch_tree_join(const PrefixPlan& p, cudaStream_t s) {
  return p.a.d == 128 ? launch<128>(p.a, s) : launch<64>(p.a, s);
}

}  // namespace wf
