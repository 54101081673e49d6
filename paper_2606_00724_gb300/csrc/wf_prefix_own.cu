// A sequence's own rows and the parts of its prompt, in one kernel (bf16).
//
// The own rows are few and differ from sequence to sequence, so their products
// are small: 16 to 64 query rows of one (sequence, key head) against tiles of 64
// keys.  A CTA of four warps takes such a block; with at most 16 or 32 rows the
// warps share the rows and divide the keys of each tile.  Blocks this size fill
// a small part of a 128-row tensor-memory tile and would pay its set-up, about
// 4 us a CTA with one CTA an SM; warp-level products (m16n8k16, fp32
// accumulators) keep S and O in registers, and four CTAs share an SM.
// The softmax is that of the prompt's kernel (base 2, running maximum), so what
// the warps found and the prompt's parts are put together with one set of
// weights 2^(m - M), and O is written here.
#include <float.h>

#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int NTH = 128;
constexpr int KT = 64;  // keys a tile

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Byte offset of 16-byte chunk ch of row r of a [rows][D] bf16 tile: chunks
// XOR-permuted by the row, so that the 8 rows of a matrix lie in 8 banks.
template <int D>
__device__ __forceinline__ uint32_t at(int r, int ch) { return (uint32_t)(r * (2 * D) + ((ch ^ (r & 7)) << 4)); }

template <int D, int WR>
constexpr size_t own_smem() {
  // Query rows, then two stages of a K and a V tile; the warps' O, m and l take
  // the stages' place.
  const size_t q = 16 * WR * D * 2, stages = 4 * KT * D * 2, o = (4 / WR) * 16 * WR * (D + 4) * 4;
  return q + (stages > o ? stages : o);
}

// WR warps along the rows, 4 / WR along the keys.
template <int D, int WR>
__global__ void __launch_bounds__(NTH) own_join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int WK = 4 / WR, RB = 16 * WR, CH = D / 8, KW = KT / WK, TILE = KT * D * 2, PO = D + 4;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float2 sml[4 * 16];  // m and l of every warp's rows
  __shared__ float sM[RB], sinv[RB];
  uint8_t* sq = smem;
  uint8_t* st = smem + RB * D * 2;
  float* so = reinterpret_cast<float*>(st);  // [WK][RB][PO]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rw = warp % WR, kw = warp / WR;
  const int nb = (a.Ro + RB - 1) / RB, u = blockIdx.x / nb, r0 = (blockIdx.x % nb) * RB, nr = min(RB, a.Ro - r0);
  const int b = u / a.H, h = u % a.H;
  grid_dep_wait();
  const int nk = own_count(a, b);
  const bf16* K = static_cast<const bf16*>(a.Kg) + b * a.gsb + h * a.gsh;
  const bf16* V = static_cast<const bf16*>(a.Vg) + b * a.gsb + h * a.gsh;

  auto fetch = [&](int t) {
    if (t * KT < nk) {
      const uint32_t base = smem_u32(st) + (t & 1) * 2 * TILE;
#pragma unroll
      for (int e = tid; e < KT * CH; e += NTH) {
        const int r = e / CH, ch = e % CH, j = t * KT + r;
        const int64_t o = j < nk ? (int64_t)j * a.gss + ch * 8 : 0;
        cp_async16_zfill(base + at<D>(r, ch), K + o, j < nk);
        cp_async16_zfill(base + TILE + at<D>(r, ch), V + o, j < nk);
      }
    }
    cp_async_commit();
  };
  if (nk > 0) {
    for (int e = tid; e < RB * CH; e += NTH) {
      const int r = e / CH, ch = e % CH;
      const RowAt w = own_row(a, u, r0 + min(r, nr - 1));
      cp_async16_zfill(smem_u32(sq) + at<D>(r, ch),
                       static_cast<const bf16*>(a.Q) + w.b * a.qsb + w.hq * a.qsh + w.i * a.qss + ch * 8, r < nr);
    }
  }
  fetch(0);
  fetch(1);

  uint32_t q[D / 16][4];
  float o[D / 8][4], m[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
#pragma unroll 1
  for (int t = 0; t * KT < nk; ++t) {
    cp_async_wait<1>();
    __syncthreads();
    if (t == 0) {
#pragma unroll
      for (int c = 0; c < D / 16; ++c) ldsm4(q[c], smem_u32(sq) + at<D>(rw * 16 + (lane & 15), 2 * c + (lane >> 4)));
    }
    const uint32_t kt = smem_u32(st) + (t & 1) * 2 * TILE, vt = kt + TILE;
    const int j0 = t * KT + kw * KW;
    if (j0 < nk) {
      float s[KW / 8][4];
#pragma unroll
      for (int n = 0; n < KW / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int n = 0; n < KW / 16; ++n) {
          uint32_t k4[4];  // keys 0-7: channels 0-7, 8-15; keys 8-15: the same
          ldsm4(k4, kt + at<D>(kw * KW + 16 * n + (lane & 7) + ((lane >> 4) << 3), 2 * c + ((lane >> 3) & 1)));
          mma16816(s[2 * n], q[c], k4[0], k4[1]);
          mma16816(s[2 * n + 1], q[c], k4[2], k4[3]);
        }
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int n = 0; n < KW / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (j0 + 8 * n + 2 * (lane & 3) + (e & 1) >= nk) s[n][e] = -INFINITY;
          top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
        top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
        const float mn = fmaxf(m[i], top[i] * a.sl2), f = ex2(m[i] - mn);
        m[i] = mn;
        l[i] *= f;
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
          o[c][2 * i] *= f;
          o[c][2 * i + 1] *= f;
        }
      }
#pragma unroll
      for (int n = 0; n < KW / 16; ++n) {
        uint32_t p[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {  // rows g (even x), g + 8; keys 0-7 (x < 2), 8-15
          const float* sv = s[2 * n + (x >> 1)] + 2 * (x & 1);
          const float p0 = ex2(fmaf(sv[0], a.sl2, -m[x & 1])), p1 = ex2(fmaf(sv[1], a.sl2, -m[x & 1]));
          l[x & 1] += p0 + p1;
          p[x] = pack_bf16(p0, p1);
        }
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
          uint32_t v4[4];  // channels 0-7: keys 0-7, 8-15; channels 8-15: the same
          ldsm4t(v4, vt + at<D>(kw * KW + 16 * n + (lane & 15), 2 * c + (lane >> 4)));
          mma16816(o[2 * c], p, v4[0], v4[1]);
          mma16816(o[2 * c + 1], p, v4[2], v4[3]);
        }
      }
    }
    __syncthreads();
    fetch(t + 2);
  }
  grid_dep_launch();
  cp_async_wait_all();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    const int r = rw * 16 + (lane >> 2) + 8 * i;
    float* row = so + (kw * RB + r) * PO + 2 * (lane & 3);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) *reinterpret_cast<float2*>(row + 8 * c) = make_float2(o[c][2 * i], o[c][2 * i + 1]);
    if ((lane & 3) == 0) sml[kw * RB + r] = make_float2(m[i], l[i]);
  }
  __syncthreads();
  // M and 1 / l of every row over the warps' and the prompt's parts, 8 threads
  // a row (RB = 16), 4 or 2.
  constexpr int TPR = NTH / RB;
  {
    const int r = tid / TPR, c = tid % TPR;
    const bool ok = r < nr;
    const int64_t flat = flat_row(a, own_row(a, u, r0 + (ok ? r : 0)));
    float M = -FLT_MAX, L = 0.f;
    auto take = [&](float2 ml) {
      if (ml.y == 0.f) return;
      const float mn = fmaxf(M, ml.x);
      L = L * ex2(M - mn) + ml.y * ex2(ml.x - mn);
      M = mn;
    };
    for (int j = c; j < WK; j += TPR) take(sml[j * RB + r]);
    for (int j = c; j < a.S; j += TPR) take(a.part_ml[j * a.rows + flat]);
#pragma unroll
    for (int x = 1; x < TPR; x *= 2) {
      const float m1 = __shfl_xor_sync(0xffffffffu, M, x), l1 = __shfl_xor_sync(0xffffffffu, L, x);
      const float mn = fmaxf(M, m1);
      L = L * ex2(M - mn) + l1 * ex2(m1 - mn);
      M = mn;
    }
    if (c == 0) {
      sM[r] = M;
      sinv[r] = L == 0.f ? 0.f : 1.f / L;
    }
  }
  __syncthreads();
  for (int e = tid; e < nr * (D / 4); e += NTH) {
    const int r = e / (D / 4), c = e % (D / 4);
    const RowAt w = own_row(a, u, r0 + r);
    const int64_t flat = flat_row(a, w);
    const float M = sM[r], inv = sinv[r];
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float2 ml, const float4& v) {
      const float f = ml.y == 0.f ? 0.f : ex2(ml.x - M) * inv;
      y.x = fmaf(f, v.x, y.x); y.y = fmaf(f, v.y, y.y); y.z = fmaf(f, v.z, y.z); y.w = fmaf(f, v.w, y.w);
    };
    for (int j = 0; j < WK; ++j)
      add(sml[j * RB + r], *reinterpret_cast<const float4*>(so + (j * RB + r) * PO + 4 * c));
#pragma unroll 4
    for (int j = 0; j < a.S; ++j)
      add(a.part_ml[j * a.rows + flat], *reinterpret_cast<const float4*>(a.part_o + (j * a.rows + flat) * D + 4 * c));
    *reinterpret_cast<uint2*>(static_cast<bf16*>(a.O) + w.b * a.osb + w.hq * a.osh + w.i * a.oss + 4 * c) =
        make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
  }
}

template <int D, int WR>
cudaError_t launch(const PrefixArgs& a, cudaStream_t s) {
  const size_t smem = own_smem<D, WR>();
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(own_join_kernel<D, WR>), smem);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)a.B * a.H * ((a.Ro + 16 * WR - 1) / (16 * WR));
  return Launch(dim3((unsigned)blocks), NTH, smem, s)(own_join_kernel<D, WR>, a);
}

template <int D>
cudaError_t launch_rows(const PrefixArgs& a, cudaStream_t s) {
  return a.Ro <= 16 ? launch<D, 1>(a, s) : a.Ro <= 32 ? launch<D, 2>(a, s) : launch<D, 4>(a, s);
}

}  // namespace

cudaError_t launch_prefix_own(const PrefixPlan& p, cudaStream_t s) {
  return p.a.d == 128 ? launch_rows<128>(p.a, s) : launch_rows<64>(p.a, s);
}

}  // namespace wf
