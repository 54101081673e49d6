// A sequence's own rows and the parts of its prompt, in one kernel (bf16).
//
// The own rows are few and differ from sequence to sequence, so their products
// are small: 16 to 64 query rows of one (sequence, key head) against tiles of 64
// keys.  A CTA of four warps takes such a block; with at most 16 or 32 rows the
// warps share the rows and divide the keys of each tile.  Blocks this size fill
// a small part of a 128-row tensor-memory tile and would pay its set-up, about
// 4 us a CTA with one CTA an SM; warp-level products (m16n8k16, fp32
// accumulators) keep S and O in registers, and four CTAs share an SM.
// P is one bf16 term, as in the prompt's kernel.
// Few prompt rows are attended here too, by every sequence for itself: one launch
// instead of two (see plan_prefix).
// The softmax is that of the prompt's kernel (base 2, running maximum), so what
// the warps found and the prompt's parts are put together with one set of
// weights 2^(m - M), and O is written here.
#include <float.h>

#include <type_traits>

#include "wf_prefix.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

using namespace sm100;

constexpr int NTH = 128;
constexpr int KT = 64;  // keys a tile

__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
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

// Query rows; one or two stages of a K and a V tile, whose place the warps' O
// take; the parts' m and l, then their weights.
template <int D, int WR>
size_t own_smem(int rows, int S, int keys) {
  const size_t q = 16 * WR * D * 2, stages = (keys > KT ? 4 : 2) * KT * D * 2;
  const size_t o = (4 / WR) * 16 * WR * (D + 4) * sizeof(float);
  return q + (stages > o ? stages : o) + (size_t)rows * (S + 4 / WR) * sizeof(float2);
}

// WR warps along the rows, 4 / WR along the keys.
template <int D, int WR>
__global__ void __launch_bounds__(NTH, WR == 4 ? 3 : 4) own_join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int WK = 4 / WR, RB = 16 * WR, CH = D / 8, KW = KT / WK, TILE = KT * D * 2, PO = D + 4;
  extern __shared__ __align__(128) uint8_t smem[];
  uint8_t* sq = smem;
  uint8_t* st = smem + RB * D * 2;
  float* so = reinterpret_cast<float*>(st);                      // [WK][RB][PO]
  const size_t room = max((size_t)(a.ng + (a.direct ? a.k : 0) > KT ? 4 : 2) * TILE, WK * RB * PO * sizeof(float));
  float2* sml = reinterpret_cast<float2*>(st + room);            // [a.ob][WK + S]: m and l, then the weight
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rw = warp % WR, kw = warp / WR;
  const int nb = (a.Ro + a.ob - 1) / a.ob, u = blockIdx.x / nb, r0 = (blockIdx.x % nb) * a.ob, nr = min(a.ob, a.Ro - r0);
  const int b = u / a.H, h = u % a.H;
  const int NP = WK + a.S;
  // Where the block's rows lie, found once.
  __shared__ int64_t row_q[RB], row_o[RB], row_flat[RB];
  if (tid < nr) {
    const RowAt w = own_row(a, b, h, r0 + tid);
    row_q[tid] = w.b * a.qsb + w.hq * a.qsh + w.i * a.qss;
    row_o[tid] = w.b * a.osb + w.hq * a.osh + w.i * a.oss;
    row_flat[tid] = flat_row(a, w);
  }
  grid_dep_wait();
  // Keys: the prompt's rows where they are attended here, then the own rows.
  const int p = b / a.each, np = a.direct ? prompt_count(a, p) : 0, nk = np + own_count(a, b);
  __syncthreads();
  // The parts' m and l and the query rows are on their way first: neither waits
  // for the length.
  for (int r = warp; r < nr; r += 4)
    for (int j = lane; j < a.S; j += 32)
      cp_async8(smem_u32(sml + r * NP + WK + j), a.part_ml + j * a.rows + row_flat[r]);
  const bf16* K = static_cast<const bf16*>(a.Kg) + b * a.gsb + h * a.gsh;
  const bf16* V = static_cast<const bf16*>(a.Vg) + b * a.gsb + h * a.gsh;
  const int64_t prompt = p * a.ksb + h * a.ksh;
  const int32_t* idx = a.idx ? a.idx + (int64_t)(p * a.H + h) * a.k : nullptr;

  auto fetch = [&](int t) {
    if (t * KT < nk) {
      const uint32_t base = smem_u32(st) + (t & 1) * 2 * TILE;
#pragma unroll
      for (int e = tid; e < KT * CH; e += NTH) {
        const int r = e / CH, ch = e % CH, j = t * KT + r;
        const bf16 *ka = K, *va = V;
        if (j < np) {
          const int64_t o = prompt + (idx ? min(max(__ldg(idx + j), 0), a.n - 1) : j) * a.kss + ch * 8;
          ka = static_cast<const bf16*>(a.K) + o;
          va = static_cast<const bf16*>(a.V) + o;
        } else if (j < nk) {
          const int64_t o = (int64_t)(j - np) * a.gss + ch * 8;
          ka += o;
          va += o;
        } else if (np) {  // no address is read past the last key; one that exists is given
          ka = static_cast<const bf16*>(a.K) + prompt;
          va = static_cast<const bf16*>(a.V) + prompt;
        }
        cp_async16_zfill(base + at<D>(r, ch), ka, j < nk);
        cp_async16_zfill(base + TILE + at<D>(r, ch), va, j < nk);
      }
    }
    cp_async_commit();
  };
  if (a.ng > 0 || a.direct) {
    for (int e = tid; e < RB * CH; e += NTH) {
      const int r = e / CH, ch = e % CH;
      cp_async16_zfill(smem_u32(sq) + at<D>(r, ch), static_cast<const bf16*>(a.Q) + row_q[min(r, nr - 1)] + ch * 8,
                       r < nr);
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
    // Without weight, O is 0 x V, which is NaN where V is not finite.
    const bool none = l[i] == 0.f;
#pragma unroll
    for (int c = 0; c < D / 8; ++c)
      *reinterpret_cast<float2*>(row + 8 * c) = none ? make_float2(0.f, 0.f) : make_float2(o[c][2 * i], o[c][2 * i + 1]);
    if ((lane & 3) == 0 && r < nr) sml[r * (WK + a.S) + kw] = make_float2(m[i], l[i]);
  }
  __syncthreads();
  // Weights 2^(m - M) / sum of 2^(m - M) l of a row's parts, 4 lanes a row; a part
  // without a key (l = 0) has weight 0.
  for (int r = tid >> 2; r < RB; r += NTH / 4) {
    float2* ml = sml + min(r, nr - 1) * NP;
    const int c = tid & 3;
    float M = -FLT_MAX, L = 0.f;
    for (int j = c; j < NP; j += 4) M = fmaxf(M, ml[j].y != 0.f ? ml[j].x : -FLT_MAX);
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 1));
    M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 2));
    for (int j = c; j < NP; j += 4) L += ml[j].y != 0.f ? ex2(ml[j].x - M) * ml[j].y : 0.f;
    L += __shfl_xor_sync(0xffffffffu, L, 1);
    L += __shfl_xor_sync(0xffffffffu, L, 2);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (r < nr)
      for (int j = c; j < NP; j += 4) ml[j].x = ml[j].y != 0.f ? ex2(ml[j].x - M) * inv : 0.f;
  }
  __syncthreads();
  // O, a group of 4 channels a thread or 4 of them, with 16 loads of parts in
  // flight either way.
  const int items = nr * (D / 4);
  auto out = [&](auto groups) {
    constexpr int EB = decltype(groups)::value, PB = 16 / EB;
    for (int e0 = tid; e0 < items; e0 += EB * NTH) {
      float4 y[EB];
      const float* po[EB];
      const float2* wt[EB];
#pragma unroll
      for (int x = 0; x < EB; ++x) {
        const int e = min(e0 + x * NTH, items - 1), r = e / (D / 4), c = e % (D / 4);
        po[x] = a.part_o + row_flat[r] * D + 4 * c;
        wt[x] = sml + r * NP;
        y[x] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      auto add = [&](int x, float f, const float4& v) {
        y[x].x = fmaf(f, v.x, y[x].x); y[x].y = fmaf(f, v.y, y[x].y);
        y[x].z = fmaf(f, v.z, y[x].z); y[x].w = fmaf(f, v.w, y[x].w);
      };
      for (int j = 0; j < a.S; j += PB) {
        float4 v[PB][EB];
#pragma unroll
        for (int k = 0; k < PB; ++k)
#pragma unroll
          for (int x = 0; x < EB; ++x)
            v[k][x] = j + k < a.S ? *reinterpret_cast<const float4*>(po[x] + (j + k) * a.rows * D)
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < PB; ++k)
#pragma unroll
          for (int x = 0; x < EB; ++x) add(x, j + k < a.S ? wt[x][WK + j + k].x : 0.f, v[k][x]);
      }
#pragma unroll
      for (int x = 0; x < EB; ++x) {
        const int e = e0 + x * NTH, r = e / (D / 4), c = e % (D / 4);
        if (e >= items) break;
#pragma unroll
        for (int j = 0; j < WK; ++j)
          add(x, wt[x][j].x, *reinterpret_cast<const float4*>(so + (j * RB + r) * PO + 4 * c));
        *reinterpret_cast<uint2*>(static_cast<bf16*>(a.O) + row_o[r] + 4 * c) =
            make_uint2(pack_bf16(y[x].x, y[x].y), pack_bf16(y[x].z, y[x].w));
      }
    }
  };
  if (items <= NTH) out(std::integral_constant<int, 1>());
  else out(std::integral_constant<int, 4>());
}

template <int D, int WR>
cudaError_t launch(const PrefixArgs& a, cudaStream_t s) {
  const size_t smem = own_smem<D, WR>(a.ob, a.S, a.ng + (a.direct ? a.k : 0));
  const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(own_join_kernel<D, WR>), smem);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)a.B * a.H * ((a.Ro + a.ob - 1) / a.ob);
  return Launch(dim3((unsigned)blocks), NTH, smem, s)(own_join_kernel<D, WR>, a);
}

template <int D>
cudaError_t launch_rows(PrefixArgs a, cudaStream_t s) {
  a.ob = prefix_own_rows(a, a.S, a.ng + (a.direct ? a.k : 0));
  return a.ob <= 16 ? launch<D, 1>(a, s) : a.ob == 32 ? launch<D, 2>(a, s) : launch<D, 4>(a, s);
}

}  // namespace

// The unit's rows, up to 64; blocks of 16 where fewer CTAs than SMs were left; down
// to 4 where the parts are more bytes than the keys that every block reads
// again (one token of 28 heads on 4, 37 parts: 15 -> 6 us).
int prefix_own_rows(const PrefixArgs& a, int S, int keys) {
  int ob = a.Ro <= 16 ? 16 : a.Ro <= 32 ? 32 : 64;
  auto blocks = [&] { return (int64_t)a.B * a.H * ((a.Ro + ob - 1) / ob); };
  while (ob > 16 && blocks() < kPrefixSms) ob /= 2;
  while (ob > 4 && blocks() < 2 * kPrefixSms && ob * S > keys) ob /= 2;
  return ob;
}

cudaError_t launch_prefix_own(const PrefixPlan& p, cudaStream_t s) {
  return p.a.d == 128 ? launch_rows<128>(p.a, s) : launch_rows<64>(p.a, s);
}

}  // namespace wf
