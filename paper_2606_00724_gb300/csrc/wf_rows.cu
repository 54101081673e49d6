// Rotary positions (wf_rotary_apply) and rows written into the pages of a cache
// with the rotation on the way (wf_paged_append).
//
// Pair i of a row turns by pos f_i: (x, y) -> (x c - y s, y c + x s).  A position
// is a whole number and a plan holds a position's turn as a fraction of 2^64, so
// their product modulo 2^64 is the angle, exactly, however far the position is;
// what is left of it is an eighth of a turn at most to either side and goes
// through fp32.
//
// Both move bytes: 16 of them a thread, so that a row is 8 to 32 lanes and a
// rotated channel's partner comes from another lane.  The angles belong to the
// row, not to a head, so a thread keeps its chunk's cosines and sines and takes
// the same chunk of several heads, whose addresses differ by a stride, UN of them on
// their way while UN are worked on.  Bound by HBM: 2 prompts of 8K and 32 heads into
// bf16 pages 89 us (6.0 TB/s), 25K rows of 32 heads rotated 73 (a plain copy of their bytes
// takes 67); into codes by instructions as well (the same prompts 79 us in 8 bits, 61 at the
// memory's rate, and 79 to 81 in 4 bits, 51).
#include <algorithm>
#include <type_traits>

#include "wf_mx.cuh"
#include "wf_rows.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

constexpr int NTH = 256;

// Cosine and sine of a fraction t / 2^64 of a turn: of the part beyond the nearest
// quarter turn, at most pi / 4 = x, by their series in x^2 (the first terms left
// out are x^12 / 12! < 2^-33 and x^11 / 11! < 2^-29).  x and its square are held in two
// numbers and what 1 - x^2 / 2 rounds off is added back, so that the last sum's rounding is
// nearly all that is lost: 0.9 of 2^-24 at most, where a plain x left 1.6, and of 67M codes of rotated keys
// 60 to 92 are other than exact arithmetic's, where that left 87 to 117.  A row's heads share it: 25K rows of 32
// heads 72.6 us for 72.1, 32 single rows 3.2 for 3.1.
__device__ __forceinline__ void turned(unsigned long long t, float& c, float& s) {
  constexpr double kUnit = 3.14159265358979323846 / 2147483648.0;  // 2 pi / 2^32
  constexpr float kHigh = (float)kUnit, kLow = (float)(kUnit - (double)kHigh);
  const uint32_t hi = (uint32_t)(t >> 32), q = (hi + 0x20000000u) >> 30;
  const int k = (int32_t)(hi - (q << 30));
  const float kf = (float)k, kl = (float)(k - (int)kf);
  const float x = __fmul_rn(kf, kHigh), xl = fmaf(kf, kHigh, -x) + fmaf(kf, kLow, kl * kHigh);
  const float y = __fmul_rn(x, x), yl = fmaf(x, x, -y);
  float c1 = -1.f / 3628800.f, s0 = 1.f / 362880.f;
  c1 = fmaf(c1, y, 1.f / 40320.f);
  s0 = fmaf(s0, y, -1.f / 5040.f);
  c1 = fmaf(c1, y, -1.f / 720.f);
  s0 = fmaf(s0, y, 1.f / 120.f);
  c1 = fmaf(c1, y, 1.f / 24.f);
  s0 = fmaf(s0, y, -1.f / 6.f);
  const float w = fmaf(-0.5f, y, 1.f), wl = fmaf(-0.5f, y, 1.f - w);
  const float c0 = __fadd_rn(w, wl + fmaf(y * y, c1, -fmaf(xl, x, 0.5f * yl)));
  s0 = __fadd_rn(x, fmaf(__fmul_rn(s0, y), x, xl * w));
  c = q & 1 ? -s0 : c0;
  s = q & 1 ? c0 : s0;
  if (q & 2) { c = -c; s = -s; }
}

// max(|a|, |b|, |c|), NaN if one of them is.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
  float r;
  asm("{\n\t.reg .f32 x, y, z;\n\t"
      "abs.f32 x, %1;\n\tabs.f32 y, %2;\n\tabs.f32 z, %3;\n\t"
      "max.NaN.f32 %0, x, y, z;\n\t}"
      : "=f"(r)
      : "f"(a), "f"(b), "f"(c));
  return r;
}

// The first head of tensor 1 in the line of both tensors' heads g, g + groups, ..
__device__ __forceinline__ int second_head(uint32_t g, const RowsArgs& a) {
  const int in = a.heads[0] - (int)g;  // line places from g to tensor 1
  return in <= 0 ? -in : (in + a.groups - 1) / a.groups * a.groups - in;
}

enum Kept { kRows, kFp8, kFp4 };

template <typename T, int KEPT, int D, int UN>
__global__ void __launch_bounds__(NTH, KEPT == kRows ? 3 : 4) rows_kernel(const __grid_constant__ RowsArgs a) {
  constexpr int N = Vec<T>::N;       // channels a thread
  constexpr int TPR = D / N;         // threads a row
  constexpr int RPC = NTH / TPR;     // rows a CTA
  constexpr bool FP4 = KEPT == kFp4;
  typedef typename Word<FP4 ? N / 2 : N>::type W;
  const T* const type = nullptr;
  const int t = threadIdx.x % TPR;
  // The CTA's heads, the same for all of its rows, so that its warps stay together.
  const uint32_t block = fastdiv(blockIdx.x, a.by_groups), g = blockIdx.x - block * a.groups;
  const uint32_t mine = block * RPC + threadIdx.x / TPR;
  bool ok = mine < a.total;
  const uint32_t r = ok ? mine : 0;
  const uint32_t b = fastdiv(r, a.by_m), i = r - b * a.by_m.d;
  sm100::grid_dep_wait();
  const int row = a.rows_at ? min(max(__ldg(a.rows_at + r), 0), a.rows - 1) : (int)i;
  // Where the row goes: row i of its batch entry, or the row of a page.
  int64_t place = i, to = b;
  if (a.pages) {
    if (a.count) ok = ok && (int)i < __ldg(a.count + b);
    place += __ldg(a.start + b);
    ok = ok && place >= 0 && place < (int64_t)a.table * a.by_ps.d;
    const uint32_t entry = ok ? fastdiv((uint32_t)place, a.by_ps) : 0;
    const int page = __ldg(a.pages + (int64_t)b * a.table + entry);
    ok = ok && page >= 0 && page < a.pool;
    to = page;
  }
  const int64_t in = a.pages ? place - (int64_t)fastdiv((uint32_t)place, a.by_ps) * a.by_ps.d : place;

  // This chunk's angles, and the chunk of the channels that it turns with.
  float c[N], s[N];
  int partner = t;
  bool turns = false;
  if (a.plan) {
    const int half = a.pairs / N;  // chunks of first (or second) channels
    turns = t < 2 * half;
    if (turns && !a.adjacent) partner = t < half ? t + half : t - half;
    if (turns) {
      const int first = a.adjacent ? t * (N / 2) : min(t, partner) * N;
#pragma unroll
      for (int e = 0; e < (N); ++e) {
        if (a.adjacent && e >= N / 2) break;
        const ulonglong2 p = __ldg(reinterpret_cast<const ulonglong2*>(a.plan) + first + e);
        const int axis = min(max((int)p.y, 0), a.axes - 1);
        const long long pos = a.pos ? __ldg(a.pos + ((int64_t)axis * a.B + b) * a.rows + row) : place;
        turned((unsigned long long)pos * p.x, c[e], s[e]);
        if (!a.adjacent && t < half) s[e] = -s[e];
      }
    }
  }

  if (!__any_sync(0xffffffffu, ok)) {  // a warp whose rows are all past their counts reads none
    sm100::grid_dep_launch();
    return;
  }
  // The thread's heads, of both tensors in one line: g, g + groups, ..  Addresses go from one to
  // the next by a stride; formed anew they were half of the instructions.
#pragma unroll 1
  for (int w = 0; w < 2; ++w) {
    const int heads = a.heads[w], h0 = w ? second_head(g, a) : (int)g;
    if (h0 >= heads) continue;
    const bool turn = a.plan && (!w || a.both);
    const int64_t sstep = a.ssh[w] * a.groups, dstep = a.dsh[w] * a.groups;
    const T* src = static_cast<const T*>(a.src[w]) + b * a.ssb[w] + h0 * a.ssh[w] + row * a.sss[w] + t * N;
    typedef typename std::conditional<KEPT == kRows, T, char>::type Out;
    Out* dst = static_cast<Out*>(a.dst[w]) + to * a.dsb[w] + h0 * a.dsh[w] + in * a.dss[w] + t * (KEPT == kRows ? N : (int)sizeof(W));
    uint8_t* scale = nullptr;
    int64_t zstep = 0;
    if (KEPT != kRows) {
      zstep = (int64_t)a.by_ps.d * (D / kMxBlock) * a.groups;
      scale = a.scales[w] + ((to * heads + h0) * (int64_t)a.by_ps.d + in) * (D / kMxBlock);
    }
    // The next UN rows are on their way while UN are worked on.
    uint4 v[UN], next[UN];
    auto load = [&](int h) {
#pragma unroll
      for (int x = 0; x < UN; ++x) {
        next[x] = make_uint4(0, 0, 0, 0);
        if (h + x * a.groups < heads) next[x] = *reinterpret_cast<const uint4*>(src + x * sstep);
      }
      src += UN * sstep;
    };
    load(h0);
#pragma unroll 1
    for (int h = h0; h < heads; h += UN * a.groups) {
#pragma unroll
      for (int x = 0; x < UN; ++x) v[x] = next[x];
      load(h + UN * a.groups);
#pragma unroll
      for (int x = 0; x < UN; ++x) {
        const bool put = ok && h + x * a.groups < heads;
        float y[N];
        widen_vec(type, v[x], y);
        if (!a.adjacent && turn) {
          uint4 u;
          u.x = __shfl_sync(0xffffffffu, v[x].x, partner, TPR);
          u.y = __shfl_sync(0xffffffffu, v[x].y, partner, TPR);
          u.z = __shfl_sync(0xffffffffu, v[x].z, partner, TPR);
          u.w = __shfl_sync(0xffffffffu, v[x].w, partner, TPR);
          float z[N];
          widen_vec(type, u, z);
          if (turns) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = fmaf(y[e], c[e], z[e] * s[e]);
          }
        } else if (turn && turns) {
#pragma unroll
          for (int e = 0; e < N / 2; ++e) {
            const float p = y[2 * e], q = y[2 * e + 1];
            y[2 * e] = fmaf(p, c[e], -q * s[e]);
            y[2 * e + 1] = fmaf(q, c[e], p * s[e]);
          }
        }
        if constexpr (KEPT == kRows) {
          if (put) st_vec(dst, y);
        } else {
          constexpr int TPB = kMxBlock / N;  // threads a block
          uint32_t top;
          if (turn) {
            float y0 = 0.f;
#pragma unroll
            for (int e = 0; e < N; e += 2) y0 = max_abs(y0, y[e], y[e + 1]);
            top = __float_as_uint(y0) & 0x7fffffffu;
          } else {
            top = top_bits(type, v[x]);
          }
#pragma unroll
          for (int d = 1; d < TPB; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
          const uint32_t byte = mx_scale_byte<FP4>(top);
          const float inv = byte == 255 ? 0.f : mx_inv_scale(byte);
          const sm100::f32x2 inv2 = sm100::pk2(inv, inv);
#pragma unroll
          for (int e = 0; e < N; e += 2) {
            const float2 p = sm100::up2(sm100::mul2(sm100::pk2(y[e], y[e + 1]), inv2));
            y[e] = p.x;
            y[e + 1] = p.y;
          }
          if (byte == 255) {  // nothing finite to keep
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = 0.f;
          }
          uint32_t bytes = byte << 8 * (t / TPB);
#pragma unroll
          for (int d = TPB; d < TPR; d *= 2) bytes |= __shfl_xor_sync(0xffffffffu, bytes, d);
          if (put) {
            *reinterpret_cast<W*>(dst) = pack_codes<FP4, N>(y);
            if (t == 0) {  // the row's scales in one store
              if (D == 128) *reinterpret_cast<uint32_t*>(scale) = bytes;
              else *reinterpret_cast<uint16_t*>(scale) = (uint16_t)bytes;
            }
          }
          scale += zstep;
        }
        dst += dstep;
      }
    }
  }
  sm100::grid_dep_launch();
}

template <typename T, int KEPT, int D>
cudaError_t launch_rows(RowsArgs& a, cudaStream_t s) {
  constexpr int TPR = D / Vec<T>::N, RPC = NTH / TPR;
  const int heads = a.heads[0] + a.heads[1];
  // Heads a thread: as many as leave about a wave of threads.
  const int64_t wave = (int64_t)sm_count() * 1536 / TPR;
  const int64_t groups = std::min<int64_t>(heads, std::max<int64_t>(1, wave / a.total));
  a.each = (int)((heads + groups - 1) / groups);
  a.groups = (heads + a.each - 1) / a.each;
  a.by_groups = make_fastdiv((uint32_t)a.groups);
  const dim3 grid((unsigned)(((int64_t)a.total + RPC - 1) / RPC * a.groups));
  Launch l(grid, NTH, 0, s);
  // Codes are bound by instructions as well, and gain more from a fourth CTA an SM than from
  // four rows in flight (two prompts of 8K, 32 heads: 88 against 92 us).
  constexpr int UN = KEPT == kRows ? 4 : 2;
  return a.each >= UN ? l(rows_kernel<T, KEPT, D, UN>, a) : l(rows_kernel<T, KEPT, D, 1>, a);
}

template <typename T, int D>
cudaError_t launch_kept(RowsArgs& a, int cache, cudaStream_t s) {
  return cache == WF_MXFP8 ? launch_rows<T, kFp8, D>(a, s)
         : cache == WF_MXFP4 ? launch_rows<T, kFp4, D>(a, s)
                             : launch_rows<T, kRows, D>(a, s);
}

}  // namespace

cudaError_t launch_rotate(RowsArgs a, int dtype, int d, cudaStream_t s) {
  const bool wide = d == 128;
  if (dtype == WF_BF16) return wide ? launch_rows<bf16, kRows, 128>(a, s) : launch_rows<bf16, kRows, 64>(a, s);
  return wide ? launch_rows<float, kRows, 128>(a, s) : launch_rows<float, kRows, 64>(a, s);
}

cudaError_t launch_append(RowsArgs a, int dtype, int cache, int d, cudaStream_t s) {
  const bool wide = d == 128;
  if (dtype == WF_BF16) return wide ? launch_kept<bf16, 128>(a, cache, s) : launch_kept<bf16, 64>(a, cache, s);
  return wide ? launch_kept<float, 128>(a, cache, s) : launch_kept<float, 64>(a, cache, s);
}

}  // namespace wf
