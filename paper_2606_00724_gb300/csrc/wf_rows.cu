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
// the same chunk of several heads, UN of them loaded before the first is used.
#include <algorithm>

#include "wf_mx.cuh"
#include "wf_rows.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

constexpr int NTH = 256;

// Cosine and sine of a fraction t / 2^64 of a turn: of the part beyond the nearest
// quarter turn, at most pi / 4 = x, by their series in x^2 (the first terms left
// out are x^12 / 12! < 2^-33 and x^11 / 11! < 2^-29).
__device__ __forceinline__ void turned(unsigned long long t, float& c, float& s) {
  const uint32_t hi = (uint32_t)(t >> 32), q = (hi + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(hi - (q << 30)) * (0x1p-31f * 3.14159265358979f), y = x * x;
  float c0 = -1.f / 3628800.f, s0 = 1.f / 362880.f;
  c0 = fmaf(c0, y, 1.f / 40320.f);
  s0 = fmaf(s0, y, -1.f / 5040.f);
  c0 = fmaf(c0, y, -1.f / 720.f);
  s0 = fmaf(s0, y, 1.f / 120.f);
  c0 = fmaf(c0, y, 1.f / 24.f);
  s0 = fmaf(s0, y, -1.f / 6.f);
  c0 = fmaf(c0, y, -0.5f);
  s0 = fmaf(s0 * y, x, x);
  c0 = fmaf(c0, y, 1.f);
  c = q & 1 ? -s0 : c0;
  s = q & 1 ? c0 : s0;
  if (q & 2) { c = -c; s = -s; }
}

enum Kept { kRows, kFp8, kFp4 };

template <typename T, int KEPT, int D, int UN>
__global__ void __launch_bounds__(NTH) rows_kernel(const __grid_constant__ RowsArgs a) {
  constexpr int N = Vec<T>::N;       // channels a thread
  constexpr int TPR = D / N;         // threads a row
  constexpr int RPC = NTH / TPR;     // rows a CTA
  constexpr bool FP4 = KEPT == kFp4;
  typedef typename Word<FP4 ? N / 2 : N>::type W;
  const T* const type = nullptr;
  const int t = threadIdx.x % TPR;
  const uint32_t item = blockIdx.x * RPC + threadIdx.x / TPR;
  bool ok = item < a.total * a.groups;
  const uint32_t at = ok ? item : 0;
  const uint32_t r = fastdiv(at, a.by_groups), g = at - r * a.groups;
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

  const int heads = a.heads[0] + a.heads[1];
#pragma unroll 1
  for (int k = 0; k < a.each; k += UN) {
    uint4 v[UN];
#pragma unroll
    for (int x = 0; x < UN; ++x) {
      const int hh = min((int)g + a.groups * (k + x), heads - 1), w = hh >= a.heads[0], h = w ? hh - a.heads[0] : hh;
      v[x] = *(reinterpret_cast<const uint4*>(static_cast<const T*>(a.src[w]) + b * a.ssb[w] + h * a.ssh[w] +
                                              row * a.sss[w]) + t);
    }
#pragma unroll
    for (int x = 0; x < UN; ++x) {
      const int hh = (int)g + a.groups * (k + x), w = hh >= a.heads[0], h = w ? hh - a.heads[0] : hh;
      const bool put = ok && hh < heads && k + x < a.each, turn = a.plan && (!w || a.both);
      float y[N];
      widen_vec(type, v[x], y);
      if (!a.adjacent && __any_sync(0xffffffffu, turn)) {  // the rows of a warp may be of both tensors
        uint4 u;
        u.x = __shfl_sync(0xffffffffu, v[x].x, partner, TPR);
        u.y = __shfl_sync(0xffffffffu, v[x].y, partner, TPR);
        u.z = __shfl_sync(0xffffffffu, v[x].z, partner, TPR);
        u.w = __shfl_sync(0xffffffffu, v[x].w, partner, TPR);
        float z[N];
        widen_vec(type, u, z);
        if (turn && turns) {
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
      if (KEPT == kRows) {
        if (put) st_vec(static_cast<T*>(a.dst[w]) + to * a.dsb[w] + h * a.dsh[w] + in * a.dss[w] + t * N, y);
      } else {
        constexpr int TPB = kMxBlock / N;  // threads a block
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
#pragma unroll
        for (int d = 1; d < TPB; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
        const uint32_t byte = mx_scale_byte<FP4>(top);
        const float inv = byte == 255 ? 0.f : mx_inv_scale(byte);
#pragma unroll
        for (int e = 0; e < N; ++e) y[e] = byte == 255 ? 0.f : y[e] * inv;
        if (put) {
          reinterpret_cast<W*>(static_cast<char*>(a.dst[w]) + to * a.dsb[w] + h * a.dsh[w] + in * a.dss[w])[t] =
              pack_codes<FP4, N>(y);
          if (t % TPB == 0)
            a.scales[w][(((to * a.heads[w]) + h) * a.by_ps.d + in) * (D / kMxBlock) + t / TPB] = (uint8_t)byte;
        }
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
  const dim3 grid((unsigned)(((int64_t)a.total * a.groups + RPC - 1) / RPC));
  Launch l(grid, NTH, 0, s);
  return a.each >= 4 ? l(rows_kernel<T, KEPT, D, 4>, a) : l(rows_kernel<T, KEPT, D, 1>, a);
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
