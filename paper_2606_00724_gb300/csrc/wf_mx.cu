// A cache in 8-bit or 4-bit codes: rows quantised as they are written
// (wf_cache_quantize) and read back (wf_cache_dequantize).
//
// Both move bytes and hardly compute, so they are bound by memory: a thread
// takes 16 bytes of the floating-point side (8 bf16 or 4 fp32 channels), so
// that a warp reads or writes 512 consecutive bytes there and the matching 128
// to 256 bytes of codes, and UN rows, all of them loaded before the first is
// used.  They are close to bound by instructions too (130 a thread and row filled
// 75 % of the issue slots), so the rows of a CTA that lie in one unit are found
// by adding strides, magnitudes are compared two at a time and codes are widened
// a word at a time.  The 4 or 8 lanes that share a block find its largest magnitude with
// shuffles, as integers: the bits of |x| are ordered as the values are, with
// infinities and NaN above them.
#include <algorithm>

#include "wf_div.cuh"
#include "wf_mx.cuh"
#include "wf_sm100.cuh"

namespace wf {
namespace {

constexpr int NTH = 256;

struct MxArgs {
  const void* src[2];    // K and V: fp32 / bf16 rows (quantise) or codes (read back)
  void* dst[2];          // codes or rows
  uint8_t* scales[2];
  int64_t fsb, fsh, fss; // strides of the fp32 / bf16 rows, in elements
  int64_t csb, csh, css; // strides of the codes, in bytes
  const int32_t* idx;    // [unit][rows] rows to read back, or null: pos + row
  int64_t pos;
  uint32_t total;        // rows of all units
  FastDiv rows, heads;   // rows a unit; heads
  int n;
};

// Unit, batch entry and head, and row within the unit of row r of all units.
struct At {
  uint32_t u, b, h, i;
};
__device__ __forceinline__ At row_at(const MxArgs& a, uint32_t r) {
  At w;
  w.u = fastdiv(r, a.rows);
  w.i = r - w.u * a.rows.d;
  w.b = fastdiv(w.u, a.heads);
  w.h = w.u - w.b * a.heads.d;
  return w;
}

// Bits of the largest magnitude of a thread's channels, as an fp32 number (a NaN
// wins over every number).
__device__ __forceinline__ uint32_t top_bits(const float*, const uint4& v) {
  return max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
}
__device__ __forceinline__ uint32_t top_bits(const bf16*, const uint4& v) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  return max(m & 0xffff0000u, m << 16);
}

template <int BYTES> struct Word;
template <> struct Word<8> { typedef uint2 type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// Codes of the N channels of one thread from their values in units of the scale.
template <bool FP4, int N>
__device__ __forceinline__ typename Word<FP4 ? N / 2 : N>::type pack_codes(const float* y) {
  constexpr int BITS = FP4 ? 8 : 16;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i * BITS / 32] |= mx_encode2<FP4>(y[2 * i], y[2 * i + 1]) << (i * BITS % 32);
  if constexpr (!FP4 && N == 8) return make_uint2(w[0], w[1]);
  else return (typename Word<FP4 ? N / 2 : N>::type)w[0];
}

// A thread's values from its codes and their scale byte, stored: bf16 by exact
// products of pairs, fp32 by way of half precision.
template <bool FP4>
__device__ __forceinline__ void put_values(bf16* out, const typename Word<FP4 ? 4 : 8>::type& c, uint32_t byte) {
  uint32_t y[4];
  if constexpr (FP4) {
    mx_pairs<true>(c, y);
  } else {
    mx_pairs<false>(c.x, y);
    mx_pairs<false>(c.y, y + 2);
  }
  const uint32_t f = mx_factor<FP4>(byte);
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = mul_bf16x2(y[i], f);
  if (byte > kMxOne<FP4>) {
    const uint32_t f2 = mx_second_factor<FP4>(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = mul_bf16x2(y[i], f2);
  }
  *reinterpret_cast<uint4*>(out) = make_uint4(y[0], y[1], y[2], y[3]);
}
template <bool FP4>
__device__ __forceinline__ void put_values(float* out, const typename Word<FP4 ? 2 : 4>::type& c, uint32_t byte) {
  const float s = mx_scale(byte);
  const float2 x = mx_decode2<FP4>(FP4 ? c & 0xffu : c & 0xffffu), y = mx_decode2<FP4>(FP4 ? c >> 8 : c >> 16);
  *reinterpret_cast<float4*>(out) = make_float4(x.x * s, x.y * s, y.x * s, y.y * s);
}

// Offsets of a thread's UN rows: of the fp32 / bf16 row, and of the row in the
// cache (unit, place).  RPC rows a pass of the CTA, first its first row.
template <int UN, int RPC>
struct Rows {
  int64_t f[UN], c[UN], s[UN];  // elements, bytes of codes, rows of scales
  __device__ __forceinline__ void find(const MxArgs& a, uint32_t first, int mine) {
    const At w = row_at(a, first);
    const uint32_t last = min(first + RPC * UN, a.total) - 1;
    if (w.i + (last - first) < a.rows.d) {  // all of one unit
      const uint32_t i0 = w.i + mine;
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        // Rows past the last repeat it.
        const uint32_t r = first + mine + RPC * i < a.total ? i0 + RPC * i : w.i + (last - first);
        f[i] = w.b * a.fsb + w.h * a.fsh + (int64_t)r * a.fss;
        c[i] = w.b * a.csb + w.h * a.csh + (a.pos + r) * a.css;
        s[i] = (int64_t)w.u * a.n + a.pos + r;
      }
    } else {
#pragma unroll
      for (int i = 0; i < UN; ++i) {
        const At x = row_at(a, min(first + mine + RPC * i, a.total - 1));
        f[i] = x.b * a.fsb + x.h * a.fsh + (int64_t)x.i * a.fss;
        c[i] = x.b * a.csb + x.h * a.csh + (a.pos + x.i) * a.css;
        s[i] = (int64_t)x.u * a.n + a.pos + x.i;
      }
    }
  }
};

template <typename T, bool FP4, int D, int UN>
__global__ void __launch_bounds__(NTH) quantize_kernel(const __grid_constant__ MxArgs a) {
  constexpr int N = Vec<T>::N;          // channels a thread
  constexpr int TPR = D / N;            // threads a row
  constexpr int TPB = kMxBlock / N;     // threads a block
  constexpr int RPC = NTH / TPR;        // rows a pass of the CTA
  typedef typename Word<FP4 ? N / 2 : N>::type W;
  const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR, y = blockIdx.y;
  const uint32_t first = blockIdx.x * (RPC * UN);
  Rows<UN, RPC> rows;
  rows.find(a, first, mine);
  sm100::grid_dep_wait();
  uint4 v[UN];
#pragma unroll
  for (int i = 0; i < UN; ++i)
    v[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.src[y]) + rows.f[i]) + t);
  sm100::grid_dep_launch();
#pragma unroll
  for (int i = 0; i < UN; ++i) {
    uint32_t top = top_bits(static_cast<const T*>(nullptr), v[i]);
#pragma unroll
    for (int s = 1; s < TPB; s *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
    const uint32_t byte = mx_scale_byte<FP4>(top);
    if (byte == 255) v[i] = make_uint4(0, 0, 0, 0);
    float x[N];
    widen_vec(static_cast<const T*>(nullptr), v[i], x);
    const float inv = mx_inv_scale(min(byte, 253u));
    const sm100::f32x2 inv2 = sm100::pk2(inv, inv);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const float2 p = sm100::up2(sm100::mul2(sm100::pk2(x[e], x[e + 1]), inv2));
      x[e] = p.x;
      x[e + 1] = p.y;
    }
    if (first + mine + RPC * i < a.total) {
      reinterpret_cast<W*>(static_cast<char*>(a.dst[y]) + rows.c[i])[t] = pack_codes<FP4, N>(x);
      if (t % TPB == 0) a.scales[y][rows.s[i] * (D / kMxBlock) + t / TPB] = (uint8_t)byte;
    }
  }
}

template <typename T, bool FP4, int D, int UN>
__global__ void __launch_bounds__(NTH) dequantize_kernel(const __grid_constant__ MxArgs a) {
  constexpr int N = Vec<T>::N, TPR = D / N, TPB = kMxBlock / N, RPC = NTH / TPR;
  typedef typename Word<FP4 ? N / 2 : N>::type W;
  const int t = threadIdx.x % TPR, mine = threadIdx.x / TPR, y = blockIdx.y;
  const uint32_t first = blockIdx.x * (RPC * UN);
  Rows<UN, RPC> rows;
  rows.find(a, first, mine);
  sm100::grid_dep_wait();
  if (a.idx) {
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int r = min(max(__ldg(a.idx + min(first + mine + RPC * i, a.total - 1)), 0), a.n - 1);
      const uint32_t u = fastdiv((uint32_t)min(first + mine + RPC * i, a.total - 1), a.rows), b = fastdiv(u, a.heads);
      rows.c[i] = b * a.csb + (u - b * a.heads.d) * a.csh + r * a.css;
      rows.s[i] = (int64_t)u * a.n + r;
    }
  }
  W c[UN];
  uint32_t byte[UN];
#pragma unroll
  for (int i = 0; i < UN; ++i) {
    c[i] = __ldg(reinterpret_cast<const W*>(static_cast<const char*>(a.src[y]) + rows.c[i]) + t);
    byte[i] = __ldg(a.scales[y] + rows.s[i] * (D / kMxBlock) + t / TPB);
  }
  sm100::grid_dep_launch();
#pragma unroll
  for (int i = 0; i < UN; ++i)
    if (first + mine + RPC * i < a.total) put_values<FP4>(static_cast<T*>(a.dst[y]) + rows.f[i] + t * N, c[i], byte[i]);
}

template <typename T, bool FP4, int D, bool BACK>
cudaError_t launch_un(const MxArgs& a, int tensors, cudaStream_t s) {
  constexpr int RPC = NTH / (D / Vec<T>::N);
  // Eight rows a thread from a wave of CTAs on (a 32K prompt of 32 heads: 127 us,
  // with four 132 to 136, with two 158); below that, as many threads as possible.
  const bool many = (int64_t)a.total * tensors > 8ll * RPC * 8 * sm_count();
  const int un = many ? 8 : 1;
  const dim3 grid((a.total + RPC * un - 1) / (RPC * un), (unsigned)tensors);
  Launch l(grid, NTH, 0, s);
  if (BACK) return many ? l(dequantize_kernel<T, FP4, D, 8>, a) : l(dequantize_kernel<T, FP4, D, 1>, a);
  return many ? l(quantize_kernel<T, FP4, D, 8>, a) : l(quantize_kernel<T, FP4, D, 1>, a);
}

template <bool BACK>
cudaError_t launch(const MxArgs& a, int dtype, int fmt, int d, int tensors, cudaStream_t s) {
  if (a.total == 0) return cudaSuccess;
  const bool fp4 = fmt == WF_MXFP4, wide = d == 128;
#define WF_MX(T)                                                                                       \
  (fp4 ? (wide ? launch_un<T, true, 128, BACK>(a, tensors, s) : launch_un<T, true, 64, BACK>(a, tensors, s)) \
       : (wide ? launch_un<T, false, 128, BACK>(a, tensors, s) : launch_un<T, false, 64, BACK>(a, tensors, s)))
  return dtype == WF_BF16 ? WF_MX(bf16) : WF_MX(float);
#undef WF_MX
}

MxArgs mx_args(const wf_tensor& f, const wf_tensor& kv) {
  MxArgs a = {};
  const int half = kv.dtype == WF_MXFP4 ? 2 : 1;  // strides of whole 16 bytes, so the division is exact
  a.fsb = f.stride_b; a.fsh = f.stride_h; a.fss = f.stride_s;
  a.csb = kv.stride_b / half; a.csh = kv.stride_h / half; a.css = kv.stride_s / half;
  a.total = (uint32_t)((int64_t)kv.batch * kv.heads * f.seq);
  a.rows = make_fastdiv((uint32_t)std::max(1, f.seq));
  a.heads = make_fastdiv((uint32_t)kv.heads);
  a.n = kv.seq;
  return a;
}

}  // namespace

cudaError_t launch_quantize(const void* Kn, const void* Vn, const wf_tensor& nt, void* Kc, void* Ks, void* Vc,
                            void* Vs, const wf_tensor& kv, int64_t pos, cudaStream_t s) {
  MxArgs a = mx_args(nt, kv);
  a.src[0] = Kn; a.src[1] = Vn;
  a.dst[0] = Kc; a.dst[1] = Vc;
  a.scales[0] = static_cast<uint8_t*>(Ks); a.scales[1] = static_cast<uint8_t*>(Vs);
  a.pos = pos;
  return launch<false>(a, nt.dtype, kv.dtype, kv.head_dim, Vn ? 2 : 1, s);
}

cudaError_t launch_dequantize(const void* Kc, const void* Ks, const void* Vc, const void* Vs, const wf_tensor& kv,
                              const int32_t* idx, int64_t pos, void* Ko, void* Vo, const wf_tensor& out,
                              cudaStream_t s) {
  MxArgs a = mx_args(out, kv);
  a.src[0] = Kc; a.src[1] = Vc;
  a.dst[0] = Ko; a.dst[1] = Vo;
  a.scales[0] = static_cast<uint8_t*>(const_cast<void*>(Ks));
  a.scales[1] = static_cast<uint8_t*>(const_cast<void*>(Vs));
  a.idx = idx;
  a.pos = pos;
  return launch<true>(a, out.dtype, kv.dtype, kv.head_dim, Vo ? 2 : 1, s);
}

}  // namespace wf
