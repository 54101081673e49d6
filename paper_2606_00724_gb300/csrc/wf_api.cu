// libwf C ABI: argument checks, workspace planning and stream-ordered
// launches.  Nothing here allocates device memory or synchronises the stream.
#include <math.h>
#include <string.h>

#include <atomic>
#include <map>
#include <mutex>
#include <utility>

#include "wf_internal.cuh"
#include "wf_mx.cuh"
#include "wf_prefix.cuh"
#include "wf_rows.cuh"
#include "wf_testing.h"

#define WF_API extern "C" __attribute__((visibility("default")))

namespace {

using wf::align_up;

int elem_size(int dtype) { return dtype == WF_BF16 ? 2 : 4; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Shape, dtype and alignment of one descriptor (seq may be 0 when allow_empty).
wf_status check_desc(const wf_tensor* t, bool allow_empty) {
  if (!t) return WF_ERR_INVALID_ARG;
  if (t->dtype != WF_F32 && t->dtype != WF_BF16) return WF_ERR_DTYPE;
  if (t->batch < 1 || t->heads < 1 || t->seq < (allow_empty ? 0 : 1)) return WF_ERR_SHAPE;
  if (t->head_dim != 64 && t->head_dim != 128) return WF_ERR_SHAPE;
  if (t->stride_b < 0 || t->stride_h < 0 || t->stride_s < 0) return WF_ERR_SHAPE;
  const int64_t es = elem_size(t->dtype);
  if ((t->stride_b * es) % 16 || (t->stride_h * es) % 16 || (t->stride_s * es) % 16) return WF_ERR_ALIGN;
  if (t->seq > 1 && t->stride_s < t->head_dim) return WF_ERR_SHAPE;
  return WF_OK;
}

bool quantised(const wf_tensor* t) { return t->dtype == WF_MXFP8 || t->dtype == WF_MXFP4; }

// The same of a quantised cache's codes (strides in elements, rows and strides
// of whole 16 bytes).
wf_status check_codes(const wf_tensor* t) {
  if (!t) return WF_ERR_INVALID_ARG;
  if (!quantised(t)) return WF_ERR_DTYPE;
  if (t->batch < 1 || t->heads < 1 || t->seq < 1) return WF_ERR_SHAPE;
  if (t->head_dim != 64 && t->head_dim != 128) return WF_ERR_SHAPE;
  if (t->stride_b < 0 || t->stride_h < 0 || t->stride_s < 0) return WF_ERR_SHAPE;
  const int64_t unit = t->dtype == WF_MXFP4 ? 32 : 16;  // elements of 16 bytes
  if (t->stride_b % unit || t->stride_h % unit || t->stride_s % unit) return WF_ERR_ALIGN;
  if (t->seq > 1 && t->stride_s < t->head_dim) return WF_ERR_SHAPE;
  return WF_OK;
}

bool same_units(const wf_tensor* a, const wf_tensor* b) {
  return a->batch == b->batch && a->heads == b->heads && a->head_dim == b->head_dim;
}

// Query heads per KV head (grouped-query attention), or 0 if the query
// descriptor q cannot be grouped onto kv.
int group_of(const wf_tensor* q, const wf_tensor* kv) {
  if (q->batch != kv->batch || q->head_dim != kv->head_dim || q->heads % kv->heads) return 0;
  return q->heads / kv->heads;
}

wf_status check_levels(const wf_tensor* kv, int levels) {
  if (levels < 1 || levels > 10) return WF_ERR_UNSUPPORTED;
  const int64_t n = kv->seq;
  if ((n >> levels) < 1 || ((n >> levels) << levels) != n) return WF_ERR_SHAPE;
  return WF_OK;
}

wf_status check_keep(int64_t n, int levels, const int32_t* keep) {
  if (!keep) return WF_ERR_INVALID_ARG;
  int64_t cnt = n >> levels;
  for (int l = levels; l >= 1; --l) {
    if (keep[l] < 1 || keep[l] > cnt) return WF_ERR_SCHEDULE;
    cnt = 2 * (int64_t)keep[l];
  }
  if (keep[0] < 1 || keep[0] > cnt) return WF_ERR_SCHEDULE;
  return WF_OK;
}

wf_status cuda_status(cudaError_t e) { return e == cudaSuccess ? WF_OK : WF_ERR_CUDA; }

// Number of SMs of the current device.
bool device_sms(int* sms) {
  *sms = wf::sm_count();
  return *sms > 0;
}

int64_t ceil_guarded(double v) { return (int64_t)ceil(v - 1e-9); }

}  // namespace

namespace wf {

cudaError_t raise_smem_limit(const void* kernel, size_t smem) {
  static std::mutex mu;
  static std::map<std::pair<int, const void*>, size_t> raised;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::lock_guard<std::mutex> lock(mu);
  size_t& cur = raised[std::make_pair(dev, kernel)];
  if (cur >= smem) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e == cudaSuccess) cur = smem;
  return e;
}

int sm_count() {
  static std::mutex mu;
  static std::map<int, int> cache;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  std::lock_guard<std::mutex> lock(mu);
  auto it = cache.find(dev);
  if (it != cache.end()) return it->second;
  int n = 0;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n = 0;
  cache.emplace(dev, n);
  return n;
}

}  // namespace wf

namespace {

wf_status check_filter_args(const wf_tensor* q, const wf_tensor* kv, int levels, const int32_t* keep) {
  wf_status st;
  if ((st = check_desc(q, false)) != WF_OK) return st;
  if ((st = check_desc(kv, false)) != WF_OK) return st;
  const int G = group_of(q, kv);
  if (!G) return WF_ERR_SHAPE;
  if (q->dtype != kv->dtype) return WF_ERR_DTYPE;
  if (q->seq > wf::kMaxQ || (int64_t)G * q->seq > wf::kMaxQR) return WF_ERR_UNSUPPORTED;
  if ((st = check_levels(kv, levels)) != WF_OK) return st;
  return check_keep(kv->seq, levels, keep);
}

wf_status check_attn_args(const wf_tensor* q, const wf_tensor* kv, int k, const wf_tensor* g, int n_g,
                          const wf_tensor* o) {
  wf_status st;
  if ((st = check_desc(q, false)) != WF_OK) return st;
  if ((st = check_desc(kv, false)) != WF_OK) return st;
  if ((st = check_desc(o, false)) != WF_OK) return st;
  if (!group_of(q, kv) || !same_units(q, o) || o->seq != q->seq) return WF_ERR_SHAPE;
  if (q->dtype != kv->dtype || o->dtype != q->dtype) return WF_ERR_DTYPE;
  if (q->seq > wf::kMaxQ) return WF_ERR_UNSUPPORTED;
  if (k < 1 || k > kv->seq || n_g < 0) return WF_ERR_INVALID_ARG;
  if (n_g > 0) {
    if ((st = check_desc(g, true)) != WF_OK) return st;
    if (!same_units(kv, g) || g->seq != n_g) return WF_ERR_SHAPE;
    if (g->dtype != q->dtype) return WF_ERR_DTYPE;
  }
  return WF_OK;
}

// The skim and scan of one layer in one launch where a plan has it (the fused
// kernel without its attention for one query head per key head, the fp32
// kernel, the grouped filter kernel), else three kernels a scale; wf_filter's
// scratch beyond the status word is used by these only.  The fp32 and the
// grouped plan compare the routes where the kernels per scale catch up; the
// fused kernel is faster wherever it applies: 32 heads x 20K tokens, filter then
// attention, 152 us with 13 launches for the filter and two for the attention,
// 57 us with one each.
cudaError_t run_filter(const wf::FilterPlan& p, const void* Q, const wf_tensor& q, const void* coeffs, const void* K,
                       const wf_tensor& kv, int levels, const int32_t* keep, int32_t* idx, int32_t* level_sets,
                       void* scratch, int* status, int sms, cudaStream_t s) {
  if (q.heads == kv.heads) {
    const wf::FusedPlan fp = wf::plan_stage(q, kv, levels, keep, -1, sms);
    if (fp.ok) {
      wf::FusedRange r{};
      r.lev_top = levels;
      r.lev_bot = fp.trim ? 0 : 1;
      r.final_sel = 1;
      return wf::launch_stage(fp, Q, q, K, nullptr, kv, nullptr, nullptr, nullptr, coeffs, levels, keep, idx,
                              level_sets, nullptr, q, status, s, &r);
    }
  }
  const wf::F32Plan f32 = wf::plan_f32(q, kv, levels, keep, -1, sms);
  if (f32.ok)
    return wf::launch_f32(f32, Q, q, K, nullptr, kv, nullptr, nullptr, nullptr, coeffs, levels, keep, idx, level_sets,
                          nullptr, q, s);
  const wf::GqaPlan gp = wf::plan_gqa(q, kv, levels, keep, sms);
  if (gp.ok) return wf::launch_gqa_filter(gp, Q, q, K, kv, coeffs, levels, keep, idx, level_sets, status, s);
  return wf::launch_filter(p, Q, q, coeffs, K, kv, idx, level_sets, scratch, status, s);
}

}  // namespace

WF_API const char* wf_status_str(int status) {
  switch (status) {
    case WF_OK: return "WF_OK";
    case WF_ERR_INVALID_ARG: return "WF_ERR_INVALID_ARG: missing pointer or bad count";
    case WF_ERR_SHAPE: return "WF_ERR_SHAPE: shapes disagree or are unsupported";
    case WF_ERR_DTYPE: return "WF_ERR_DTYPE: unknown or mixed dtypes";
    case WF_ERR_ALIGN: return "WF_ERR_ALIGN: pointer or stride not 16-byte aligned";
    case WF_ERR_WORKSPACE: return "WF_ERR_WORKSPACE: buffer too small";
    case WF_ERR_CUDA: return "WF_ERR_CUDA: CUDA runtime or launch failure";
    case WF_ERR_TIMEOUT: return "WF_ERR_TIMEOUT: a bounded device wait gave up";
    case WF_ERR_UNSUPPORTED: return "WF_ERR_UNSUPPORTED: outside what this build implements";
    case WF_ERR_SCHEDULE: return "WF_ERR_SCHEDULE: kept counts infeasible";
    default: return "unknown wf_status";
  }
}

WF_API size_t wf_coeffs_bytes(const wf_tensor* kv, int levels) {
  if (check_desc(kv, false) != WF_OK || check_levels(kv, levels) != WF_OK) return 0;
  const int64_t rows = (int64_t)kv->seq - ((int64_t)kv->seq >> levels);
  return (size_t)kv->batch * kv->heads * rows * kv->head_dim * elem_size(kv->dtype);
}

WF_API wf_status wf_dwt_build(const void* K, const void* V, const wf_tensor* kv, int levels, void* coeffs,
                              size_t coeffs_bytes, void* stream) {
  wf_status st;
  if ((st = check_desc(kv, false)) != WF_OK) return st;
  if ((st = check_levels(kv, levels)) != WF_OK) return st;
  if (!K || !coeffs || V) return WF_ERR_INVALID_ARG;
  if (!aligned16(K) || !aligned16(coeffs)) return WF_ERR_ALIGN;
  if (coeffs_bytes < wf_coeffs_bytes(kv, levels)) return WF_ERR_WORKSPACE;
  return cuda_status(wf::launch_dwt(K, *kv, levels, coeffs, static_cast<cudaStream_t>(stream)));
}

WF_API wf_status wf_cache_update(const void* Knew, const void* Vnew, const wf_tensor* nt, void* K, void* V,
                                 const wf_tensor* kv, int64_t pos, int levels, void* coeffs, size_t coeffs_bytes,
                                 void* stream) {
  wf_status st;
  if ((st = check_desc(kv, false)) != WF_OK) return st;
  if ((st = check_desc(nt, false)) != WF_OK) return st;
  if ((st = check_levels(kv, levels)) != WF_OK) return st;
  if (!same_units(kv, nt)) return WF_ERR_SHAPE;
  if (kv->dtype != nt->dtype) return WF_ERR_DTYPE;
  if (!Knew || !K || !coeffs || (!Vnew) != (!V)) return WF_ERR_INVALID_ARG;
  if (pos < 0 || pos + (int64_t)nt->seq > (int64_t)kv->seq) return WF_ERR_INVALID_ARG;
  if (!aligned16(Knew) || !aligned16(K) || !aligned16(coeffs) || (V && (!aligned16(V) || !aligned16(Vnew))))
    return WF_ERR_ALIGN;
  if (coeffs_bytes < wf_coeffs_bytes(kv, levels)) return WF_ERR_WORKSPACE;
  return cuda_status(
      wf::launch_cache_update(Knew, Vnew, *nt, K, V, *kv, pos, levels, coeffs, static_cast<cudaStream_t>(stream)));
}

WF_API wf_status wf_default_schedule(int64_t n, int levels, int64_t k, int32_t* keep) {
  if (!keep || levels < 1 || levels > 30 || n < 1 || k < 1 || k > n) return WF_ERR_INVALID_ARG;
  if ((n >> levels) < 1 || ((n >> levels) << levels) != n) return WF_ERR_SHAPE;
  const double m = pow((double)k / (double)n, 1.0 / levels);
  int64_t cnt = n >> levels;
  for (int l = levels; l >= 2; --l) {
    int64_t kb = ceil_guarded(m * (double)cnt);
    kb = kb < 1 ? 1 : (kb > cnt ? cnt : kb);
    keep[l] = (int32_t)kb;
    cnt = 2 * kb;
  }
  const int64_t k1 = (k + 1) / 2;
  if (k1 > cnt) return WF_ERR_SCHEDULE;
  keep[1] = (int32_t)k1;
  keep[0] = (int32_t)k;
  return WF_OK;
}

WF_API wf_status wf_level0_schedule(int64_t n, int levels, int64_t k, int32_t* keep) {
  if (!keep || levels < 1 || levels > 30 || n < 1 || k < 1 || k > n) return WF_ERR_INVALID_ARG;
  if ((n >> levels) < 1 || ((n >> levels) << levels) != n) return WF_ERR_SHAPE;
  const double m = pow((double)k / (double)n, 1.0 / (levels + 1));  // L pyramid scans + the token scan
  int64_t cnt = n >> levels;
  for (int l = levels; l >= 1; --l) {
    int64_t kb = ceil_guarded(m * (double)cnt);
    kb = kb < 1 ? 1 : (kb > cnt ? cnt : kb);
    keep[l] = (int32_t)kb;
    cnt = 2 * kb;
  }
  if (k > cnt) return WF_ERR_SCHEDULE;
  keep[0] = (int32_t)k;
  return WF_OK;
}

WF_API wf_status wf_schedule_from_proportions(int64_t n, int levels, const double* m, int32_t* keep) {
  if (!keep || !m || levels < 1 || levels > 30 || n < 1) return WF_ERR_INVALID_ARG;
  if ((n >> levels) < 1 || ((n >> levels) << levels) != n) return WF_ERR_SHAPE;
  int64_t cnt = n >> levels;
  for (int l = levels; l >= 1; --l) {
    if (!(m[l] > 0.0 && m[l] <= 1.0)) return WF_ERR_SCHEDULE;
    int64_t kb = ceil_guarded(m[l] * (double)cnt);
    kb = kb < 1 ? 1 : (kb > cnt ? cnt : kb);
    keep[l] = (int32_t)kb;
    cnt = 2 * kb;
  }
  keep[0] = 2 * keep[1];
  return WF_OK;
}

WF_API size_t wf_filter_workspace_bytes(const wf_tensor* q, const wf_tensor* kv, int levels, const int32_t* keep) {
  if (check_filter_args(q, kv, levels, keep) != WF_OK) return 0;
  return wf::plan_filter(*q, *kv, levels, keep).total;
}

WF_API wf_status wf_filter(const void* Q, const wf_tensor* q, const void* coeffs, const void* K,
                           const wf_tensor* kv, int levels, const int32_t* keep, int32_t* idx, int32_t* level_sets,
                           void* ws, size_t ws_bytes, void* stream) {
  wf_status st = check_filter_args(q, kv, levels, keep);
  if (st != WF_OK) return st;
  if (!Q || !coeffs || !K || !idx || !ws) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(coeffs) || !aligned16(K)) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(idx) & 3u) != 0 || (reinterpret_cast<uintptr_t>(level_sets) & 3u) != 0)
    return WF_ERR_ALIGN;
  const wf::FilterPlan p = wf::plan_filter(*q, *kv, levels, keep);
  if (ws_bytes < p.total) return WF_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if (!device_sms(&sms)) return WF_ERR_CUDA;
  return cuda_status(run_filter(p, Q, *q, coeffs, K, *kv, levels, keep, idx, level_sets, ws, static_cast<int*>(ws),
                                sms, s));
}

WF_API wf_status wf_wavelet_approx(const void* K, const wf_tensor* kv, const int32_t* cand, int m, int level,
                                   int wavelet, void* out, size_t out_bytes, void* stream) {
  wf_status st;
  if ((st = check_desc(kv, false)) != WF_OK) return st;
  if (!wf::wavelet_taps(wavelet) || level < 1 || level > wf::wavelet_max_level(wavelet)) return WF_ERR_UNSUPPORTED;
  if ((st = check_levels(kv, level)) != WF_OK) return st;
  if (!K || !out || m < 1 || (!cand && m != (kv->seq >> level))) return WF_ERR_INVALID_ARG;
  if (!aligned16(K) || !aligned16(out) || (reinterpret_cast<uintptr_t>(cand) & 3u) != 0) return WF_ERR_ALIGN;
  if (out_bytes < (size_t)kv->batch * kv->heads * m * kv->head_dim * elem_size(kv->dtype)) return WF_ERR_WORKSPACE;
  return cuda_status(wf::launch_wavelet_approx(K, *kv, cand, m, m, level, wavelet, out, (int64_t)m * kv->head_dim,
                                               static_cast<cudaStream_t>(stream)));
}

WF_API size_t wf_filter_wavelet_workspace_bytes(const wf_tensor* q, const wf_tensor* kv, int levels,
                                                const int32_t* keep, int wavelet) {
  if (check_filter_args(q, kv, levels, keep) != WF_OK) return 0;
  if (!wf::wavelet_taps(wavelet) || levels > wf::wavelet_max_level(wavelet)) return 0;
  return wf::wavelet_filter_bytes(wf::plan_filter(*q, *kv, levels, keep));
}

WF_API wf_status wf_filter_wavelet(const void* Q, const wf_tensor* q, const void* top, const void* K,
                                   const wf_tensor* kv, int levels, const int32_t* keep, int wavelet, int32_t* idx,
                                   int32_t* level_sets, void* ws, size_t ws_bytes, void* stream) {
  wf_status st = check_filter_args(q, kv, levels, keep);
  if (st != WF_OK) return st;
  if (!wf::wavelet_taps(wavelet) || levels > wf::wavelet_max_level(wavelet)) return WF_ERR_UNSUPPORTED;
  if (!Q || !top || !K || !idx || !ws) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(top) || !aligned16(K)) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(idx) & 3u) != 0 || (reinterpret_cast<uintptr_t>(level_sets) & 3u) != 0)
    return WF_ERR_ALIGN;
  const wf::FilterPlan p = wf::plan_filter(*q, *kv, levels, keep);
  if (ws_bytes < wf::wavelet_filter_bytes(p)) return WF_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if (!device_sms(&sms)) return WF_ERR_CUDA;
  const wf::FusedPlan fp = wf::plan_fused(*q, *kv, levels, keep, -1, sms, true);
  if (fp.ok && q->heads == kv->heads)
    return cuda_status(wf::launch_literal_fused(fp, p, Q, *q, top, K, nullptr, *kv, nullptr, nullptr, nullptr,
                                                wavelet, idx, level_sets, nullptr, nullptr, ws,
                                                static_cast<int*>(ws), s));
  return cuda_status(wf::launch_filter_wavelet(p, Q, *q, top, K, *kv, wavelet, idx, level_sets, ws,
                                               static_cast<int*>(ws), s));
}

WF_API size_t wf_attn_workspace_bytes(const wf_tensor* q, int k, int n_g) {
  if (check_desc(q, false) != WF_OK || k < 1 || n_g < 0 || q->seq > wf::kMaxQ) return 0;
  return wf::plan_attn(*q, k, n_g, 1).total;  // the size does not depend on the grouping
}

WF_API wf_status wf_sparse_attn(const void* Q, const wf_tensor* q, const void* K, const void* V,
                                const wf_tensor* kv, const int32_t* idx, int k, const void* Kg, const void* Vg,
                                const wf_tensor* g, void* O, const wf_tensor* o, float scale, void* ws,
                                size_t ws_bytes, void* stream) {
  const int n_g = g ? g->seq : 0;
  wf_status st = check_attn_args(q, kv, k, g, n_g, o);
  if (st != WF_OK) return st;
  if (!Q || !K || !V || !idx || !O || !ws) return WF_ERR_INVALID_ARG;
  if (n_g > 0 && (!Kg || !Vg)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return WF_ERR_ALIGN;
  if (n_g > 0 && (!aligned16(Kg) || !aligned16(Vg))) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || (reinterpret_cast<uintptr_t>(idx) & 3u) != 0)
    return WF_ERR_ALIGN;
  if (!(scale >= 0.f) || isinf(scale)) return WF_ERR_INVALID_ARG;
  const wf::AttnPlan p = wf::plan_attn(*q, k, n_g, group_of(q, kv));
  if (ws_bytes < p.total) return WF_ERR_WORKSPACE;
  const float sc = scale == 0.f ? 1.0f / sqrtf((float)q->head_dim) : scale;
  return cuda_status(wf::launch_attn(p, Q, *q, K, V, *kv, idx, Kg, Vg, n_g > 0 ? g : nullptr, O, *o, sc, ws,
                                     static_cast<int*>(ws), static_cast<cudaStream_t>(stream)));
}

// wf_step keeps a 256-byte status block at the start of its workspace (the
// fused kernel's bounded waits report there); the rest is the scratch of the
// per-stage kernels when the fused kernel does not apply.
constexpr size_t kStatusBytes = 256;

WF_API size_t wf_step_workspace_bytes(const wf_tensor* q, const wf_tensor* kv, int levels, const int32_t* keep,
                                      int n_g) {
  if (check_filter_args(q, kv, levels, keep) != WF_OK || n_g < 0) return 0;
  const size_t f = wf::plan_filter(*q, *kv, levels, keep).total;
  const size_t a = wf::plan_attn(*q, keep[0], n_g, 1).total;
  return kStatusBytes + (f > a ? f : a);
}

WF_API wf_status wf_step(const void* Q, const wf_tensor* q, const void* K, const void* V, const wf_tensor* kv,
                         const void* Kg, const void* Vg, const wf_tensor* g, void* coeffs, size_t coeffs_bytes,
                         int refresh_coeffs, int levels, const int32_t* keep, int32_t* idx, int32_t* level_sets,
                         void* O, const wf_tensor* o, void* ws, size_t ws_bytes, void* stream) {
  wf_status st = check_filter_args(q, kv, levels, keep);
  if (st != WF_OK) return st;
  const int n_g = g ? g->seq : 0;
  if ((st = check_attn_args(q, kv, keep[0], g, n_g, o)) != WF_OK) return st;
  if (!Q || !K || !V || !coeffs || !idx || !O || !ws) return WF_ERR_INVALID_ARG;
  if (n_g > 0 && (!Kg || !Vg)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned16(coeffs)) return WF_ERR_ALIGN;
  if (n_g > 0 && (!aligned16(Kg) || !aligned16(Vg))) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || (reinterpret_cast<uintptr_t>(idx) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(level_sets) & 3u) != 0)
    return WF_ERR_ALIGN;
  if (coeffs_bytes < wf_coeffs_bytes(kv, levels)) return WF_ERR_WORKSPACE;
  if (ws_bytes < wf_step_workspace_bytes(q, kv, levels, keep, n_g)) return WF_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if (!device_sms(&sms)) return WF_ERR_CUDA;
  int* status = static_cast<int*>(ws);  // set by the fused kernel on a timeout; read and cleared by wf_workspace_status
  void* scratch = static_cast<char*>(ws) + kStatusBytes;
  cudaError_t e = cudaSuccess;
  if (refresh_coeffs && (e = wf::launch_dwt(K, *kv, levels, coeffs, s)) != cudaSuccess) return WF_ERR_CUDA;
  // The fused kernel takes one query head per KV head.
  const wf::FusedPlan fp = wf::plan_fused(*q, *kv, levels, keep, n_g, sms, false);
  if (fp.ok && q->heads == kv->heads) {
    e = wf::launch_fused(fp, Q, *q, K, V, *kv, Kg, Vg, n_g > 0 ? g : nullptr, coeffs, levels, keep, idx,
                         level_sets, O, *o, status, s, nullptr);
    return cuda_status(e);
  }
  const wf::F32Plan f32 = wf::plan_f32(*q, *kv, levels, keep, n_g, sms);
  if (f32.ok)
    return cuda_status(wf::launch_f32(f32, Q, *q, K, V, *kv, Kg, Vg, n_g > 0 ? g : nullptr, coeffs, levels, keep, idx,
                                      level_sets, O, *o, s));
  // Otherwise the filter (wf_filter's kernels), then the per-stage attention.
  const wf::FilterPlan fl = wf::plan_filter(*q, *kv, levels, keep);
  if ((e = run_filter(fl, Q, *q, coeffs, K, *kv, levels, keep, idx, level_sets, scratch, status, sms, s)) !=
      cudaSuccess)
    return WF_ERR_CUDA;
  const wf::AttnPlan ap = wf::plan_attn(*q, keep[0], n_g, group_of(q, kv));
  const float sc = 1.0f / sqrtf((float)q->head_dim);
  e = wf::launch_attn(ap, Q, *q, K, V, *kv, idx, Kg, Vg, n_g > 0 ? g : nullptr, O, *o, sc, scratch, status, s);
  return cuda_status(e);
}

WF_API size_t wf_step_wavelet_workspace_bytes(const wf_tensor* q, const wf_tensor* kv, int levels,
                                              const int32_t* keep, int wavelet, int n_g) {
  if (check_filter_args(q, kv, levels, keep) != WF_OK || n_g < 0) return 0;
  if (!wf::wavelet_taps(wavelet) || levels > wf::wavelet_max_level(wavelet)) return 0;
  const size_t f = wf::wavelet_filter_bytes(wf::plan_filter(*q, *kv, levels, keep));
  const size_t a = wf::plan_attn(*q, keep[0], n_g, 1).total;
  return kStatusBytes + (f > a ? f : a);
}

WF_API wf_status wf_step_wavelet(const void* Q, const wf_tensor* q, const void* top, const void* K, const void* V,
                                 const wf_tensor* kv, const void* Kg, const void* Vg, const wf_tensor* g, int levels,
                                 const int32_t* keep, int wavelet, int32_t* idx, int32_t* level_sets, void* O,
                                 const wf_tensor* o, void* ws, size_t ws_bytes, void* stream) {
  wf_status st = check_filter_args(q, kv, levels, keep);
  if (st != WF_OK) return st;
  if (!wf::wavelet_taps(wavelet) || levels > wf::wavelet_max_level(wavelet)) return WF_ERR_UNSUPPORTED;
  const int n_g = g ? g->seq : 0;
  if ((st = check_attn_args(q, kv, keep[0], g, n_g, o)) != WF_OK) return st;
  if (!Q || !top || !K || !V || !idx || !O || !ws) return WF_ERR_INVALID_ARG;
  if (n_g > 0 && (!Kg || !Vg)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(top) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return WF_ERR_ALIGN;
  if (n_g > 0 && (!aligned16(Kg) || !aligned16(Vg))) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || (reinterpret_cast<uintptr_t>(idx) & 3u) != 0 ||
      (reinterpret_cast<uintptr_t>(level_sets) & 3u) != 0)
    return WF_ERR_ALIGN;
  if (ws_bytes < wf_step_wavelet_workspace_bytes(q, kv, levels, keep, wavelet, n_g)) return WF_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int sms = 0;
  if (!device_sms(&sms)) return WF_ERR_CUDA;
  int* status = static_cast<int*>(ws);
  void* scratch = static_cast<char*>(ws) + kStatusBytes;
  const wf::FilterPlan fl = wf::plan_filter(*q, *kv, levels, keep);
  const wf::FusedPlan fp = wf::plan_fused(*q, *kv, levels, keep, n_g, sms, true);
  if (fp.ok && q->heads == kv->heads)
    return cuda_status(wf::launch_literal_fused(fp, fl, Q, *q, top, K, V, *kv, Kg, Vg, n_g > 0 ? g : nullptr, wavelet,
                                                idx, level_sets, O, o, scratch, status, s));
  cudaError_t e = wf::launch_filter_wavelet(fl, Q, *q, top, K, *kv, wavelet, idx, level_sets, scratch, status, s);
  if (e != cudaSuccess) return WF_ERR_CUDA;
  const wf::AttnPlan ap = wf::plan_attn(*q, keep[0], n_g, group_of(q, kv));
  const float sc = 1.0f / sqrtf((float)q->head_dim);
  e = wf::launch_attn(ap, Q, *q, K, V, *kv, idx, Kg, Vg, n_g > 0 ? g : nullptr, O, *o, sc, scratch, status, s);
  return cuda_status(e);
}

// ---------------------------------------------------------------------------
// The quantised cache.
// ---------------------------------------------------------------------------
namespace {

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The row counts that the kernels' 32-bit row numbers take.
bool too_many_rows(int64_t units, int64_t rows) { return units * rows >= (int64_t)1 << 30; }

// Descriptors and sizes of a call that moves rows (f) into or out of a cache.
wf_status check_mx_args(const wf_tensor* f, const wf_tensor* kv, size_t scales_bytes) {
  wf_status st;
  if ((st = check_codes(kv)) != WF_OK) return st;
  if ((st = check_desc(f, true)) != WF_OK) return st;
  if (!same_units(f, kv)) return WF_ERR_SHAPE;
  if (too_many_rows((int64_t)kv->batch * kv->heads, f->seq)) return WF_ERR_UNSUPPORTED;
  return scales_bytes < wf_scales_bytes(kv) ? WF_ERR_WORKSPACE : WF_OK;
}

}  // namespace

WF_API size_t wf_scales_bytes(const wf_tensor* kv) {
  if (check_codes(kv) != WF_OK) return 0;
  return (size_t)kv->batch * kv->heads * kv->seq * (kv->head_dim / 32);
}

WF_API wf_status wf_cache_quantize(const void* Knew, const void* Vnew, const wf_tensor* nt, void* Kc, void* Ks,
                                   void* Vc, void* Vs, const wf_tensor* kv, size_t scales_bytes, int64_t pos,
                                   void* stream) {
  const wf_status st = check_mx_args(nt, kv, scales_bytes);
  if (st != WF_OK) return st;
  if (pos < 0 || pos > kv->seq || nt->seq > kv->seq - pos) return WF_ERR_INVALID_ARG;
  if (nt->seq == 0) return WF_OK;  // a tensor without rows may have no address
  if (!Knew || !Kc || !Ks) return WF_ERR_INVALID_ARG;
  if ((Vnew != nullptr) != (Vc != nullptr) || (Vnew != nullptr) != (Vs != nullptr)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Knew) || !aligned16(Vnew) || !aligned16(Kc) || !aligned16(Vc) || !aligned4(Ks) || !aligned4(Vs))
    return WF_ERR_ALIGN;
  return cuda_status(wf::launch_quantize(Knew, Vnew, *nt, Kc, Ks, Vc, Vs, *kv, pos, static_cast<cudaStream_t>(stream)));
}

WF_API wf_status wf_cache_dequantize(const void* Kc, const void* Ks, const void* Vc, const void* Vs,
                                     const wf_tensor* kv, size_t scales_bytes, const int32_t* idx, int64_t pos,
                                     void* Kout, void* Vout, const wf_tensor* out, void* stream) {
  const wf_status st = check_mx_args(out, kv, scales_bytes);
  if (st != WF_OK) return st;
  if (idx ? pos != 0 : (pos < 0 || pos > kv->seq || out->seq > kv->seq - pos)) return WF_ERR_INVALID_ARG;
  if (out->seq == 0) return WF_OK;
  if (!Kc || !Ks || !Kout) return WF_ERR_INVALID_ARG;
  if ((Vout != nullptr) != (Vc != nullptr) || (Vout != nullptr) != (Vs != nullptr)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Kout) || !aligned16(Vout) || !aligned16(Kc) || !aligned16(Vc) || !aligned4(Ks) || !aligned4(Vs) ||
      !aligned4(idx))
    return WF_ERR_ALIGN;
  return cuda_status(
      wf::launch_dequantize(Kc, Ks, Vc, Vs, *kv, idx, pos, Kout, Vout, *out, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// Attention over shared prompts.
// ---------------------------------------------------------------------------
namespace {

wf_status check_prefix_args(const wf_tensor* q, const wf_tensor* kv, int k, int n_g) {
  wf_status st;
  if ((st = check_desc(q, false)) != WF_OK) return st;
  if (!kv) return WF_ERR_INVALID_ARG;
  if ((st = quantised(kv) ? check_codes(kv) : check_desc(kv, false)) != WF_OK) return st;
  if (!quantised(kv) && kv->dtype != q->dtype) return WF_ERR_DTYPE;
  if (kv->head_dim != q->head_dim || q->heads % kv->heads || q->batch % kv->batch) return WF_ERR_SHAPE;
  if (k < 0 || k > kv->seq || n_g < 0) return WF_ERR_INVALID_ARG;
  if (too_many_rows((int64_t)q->batch * q->heads, q->seq)) return WF_ERR_UNSUPPORTED;
  // A range of keys ends at a multiple of its tiles, past the count.
  if (too_many_rows(1, k) || too_many_rows(1, n_g)) return WF_ERR_UNSUPPORTED;
  return WF_OK;
}

// Outputs and, where there are any, own rows (g) of the queries q over key heads kv.
wf_status check_attn_rows(const wf_tensor* q, const wf_tensor* kv, const wf_tensor* g, const wf_tensor* o) {
  wf_status st;
  if ((st = check_desc(o, false)) != WF_OK) return st;
  if (!same_units(q, o) || o->seq != q->seq) return WF_ERR_SHAPE;
  if (o->dtype != q->dtype) return WF_ERR_DTYPE;
  if (g) {
    if ((st = check_desc(g, true)) != WF_OK) return st;
    if (g->batch != q->batch || g->heads != kv->heads || g->head_dim != q->head_dim) return WF_ERR_SHAPE;
    if (g->dtype != q->dtype) return WF_ERR_DTYPE;
  }
  return WF_OK;
}

void fill_prefix(wf::PrefixPlan& p, const void* Q, const wf_tensor* q, const void* K, const void* V,
                 const wf_tensor* kv, const void* Ks, const void* Vs, const void* Kg, const void* Vg,
                 const wf_tensor* g, void* O, const wf_tensor* o, float scale, void* ws) {
  wf::PrefixArgs& a = p.a;
  const int64_t code = kv->dtype == WF_MXFP4 ? 2 : 1;  // elements a byte of the codes' strides
  a.Q = Q; a.qsb = q->stride_b; a.qsh = q->stride_h; a.qss = q->stride_s;
  a.K = K; a.V = V;
  a.ksb = kv->stride_b / code; a.ksh = kv->stride_h / code; a.kss = kv->stride_s / code;
  a.Ks = static_cast<const uint8_t*>(Ks); a.Vs = static_cast<const uint8_t*>(Vs);
  a.Kg = Kg; a.Vg = Vg;
  if (a.ng > 0) { a.gsb = g->stride_b; a.gsh = g->stride_h; a.gss = g->stride_s; }
  a.O = O; a.osb = o->stride_b; a.osh = o->stride_h; a.oss = o->stride_s;
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + p.off_ml);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + p.off_o);
  a.sl2 = 1.4426950408889634f * (scale == 0.f ? 1.0f / sqrtf((float)q->head_dim) : scale);
  a.status = static_cast<int*>(ws);
  const wf::WaitControls wc = wf::wait_controls();
  a.wait_limit = wc.limit;
  a.stall = wc.stall;
}

}  // namespace

WF_API size_t wf_prefix_attn_workspace_bytes(const wf_tensor* q, const wf_tensor* kv, int k, int n_g) {
  if (check_prefix_args(q, kv, k, n_g) != WF_OK) return 0;
  return wf::plan_prefix(*q, *kv, k, n_g).total;
}

WF_API wf_status wf_prefix_attn(const void* Q, const wf_tensor* q, const void* K, const void* V, const wf_tensor* kv,
                                const void* Ks, const void* Vs, const int32_t* idx, int k, const int32_t* prefix_len,
                                const void* Kg, const void* Vg, const wf_tensor* g, const int32_t* gen_len, void* O,
                                const wf_tensor* o, float scale, void* ws, size_t ws_bytes, void* stream) {
  const int n_g = g ? g->seq : 0;
  wf_status st = check_prefix_args(q, kv, k, n_g);
  if (st != WF_OK) return st;
  if ((st = check_attn_rows(q, kv, g, o)) != WF_OK) return st;
  if (!Q || !K || !V || !O || !ws) return WF_ERR_INVALID_ARG;
  if (quantised(kv) ? (!Ks || !Vs) : (Ks || Vs)) return WF_ERR_INVALID_ARG;
  if (n_g > 0 && (!Kg || !Vg)) return WF_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || isinf(scale)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned4(Ks) || !aligned4(Vs))
    return WF_ERR_ALIGN;
  if (n_g > 0 && (!aligned16(Kg) || !aligned16(Vg))) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || !aligned4(idx) || !aligned4(prefix_len) || !aligned4(gen_len))
    return WF_ERR_ALIGN;
  wf::PrefixPlan p = wf::plan_prefix(*q, *kv, k, n_g);
  if (ws_bytes < p.total) return WF_ERR_WORKSPACE;
  fill_prefix(p, Q, q, K, V, kv, Ks, Vs, Kg, Vg, g, O, o, scale, ws);
  p.a.idx = idx; p.a.plen = prefix_len; p.a.glen = gen_len;
  return cuda_status(wf::launch_prefix(p, static_cast<cudaStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// A cache in pages.
// ---------------------------------------------------------------------------
namespace {

// 2^192 / (2 pi) rounded down, in 32-bit digits, the most significant first.
constexpr uint32_t kTurn[] = {0x28be60dbu, 0x9391054au, 0x7f09d5f4u, 0x7d4d3770u, 0x36d8a566u, 0x4f10e410u};

// f / (2 pi) modulo 1, as a fraction of 2^64, to nearest.  f = m 2^e with a whole m of 53
// bits, so the fraction is m times the digits above, shifted; of |f| < 2^32 no
// digit that counts is left out.
uint64_t turns_of(double f) {
  int e;
  const double x = frexp(fabs(f), &e);
  const uint64_t m = (uint64_t)ldexp(x, 53);
  e -= 53;  // f = m 2^e, e <= -21
  // m / (2 pi) in units of 2^-192, eight digits, the least significant first.
  uint32_t y[9] = {0};
  for (int part = 0; part < 2; ++part) {
    const uint64_t d = part ? m >> 32 : m & 0xffffffffu;
    uint64_t carry = 0;
    for (int i = 0; i < 6; ++i) {
      const uint64_t t = d * kTurn[5 - i] + y[i + part] + carry;
      y[i + part] = (uint32_t)t;
      carry = t >> 32;
    }
    y[6 + part] += (uint32_t)carry;
  }
  // 2^64 f / (2 pi) = y 2^(e - 128): bits [s, s + 64) of y, s = 128 - e, rounded at bit s - 1.
  const int s = 128 - e;
  if (s > 256) return 0;
  auto bit = [&](int i) { return i < 0 || i >= 288 ? 0u : y[i >> 5] >> (i & 31) & 1u; };
  uint64_t r = 0;
  for (int i = 0; i < 64; ++i) r |= (uint64_t)bit(s + i) << i;
  r += bit(s - 1);
  return f < 0 ? 0 - r : r;
}

wf_status check_plan(const int64_t* plan, int pairs, int d) {
  if (!plan) return WF_ERR_INVALID_ARG;
  if (pairs < 8 || pairs % 8 || pairs > d / 2) return WF_ERR_SHAPE;
  return aligned16(plan) ? WF_OK : WF_ERR_ALIGN;
}

// A pool of pages and the tables of its sequences.
wf_status check_pool(const wf_tensor* pool, int table) {
  if (!pool) return WF_ERR_INVALID_ARG;
  const wf_status st = quantised(pool) ? check_codes(pool) : check_desc(pool, false);
  if (st != WF_OK) return st;
  if (table < 1) return WF_ERR_INVALID_ARG;
  const int64_t most = (int64_t)1 << 31;
  if ((int64_t)pool->batch * pool->seq >= most || (int64_t)table * pool->seq >= most) return WF_ERR_UNSUPPORTED;
  return WF_OK;
}

void fill_rows(wf::RowsArgs& a, int x, const void* src, const wf_tensor* from, void* dst, const wf_tensor* to) {
  const int64_t code = to->dtype == WF_MXFP4 ? 2 : 1;
  a.src[x] = src;
  a.ssb[x] = from->stride_b; a.ssh[x] = from->stride_h; a.sss[x] = from->stride_s;
  a.dst[x] = dst;
  a.dsb[x] = to->stride_b / code; a.dsh[x] = to->stride_h / code; a.dss[x] = to->stride_s / code;
  a.heads[x] = from->heads;
}

// The shapes of a wf_tree_attn call, and what wf_prefix_attn's plan takes for them: a
// cache of n rows a sequence.
wf_status check_tree(const wf_tensor* q, const wf_tensor* pool, int n, int n_t, wf_tensor* cache) {
  wf_status st;
  if ((st = check_desc(q, false)) != WF_OK) return st;
  if ((st = check_pool(pool, 1)) != WF_OK) return st;
  if (!quantised(pool) && pool->dtype != q->dtype) return WF_ERR_DTYPE;
  if (pool->head_dim != q->head_dim || q->heads % pool->heads) return WF_ERR_SHAPE;
  if (n < 0 || n_t < 0) return WF_ERR_INVALID_ARG;
  if (too_many_rows((int64_t)q->batch * q->heads, q->seq) || too_many_rows(1, n) || too_many_rows(1, n_t))
    return WF_ERR_UNSUPPORTED;
  // All key tiles, and empty places between them, lie in one line of less than 2^31 (see wf::Walk).
  const int64_t group = q->heads / pool->heads, tiles = (group * q->seq + 255) / 256;
  if ((int64_t)q->batch * pool->heads * tiles * ((int64_t)n + n_t + 1024) >= (int64_t)1 << 37) return WF_ERR_UNSUPPORTED;
  *cache = *pool;
  cache->batch = q->batch;
  cache->seq = n;
  return WF_OK;
}

}  // namespace

WF_API wf_status wf_rotary_plan(const double* freq, const int32_t* axis, int pairs, int64_t* plan) {
  if (!freq || !plan || pairs < 1) return WF_ERR_INVALID_ARG;
  for (int i = 0; i < pairs; ++i) {
    if (!(fabs(freq[i]) < 4294967296.0) || (axis && (axis[i] < 0 || axis[i] >= 64))) return WF_ERR_INVALID_ARG;
  }
  for (int i = 0; i < pairs; ++i) {
    plan[2 * i] = (int64_t)turns_of(freq[i]);
    plan[2 * i + 1] = axis ? axis[i] : 0;
  }
  return WF_OK;
}

WF_API wf_status wf_rotary_apply(const void* Q, const wf_tensor* q, const void* K, const wf_tensor* k,
                                 const int64_t* plan, int pairs, int adjacent, const int32_t* pos, int axes,
                                 void* Qout, const wf_tensor* qo, void* Kout, const wf_tensor* ko, void* stream) {
  wf_status st;
  if ((st = check_desc(q, true)) != WF_OK || (st = check_desc(qo, true)) != WF_OK) return st;
  if ((K != nullptr) != (Kout != nullptr)) return WF_ERR_INVALID_ARG;
  if (!same_units(q, qo) || q->seq != qo->seq) return WF_ERR_SHAPE;
  if (q->dtype != qo->dtype) return WF_ERR_DTYPE;
  if (K) {
    if ((st = check_desc(k, true)) != WF_OK || (st = check_desc(ko, true)) != WF_OK) return st;
    if (!same_units(k, ko) || k->seq != ko->seq || k->batch != q->batch || k->head_dim != q->head_dim ||
        k->seq != q->seq)
      return WF_ERR_SHAPE;
    if (k->dtype != q->dtype || ko->dtype != q->dtype) return WF_ERR_DTYPE;
  }
  if (too_many_rows((int64_t)q->batch * (q->heads + (int64_t)(K ? k->heads : 0)), q->seq)) return WF_ERR_UNSUPPORTED;
  if ((st = check_plan(plan, pairs, q->head_dim)) != WF_OK) return st;
  if (axes < 1) return WF_ERR_INVALID_ARG;
  if (q->seq == 0) return WF_OK;
  if (!Q || !Qout || !pos) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(Qout) || !aligned16(Kout) || !aligned4(pos)) return WF_ERR_ALIGN;
  wf::RowsArgs a = {};
  fill_rows(a, 0, Q, q, Qout, qo);
  if (K) fill_rows(a, 1, K, k, Kout, ko);
  a.both = 1;
  a.plan = reinterpret_cast<const wf::RotaryPair*>(plan);
  a.pairs = pairs; a.adjacent = adjacent != 0;
  a.pos = pos; a.axes = axes; a.B = q->batch; a.rows = q->seq;
  a.by_m = wf::make_fastdiv((uint32_t)q->seq);
  a.total = (uint32_t)q->batch * (uint32_t)q->seq;
  return cuda_status(wf::launch_rotate(a, q->dtype, q->head_dim, static_cast<cudaStream_t>(stream)));
}

WF_API wf_status wf_paged_append(const void* Knew, const void* Vnew, const wf_tensor* nt, const int32_t* rows_at, int m,
                                 const int32_t* start, const int32_t* count, const int64_t* plan, int pairs,
                                 int adjacent, const int32_t* pos, int axes, void* K, void* V, void* Ks, void* Vs,
                                 const wf_tensor* pool, size_t scales_bytes, const int32_t* pages, int table,
                                 void* stream) {
  wf_status st;
  if ((st = check_pool(pool, table)) != WF_OK || (st = check_desc(nt, true)) != WF_OK) return st;
  if (!quantised(pool) && pool->dtype != nt->dtype) return WF_ERR_DTYPE;
  if (nt->heads != pool->heads || nt->head_dim != pool->head_dim) return WF_ERR_SHAPE;
  if (m < 0 || (rows_at ? nt->seq < 1 && m > 0 : m != nt->seq)) return WF_ERR_INVALID_ARG;
  if (too_many_rows((int64_t)nt->batch * nt->heads * 2, nt->seq) || too_many_rows((int64_t)nt->batch * nt->heads * 2, m))
    return WF_ERR_UNSUPPORTED;
  if (quantised(pool) && scales_bytes < wf_scales_bytes(pool)) return WF_ERR_WORKSPACE;
  if (plan && (st = check_plan(plan, pairs, nt->head_dim)) != WF_OK) return st;
  if (pos && axes < 1) return WF_ERR_INVALID_ARG;
  if (m == 0) return WF_OK;
  if (!Knew || !K || !start || !pages) return WF_ERR_INVALID_ARG;
  if ((Vnew != nullptr) != (V != nullptr)) return WF_ERR_INVALID_ARG;
  if (quantised(pool) ? (!Ks || (Vs != nullptr) != (V != nullptr)) : (Ks || Vs)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Knew) || !aligned16(Vnew) || !aligned16(K) || !aligned16(V) || !aligned4(Ks) || !aligned4(Vs) ||
      !aligned4(rows_at) || !aligned4(start) || !aligned4(count) || !aligned4(pos) || !aligned4(pages))
    return WF_ERR_ALIGN;
  wf::RowsArgs a = {};
  fill_rows(a, 0, Knew, nt, K, pool);
  if (V) fill_rows(a, 1, Vnew, nt, V, pool);
  a.scales[0] = static_cast<uint8_t*>(Ks); a.scales[1] = static_cast<uint8_t*>(Vs);
  a.plan = reinterpret_cast<const wf::RotaryPair*>(plan);
  a.pairs = pairs; a.adjacent = adjacent != 0;
  a.pos = pos; a.axes = pos ? axes : 64; a.B = nt->batch; a.rows = nt->seq;
  a.pages = pages; a.start = start; a.rows_at = rows_at; a.count = count;
  a.table = table; a.pool = pool->batch;
  a.by_ps = wf::make_fastdiv((uint32_t)pool->seq);
  a.by_m = wf::make_fastdiv((uint32_t)m);
  a.total = (uint32_t)nt->batch * (uint32_t)m;
  return cuda_status(wf::launch_append(a, nt->dtype, pool->dtype, nt->head_dim, static_cast<cudaStream_t>(stream)));
}

WF_API size_t wf_tree_attn_workspace_bytes(const wf_tensor* q, const wf_tensor* pool, int n, int n_t) {
  wf_tensor cache;
  if (check_tree(q, pool, n, n_t, &cache) != WF_OK) return 0;
  return wf::plan_tree(*q, cache, n, n_t).total;
}

WF_API wf_status wf_tree_attn(const void* Q, const wf_tensor* q, const void* K, const void* V, const wf_tensor* pool,
                              const void* Ks, const void* Vs, const int32_t* pages, int table, int n,
                              const int32_t* cache_len, const void* Kt, const void* Vt, const wf_tensor* t,
                              const int32_t* tree_len, const int32_t* mask, void* O, const wf_tensor* o, float scale,
                              void* ws, size_t ws_bytes, void* stream) {
  const int n_t = t ? t->seq : 0;
  wf_tensor cache;
  wf_status st = check_tree(q, pool, n, n_t, &cache);
  if (st != WF_OK || (st = check_pool(pool, table)) != WF_OK) return st;
  if (n > (int64_t)table * pool->seq) return WF_ERR_INVALID_ARG;
  if ((st = check_attn_rows(q, pool, t, o)) != WF_OK) return st;
  if (!Q || !K || !V || !O || !ws || !pages) return WF_ERR_INVALID_ARG;
  if (quantised(pool) ? (!Ks || !Vs) : (Ks || Vs)) return WF_ERR_INVALID_ARG;
  if (n_t > 0 && (!Kt || !Vt)) return WF_ERR_INVALID_ARG;
  if (!(scale >= 0.f) || isinf(scale)) return WF_ERR_INVALID_ARG;
  if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O) || !aligned4(Ks) || !aligned4(Vs))
    return WF_ERR_ALIGN;
  if (n_t > 0 && (!aligned16(Kt) || !aligned16(Vt))) return WF_ERR_ALIGN;
  if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0 || !aligned4(pages) || !aligned4(cache_len) ||
      !aligned4(tree_len) || !aligned4(mask))
    return WF_ERR_ALIGN;
  wf::PrefixPlan p = wf::plan_tree(*q, cache, n, n_t);
  if (ws_bytes < p.total) return WF_ERR_WORKSPACE;
  fill_prefix(p, Q, q, K, V, pool, Ks, Vs, Kt, Vt, t, O, o, scale, ws);
  wf::PrefixArgs& a = p.a;
  a.plen = cache_len; a.glen = tree_len;
  a.pages = pages; a.table = table; a.pool = pool->batch;
  a.by_ps = wf::make_fastdiv((uint32_t)pool->seq);
  a.kx = a.ksb - (int64_t)pool->seq * a.kss;
  a.mask = n_t > 0 ? reinterpret_cast<const uint32_t*>(mask) : nullptr;
  a.mw = (n_t + 31) / 32;
  if (p.off_info) {
    const size_t items = (size_t)a.B * a.H * a.mt;
    a.info = reinterpret_cast<int2*>(static_cast<char*>(ws) + p.off_info);
    a.flags = reinterpret_cast<int*>(a.info + items);
  }
  return cuda_status(wf::launch_tree(p, static_cast<cudaStream_t>(stream)));
}

WF_API wf_status wf_workspace_status(void* ws, void* stream) {
  if (!ws) return WF_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int h = 0;
  if (cudaMemcpyAsync(&h, ws, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess) return WF_ERR_CUDA;
  if (cudaStreamSynchronize(s) != cudaSuccess) return WF_ERR_CUDA;
  if (h != 0) {
    if (cudaMemsetAsync(ws, 0, sizeof(int), s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)
      return WF_ERR_CUDA;
    return WF_ERR_TIMEOUT;
  }
  return WF_OK;
}

// ---------------------------------------------------------------------------
// Test-only wait-failure controls (include/wf_testing.h).
// ---------------------------------------------------------------------------
namespace {
std::atomic<int> g_test_stall{0};
std::atomic<long long> g_test_wait_limit{0};
}  // namespace

namespace wf {
WaitControls wait_controls() {
  WaitControls c;
  c.stall = g_test_stall.load(std::memory_order_relaxed);
  const long long lim = g_test_wait_limit.load(std::memory_order_relaxed);
  c.limit = lim > 0 ? lim : kDefaultWaitLimit;
  return c;
}
}  // namespace wf

WF_API wf_status wf_testing_set_wait_failure(int stall, long long wait_limit_cycles) {
  if (wait_limit_cycles < 0) return WF_ERR_INVALID_ARG;
  g_test_wait_limit.store(wait_limit_cycles, std::memory_order_relaxed);
  g_test_stall.store(stall != 0, std::memory_order_relaxed);
  return WF_OK;
}

WF_API wf_status wf_testing_prefix_plan(const wf_tensor* q, const wf_tensor* kv, int k, int n_g,
                                        wf_testing_plan* plan) {
  const wf_status st = check_prefix_args(q, kv, k, n_g);
  if (st != WF_OK) return st;
  if (!plan) return WF_ERR_INVALID_ARG;
  const wf::PrefixPlan p = wf::plan_prefix(*q, *kv, k, n_g);
  plan->workspace_used = (long long)p.used;
  plan->prompt_parts = p.a.S;
  plan->own_parts = p.a.So;
  plan->key_tile = p.tk;
  plan->prompt_rows = p.tr < p.a.R ? p.tr : p.a.R;
  plan->joined = p.fold;
  plan->direct = p.a.direct;
  plan->join_rows = p.fold ? wf::prefix_own_rows(p.a, p.a.S, n_g + (p.a.direct ? k : 0)) : 0;
  return WF_OK;
}
