// extern "C" entry points of the quantised cache and of the attention over it: argument validation and dispatch.
// As in api.cu, every check that can fail happens before the first launch.
#include <math.h>

#include "common.cuh"

namespace {

using namespace kvc;

constexpr int kMaxHeadDim = 256;
constexpr int kMaxNew = 1024;
constexpr int kMaxPageSize = 1024;
constexpr uint32_t kWaitPolls = 1u << 20, kShortWaitPolls = 1u << 12;   // limits of a barrier wait
constexpr long long kMaxStep = 1LL << 31;            // bytes from one token to the next, in the attention kernels

// Is it that far from one token to the next?  stride: in elements of `bits`.
bool too_far(long long stride, int bits) { return stride >= kMaxStep * 8 / bits; }
int element_bits(int dtype) { return dtype == KVCRUSH_INT4 ? 4 : dtype == KVCRUSH_INT8 || dtype == KVCRUSH_E4M3 ? 8 : 8 * elt_bytes(dtype); }

// A tensor that nothing is read from or written to may have no memory.
alignas(16) const unsigned char kNowhere[16] = {};
int make_view(const kvcrush_tensor_t* t, int head_dim, bool empty, TensorView* v) {
  kvcrush_tensor_t some;
  if (empty && t && !t->ptr_dev) {
    some = *t;
    some.ptr_dev = const_cast<unsigned char*>(kNowhere);
    t = &some;
  }
  return view_from_tensor(t, head_dim, v);
}

// Values (scales NULL) or codes with their scales.  `empty`: no row of it is read, so that it may have no memory.
int make_cache(const kvcrush_tensor_t* t, const kvcrush_scales_t* scales, int head_dim, bool empty, CacheView* c) {
  kvcrush_tensor_t some;
  kvcrush_scales_t some_scales;
  if (empty && t && !t->ptr_dev) {
    some = *t;
    some.ptr_dev = const_cast<unsigned char*>(kNowhere);
    t = &some;
  }
  if (empty && scales && !scales->ptr_dev) {
    some_scales = *scales;
    some_scales.ptr_dev = reinterpret_cast<float*>(const_cast<unsigned char*>(kNowhere));
    scales = &some_scales;
  }
  if (!scales) {
    TensorView v;
    const int rc = view_from_tensor(t, head_dim, &v);
    if (rc != KVCRUSH_OK) return rc;
    *c = CacheView{v.ptr, v.dtype, v.sl, v.st, v.sh, nullptr, 0, 0, 0};
    return KVCRUSH_OK;
  }
  if (!t || !t->ptr_dev || !scales->ptr_dev) return KVCRUSH_ERR_INVALID_ARG;
  if (t->dtype != KVCRUSH_INT8 && t->dtype != KVCRUSH_E4M3 && t->dtype != KVCRUSH_INT4) return KVCRUSH_ERR_INVALID_ARG;
  const bool int4 = t->dtype == KVCRUSH_INT4;
  const long long strides[3] = {t->stride_layer, t->stride_token, t->stride_head};
  const long long scale_strides[3] = {scales->stride_layer, scales->stride_token, scales->stride_head};
  if (reinterpret_cast<uintptr_t>(t->ptr_dev) % 16 || reinterpret_cast<uintptr_t>(scales->ptr_dev) % (int4 ? 8 : 4))
    return KVCRUSH_ERR_MISALIGNED;
  const int unit = int4 ? 32 : 16;                    // channels of 16 bytes
  for (int i = 0; i < 3; ++i) {
    if (strides[i] < 0 || scale_strides[i] < 0) return KVCRUSH_ERR_INVALID_ARG;
    if (strides[i] % unit || (int4 && scale_strides[i] % 2)) return KVCRUSH_ERR_MISALIGNED;
  }
  if (head_dim % unit) return KVCRUSH_ERR_UNSUPPORTED;
  *c = CacheView{t->ptr_dev, t->dtype, strides[0], strides[1], strides[2], scales->ptr_dev, scale_strides[0], scale_strides[1],
                 scale_strides[2]};
  return KVCRUSH_OK;
}

int convert_entry(const kvcrush_problem_t* problem, bool quantize, const kvcrush_tensor_t* K_val, const kvcrush_tensor_t* V_val,
                  const kvcrush_tensor_t* K_codes, const kvcrush_scales_t* K_scales, const kvcrush_tensor_t* V_codes,
                  const kvcrush_scales_t* V_scales, const int32_t* cu_kept_dev, const int32_t* idx_dev, int64_t total_kept,
                  const int32_t* in_begin_dev, const int32_t* out_begin_dev, int32_t* status_dev, void* stream) {
  Shape s;
  int rc = shape_from_problem(problem, &s);
  if (rc != KVCRUSH_OK) return rc;
  if (!status_dev || !K_scales) return KVCRUSH_ERR_INVALID_ARG;
  if ((V_val == nullptr) != (V_codes == nullptr) || (V_val == nullptr) != (V_scales == nullptr)) return KVCRUSH_ERR_INVALID_ARG;
  if (cu_kept_dev ? total_kept < 0 : idx_dev != nullptr) return KVCRUSH_ERR_INVALID_ARG;
  if (s.D > kMaxHeadDim || s.D % 8) return KVCRUSH_ERR_UNSUPPORTED;
  const RowList rows{cu_kept_dev, idx_dev, cu_kept_dev ? (long long)total_kept : (long long)s.n_layers * s.T, in_begin_dev, out_begin_dev};
  const bool none = rows.total == 0;
  CacheView kv{}, vv{}, kc{}, vc{};
  if ((rc = make_cache(K_val, nullptr, s.D, none, &kv)) != KVCRUSH_OK) return rc;
  if ((rc = make_cache(K_codes, K_scales, s.D, none, &kc)) != KVCRUSH_OK) return rc;
  if (V_val) {
    if ((rc = make_cache(V_val, nullptr, s.D, none, &vv)) != KVCRUSH_OK) return rc;
    if ((rc = make_cache(V_codes, V_scales, s.D, none, &vc)) != KVCRUSH_OK) return rc;
    if (vv.dtype != kv.dtype || vc.dtype != kc.dtype) return KVCRUSH_ERR_INVALID_ARG;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return quantize ? launch_convert_rows(s, kv, vv, rows, kc, vc, st) : launch_convert_rows(s, kc, vc, rows, kv, vv, st);
}

int make_new_tokens(const kvcrush_new_tokens_t* n, int n_seqs, NewTokens* out) {
  if (!n || !n->cu_new_host || !n->cu_new_dev || n->total_new < 0 || n->max_new < 0 || n->mask_words < 0) return KVCRUSH_ERR_INVALID_ARG;
  if (n->cu_new_host[0] != 0 || n->cu_new_host[n_seqs] != n->total_new) return KVCRUSH_ERR_INVALID_ARG;
  for (int i = 0; i < n_seqs; ++i) {
    const int len = n->cu_new_host[i + 1] - n->cu_new_host[i];
    if (len < 0 || len > n->max_new) return KVCRUSH_ERR_INVALID_ARG;
  }
  if (n->mask_dev && n->max_new > 32LL * n->mask_words) return KVCRUSH_ERR_INVALID_ARG;
  if (n->max_new > kMaxNew) return KVCRUSH_ERR_UNSUPPORTED;
  *out = NewTokens{n->total_new, n->max_new, n->mask_words, n->cu_new_dev, n->mask_dev};
  return KVCRUSH_OK;
}

// What kvcrush_attend and kvcrush_attend_pages share; fills everything but K_new, V_new and the pages.
int make_attend(const kvcrush_problem_t* problem, const kvcrush_new_tokens_t* new_tokens, const kvcrush_tensor_t* Q,
                const kvcrush_tensor_t* K, const kvcrush_scales_t* K_scales, const kvcrush_tensor_t* V,
                const kvcrush_scales_t* V_scales, const int32_t* row_begin_dev, const int32_t* row_count_dev,
                const kvcrush_tensor_t* O, float* lse_out_dev, int32_t* status_dev, AttendArgs* a) {
  int rc = shape_from_problem(problem, &a->s);
  if (rc != KVCRUSH_OK) return rc;
  const Shape& s = a->s;
  if ((rc = make_new_tokens(new_tokens, s.n_seqs, &a->fresh)) != KVCRUSH_OK) return rc;
  if (!status_dev || (K_scales == nullptr) != (V_scales == nullptr) || (row_begin_dev == nullptr) != (row_count_dev == nullptr))
    return KVCRUSH_ERR_INVALID_ARG;
  if (s.D > kMaxHeadDim || s.D % 8) return KVCRUSH_ERR_UNSUPPORTED;
  if (a->fresh.total == 0) return KVCRUSH_OK;         // nothing to do, and the tensors may have no memory
  if ((rc = view_from_tensor(Q, s.D, &a->Q)) != KVCRUSH_OK) return rc;
  if ((rc = view_from_tensor(O, s.D, &a->O)) != KVCRUSH_OK) return rc;
  if ((rc = make_cache(K, K_scales, s.D, s.T == 0, &a->K)) != KVCRUSH_OK) return rc;
  if ((rc = make_cache(V, V_scales, s.D, s.T == 0, &a->V)) != KVCRUSH_OK) return rc;
  if (a->O.dtype != a->Q.dtype || a->K.dtype != a->V.dtype || (!K_scales && a->K.dtype != a->Q.dtype)) return KVCRUSH_ERR_INVALID_ARG;
  const int bits = element_bits(a->K.dtype);
  if (too_far(a->K.st, bits) || too_far(a->V.st, bits) || too_far(a->K.sct, 32) || too_far(a->V.sct, 32)) return KVCRUSH_ERR_UNSUPPORTED;
  a->group_magic = s.G > 1 ? 0xFFFFFFFFu / (uint32_t)s.G + 1u : 0u;
  a->row_begin = row_begin_dev;
  a->row_count = row_count_dev;
  a->lse = lse_out_dev;
  a->status = status_dev;
  a->polls = kWaitPolls;
  const float scale = problem->softmax_scale != 0.f ? problem->softmax_scale : 1.f / sqrtf((float)s.D);
  a->scale_log2 = scale * 1.4426950408889634f;
  return KVCRUSH_OK;
}

int dispatch_attend(const AttendArgs& a, void* stream) {
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (a.Q.dtype == KVCRUSH_FP32) return launch_attend_simt(a, st);
  if (attend_tree_fits(a)) {
    bool taken = false;
    const int rc = launch_attend_tree(a, &taken, st);
    if (taken) return rc;
  }
  switch (a.K.dtype) {
    case KVCRUSH_BF16: return launch_attend_bf16(a, st);
    case KVCRUSH_FP16: return launch_attend_fp16(a, st);
    case KVCRUSH_INT8: return launch_attend_int8(a, st);
    case KVCRUSH_E4M3: return launch_attend_e4m3(a, st);
    default: return launch_attend_int4(a, st);
  }
}

int pages_of(const Shape& s, int page_size) { return (int)(((long long)s.max_seqlen + page_size - 1) / page_size); }

}  // namespace

extern "C" {

int kvcrush_quantize(const kvcrush_problem_t* problem, const kvcrush_tensor_t* K, const kvcrush_tensor_t* V,
                     const int32_t* cu_kept_dev, const int32_t* idx_dev, int64_t total_kept,
                     const int32_t* in_begin_dev, const int32_t* out_begin_dev,
                     const kvcrush_tensor_t* K_codes, const kvcrush_scales_t* K_scales,
                     const kvcrush_tensor_t* V_codes, const kvcrush_scales_t* V_scales,
                     int32_t* status_dev, void* stream) {
  return convert_entry(problem, true, K, V, K_codes, K_scales, V_codes, V_scales, cu_kept_dev, idx_dev, total_kept, in_begin_dev,
                       out_begin_dev, status_dev, stream);
}

int kvcrush_dequantize(const kvcrush_problem_t* problem, const kvcrush_tensor_t* K_codes, const kvcrush_scales_t* K_scales,
                       const kvcrush_tensor_t* V_codes, const kvcrush_scales_t* V_scales,
                       const int32_t* cu_kept_dev, const int32_t* idx_dev, int64_t total_kept,
                       const int32_t* in_begin_dev, const int32_t* out_begin_dev,
                       const kvcrush_tensor_t* K, const kvcrush_tensor_t* V, int32_t* status_dev, void* stream) {
  return convert_entry(problem, false, K, V, K_codes, K_scales, V_codes, V_scales, cu_kept_dev, idx_dev, total_kept, in_begin_dev,
                       out_begin_dev, status_dev, stream);
}

}  // extern "C"

namespace {

int attend_entry(const kvcrush_problem_t* problem, const kvcrush_new_tokens_t* new_tokens, const kvcrush_tensor_t* Q,
                 const kvcrush_tensor_t* K, const kvcrush_scales_t* K_scales,
                 const kvcrush_tensor_t* V, const kvcrush_scales_t* V_scales,
                 const kvcrush_tensor_t* K_new, const kvcrush_tensor_t* V_new,
                 const int32_t* row_begin_dev, const int32_t* row_count_dev,
                 const kvcrush_tensor_t* O, float* lse_out_dev, int32_t* status_dev, void* stream, bool short_waits, bool withhold) {
  AttendArgs a{};
  int rc = make_attend(problem, new_tokens, Q, K, K_scales, V, V_scales, row_begin_dev, row_count_dev, O, lse_out_dev, status_dev, &a);
  if (rc != KVCRUSH_OK || a.fresh.total == 0) return rc;
  if ((K_new == nullptr) != (V_new == nullptr) || (!K_new && a.fresh.mask)) return KVCRUSH_ERR_INVALID_ARG;
  if (K_new) {
    if ((rc = view_from_tensor(K_new, a.s.D, &a.K_new)) != KVCRUSH_OK) return rc;
    if ((rc = view_from_tensor(V_new, a.s.D, &a.V_new)) != KVCRUSH_OK) return rc;
    if (a.K_new.dtype != a.Q.dtype || a.V_new.dtype != a.Q.dtype) return KVCRUSH_ERR_INVALID_ARG;
    if (too_far(a.K_new.st, element_bits(a.Q.dtype)) || too_far(a.V_new.st, element_bits(a.Q.dtype))) return KVCRUSH_ERR_UNSUPPORTED;
  }
  if (short_waits) a.polls = kShortWaitPolls;
  a.withhold = withhold;
  return dispatch_attend(a, stream);
}

}  // namespace

extern "C" {

int kvcrush_attend(const kvcrush_problem_t* problem, const kvcrush_new_tokens_t* new_tokens, const kvcrush_tensor_t* Q,
                   const kvcrush_tensor_t* K, const kvcrush_scales_t* K_scales,
                   const kvcrush_tensor_t* V, const kvcrush_scales_t* V_scales,
                   const kvcrush_tensor_t* K_new, const kvcrush_tensor_t* V_new,
                   const int32_t* row_begin_dev, const int32_t* row_count_dev,
                   const kvcrush_tensor_t* O, float* lse_out_dev, int32_t* status_dev, void* stream) {
  return attend_entry(problem, new_tokens, Q, K, K_scales, V, V_scales, K_new, V_new, row_begin_dev, row_count_dev, O, lse_out_dev,
                      status_dev, stream, false, false);
}

// Not part of the public ABI (the header does not declare it): kvcrush_attend for the test that makes a bounded wait run out.
// short_waits: the barrier waits of the kernel for many query rows give up after a few thousand polls; withhold: its producer
// stops before its first copy, so that the other roles' first waits run out with nothing in flight and every block returns with
// status = {KVCRUSH_DEV_TIMEOUT, kernel id, block, 0}.  Other kernels have no such waits.
int kvcrush_diag_attend(const kvcrush_problem_t* problem, const kvcrush_new_tokens_t* new_tokens, const kvcrush_tensor_t* Q,
                        const kvcrush_tensor_t* K, const kvcrush_tensor_t* V, const kvcrush_tensor_t* K_new, const kvcrush_tensor_t* V_new,
                        const kvcrush_tensor_t* O, int32_t* status_dev, void* stream, int short_waits, int withhold) {
  return attend_entry(problem, new_tokens, Q, K, nullptr, V, nullptr, K_new, V_new, nullptr, nullptr, O, nullptr, status_dev, stream,
                      short_waits != 0, withhold != 0);
}

int kvcrush_page_bounds(const kvcrush_problem_t* problem, const kvcrush_tensor_t* K, int page_size, int recent_pages,
                        const int32_t* row_begin_dev, const int32_t* row_count_dev,
                        const kvcrush_tensor_t* lo, const kvcrush_tensor_t* hi, int32_t* status_dev, void* stream) {
  Shape s;
  int rc = shape_from_problem(problem, &s);
  if (rc != KVCRUSH_OK) return rc;
  if (!status_dev || page_size < 1 || recent_pages < 0 || (row_begin_dev == nullptr) != (row_count_dev == nullptr))
    return KVCRUSH_ERR_INVALID_ARG;
  TensorView k, l, h;
  if ((rc = make_view(K, s.D, s.T == 0, &k)) != KVCRUSH_OK) return rc;
  if ((rc = make_view(lo, s.D, s.T == 0, &l)) != KVCRUSH_OK) return rc;
  if ((rc = make_view(hi, s.D, s.T == 0, &h)) != KVCRUSH_OK) return rc;
  if (l.dtype != k.dtype || h.dtype != k.dtype) return KVCRUSH_ERR_INVALID_ARG;
  if (page_size % 8 || page_size > kMaxPageSize || s.D > kMaxHeadDim || s.D % 8) return KVCRUSH_ERR_UNSUPPORTED;
  if (s.T == 0) return KVCRUSH_OK;
  return launch_page_bounds(s, k, page_size, recent_pages, row_begin_dev, row_count_dev, l, h, static_cast<cudaStream_t>(stream));
}

int kvcrush_attend_pages(const kvcrush_problem_t* problem, const kvcrush_new_tokens_t* new_tokens, const kvcrush_tensor_t* Q,
                         const kvcrush_tensor_t* K, const kvcrush_scales_t* K_scales,
                         const kvcrush_tensor_t* V, const kvcrush_scales_t* V_scales,
                         int page_size, const kvcrush_tensor_t* lo, const kvcrush_tensor_t* hi, int budget,
                         int keep_initial, int keep_recent, const int32_t* row_begin_dev, const int32_t* row_count_dev,
                         int32_t* page_idx_dev, int32_t* n_pages_dev,
                         const kvcrush_tensor_t* O, float* lse_out_dev, int32_t* status_dev, void* stream) {
  AttendArgs a{};
  int rc = make_attend(problem, new_tokens, Q, K, K_scales, V, V_scales, row_begin_dev, row_count_dev, O, lse_out_dev, status_dev, &a);
  if (rc != KVCRUSH_OK || a.fresh.total == 0) return rc;
  if (a.fresh.mask || page_size < 1 || budget < 1 || keep_initial < 0 || keep_recent < 0) return KVCRUSH_ERR_INVALID_ARG;
  PageChoice& p = a.pages;
  if ((rc = make_view(lo, a.s.D, a.s.T == 0, &p.lo)) != KVCRUSH_OK) return rc;
  if ((rc = make_view(hi, a.s.D, a.s.T == 0, &p.hi)) != KVCRUSH_OK) return rc;
  if (p.lo.dtype != a.Q.dtype || p.hi.dtype != a.Q.dtype) return KVCRUSH_ERR_INVALID_ARG;
  if (page_size % 8 || page_size > kMaxPageSize || pages_of(a.s, page_size) > kMaxPagesPerSeq) return KVCRUSH_ERR_UNSUPPORTED;
  p.page_size = page_size; p.budget = budget; p.keep_initial = keep_initial; p.keep_recent = keep_recent;
  p.max_pages = pages_of(a.s, page_size);
  p.page_idx = page_idx_dev; p.n_pages = n_pages_dev;
  return dispatch_attend(a, stream);
}

}  // extern "C"
