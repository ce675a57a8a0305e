// Rows of a cache on their way into 8 or 4 bits and back (Sec. 3.2 of the paper: the kept tokens form the final cache; the
// representation of that cache is independent of which tokens are kept).
//
// Bound by HBM bandwidth: every row is read once, gathered by the kept list, and written once.  A row (one token, one KV
// head) belongs to 8, 16 or 32 lanes of eight channels each; its largest magnitude (INT4: least and largest value) is
// found by shuffles while the row stays in registers.
//
// Codes are quotients rounded to the nearest code.  Rows of 16-bit values have few significant bits, so that quotients often
// lie on the border between two codes exactly, and a product with a rounded reciprocal would fall on either side.  The
// quotient is therefore corrected by its remainder (one Newton step, Markstein 1990: q' = q + (a - q b) / b with both steps as
// fused multiply-adds), which gives the nearest float32 to a / b and so exact ties.
#include "cache_format.cuh"

namespace kvc {

namespace {

using namespace fmt;

constexpr int kWarps = 8;
constexpr int kSteps = 4;                    // rows of a lane group in flight

struct ConvertArgs {
  CacheView in[2], out[2];
  RowList rows;
  int items_per_row;                         // of one tensor
};

template <int F> __device__ constexpr float top_code() { return F == KVCRUSH_INT8 ? 127.f : F == KVCRUSH_E4M3 ? 448.f : 15.f; }

// a / b, correctly rounded but for results near the ends of the range; inv: 1 / b rounded.
__device__ __forceinline__ float quotient(float a, float b, float inv) {
  const float q = a * inv;
  return fmaf(fmaf(-q, b, a), inv, q);
}

// Codes of eight channels of a row whose kLanes lanes call this together; scale (and zero) come back in every lane.
template <int F, int kLanes>
__device__ __forceinline__ void quantize8(float (&x)[8], int lanes_used, Raw8<F>& codes, float& scale, float& zero) {
  uint32_t big = 0;                          // order of magnitudes as integers: NaN behind infinity behind the rest
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    big = max(big, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    if (F == KVCRUSH_INT4) { lo = fminf(lo, x[i]); hi = fmaxf(hi, x[i]); }
  }
  const bool used = (threadIdx.x & (kLanes - 1)) < lanes_used;
  if (!used) { big = 0; lo = FLT_MAX; hi = -FLT_MAX; }
#pragma unroll
  for (int d = 1; d < kLanes; d <<= 1) {
    big = max(big, __shfl_xor_sync(0xFFFFFFFFu, big, d));
    if (F == KVCRUSH_INT4) {
      lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, d));
      hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, d));
    }
  }
  zero = F == KVCRUSH_INT4 ? lo : 0.f;
  const float span = F == KVCRUSH_INT4 ? hi - lo : __uint_as_float(big);
  scale = span * (1.f / top_code<F>());
  const bool bad = big >= 0x7F800000u || !(span <= FLT_MAX);
  if (bad) scale = zero = __uint_as_float(0x7FC00000u);
  else if (scale < 0x1p-126f) scale = 0.f;
  // a power of two that keeps products and remainders away from both ends of the range
  const float shift = span > 0x1p64f ? 0x1p-64f : span < 0x1p-64f ? 0x1p64f : 1.f;
  const float num = top_code<F>() * shift, den = span * shift;
  const float inv = __frcp_rn(den);
  const bool none = bad || scale == 0.f;
  uint32_t c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = quotient((F == KVCRUSH_INT4 ? x[i] - lo : x[i]) * num, den, inv);
    if (F == KVCRUSH_E4M3) c[i] = __float_as_uint(none ? 0.f : y);
    else c[i] = none ? 0u : __float_as_uint(y + 12582912.f);       // 1.5 * 2^23: the nearest integer in the low bits, ties to even
  }
  if constexpr (F == KVCRUSH_INT8) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      codes.w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
  } else if constexpr (F == KVCRUSH_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(c[4 * i]), __uint_as_float(c[4 * i + 1])), __NV_SATFINITE, __NV_E4M3);
      const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(c[4 * i + 2]), __uint_as_float(c[4 * i + 3])), __NV_SATFINITE, __NV_E4M3);
      codes.w[i] = a | b << 16;
    }
  } else {
    codes.w[0] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) codes.w[0] |= (c[i] & 15u) << (4 * i);
  }
}

// One warp: kSteps * 32 / kLanes heads of one token of one tensor.
template <int FI, int FO, int kLanes>
__global__ void __launch_bounds__(kWarps * 32)
convert_kernel(Shape s, ConvertArgs a, int n_tensors) {
  chain_wait();
  chain_trigger();
  constexpr int kRowsPerStep = 32 / kLanes;
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int per_row = a.items_per_row * n_tensors;
  const long long row = item / per_row;
  if (row >= a.rows.total) return;
  const int part = (int)(item - row * per_row), ten = part / a.items_per_row, chunk = part - ten * a.items_per_row;
  int layer, seq;
  long long src, dst;
  if (a.rows.cu_kept) {
    const int n_seg = s.n_layers * s.n_seqs;
    if (row >= __ldg(a.rows.cu_kept + n_seg)) return;               // `total` is an upper bound
    const int seg = warp_segment_of_row(a.rows.cu_kept, n_seg, row, lane);
    layer = seg / s.n_seqs;
    seq = seg - layer * s.n_seqs;
    const int first = __ldg(a.rows.cu_kept + seg);
    src = a.rows.idx ? (long long)__ldg(a.rows.idx + row) : row - first;
    dst = row - first;
    src += a.rows.in_begin ? __ldg(a.rows.in_begin + seg) : __ldg(s.cu_seqlens + seq);
    dst += a.rows.out_begin ? __ldg(a.rows.out_begin + seg) : first - __ldg(a.rows.cu_kept + layer * s.n_seqs);
  } else {
    layer = (int)(row / s.T);
    const int tok = (int)(row - (long long)layer * s.T);
    src = dst = tok;
    if (a.rows.in_begin || a.rows.out_begin) {
      seq = seq_of_token(s.cu_seqlens, s.n_seqs, tok);
      const int seg = layer * s.n_seqs + seq, off = tok - __ldg(s.cu_seqlens + seq);
      if (a.rows.in_begin) src = __ldg(a.rows.in_begin + seg) + (long long)off;
      if (a.rows.out_begin) dst = __ldg(a.rows.out_begin + seg) + (long long)off;
    }
  }
  const CacheView in = a.in[ten], out = a.out[ten];
  const int sub = lane & (kLanes - 1), lanes_used = s.D / 8, ch = sub * 8;
  const unsigned char* ip = static_cast<const unsigned char*>(in.ptr) + bytes_of<FI>(layer * in.sl + src * in.st + ch);
  unsigned char* op = static_cast<unsigned char*>(const_cast<void*>(out.ptr)) + bytes_of<FO>(layer * out.sl + dst * out.st + ch);
  const int h0 = chunk * kSteps * kRowsPerStep + lane / kLanes;
  Raw8<FI> raw[kSteps];
  float2 sc[kSteps];
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int h = h0 + u * kRowsPerStep;
#pragma unroll
    for (int i = 0; i < Raw8<FI>::kWords; ++i) raw[u].w[i] = 0;
    if (h < s.Hkv && sub < lanes_used) {
      raw[u].load(ip + bytes_of<FI>(h * in.sh));
      if constexpr (kQuantized<FI>) {
        const float* p = in.scales + layer * in.scl + src * in.sct + h * in.sch;
        if constexpr (FI == KVCRUSH_INT4) sc[u] = __ldg(reinterpret_cast<const float2*>(p)); else sc[u].x = __ldg(p);
      }
    }
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int h = h0 + u * kRowsPerStep;
    const bool there = h < s.Hkv && sub < lanes_used;
    float x[8];
    raw[u].widen(x);
    if constexpr (kQuantized<FO>) {
      Raw8<FO> codes;
      float scale, zero;
      quantize8<FO, kLanes>(x, lanes_used, codes, scale, zero);
      if (there) codes.store(op + bytes_of<FO>(h * out.sh));
      if (there && sub == 0) {
        float* p = out.scales + layer * out.scl + dst * out.sct + h * out.sch;
        if constexpr (FO == KVCRUSH_INT4) *reinterpret_cast<float2*>(p) = make_float2(scale, zero); else *p = scale;
      }
    } else if (there) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = FI == KVCRUSH_INT4 ? fmaf(x[i], sc[u].x, sc[u].y) : x[i] * sc[u].x;
      Raw8<FO> v;
      v.narrow(x);
      v.store(op + bytes_of<FO>(h * out.sh));
    }
  }
}

template <int FI, int FO, int kLanes>
int launch_lanes(const Shape& s, ConvertArgs& a, int n_tensors, cudaStream_t stream) {
  constexpr int heads = kSteps * 32 / kLanes;
  a.items_per_row = (s.Hkv + heads - 1) / heads;
  const long long blocks = (a.rows.total * a.items_per_row * n_tensors + kWarps - 1) / kWarps;
  if (blocks > 0x7FFFFFFFLL) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(convert_kernel<FI, FO, kLanes>, dim3((unsigned)blocks), dim3(kWarps * 32), 0, stream, 1, s, a, n_tensors);
}

template <int FI, int FO>
int launch_formats(const Shape& s, ConvertArgs& a, int n_tensors, cudaStream_t stream) {
  if (s.D <= 64) return launch_lanes<FI, FO, 8>(s, a, n_tensors, stream);
  if (s.D <= 128) return launch_lanes<FI, FO, 16>(s, a, n_tensors, stream);
  return launch_lanes<FI, FO, 32>(s, a, n_tensors, stream);
}

template <int V>
int launch_values(const Shape& s, ConvertArgs& a, int n_tensors, bool quantize, int code, cudaStream_t stream) {
  switch (code) {
    case KVCRUSH_INT8: return quantize ? launch_formats<V, KVCRUSH_INT8>(s, a, n_tensors, stream) : launch_formats<KVCRUSH_INT8, V>(s, a, n_tensors, stream);
    case KVCRUSH_E4M3: return quantize ? launch_formats<V, KVCRUSH_E4M3>(s, a, n_tensors, stream) : launch_formats<KVCRUSH_E4M3, V>(s, a, n_tensors, stream);
    default: return quantize ? launch_formats<V, KVCRUSH_INT4>(s, a, n_tensors, stream) : launch_formats<KVCRUSH_INT4, V>(s, a, n_tensors, stream);
  }
}

}  // namespace

int launch_convert_rows(const Shape& s, const CacheView& K_in, const CacheView& V_in, const RowList& rows, const CacheView& K_out,
                        const CacheView& V_out, cudaStream_t stream) {
  if (rows.total == 0) return KVCRUSH_OK;
  ConvertArgs a{};
  a.in[0] = K_in; a.in[1] = V_in; a.out[0] = K_out; a.out[1] = V_out;
  a.rows = rows;
  const int n_tensors = V_in.ptr ? 2 : 1;
  const bool quantize = K_out.scales != nullptr;
  const int code = quantize ? K_out.dtype : K_in.dtype;
  switch (quantize ? K_in.dtype : K_out.dtype) {
    case KVCRUSH_BF16: return launch_values<KVCRUSH_BF16>(s, a, n_tensors, quantize, code, stream);
    case KVCRUSH_FP16: return launch_values<KVCRUSH_FP16>(s, a, n_tensors, quantize, code, stream);
    default: return launch_values<KVCRUSH_FP32>(s, a, n_tensors, quantize, code, stream);
  }
}

}  // namespace kvc
