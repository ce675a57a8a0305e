// Rows of a cache on their way into 8 or 4 bits and back (Sec. 3.2 of the paper: the kept tokens form the final cache; the
// representation of that cache is independent of which tokens are kept).
//
// Bound by HBM bandwidth: every row is read once, gathered by the kept list, and written once.  A row (one token, one KV
// head) belongs to 4, 8 or 16 lanes with one to three pieces of eight channels each; its largest magnitude (INT4: least and
// largest value) is found by shuffles while the row stays in registers.
//
// 32 layers x 2048 rows x 32 heads of 128, both tensors: bf16 to 8 bits 278 us = 5.8 TB/s
// (591 with a row to 16 lanes, one row a warp and unpaired arithmetic), to 4 bits 319 = 4.3 TB/s; back 257 = 6.3 TB/s and 233.  What keeps
// the way in below the way out is arithmetic: about 12.6 instructions a value to 8 bits, 17 to 4 bits (301 us with codes that are not
// always the nearest, see below); issue slots are 72 % busy there, DRAM 41 %.
//
// Codes are quotients rounded to the nearest code.  Rows of 16-bit values have few significant bits, so that quotients often
// lie on the border between two codes exactly, and a product with a rounded reciprocal would fall on either side.  The
// quotient is therefore corrected by its remainder (one Newton step, Markstein 1990: q' = q + (a - q b) / b with both steps as
// fused multiply-adds), which gives the nearest float32 to a / b.  For 8-bit codes of 16-bit rows that decides: a = 127 x or 448 x is
// exact (18 bits), and where a / b is not on a border it is 2^-19 of its size or more beside one.  4-bit codes: codes_by_borders.
// The quotients of float32 rows are off by 2^-21 of their size (x - lo, a, the span and the quotient: 2.5 steps of 2^-23 at most).
#include "cache_format.cuh"
#include "tc_ptx.cuh"

namespace kvc {

namespace {

using namespace fmt;

constexpr int kWarps = 8;

struct ConvertArgs {
  CacheView in[2], out[2];
  RowList rows;
  int chunks;                                // groups of heads of a row that a warp takes at a time
  int rows_per_warp;                         // 1 .. 16 rows of the list
};

template <int F> __device__ constexpr float top_code() { return F == KVCRUSH_INT8 ? 127.f : F == KVCRUSH_E4M3 ? 448.f : 15.f; }

// Two quotients a / b to the nearest float32 but near the ends of the range; inv: 1 / b to an ulp.
__device__ __forceinline__ tc::f32x2 quotient2(tc::f32x2 a, tc::f32x2 minus_b, tc::f32x2 inv) {
  const tc::f32x2 q = tc::mul2(a, inv);
  return tc::fma2(tc::fma2(q, minus_b, a), inv, q);
}
__device__ __forceinline__ float reciprocal(float b) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(b));
  return fmaf(fmaf(-r, b, 1.f), r, r);
}
// the larger magnitude; NaN if either is NaN
__device__ __forceinline__ float larger(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

__device__ __forceinline__ float larger3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float least3(float a, float b, float c) {
  float d;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// ---- 4-bit codes of 16-bit rows -------------------------------------------------------------------------------
// x - lo need not be a float32 (lo = -1, x = -2^-30), and a quotient of rounded numbers can land on a border beside which it lies.
// So the quotient only names a border that is next to it, k + 1/2, and the code is k, k + 1 or, on the border, the even one by the sign of
//   r = 15 x - [(k + 1/2) hi + (29/2 - k) lo].
// The bracket is exact where both ends are zero or at least 2^-7 of the span: multiples of half the smaller end's last place, less
// than 2^24 of them.  r is then one rounding of the exact value, which keeps its sign.  Where an end is smaller, the bracket is off by
// 2^-18 of the span at most (half steps of float32: 14.5 and 15 for its constants, 15 for itself), and so is the quotient that decides.
// 0, 1/2 or 1 for a negative, zero or positive x
__device__ __forceinline__ float side(float x) {
  float d;
  asm("fma.rn.sat.f32 %0, %1, %2, 0f3F000000;" : "=f"(d) : "f"(x), "f"(0x1p127f));
  return d;
}

__device__ __forceinline__ void codes_by_borders(const float (&x)[8], float lo, float hi, float shift, float inv, uint32_t (&c)[8]) {
  const tc::f32x2 magic = tc::splat2(12582912.f), minus_magic = tc::splat2(-12582912.f);     // as in quantize_row
  const tc::f32x2 factor = tc::splat2(15.f * shift * inv), first = tc::splat2(fmaf(-lo, 15.f * shift * inv, -0.5f)), num = tc::splat2(15.f * shift);
  const tc::f32x2 step = tc::splat2((lo - hi) * shift), start = tc::splat2(fmaf(-14.5f, lo * shift, -0.5f * (hi * shift)));
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const tc::f32x2 y = tc::pack2f(x[i], x[i + 1]);
    tc::f32x2 n = tc::add2(tc::fma2(y, factor, first), magic);
    float r0, r1;
    tc::unpack2(tc::fma2(y, num, tc::fma2(tc::add2(n, minus_magic), step, start)), r0, r1);
    n = tc::add2(n, tc::pack2f(side(r0), side(r1)));           // ties to even
    tc::unpack2(n, r0, r1);
    c[i] = __float_as_uint(r0); c[i + 1] = __float_as_uint(r1);
  }
}

// Codes of the pieces of a row whose kLanes lanes call this together; scale (and zero) come back in every lane.  there: which of
// the lane's pieces exist.  FI: type of the values.
template <int FI, int F, int kLanes, int kVecs>
__device__ __forceinline__ void quantize_row(const float (&x)[kVecs][8], const bool (&there)[kVecs], Raw8<F> (&codes)[kVecs], float& scale,
                                             float& zero) {
  float big = 0.f, lo = FLT_MAX, hi = -FLT_MAX;      // pieces that do not exist are zeros
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    float l = x[v][0], h = x[v][0];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      if (F == KVCRUSH_INT4) { l = least3(l, x[v][i], x[v][i + 1]); h = larger3(h, x[v][i], x[v][i + 1]); }
      else big = larger(larger(big, fabsf(x[v][i])), fabsf(x[v][i + 1]));
    }
    if (F == KVCRUSH_INT4 && there[v]) { lo = fminf(lo, l); hi = larger(hi, h); }
  }
#pragma unroll
  for (int d = 1; d < kLanes; d <<= 1) {
    if (F == KVCRUSH_INT4) {
      lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, d));
      hi = larger(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, d));
    } else {
      big = larger(big, __shfl_xor_sync(0xFFFFFFFFu, big, d));
    }
  }
  const float span = F == KVCRUSH_INT4 ? hi - lo : big;
  scale = span * (1.f / top_code<F>());
  zero = F == KVCRUSH_INT4 ? lo : 0.f;
  const bool bad = !(span <= FLT_MAX);               // a NaN or an infinity, or INT4's span overflows
  if (scale < 0x1p-126f) scale = 0.f;
  if (bad) scale = zero = __uint_as_float(0x7FC00000u);
  // a power of two that keeps products and remainders away from both ends of the range
  const float shift = span > 0x1p64f ? 0x1p-64f : span < 0x1p-64f ? 0x1p64f : 1.f;
  const uint32_t keep = bad || scale == 0.f ? 0u : ~0u;
  const float den = span * shift;
  const float inv1 = reciprocal(den);
  const tc::f32x2 num = tc::splat2(top_code<F>() * shift), minus_den = tc::splat2(-den), inv = tc::splat2(inv1), minus_lo = tc::splat2(-lo);
  const tc::f32x2 magic = tc::splat2(12582912.f);    // 1.5 * 2^23 on top: the nearest integer in the low bits, ties to even
  constexpr bool kBorders = F == KVCRUSH_INT4 && FI != KVCRUSH_FP32;
#pragma unroll
  for (int v = 0; v < kVecs; ++v) {
    uint32_t c[8];
    if constexpr (kBorders) {
      codes_by_borders(x[v], lo, hi, shift, inv1, c);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        tc::f32x2 y = tc::pack2f(x[v][i], x[v][i + 1]);
        if (F == KVCRUSH_INT4) y = tc::add2(y, minus_lo);
        y = quotient2(tc::mul2(y, num), minus_den, inv);
        if (F != KVCRUSH_E4M3) y = tc::add2(y, magic);
        float y0, y1;
        tc::unpack2(y, y0, y1);
        c[i] = __float_as_uint(y0); c[i + 1] = __float_as_uint(y1);
      }
    }
    Raw8<F>& out = codes[v];
    if constexpr (F == KVCRUSH_INT8) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        out.w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410) & keep;
    } else if constexpr (F == KVCRUSH_E4M3) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(c[4 * i]), __uint_as_float(c[4 * i + 1])), __NV_SATFINITE, __NV_E4M3);
        const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(c[4 * i + 2]), __uint_as_float(c[4 * i + 3])), __NV_SATFINITE, __NV_E4M3);
        out.w[i] = (a | b << 16) & keep;
      }
    } else {
      // nibbles of four channels pair up by a shift, bytes by a permutation
      uint32_t p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = c[2 * i + 1] * 16u + c[2 * i];    // the low byte
      out.w[0] = __byte_perm(__byte_perm(p[0], p[1], 0x0040), __byte_perm(p[2], p[3], 0x0040), 0x5410) & keep;
    }
  }
}

// A row has kLanes lanes of kVecs pieces.  One warp: kSteps * 32 / kLanes heads of one tensor, for a few consecutive rows of the list.  Where the rows come from and go
// to is found for all of them at once, a lane a row, since it takes a chain of dependent loads.
template <int FI, int FO, int kLanes, int kVecs, int kSteps>
__global__ void __launch_bounds__(kWarps * 32, 3)
convert_kernel(Shape s, ConvertArgs a, int n_tensors) {
  chain_wait();
  chain_trigger();
  constexpr int kRowsPerStep = 32 / kLanes;
  const int lane = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5);
  const int per_group = a.chunks * n_tensors;
  const long long row0 = (item <= 0x7FFFFFFF ? (long long)((unsigned)item / (unsigned)per_group) : item / per_group) * a.rows_per_warp;
  long long end = a.rows.total;
  const int n_seg = s.n_layers * s.n_seqs;
  if (a.rows.cu_kept) end = min(end, (long long)__ldg(a.rows.cu_kept + n_seg));      // `total` is an upper bound
  if (row0 >= end) return;
  const int part = (int)(item % per_group), ten = part / a.chunks, chunk = part - ten * a.chunks;
  const int n_rows = (int)min((long long)a.rows_per_warp, end - row0);
  int layer = 0;
  long long src = 0, dst = 0;
  int seg = a.rows.cu_kept ? warp_segment_of_row(a.rows.cu_kept, n_seg, row0, lane) : 0;
  if (lane < n_rows) {
    const long long row = row0 + lane;
    if (a.rows.cu_kept) {
      while (seg + 1 < n_seg && (long long)__ldg(a.rows.cu_kept + seg + 1) <= row) ++seg;   // later rows may belong to a later segment
      layer = seg / s.n_seqs;
      const int seq = seg - layer * s.n_seqs, first = __ldg(a.rows.cu_kept + seg);
      src = (a.rows.idx ? (long long)__ldg(a.rows.idx + row) : row - first) + (a.rows.in_begin ? __ldg(a.rows.in_begin + seg) : __ldg(s.cu_seqlens + seq));
      dst = row - first + (a.rows.out_begin ? __ldg(a.rows.out_begin + seg) : first - __ldg(a.rows.cu_kept + layer * s.n_seqs));
    } else {
      layer = (int)(row / s.T);
      const int tok = (int)(row - (long long)layer * s.T);
      src = dst = tok;
      if (a.rows.in_begin || a.rows.out_begin) {
        const int seq = seq_of_token(s.cu_seqlens, s.n_seqs, tok), off = tok - __ldg(s.cu_seqlens + seq);
        seg = layer * s.n_seqs + seq;
        if (a.rows.in_begin) src = __ldg(a.rows.in_begin + seg) + (long long)off;
        if (a.rows.out_begin) dst = __ldg(a.rows.out_begin + seg) + (long long)off;
      }
    }
  }
  const CacheView in = a.in[ten], out = a.out[ten];
  const int sub = lane & (kLanes - 1);
  const int h0 = chunk * kSteps * kRowsPerStep + lane / kLanes;
  // offsets of the lane's first row: in and out in channels, scales of the quantised side in floats
  const long long ib = layer * in.sl + src * in.st, ob = layer * out.sl + dst * out.st;
  const long long sb = kQuantized<FI> ? layer * in.scl + src * in.sct : layer * out.scl + dst * out.sct;
  const unsigned char* ip = static_cast<const unsigned char*>(in.ptr) + bytes_of<FI>(sub * 8);
  unsigned char* op = static_cast<unsigned char*>(const_cast<void*>(out.ptr)) + bytes_of<FO>(sub * 8);
  constexpr int kPiece = kLanes * 8;                 // channels from a lane's piece to its next
  bool exists[kVecs];
#pragma unroll
  for (int v = 0; v < kVecs; ++v) exists[v] = sub * 8 + v * kPiece < s.D;
  Raw8<FI> next[kSteps][kVecs];
  float2 next_sc[kSteps];
  auto load = [&](int r) {
    const long long ir = __shfl_sync(0xFFFFFFFFu, ib, r), sr = __shfl_sync(0xFFFFFFFFu, sb, r);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int h = h0 + u * kRowsPerStep;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
#pragma unroll
        for (int i = 0; i < Raw8<FI>::kWords; ++i) next[u][v].w[i] = 0;
        if (h < s.Hkv && exists[v]) next[u][v].load(ip + bytes_of<FI>(ir + h * in.sh + v * kPiece));
      }
      if constexpr (kQuantized<FI>) {
        const float* p = in.scales + sr + h * in.sch;
        next_sc[u] = make_float2(0.f, 0.f);
        if (h < s.Hkv) { if constexpr (FI == KVCRUSH_INT4) next_sc[u] = __ldg(reinterpret_cast<const float2*>(p)); else next_sc[u].x = __ldg(p); }
      }
    }
  };
  load(0);
  for (int r = 0; r < n_rows; ++r) {
    // the next row is under way while this one is converted
    const long long orow = __shfl_sync(0xFFFFFFFFu, ob, r), sr = __shfl_sync(0xFFFFFFFFu, sb, r);
    Raw8<FI> raw[kSteps][kVecs];
    float2 sc[kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      if constexpr (kQuantized<FI>) sc[u] = next_sc[u];
#pragma unroll
      for (int v = 0; v < kVecs; ++v) raw[u][v] = next[u][v];
    }
    if (r + 1 < n_rows) load(r + 1);
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int h = h0 + u * kRowsPerStep;
      float x[kVecs][8];
#pragma unroll
      for (int v = 0; v < kVecs; ++v) raw[u][v].widen(x[v]);
      if constexpr (kQuantized<FO>) {
        Raw8<FO> codes[kVecs];
        float scale, zero;
        quantize_row<FI, FO, kLanes, kVecs>(x, exists, codes, scale, zero);
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
          if (h < s.Hkv && exists[v]) codes[v].store(op + bytes_of<FO>(orow + h * out.sh + v * kPiece));
        if (h < s.Hkv && sub == 0) {
          float* p = out.scales + sr + h * out.sch;
          if constexpr (FO == KVCRUSH_INT4) *reinterpret_cast<float2*>(p) = make_float2(scale, zero); else *p = scale;
        }
      } else {
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
          if (h < s.Hkv && exists[v]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[v][i] = FI == KVCRUSH_INT4 ? fmaf(x[v][i], sc[u].x, sc[u].y) : x[v][i] * sc[u].x;
            Raw8<FO> w;
            w.narrow(x[v]);
            w.store(op + bytes_of<FO>(orow + h * out.sh + v * kPiece));
          }
        }
      }
    }
  }
}

template <int FI, int FO, int kLanes, int kVecs>
int launch_lanes(const Shape& s, ConvertArgs& a, int n_tensors, cudaStream_t stream) {
  // Half as many rows in flight on the way to 4 bits, whose constants need the registers: with as many as elsewhere, and spills, 32
  // heads of 128 took 173 us for 157, heads of 64 123 for 66.
  constexpr int kInFlight = FO == KVCRUSH_INT4 ? 2 : 4, kSteps = kVecs == 1 ? kInFlight : kVecs == 2 ? kInFlight / 2 : 1, heads = kSteps * 32 / kLanes;
  a.chunks = (s.Hkv + heads - 1) / heads;
  // as many rows a warp as leave the chip several times the warps it holds
  a.rows_per_warp = 1;
  while (a.rows_per_warp < 16 && a.rows.total * a.chunks * n_tensors > 256LL * sm_count() * a.rows_per_warp) a.rows_per_warp *= 2;
  const long long groups = (a.rows.total + a.rows_per_warp - 1) / a.rows_per_warp;
  const long long blocks = (groups * a.chunks * n_tensors + kWarps - 1) / kWarps;
  if (blocks > 0x7FFFFFFFLL) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(convert_kernel<FI, FO, kLanes, kVecs, kSteps>, dim3((unsigned)blocks), dim3(kWarps * 32), 0, stream, 1, s, a, n_tensors);
}

// Lanes and pieces of a row: few lanes with several pieces, so that the row's statistics cost little.
template <int FI, int FO>
int launch_formats(const Shape& s, ConvertArgs& a, int n_tensors, cudaStream_t stream) {
  if (s.D <= 32) return launch_lanes<FI, FO, 4, 1>(s, a, n_tensors, stream);
  if (s.D <= 64) return launch_lanes<FI, FO, 4, 2>(s, a, n_tensors, stream);
  if (s.D <= 96) return launch_lanes<FI, FO, 4, 3>(s, a, n_tensors, stream);
  if (s.D <= 128) return launch_lanes<FI, FO, 8, 2>(s, a, n_tensors, stream);
  if (s.D <= 192) return launch_lanes<FI, FO, 8, 3>(s, a, n_tensors, stream);
  return launch_lanes<FI, FO, 16, 2>(s, a, n_tensors, stream);
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
