// Element types of a cache in registers: 16-bit and 32-bit values, 8- and 4-bit codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>

#include "common.cuh"

namespace kvc {
namespace fmt {

// Channels of one byte address: bytes per channel as a fraction.
template <int F> struct Bits { static constexpr int value = F == KVCRUSH_FP32 ? 32 : F == KVCRUSH_INT4 ? 4 : F == KVCRUSH_INT8 || F == KVCRUSH_E4M3 ? 8 : 16; };
template <int F> constexpr bool kQuantized = F >= KVCRUSH_INT8;
template <int F> __host__ __device__ constexpr long long bytes_of(long long channels) { return channels * Bits<F>::value / 8; }

__device__ __forceinline__ float2 unpack_bf16(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
__device__ __forceinline__ float2 unpack_fp16(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_fp16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Byte `i` of codes as 2^23 + byte, exactly: the byte becomes the low mantissa bits.
__device__ __forceinline__ float biased_byte(uint32_t codes, int i) { return __uint_as_float(__byte_perm(codes, 0x4B000000u, 0x7440u + i)); }

// N channels (a multiple of 4) from the registers of their codes, without scale; INT4: codes as they are, 0 .. 15.
template <int F>
__device__ __forceinline__ void codes4(uint32_t v, float (&out)[4]) {
  if constexpr (F == KVCRUSH_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = biased_byte(v ^ 0x80808080u, i) - 8388736.f;
  } else if constexpr (F == KVCRUSH_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> (16 * i)), __NV_E4M3);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      out[2 * i] = f.x; out[2 * i + 1] = f.y;
    }
  } else {                                           // the low 16 bits of v
    const uint32_t low = v & 0x0F0F0F0Fu, high = (v >> 4) & 0x0F0F0F0Fu;
    out[0] = biased_byte(low, 0) - 8388608.f; out[1] = biased_byte(high, 0) - 8388608.f;
    out[2] = biased_byte(low, 1) - 8388608.f; out[3] = biased_byte(high, 1) - 8388608.f;
  }
}

// Eight consecutive channels as they lie in memory.
template <int F>
struct Raw8 {
  static constexpr int kWords = Bits<F>::value / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const unsigned char* p) {
    if constexpr (kWords == 1) w[0] = __ldcs(reinterpret_cast<const unsigned int*>(p));
    else if constexpr (kWords == 2) { const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p)); w[0] = v.x; w[1] = v.y; }
    else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p) + i / 4);
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void store(unsigned char* p) const {
    if constexpr (kWords == 1) __stcs(reinterpret_cast<unsigned int*>(p), w[0]);
    else if constexpr (kWords == 2) __stcs(reinterpret_cast<uint2*>(p), make_uint2(w[0], w[1]));
    else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) __stcs(reinterpret_cast<uint4*>(p) + i / 4, make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
    }
  }
  // values, or codes without their scale
  __device__ __forceinline__ void widen(float (&x)[8]) const {
    if constexpr (F == KVCRUSH_FP32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else if constexpr (F == KVCRUSH_BF16 || F == KVCRUSH_FP16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = F == KVCRUSH_BF16 ? unpack_bf16(w[i]) : unpack_fp16(w[i]);
        x[2 * i] = f.x; x[2 * i + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float c[4];
        codes4<F>(F == KVCRUSH_INT4 ? w[0] >> (16 * i) : w[F == KVCRUSH_INT4 ? 0 : i], c);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * i + j] = c[j];
      }
    }
  }
  __device__ __forceinline__ void narrow(const float (&x)[8]) {      // value types only
    if constexpr (F == KVCRUSH_FP32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = F == KVCRUSH_BF16 ? pack_bf16(x[2 * i], x[2 * i + 1]) : pack_fp16(x[2 * i], x[2 * i + 1]);
    }
  }
};

}  // namespace fmt
}  // namespace kvc
