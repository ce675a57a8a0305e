// Attention of new tokens over a cache of 16-bit values or 8- or 4-bit codes, on the tensor cores.
//
// Bound by reading the cache, which passes through the chip once for every block of 8 to 32 query rows.  A cluster shares one
// (layer, sequence, KV head) and a block of its query rows (new tokens x query heads of the group); a warp takes tiles of 16
// keys.  Both products run as mma.sync with the cache as the left operand, which needs no staging of the cache:
//   logits   S^T[16 keys x 8 rows] = K Q^T: a lane's 16-byte piece of a key row is used as the operand registers of its
//            steps as it arrives; the channels may come in any order as long as the queries' registers do too
//   output   O^T[16 channels x 8 rows] += V^T P^T: a lane holds the same channels of four keys and pairs them up with byte
//            permutations; the weights are turned around by one 8x8 transposition a half tile
// Codes are used as exact 16-bit integers; a row's scale multiplies the logit, and the weight on the other side, so that no
// value is ever dequantised.  Weights that carry a scale have a maximum of their own (below), since the largest weight
// need not belong to the largest product of weight and scale.
#pragma once

#include <atomic>

#include "attend_common.cuh"

namespace kvc {
namespace att {

using namespace fmt;

constexpr int kMaxDevices = 64;

// ---- registers of a tile -----------------------------------------------------------------------------------

// 16-bit type that codes and weights are multiplied in
template <int F, int FQ> constexpr int kArith = kQuantized<F> ? KVCRUSH_FP16 : FQ;

template <int A>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (A == KVCRUSH_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

__device__ __forceinline__ uint32_t sub_half2(uint32_t a, uint32_t b) {
  const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint32_t fma_half2(uint32_t a, uint32_t b, uint32_t c) {
  const __half2 d = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ uint32_t e4m3_half2(uint32_t two_codes) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two_codes, __NV_E4M3);
  return (uint32_t)h.x | (uint32_t)h.y << 16;
}
// Integers as half-precision numbers: the bits of 1024 + n with n in the low mantissa bits, less 1024 and the offset.
constexpr uint32_t k1024 = 0x64006400u, k1032 = 0x64086408u, k1152 = 0x64806480u, kSixteenth = 0x2C002C00u, kMinus72 = 0xD480D480u;
// bytes 0 and 1 (hi: 2 and 3) of a word of signed bytes, offset by 128
template <bool kHi> __device__ __forceinline__ uint32_t int8_half2(uint32_t offset_bytes) {
  return sub_half2(__byte_perm(offset_bytes, k1024, kHi ? 0x7372 : 0x7170), k1152);
}
// the codes (less 8) in bits 4 i of either half word
template <int I> __device__ __forceinline__ uint32_t int4_half2(uint32_t v) {
  const uint32_t s = I >= 2 ? v >> 8 : v;
  if constexpr (I % 2 == 0) return sub_half2((s & 0x000F000Fu) | k1024, k1032);
  else return fma_half2((s & 0x00F000F0u) | k1024, kSixteenth, kMinus72);
}

// Where the channels of a head lie in a lane's registers.  DP: channels rounded up to 64, 128 or 256.
template <int F, int DP>
struct Layout {
  static constexpr int kBits = Bits<F>::value;
  // keys: pieces of at most 16 bytes; lane c of a quad holds kChannels channels from piece * 4 kChannels + c * kChannels on
  static constexpr int kChannels = kBits == 16 ? 8 : kBits == 8 ? 16 : DP == 64 ? 16 : 32;
  static constexpr int kPieces = DP / (4 * kChannels);
  static constexpr int kWords = kChannels * kBits / 32;
  // values: pieces of at most 16 bytes; lane g of eight holds kVChannels channels from piece * 8 kVChannels + g * kVChannels on
  static constexpr int kVChannels = kBits == 16 ? 8 : kBits == 8 ? (DP >= 128 ? 16 : 8) : DP / 8;
  static constexpr int kVPieces = DP / (8 * kVChannels);
  static constexpr int kVWords = kVChannels * kBits / 32;
  __device__ static __forceinline__ int k_channel(int piece, int c) { return (piece * 4 + c) * kChannels; }
  __device__ static __forceinline__ int v_channel(int piece, int g) { return (piece * 8 + g) * kVChannels; }
  // first of the two channels of m-tile mt that lane g holds (rows g and g + 8 of the operand)
  __device__ static __forceinline__ int out_channel(int mt, int g) { return v_channel(mt / (kVChannels / 2), g) + 2 * (mt % (kVChannels / 2)); }
};

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const unsigned char* p, bool there) {
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = 0u;
  if (there) {
    if constexpr (N == 4) { const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p)); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else if constexpr (N == 2) { const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p)); w[0] = v.x; w[1] = v.y; }
    else w[0] = __ldcs(reinterpret_cast<const unsigned int*>(p));
  }
}

// Where a tile's rows are: row numbers of its two halves of eight keys, and how many of each exist.
struct Halves {
  int row[2];
  int n[2];
};
struct Source {
  const unsigned char *k, *v;                // of the layer and head
  uint32_t k_st, v_st;                       // bytes, below 2^31
  const float *ks, *vs;
  uint32_t k_sct, v_sct;                     // floats
};
template <class T> __device__ __forceinline__ const T* at_row(const T* base, int row, uint32_t stride) {
  return base + (unsigned long long)(uint32_t)row * stride;
}

template <int F, int DP>
struct KeyTile {
  using L = Layout<F, DP>;
  uint32_t a[2][L::kPieces][L::kWords];      // keys g and g + 8
  float2 sc[2];                              // scale (and zero)
  // kFull: all 16 keys exist
  template <bool kFull>
  __device__ __forceinline__ void load(const Source& s, const Halves& h, int D, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const bool there = kFull || g < h.n[j];
      const unsigned char* p = at_row(s.k, h.row[j] + g, s.k_st);
#pragma unroll
      for (int i = 0; i < L::kPieces; ++i) load_words(a[j][i], p + bytes_of<F>(L::k_channel(i, c)), there && L::k_channel(i, c) < D);
      if constexpr (kQuantized<F>) {
        sc[j] = make_float2(0.f, 0.f);
        const float* sp = at_row(s.ks, h.row[j] + g, s.k_sct);
        if (there) { if (F == KVCRUSH_INT4) sc[j] = __ldg(reinterpret_cast<const float2*>(sp)); else sc[j].x = __ldg(sp); }
      }
    }
  }
  // Operand pairs of word i of a piece: two channels each.
  __device__ static __forceinline__ void pairs(uint32_t w, uint32_t (&p)[32 / L::kBits / 2]) {
    if constexpr (F == KVCRUSH_INT8) { p[0] = int8_half2<false>(w ^ 0x80808080u); p[1] = int8_half2<true>(w ^ 0x80808080u); }
    else if constexpr (F == KVCRUSH_E4M3) { p[0] = e4m3_half2(w & 0xFFFFu); p[1] = e4m3_half2(w >> 16); }
    else if constexpr (F == KVCRUSH_INT4) { p[0] = int4_half2<0>(w); p[1] = int4_half2<1>(w); p[2] = int4_half2<2>(w); p[3] = int4_half2<3>(w); }
    else p[0] = w;
  }
};
// FO: whose layout the output has.  Values of another type than the cache's (those of new tokens, 16-bit) are loaded eight
// channels at a time from where the cache's layout has them.
template <int F, int DP, int FO = F>
struct ValueTile {
  using L = Layout<F, DP>;
  __device__ static __forceinline__ int channel(int piece, int g) {
    if constexpr (F == FO) return L::v_channel(piece, g);
    else return Layout<FO, DP>::out_channel(4 * piece, g);
  }
  uint32_t a[4][L::kVPieces][L::kVWords];    // keys 2c, 2c + 1, 2c + 8, 2c + 9
  float2 sc[2];                              // keys g and g + 8
  template <bool kFull>
  __device__ __forceinline__ void load(const Source& s, const Halves& h, int D, int lane) {
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool there = kFull || 2 * c + (j & 1) < h.n[j >> 1];
      const unsigned char* p = at_row(s.v, h.row[j >> 1] + 2 * c + (j & 1), s.v_st);
#pragma unroll
      for (int i = 0; i < L::kVPieces; ++i) load_words(a[j][i], p + bytes_of<F>(channel(i, g)), there && channel(i, g) < D);
    }
    if constexpr (kQuantized<F>) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        sc[j] = make_float2(0.f, 0.f);
        const float* sp = at_row(s.vs, h.row[j] + g, s.v_sct);
        if (kFull || g < h.n[j]) { if (F == KVCRUSH_INT4) sc[j] = __ldg(reinterpret_cast<const float2*>(sp)); else sc[j].x = __ldg(sp); }
      }
    }
  }
  // Operand pairs (key a, key b) of the channels of word i of both keys.
  __device__ static __forceinline__ void pairs(uint32_t wa, uint32_t wb, uint32_t (&p)[32 / L::kBits]) {
    if constexpr (F == KVCRUSH_INT8) {
      const uint32_t lo = __byte_perm(wa, wb, 0x5140) ^ 0x80808080u, hi = __byte_perm(wa, wb, 0x7362) ^ 0x80808080u;
      p[0] = int8_half2<false>(lo); p[1] = int8_half2<true>(lo); p[2] = int8_half2<false>(hi); p[3] = int8_half2<true>(hi);
    } else if constexpr (F == KVCRUSH_E4M3) {
      const uint32_t lo = __byte_perm(wa, wb, 0x5140), hi = __byte_perm(wa, wb, 0x7362);
      p[0] = e4m3_half2(lo & 0xFFFFu); p[1] = e4m3_half2(lo >> 16); p[2] = e4m3_half2(hi & 0xFFFFu); p[3] = e4m3_half2(hi >> 16);
    } else if constexpr (F == KVCRUSH_INT4) {
      const uint32_t lo = __byte_perm(wa, wb, 0x5410), hi = __byte_perm(wa, wb, 0x7632);
      p[0] = int4_half2<0>(lo); p[1] = int4_half2<1>(lo); p[2] = int4_half2<2>(lo); p[3] = int4_half2<3>(lo);
      p[4] = int4_half2<0>(hi); p[5] = int4_half2<1>(hi); p[6] = int4_half2<2>(hi); p[7] = int4_half2<3>(hi);
    } else {
      p[0] = __byte_perm(wa, wb, 0x5410); p[1] = __byte_perm(wa, wb, 0x7632);
    }
  }
};

// One channel of a value row, codes without their scale (INT4: less 8).
template <int F>
__device__ __forceinline__ float value_at(const unsigned char* row, int channel) {
  if constexpr (F == KVCRUSH_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(row)[channel]);
  else if constexpr (F == KVCRUSH_FP16) return __half2float(reinterpret_cast<const __half*>(row)[channel]);
  else if constexpr (F == KVCRUSH_INT8) return (float)reinterpret_cast<const signed char*>(row)[channel];
  else if constexpr (F == KVCRUSH_E4M3) return __low2float(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)row[channel], __NV_E4M3)));
  else return (float)(int)((row[channel >> 1] >> (4 * (channel & 1))) & 15) - 8.f;
}
// Is any of the four numbers (or two, of 16 bits) of a word not finite?
template <int F>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  if constexpr (F == KVCRUSH_BF16 || F == KVCRUSH_FP16) {
    constexpr uint32_t e = F == KVCRUSH_BF16 ? 0x7F80u : 0x7C00u;
    return (w & e) == e || (w >> 16 & e) == e;
  } else if constexpr (F == KVCRUSH_E4M3) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (w >> (8 * i) & 0x7Fu) == 0x7Fu;
    return bad;
  } else {
    return false;
  }
}

// ---- state of a warp ------------------------------------------------------------------------------------------

// Rows 2c and 2c + 1 of each of NB blocks of eight rows.  m, l: maximum of the logits (log2 domain) and sum of 2^(x - m).
// m2: what the output is relative to; for a quantised cache the maximum of x + log2(scale of the value row), otherwise m.
// b: sum of 2^(x - m) * zero of the value row (INT4).
template <int NB, int DP, bool kScaled>
struct Running {
  float m[NB][2], l[NB][2], m2[NB][2], b[NB][2];
  float o[NB][DP / 16][4];
};

// Queries as operands of the logits: rows of `stride` bytes in shared memory, in the order of the cache's channels.
struct Queries {
  const unsigned char* sh;
  int stride;
};

// Multiplies a tile of keys with 8 NB query rows.
template <int F, int A, int DP, int NB, bool kRegs, int kQRegs>
__device__ __forceinline__ void logits(const KeyTile<F, DP>& K, const Queries& q, const uint32_t (&qr)[kQRegs], int lane, float (&x)[NB][4]) {
  using L = Layout<F, DP>;
  constexpr int kPairs = 32 / L::kBits / 2 < 1 ? 1 : 32 / L::kBits / 2;   // of a word
  const int g = lane >> 2, c = lane & 3;
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[n][i] = 0.f;
#pragma unroll
  for (int i = 0; i < L::kPieces; ++i) {
    uint32_t pa[L::kChannels / 2], pb[L::kChannels / 2];
#pragma unroll
    for (int w = 0; w < L::kWords; ++w) {
      uint32_t p[kPairs], r[kPairs];
      KeyTile<F, DP>::pairs(K.a[0][i][w], p);
      KeyTile<F, DP>::pairs(K.a[1][i][w], r);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) { pa[w * kPairs + j] = p[j]; pb[w * kPairs + j] = r[j]; }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int e = 0; e < L::kChannels / 8; ++e) {                   // eight channels: two steps
        uint32_t b[4];
        if constexpr (kRegs) {
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = qr[((n * L::kPieces + i) * (L::kChannels / 8) + e) * 4 + j];
        } else {
          const uint4 v = *reinterpret_cast<const uint4*>(q.sh + (n * 8 + g) * q.stride + (L::k_channel(i, c) + 8 * e) * 2);
          b[0] = v.x; b[1] = v.y; b[2] = v.z; b[3] = v.w;
        }
        mma<A>(x[n], pa[4 * e], pb[4 * e], pa[4 * e + 1], pb[4 * e + 1], b[0], b[1]);
        mma<A>(x[n], pa[4 * e + 2], pb[4 * e + 2], pa[4 * e + 3], pb[4 * e + 3], b[2], b[3]);
      }
    }
  }
}

// Adds a tile to the running state.  x: logits (log2 domain), -inf where a key is not seen (then `hidden`, bit 4 n + i, says
// so); F, A: the tile's type and the type it is multiplied in; kScaled: the state's output has a maximum of its own;
// kFull: every key exists and is seen by all rows.  Maxima start at the lowest finite number, so that a logit of -inf
// has weight 0 whatever came before.
template <int F, int FO, int A, int DP, int NB, bool kScaled, bool kFull>
__device__ __forceinline__ void add_tile(const ValueTile<F, DP, FO>& V, const Source& src, const Halves& h, int D, float (&x)[NB][4], uint32_t hidden,
                                         bool masked, Running<NB, DP, kScaled>& run, int lane) {
  using L = Layout<F, DP>;
  // log2 of the value rows' scales
  float lv[2] = {0.f, 0.f}, vz[2] = {0.f, 0.f};
  if constexpr (kQuantized<F>) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      lv[j] = __log2f(V.sc[j].x);
      if (F == KVCRUSH_INT4) vz[j] = fmaf(8.f, V.sc[j].x, V.sc[j].y);
    }
  }
  float d[NB][4], d2[NB][4];
  auto differences = [&] {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        d[n][i] = x[n][i] - run.m[n][i & 1];
        if (kScaled) d2[n][i] = (x[n][i] + lv[i >> 1]) - run.m2[n][i & 1];
      }
  };
  differences();
  // The maximum of a row seldom moves: the reduction over the tile's keys is done where any lane has a larger logit.
  float most = 0.f;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    most = fmaxf(fmaxf(most, fmaxf(d[n][0], d[n][1])), fmaxf(d[n][2], d[n][3]));
    if (kScaled) most = fmaxf(fmaxf(most, fmaxf(d2[n][0], d2[n][1])), fmaxf(d2[n][2], d2[n][3]));
  }
  if (__any_sync(kAll, most > 0.f)) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float big = fmaxf(x[n][i], x[n][i + 2]), big2 = kScaled ? fmaxf(x[n][i] + lv[0], x[n][i + 2] + lv[1]) : 0.f;
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) {
          big = fmaxf(big, __shfl_xor_sync(kAll, big, k));
          if (kScaled) big2 = fmaxf(big2, __shfl_xor_sync(kAll, big2, k));
        }
        const float m = fmaxf(run.m[n][i], big), f = ex2(run.m[n][i] - m);
        run.m[n][i] = m;
        run.l[n][i] *= f;
        if (kScaled) run.b[n][i] *= f;
        float f2 = f;
        if constexpr (kScaled) {
          const float m2 = fmaxf(run.m2[n][i], big2);
          f2 = ex2(run.m2[n][i] - m2);
          run.m2[n][i] = m2;
        }
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) { run.o[n][t][i] *= f2; run.o[n][t][i + 2] *= f2; }
      }
    differences();
  }
  uint32_t b0[NB], b1[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = ex2(d[n][i]);
      const bool unseen = !kFull && (hidden >> (4 * n + i) & 1u);
      run.l[n][i & 1] += p;
      w[i] = p;
      if constexpr (kScaled) {
        if (F == KVCRUSH_INT4) run.b[n][i & 1] = fmaf(p, unseen ? 0.f : vz[i >> 1], run.b[n][i & 1]);
        w[i] = kQuantized<F> && unseen ? 0.f : ex2(d2[n][i]);
      }
    }
    x[n][0] = w[0]; x[n][1] = w[1]; x[n][2] = w[2]; x[n][3] = w[3];
    b0[n] = transpose8x8(A == KVCRUSH_BF16 ? pack_bf16(w[0], w[1]) : pack_fp16(w[0], w[1]));
    b1[n] = transpose8x8(A == KVCRUSH_BF16 ? pack_bf16(w[2], w[3]) : pack_fp16(w[2], w[3]));
  }
  if (!kFull && masked) {
    // A weight of 0 takes a value that is not finite along: where there is one, every row adds up the keys that it sees.
    bool bad = false;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < L::kVPieces; ++i)
#pragma unroll
        for (int k = 0; k < L::kVWords; ++k) bad |= not_finite<F>(V.a[j][i][k]);
    if (__any_sync(kAll, bad)) {
      const int g = lane >> 2, c = lane & 3;
#pragma unroll 1
      for (int key = 0; key < kTile; ++key) {
        if ((key & 7) >= h.n[key >> 3]) continue;
        const unsigned char* row = at_row(src.v, h.row[key >> 3] + (key & 7), src.v_st);
        const uint32_t hid = __shfl_sync(kAll, hidden, (key & 7) * 4 + c);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float w[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float lo = __shfl_sync(kAll, x[n][i], (key & 7) * 4 + c), hi = __shfl_sync(kAll, x[n][i + 2], (key & 7) * 4 + c);
            w[i] = key < 8 ? lo : hi;
          }
#pragma unroll
          for (int t = 0; t < DP / 16; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int ch = Layout<FO, DP>::out_channel(t, g) + (i >> 1);
              const bool unseen = hid >> (4 * n + (key < 8 ? 0 : 2) + (i & 1)) & 1u;
              if (ch < D && !unseen) run.o[n][t][i] = fmaf(w[i & 1], value_at<F>(row, ch), run.o[n][t][i]);
            }
        }
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < L::kVPieces; ++i)
#pragma unroll
    for (int k = 0; k < L::kVWords; ++k) {
      constexpr int kPairs = 32 / L::kBits;
      uint32_t p[kPairs], r[kPairs];
      ValueTile<F, DP, FO>::pairs(V.a[0][i][k], V.a[1][i][k], p);
      ValueTile<F, DP, FO>::pairs(V.a[2][i][k], V.a[3][i][k], r);
#pragma unroll
      for (int j = 0; j < kPairs; j += 2) {
        const int t = ((i * L::kVWords + k) * kPairs + j) / 2;
#pragma unroll
        for (int n = 0; n < NB; ++n) mma<A>(run.o[n][t], p[j], p[j + 1], r[j], r[j + 1], b0[n], b1[n]);
      }
    }
}

// ---- the kernel ---------------------------------------------------------------------------------------------------

// Byte offsets in dynamic shared memory.
template <int F, int FQ, int DP, int NB, int kWarps>
struct Mem {
  static constexpr int kRows = 8 * NB;
  static constexpr int kQStride = DP * 2 + 16, kOStride = DP + 4;
  static constexpr int kQ = 0;                                                    // queries in the cache's order
  static constexpr int kQNew = kQuantized<F> ? kQ + kRows * kQStride : kQ;        // queries as they are
  static constexpr int kRowScale = kQNew + kRows * kQStride;                      // [kRows] factor and sum of the queries
  static constexpr int kPart = kRowScale + kRows * 8;                             // [kWarps + 1][kRows] Part
  static constexpr int kFactor = kPart + (kWarps + 1) * kRows * (int)sizeof(Part);
  static constexpr int kO = (kFactor + kRows * (kMaxCluster + 1) * 4 + 15) / 16 * 16;
  static constexpr int kEnd = kO + kWarps * kRows * kOStride * 4;
};

template <int F, int FQ, int DP, int NB, int kWarps, int kBlocks, bool kPages>
__global__ void __launch_bounds__(kWarps * 32, kBlocks)
attend_kernel(AttendArgs a) {
  using M = Mem<F, FQ, DP, NB, kWarps>;
  using L = Layout<F, DP>;
  constexpr bool kScaled = kQuantized<F>;
  constexpr int A = kArith<F, FQ>, kRows = M::kRows;
  // Keys of a tile that take few registers are loaded a tile ahead; otherwise other warps' loads fill the time.
  constexpr bool kAhead = DP * Bits<F>::value <= 1024;
  constexpr bool kRegs = NB * DP <= 128 && kAhead;             // queries in registers
  extern __shared__ __align__(16) unsigned char sh[];
  chain_wait();
  chain_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const int n_blk = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const Shape& s = a.s;
  Unit w;
  if (!unit_of<kPages>(a, blockIdx.x / n_blk, kRows, w)) return;
  PageMem pages{};
  int n_chosen = 0;
  if constexpr (kPages) {
    pages = page_mem(sh + (M::kEnd + 15) / 16 * 16, a.pages.max_pages, a.pages.budget, s.D);
    n_chosen = choose_pages<FQ, kWarps * 32>(a, w, cluster, n_blk, rank, pages);
  }
  float2* row_scale = reinterpret_cast<float2*>(sh + M::kRowScale);
  // queries: a warp takes a row
  for (int r = warp; r < kRows; r += kWarps) {
    const unsigned char* q = static_cast<const unsigned char*>(a.Q.ptr);
    if (r < w.rows) q += bytes_of<FQ>(w.layer * a.Q.sl + (w.first + w.token(s.G, r)) * a.Q.st + (w.hk * s.G + w.head(s.G, r)) * a.Q.sh);
    float v[DP / 32], big = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
      const int d = 32 * i + lane;
      v[i] = r < w.rows && d < s.D ? value_at<FQ>(q, d) : 0.f;
      reinterpret_cast<uint16_t*>(sh + M::kQNew + r * M::kQStride)[d] = (uint16_t)(FQ == KVCRUSH_BF16 ? pack_bf16(v[i], 0.f) : pack_fp16(v[i], 0.f));
      big = fmaxf(big, fabsf(v[i]));
      sum += v[i];
    }
    if constexpr (kScaled) {
      // bf16 queries are multiplied as half precision: a power of two that brings the row's largest value just under 2^15
      // keeps all their bits (those 2^-29 below the largest fade out)
      float f = 1.f;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) { big = fmaxf(big, __shfl_xor_sync(kAll, big, d)); sum += __shfl_xor_sync(kAll, sum, d); }
      if (FQ == KVCRUSH_BF16 && big > 0.f) {
        const int e = min((int)(__float_as_uint(big) >> 23), 254) - 127;
        f = __uint_as_float((uint32_t)(min(14 - e, 126) + 127) << 23);
      }
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) {
        int d = 32 * i + lane;
        if (F == KVCRUSH_INT4) d = (d & ~7) | (d & 3) << 1 | (d >> 2 & 1);           // codes of a word pair up as 0 4, 1 5, 2 6, 3 7
        reinterpret_cast<uint16_t*>(sh + M::kQ + r * M::kQStride)[d] = (uint16_t)pack_fp16(v[i] * f, 0.f);
      }
      if (lane == 0) row_scale[r] = make_float2(a.scale_log2 / f, sum * a.scale_log2);
    }
  }
  __syncthreads();
  const Queries q{sh + M::kQ, M::kQStride}, q_new{sh + M::kQNew, M::kQStride};
  constexpr int kQRegs = kRegs ? NB * DP / 8 : 1;
  uint32_t qr[kQRegs];
  if constexpr (kRegs) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < L::kPieces; ++i)
#pragma unroll
        for (int e = 0; e < L::kChannels / 8; ++e) {
          const uint4 v = *reinterpret_cast<const uint4*>(q.sh + (n * 8 + g) * q.stride + (L::k_channel(i, c) + 8 * e) * 2);
          const int at = ((n * L::kPieces + i) * (L::kChannels / 8) + e) * 4;
          qr[at] = v.x; qr[at + 1] = v.y; qr[at + 2] = v.z; qr[at + 3] = v.w;
        }
  }
  float2 rs[NB][2];
  if constexpr (kScaled) {
#pragma unroll
    for (int n = 0; n < NB; ++n) { rs[n][0] = row_scale[n * 8 + 2 * c]; rs[n][1] = row_scale[n * 8 + 2 * c + 1]; }
  }

  Running<NB, DP, kScaled> run;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
#pragma unroll
    for (int i = 0; i < 2; ++i) { run.m[n][i] = run.m2[n][i] = -FLT_MAX; run.l[n][i] = run.b[n][i] = 0.f; }
#pragma unroll
    for (int t = 0; t < DP / 16; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) run.o[n][t][i] = 0.f;
  }

  const Source src{static_cast<const unsigned char*>(a.K.ptr) + bytes_of<F>(w.layer * a.K.sl + w.hk * a.K.sh),
                   static_cast<const unsigned char*>(a.V.ptr) + bytes_of<F>(w.layer * a.V.sl + w.hk * a.V.sh),
                   (uint32_t)bytes_of<F>(a.K.st), (uint32_t)bytes_of<F>(a.V.st), a.K.scales + w.layer * a.K.scl + w.hk * a.K.sch,
                   a.V.scales + w.layer * a.V.scl + w.hk * a.V.sch, (uint32_t)a.K.sct, (uint32_t)a.V.sct};
  const int halves_per_page = kPages ? a.pages.page_size / 8 : 1;
  const int cached = kPages ? (n_chosen * halves_per_page + 1) / 2 : (w.seen + kTile - 1) / kTile;
  const int n_tiles = cached + (w.own + kTile - 1) / kTile;
  const int per = (n_tiles + n_blk - 1) / n_blk, lo = min(n_tiles, rank * per), hi = min(n_tiles, lo + per), hi_cached = min(hi, cached);
  // tiles whose keys all exist and are seen by every query row; of the chosen pages only the last may be short
  int full;
  if (kPages) {
    const int last = n_chosen ? pages.chosen[n_chosen - 1] : 0;
    full = n_chosen ? ((n_chosen - 1) * a.pages.page_size + min(a.pages.page_size, w.seen - last * a.pages.page_size)) / kTile : 0;
  } else {
    full = (w.own ? w.seen : w.limit(s.G, 0)) / kTile;
  }
  const int hi_full = min(hi, full);
  auto halves = [&](int t) {
    Halves h;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int pos = t * kTile + j * 8;
      bool there = true;
      if constexpr (kPages) {
        const int hn = 2 * t + j, page = hn / halves_per_page;
        there = page < n_chosen;
        pos = there ? pages.chosen[page] * a.pages.page_size + (hn - page * halves_per_page) * 8 : 0;
      }
      h.n[j] = there ? min(8, max(0, w.seen - pos)) : 0;
      h.row[j] = w.begin + pos;
    }
    return h;
  };
  auto scale_logits = [&](const KeyTile<F, DP>& K, float (&x)[NB][4]) {
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kScaled) {
          x[n][i] *= rs[n][i & 1].x * K.sc[i >> 1].x;
          if (F == KVCRUSH_INT4) x[n][i] = fmaf(fmaf(8.f, K.sc[i >> 1].x, K.sc[i >> 1].y), rs[n][i & 1].y, x[n][i]);
        } else {
          x[n][i] *= a.scale_log2;
        }
      }
  };
  {
    auto step = [&](const Halves& h, const KeyTile<F, DP>& K, auto&& prefetch) {
      ValueTile<F, DP> V;
      V.template load<true>(src, h, s.D, lane);
      prefetch();
      float x[NB][4];
      logits<F, A, DP, NB, kRegs>(K, q, qr, lane, x);
      scale_logits(K, x);
      add_tile<F, F, A, DP, NB, kScaled, true>(V, src, h, s.D, x, 0u, false, run, lane);
    };
    int t = lo + warp;
    if constexpr (kAhead) {
      // while a tile is multiplied the next one's keys are in flight
      KeyTile<F, DP> k0, k1;
      Halves h0, h1;
      if (t < hi_full) { h0 = halves(t); k0.template load<true>(src, h0, s.D, lane); }
      for (; t < hi_full; t += 2 * kWarps) {
        step(h0, k0, [&] { if (t + kWarps < hi_full) { h1 = halves(t + kWarps); k1.template load<true>(src, h1, s.D, lane); } });
        if (t + kWarps >= hi_full) break;
        step(h1, k1, [&] { if (t + 2 * kWarps < hi_full) { h0 = halves(t + 2 * kWarps); k0.template load<true>(src, h0, s.D, lane); } });
      }
    } else {
      for (; t < hi_full; t += kWarps) {
        const Halves h = halves(t);
        KeyTile<F, DP> K;
        K.template load<true>(src, h, s.D, lane);
        step(h, K, [] {});
      }
    }
  }
  // short tiles, and those that some rows see only a part of
  for (int t = max(lo, full) + warp; t < hi_cached; t += kWarps) {
    const Halves h = halves(t);
    KeyTile<F, DP> K;
    ValueTile<F, DP> V;
    K.template load<false>(src, h, s.D, lane);
    V.template load<false>(src, h, s.D, lane);
    float x[NB][4];
    logits<F, A, DP, NB, kRegs>(K, q, qr, lane, x);
    scale_logits(K, x);
    uint32_t hidden = 0;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = n * 8 + 2 * c + (i & 1);
        if (g >= h.n[i >> 1] || (!kPages && t * kTile + g + (i >> 1) * 8 >= w.limit(s.G, min(r, w.rows - 1)))) {
          x[n][i] = neg_inf();
          hidden |= 1u << (4 * n + i);
        }
      }
    add_tile<F, F, A, DP, NB, kScaled, false>(V, src, h, s.D, x, hidden, true, run, lane);
  }
  // keys among the new tokens
  if (!kPages && w.own && hi > cached) {
    const Source fresh{static_cast<const unsigned char*>(a.K_new.ptr) + bytes_of<FQ>(w.layer * a.K_new.sl + w.hk * a.K_new.sh),
                       static_cast<const unsigned char*>(a.V_new.ptr) + bytes_of<FQ>(w.layer * a.V_new.sl + w.hk * a.V_new.sh),
                       (uint32_t)bytes_of<FQ>(a.K_new.st), (uint32_t)bytes_of<FQ>(a.V_new.st), nullptr, nullptr, 0, 0};
    for (int t = max(lo, cached) + warp; t < hi; t += kWarps) {
      const int first = (t - cached) * kTile;
      Halves h;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        h.row[j] = w.first + first + j * 8;
        h.n[j] = min(8, max(0, w.own - first - j * 8));
      }
      KeyTile<FQ, DP> K;
      ValueTile<FQ, DP, F> V;
      K.template load<false>(fresh, h, s.D, lane);
      V.template load<false>(fresh, h, s.D, lane);
      float x[NB][4];
      const uint32_t none[1] = {0u};
      logits<FQ, FQ, DP, NB, false>(K, q_new, none, lane, x);
      uint32_t hidden = 0;
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = min(n * 8 + 2 * c + (i & 1), w.rows - 1), key = g + (i >> 1) * 8;
          x[n][i] *= a.scale_log2;
          if (g >= h.n[i >> 1] || !sees_new(a, w, w.token(s.G, r), first + key)) {
            x[n][i] = neg_inf();
            hidden |= 1u << (4 * n + i);
          }
        }
      add_tile<FQ, F, FQ, DP, NB, kScaled, false>(V, fresh, h, s.D, x, hidden, true, run, lane);
    }
  }

  // the block's warps
  Part* part = reinterpret_cast<Part*>(sh + M::kPart);
  Part* warp_part = part + kRows;
  float* o = reinterpret_cast<float*>(sh + M::kO);
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        run.l[n][i] += __shfl_xor_sync(kAll, run.l[n][i], d);
        if (F == KVCRUSH_INT4) run.b[n][i] += __shfl_xor_sync(kAll, run.b[n][i], d);
      }
      if (g == 0) warp_part[warp * kRows + n * 8 + 2 * c + i] = Part{run.m[n][i], run.l[n][i], kScaled ? run.m2[n][i] : run.m[n][i], run.b[n][i]};
#pragma unroll
      for (int t = 0; t < DP / 16; ++t) {
        float* at = o + (warp * kRows + n * 8 + 2 * c + i) * M::kOStride;
        // the two channels are neighbours
        *reinterpret_cast<float2*>(at + L::out_channel(t, g)) = make_float2(run.o[n][t][i], run.o[n][t][i + 2]);
      }
    }
  __syncthreads();
  if (tid < kRows) {
    float m = -FLT_MAX, l = 0.f, m2 = -FLT_MAX, b = 0.f;
    for (int k = 0; k < kWarps; ++k) { m = fmaxf(m, warp_part[k * kRows + tid].m); m2 = fmaxf(m2, warp_part[k * kRows + tid].m2); }
    for (int k = 0; k < kWarps; ++k) {
      Part& p = warp_part[k * kRows + tid];
      const float f = ex2(p.m - m);
      l = fmaf(p.l, f, l);
      b = fmaf(p.b, f, b);
      p.b = ex2(p.m2 - m2);                              // factor of the warp's output
    }
    part[tid] = Part{m, l, m2, b};
  }
  __syncthreads();
  for (int e = tid; e < w.rows * (DP / 4); e += kWarps * 32) {
    const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float f = warp_part[k * kRows + r].b;
      const float4 v = *reinterpret_cast<const float4*>(o + (k * kRows + r) * M::kOStride + d);
      sum.x = fmaf(v.x, f, sum.x); sum.y = fmaf(v.y, f, sum.y); sum.z = fmaf(v.z, f, sum.z); sum.w = fmaf(v.w, f, sum.w);
    }
    *reinterpret_cast<float4*>(o + r * M::kOStride + d) = sum;
  }
  join_and_write<FQ, kWarps * 32>(a, w, cluster, n_blk, rank, o, M::kOStride, part, reinterpret_cast<float*>(sh + M::kFactor));
}

// ---- host -----------------------------------------------------------------------------------------------------

// Largest cluster of this kernel that the device runs (write-once cache per device): 16 blocks are more than every device
// grants.
template <class Kernel>
int largest_cluster(Kernel kern, int threads, size_t dyn, std::atomic<int>* known) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return 8; }
  int n = known[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  n = 8;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(kMaxCluster);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = dyn;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kMaxCluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  int resident = 0;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
      cudaOccupancyMaxActiveClusters(&resident, kern, &cfg) == cudaSuccess && resident > 0)
    n = kMaxCluster;
  else
    cudaGetLastError();
  known[dev].store(n, std::memory_order_relaxed);
  return n;
}

template <int F, int FQ, int DP, int NB, bool kPages>
int launch_one(AttendArgs& a, cudaStream_t stream) {
  // Two blocks an SM at least: a chip has room for 14 clusters of 16 then, with one only for 7.
  constexpr int kWarps = NB * DP <= 128 ? 8 : 4, kBlocks = NB * DP == 256 ? 3 : 2;
  auto kern = attend_kernel<F, FQ, DP, NB, kWarps, kBlocks, kPages>;
  using M = Mem<F, FQ, DP, NB, kWarps>;
  const Shape& s = a.s;
  const long long rows = (long long)(kPages ? 1 : a.fresh.most) * s.G;
  a.row_blocks = (int)((rows + M::kRows - 1) / M::kRows);
  const long long units = (long long)s.n_layers * (kPages ? a.fresh.total : s.n_seqs) * s.Hkv * a.row_blocks;
  const long long keys = kPages ? (long long)(a.pages.budget < a.pages.max_pages ? a.pages.budget : a.pages.max_pages) * a.pages.page_size
                                : (long long)s.max_seqlen + (a.K_new.ptr ? a.fresh.most : 0);
  constexpr int most = (M::kEnd + 15) / 16 * 16;
  const size_t dyn = most + (kPages ? page_mem_bytes(a.pages.max_pages, a.pages.budget, s.D) : 0);
  constexpr int bound = most + (kPages ? kMaxPagesPerSeq * 12 + 256 * 16 + 2048 : 0);
  if (allow_dynamic_smem(kern, bound) != KVCRUSH_OK) return KVCRUSH_ERR_CUDA;
  static std::atomic<int> known[kMaxDevices];
  const int n_blk = cluster_size(units, (int)((keys + kTile - 1) / kTile), kWarps, largest_cluster(kern, kWarps * 32, bound, known), 4 * sm_count());
  if (units * n_blk > 0x7FFFFFFFLL) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(kern, dim3((unsigned)(units * n_blk)), dim3(kWarps * 32), dyn, stream, n_blk, a);
}

// Query rows of a block: as many as there are, up to 32 (16 with more than 128 channels, whose output takes the registers).
template <int F, int FQ, int DP>
int launch_rows(AttendArgs& a, cudaStream_t stream) {
  const long long rows = (long long)(a.pages.page_size ? 1 : a.fresh.most) * a.s.G;
  if (a.pages.page_size) return rows <= 8 ? launch_one<F, FQ, DP, 1, true>(a, stream) : launch_one<F, FQ, DP, 2, true>(a, stream);
  if (rows <= 8) return launch_one<F, FQ, DP, 1, false>(a, stream);
  if constexpr (DP <= 128) {
    if (rows > 16) return launch_one<F, FQ, DP, 4, false>(a, stream);
  }
  return launch_one<F, FQ, DP, 2, false>(a, stream);
}

template <int F, int FQ>
int launch_width(AttendArgs& a, cudaStream_t stream) {
  if (a.s.D <= 64) return launch_rows<F, FQ, 64>(a, stream);
  if (a.s.D <= 128) return launch_rows<F, FQ, 128>(a, stream);
  return launch_rows<F, FQ, 256>(a, stream);
}

template <int F>
int launch_queries(AttendArgs& a, cudaStream_t stream) {
  return a.Q.dtype == KVCRUSH_BF16 ? launch_width<F, KVCRUSH_BF16>(a, stream) : launch_width<F, KVCRUSH_FP16>(a, stream);
}

}  // namespace att
}  // namespace kvc
