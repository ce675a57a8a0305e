// Attention of new tokens over a cache of 16-bit values or 8- or 4-bit codes, on the tensor cores.
//
// Bound by reading the cache, which passes through the chip once for every block of 8 to 32 query rows.  A cluster shares one
// (layer, sequence, KV head) and a block of its query rows (new tokens x query heads of the group); a warp takes tiles of 16
// keys, which it copies ahead into a ring of its own in shared memory (cp.async; rows and channels that do not exist
// arrive as zeros), so that no warp waits for another.  Both products run as mma.sync with the cache as the left operand:
//   logits   S^T[16 keys x 8 rows] = K Q^T
//   output   O^T[16 channels x 8 rows] += V^T P^T, the weights turned around by one 8x8 transposition a half tile
// 16-bit values become operands by ldmatrix.  Codes are used as exact half-precision integers: the channels of a product may
// come in any order, so a lane takes whole words of codes and pairs them up by byte permutations; a row's scale multiplies the
// logit, and the weight on the other side, so that no value is ever dequantised.  Weights that carry a scale have a
// maximum of their own (below), since the largest weight need not belong to the largest product of weight and scale.
// Measured, 8 KV heads of 128 with 4 query heads each: one token over 2048 bf16 rows 6.4 us, over 32768 4-bit rows 25 us
// (37.7 MB), over 16 ragged sequences of 8-bit rows 25 us (80 MB, 3.2 TB/s); 15 tokens of 32 heads of 96 over the same sequences
// in float16 103 us (472 MB, 4.6 TB/s).  Few units are bound by what one warp does for a tile one thing after the other (about
// 300 instructions and 1400 to 1700 clocks for 4-bit codes, 208 instructions for 16-bit values, at 7 to 8 warps an SM) and by what a block
// does once: 750 to 1000 clocks to find its unit, 1000 to 5000 for queries and first tiles, 2800 to 10000 for the join, which
// waits for the slowest block.
// Blocks of 32 rows over codes spill (128 channels: 488 bytes for 4-bit codes, 392 and 68 for 8-bit ones, at 255 registers), and so do
// those of 16 rows of 64 channels with eight warps (56 to 104 bytes at 128).  Many rows over codes are slow for that and because every
// block unpacks the cache again: 63 tokens of the heads above over 32768 rows take 309 us in INT8, 198 in E4M3, 281 in INT4, where
// bf16 goes through attend_tree.cu in 63; 15 tokens 110, 71 and 100 for 42.
#pragma once

#include "attend_common.cuh"

namespace kvc {
namespace att {

using namespace fmt;


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

__device__ __forceinline__ uint32_t e4m3_half2(uint32_t two_codes) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two_codes, __NV_E4M3);
  return (uint32_t)h.x | (uint32_t)h.y << 16;
}
// Integers as half-precision numbers: a byte or nibble in the low bits of a half word is a subnormal number, n * 2^-24, exactly,
// and the tensor cores multiply those as they are.  Codes are made unsigned that way: 8-bit ones carry 128 too much, 4-bit ones are
// taken less 8; what that adds to a sum over channels is known from the queries, and what it adds to a sum over keys from
// a product with ones.  4-bit codes of odd channels stand four bits higher and count 16 times: their queries are divided by 16,
// and their outputs.
constexpr uint32_t kOnes = 0x3C003C00u;
template <int F> constexpr float kOffset = F == KVCRUSH_INT8 ? 128.f : F == KVCRUSH_INT4 ? 8.f : 0.f;
template <int F> constexpr bool kInteger = F == KVCRUSH_INT8 || F == KVCRUSH_INT4;
// bytes 0 and 1 (hi: 2 and 3) of a word
template <bool kHi> __device__ __forceinline__ uint32_t byte_half2(uint32_t bytes) { return __byte_perm(bytes, 0u, kHi ? 0x4342 : 0x4140); }
// the codes in bits 4 I of either half word
template <int I> __device__ __forceinline__ uint32_t int4_half2(uint32_t v) { return (I >= 2 ? v >> 8 : v) & (I % 2 ? 0x00F000F0u : 0x000F000Fu); }

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
  // (16-bit values come through ldmatrix: channels g and g + 8 of sixteen)
  static constexpr int kPairStep = kBits == 16 ? 8 : 1;
  __device__ static __forceinline__ int out_channel(int mt, int g) {
    return kBits == 16 ? 16 * mt + g : v_channel(mt / (kVChannels / 2), g) + 2 * (mt % (kVChannels / 2));
  }
};

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

// Operand pairs of a word of a key row: two channels each.
template <int F>
__device__ __forceinline__ void key_pairs(uint32_t w, uint32_t (&p)[16 / Bits<F>::value]) {
  if constexpr (F == KVCRUSH_INT8) { p[0] = byte_half2<false>(w ^ 0x80808080u); p[1] = byte_half2<true>(w ^ 0x80808080u); }
  else if constexpr (F == KVCRUSH_E4M3) { p[0] = e4m3_half2(w & 0xFFFFu); p[1] = e4m3_half2(w >> 16); }
  else { p[0] = int4_half2<0>(w); p[1] = int4_half2<1>(w); p[2] = int4_half2<2>(w); p[3] = int4_half2<3>(w); }
}
// Operand pairs (key a, key b) of the channels of a word of both keys' value rows.
template <int F>
__device__ __forceinline__ void value_pairs(uint32_t wa, uint32_t wb, uint32_t (&p)[32 / Bits<F>::value]) {
  if constexpr (F == KVCRUSH_INT8) {
    const uint32_t lo = __byte_perm(wa, wb, 0x5140) ^ 0x80808080u, hi = __byte_perm(wa, wb, 0x7362) ^ 0x80808080u;
    p[0] = byte_half2<false>(lo); p[1] = byte_half2<true>(lo); p[2] = byte_half2<false>(hi); p[3] = byte_half2<true>(hi);
  } else if constexpr (F == KVCRUSH_E4M3) {
    const uint32_t lo = __byte_perm(wa, wb, 0x5140), hi = __byte_perm(wa, wb, 0x7362);
    p[0] = e4m3_half2(lo & 0xFFFFu); p[1] = e4m3_half2(lo >> 16); p[2] = e4m3_half2(hi & 0xFFFFu); p[3] = e4m3_half2(hi >> 16);
  } else {
    const uint32_t lo = __byte_perm(wa, wb, 0x5410), hi = __byte_perm(wa, wb, 0x7632);
    p[0] = int4_half2<0>(lo); p[1] = int4_half2<1>(lo); p[2] = int4_half2<2>(lo); p[3] = int4_half2<3>(lo);
    p[4] = int4_half2<0>(hi); p[5] = int4_half2<1>(hi); p[6] = int4_half2<2>(hi); p[7] = int4_half2<3>(hi);
  }
}

// ---- a tile in shared memory -------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16_ahead(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// kBytes of 4, 8 or 16; nothing is read and zeros are written unless there
template <int kBytes>
__device__ __forceinline__ void copy_ahead(uint32_t dst, const void* src, bool there) {
  const int n = there ? kBytes : 0;
  if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(kBytes), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <bool kTrans>
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  if constexpr (kTrans) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
  else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <int N>
__device__ __forceinline__ void shared_words(uint32_t (&w)[N], uint32_t addr) {
  if constexpr (N == 4) asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
  else if constexpr (N == 2) asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr) : "memory");
  else asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(addr) : "memory");
}

// Keys, then values, 16 rows each, then their scales.  Rows of 128 bytes or more have their 16-byte chunks permuted so that
// neither product's reads meet in a bank; shorter ones are 16 bytes apart.
template <int F, int DP>
struct Stage {
  static constexpr int kRowBytes = DP * Bits<F>::value / 8, kChunks = kRowBytes / 16;
  static constexpr bool kPermuted = kRowBytes >= 128;
  static constexpr int kPitch = kPermuted ? kRowBytes : kRowBytes + 16, kTileBytes = kTile * kPitch;
  static constexpr int kScaleBytes = F == KVCRUSH_INT4 ? 8 : 4;
  static constexpr int kScales = 2 * kTileBytes, kBytes = kScales + (kQuantized<F> ? 2 * kTile * kScaleBytes : 0);
  // 16-bit rows are read eight rows to a chunk; codes by pairs of rows (keys) and by every other row (values)
  __device__ static constexpr int permutation(int row) { return !kPermuted ? 0 : kQuantized<F> ? (row & 6) ^ (row & 1) << 2 : row & 7; }
  __device__ static __forceinline__ uint32_t at(int row, int chunk) { return (uint32_t)(row * kPitch + (chunk ^ permutation(row)) * 16); }

  // A lane copies the same chunk of every kRowsPerCopy-th row.
  static constexpr int kRowsPerCopy = 32 / kChunks;
  struct Lane {
    const unsigned char *k, *v;              // its chunk of its first row
    const float* scales;                     // lanes 0 .. 15: of the keys, 16 .. 31: of the values
    uint32_t k_st, v_st, scale_st;           // strides
    uint32_t dst;                            // where its first row goes, without the chunk
    int chunk;                               // permuted as in its first row
    bool used;                               // the head has these channels
  };
  static __device__ __forceinline__ Lane lane_of(const Source& s, int D, int lane) {
    Lane l;
    const int row = lane / kChunks, chunk = lane % kChunks;
    l.k = at_row(s.k, row, s.k_st) + chunk * 16;
    l.v = at_row(s.v, row, s.v_st) + chunk * 16;
    l.k_st = s.k_st; l.v_st = s.v_st;
    l.scales = lane < 16 ? s.ks : s.vs;
    l.scale_st = lane < 16 ? s.k_sct : s.v_sct;
    l.dst = row * kPitch;
    l.chunk = chunk ^ permutation(row & 7);
    l.used = chunk * 16 < (int)bytes_of<F>(D);
    return l;
  }
  // kFull: all 16 rows exist; otherwise zeros take the place of those that do not.
  template <bool kFull>
  static __device__ __forceinline__ void fetch(uint32_t stage, const Lane& l, const Halves& h, int lane) {
    if (l.used) {
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const unsigned char* base = kv ? l.v : l.k;
        const uint32_t stride = kv ? l.v_st : l.k_st;
        const uint32_t to = stage + kv * kTileBytes + l.dst;
        const unsigned char* p = base;
#pragma unroll
        for (int i = 0; i < kTile / kRowsPerCopy; ++i) {
          const int first = i * kRowsPerCopy;                        // of the rows of this copy
          if (kRowsPerCopy == 16) p = at_row(base, lane / kChunks < 8 ? h.row[0] : h.row[1] - 8, stride);
          else if (first % 8 == 0) p = at_row(base, h.row[first / 8], stride);
          const uint32_t dst = to + first * kPitch + ((l.chunk ^ permutation(first & 7)) << 4);
          if (kFull) {
            copy16_ahead(dst, p);
          } else {
            const int row = lane / kChunks + first;
            const bool there = (row & 7) < (row < 8 ? h.n[0] : h.n[1]);
            copy_ahead<16>(dst, there ? p : base, there);
          }
          p += (unsigned long long)kRowsPerCopy * stride;
        }
      }
    }
    if constexpr (kQuantized<F>) {
      const int row = lane & 15, first = row < 8 ? h.row[0] : h.row[1] - 8;
      const bool there = kFull || (row & 7) < (row < 8 ? h.n[0] : h.n[1]);
      copy_ahead<kScaleBytes>(stage + kScales + lane * kScaleBytes, there ? at_row(l.scales, first + row, l.scale_st) : l.scales, there);
    }
  }
  // scale (and zero) of keys or values row `row`
  static __device__ __forceinline__ float2 scale(uint32_t stage, bool values, int row) {
    float2 v = make_float2(0.f, 0.f);
    const uint32_t p = stage + kScales + (values ? kTile + row : row) * kScaleBytes;
    if constexpr (F == KVCRUSH_INT4) asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(p) : "memory");
    else asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v.x) : "r"(p) : "memory");
    return v;
  }
};

// One channel of row `row` of the values at `tile`, of the types that have numbers that are not finite; codes without their scale.
template <int F, int DP>
__device__ __forceinline__ float value_at(uint32_t tile, int row, int channel) {
  using T = Stage<F, DP>;
  const int byte = channel * Bits<F>::value / 8;
  uint32_t w[1];
  shared_words(w, tile + T::at(row, byte >> 4) + (byte & 12));
  if constexpr (F == KVCRUSH_BF16) return (channel & 1) ? unpack_bf16(w[0]).y : unpack_bf16(w[0]).x;
  else if constexpr (F == KVCRUSH_FP16) return (channel & 1) ? unpack_fp16(w[0]).y : unpack_fp16(w[0]).x;
  else return unpack_fp16(e4m3_half2(w[0] >> (8 * (channel & 3)) & 0xFFu)).x;
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
// b: sum of 2^(x - m) * zero of the value row (INT4).  ones: sum of the rounded weights, as an m-tile of ones gives it (all
// its rows are alike).
template <int NB, int DP, bool kScaled>
struct Running {
  float m[NB][2], l[NB][2], m2[NB][2], b[NB][2];
  float o[NB][DP / 16][4], ones[NB][4];
};

constexpr float kSlack = 8.f;

// Queries as operands: rows of `stride` bytes in shared memory, in the order of the cache's channels.
struct Queries {
  uint32_t sh;
  int stride;
};

// Multiplies a tile of keys with 8 NB query rows.  kRegs: the queries' operands are in qr, otherwise in shared memory.
template <int F, int A, int DP, int NB, bool kRegs, int kQRegs>
__device__ __forceinline__ void logits(uint32_t stage, const Queries& q, const uint32_t (&qr)[kQRegs], int lane, float (&x)[NB][4]) {
  using L = Layout<F, DP>;
  using T = Stage<F, DP>;
  const int g = lane >> 2, c = lane & 3;
  float y[NB][4];                            // a second chain of sums: half the latency
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[n][i] = y[n][i] = 0.f;
  if constexpr (!kQuantized<F>) {
    const int key = lane & 15;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {      // 32 channels: two steps
      uint32_t a[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) ldmatrix4<false>(a[j], stage + T::at(key, 4 * i + 2 * j + (lane >> 4)));
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        uint32_t b[4];
        if constexpr (kRegs) {
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = qr[(n * (DP / 32) + i) * 4 + j];
        } else {
          ldmatrix4<false>(b, q.sh + (n * 8 + (lane & 7)) * q.stride + (4 * i + (lane >> 3)) * 16);
        }
        mma<A>(x[n], a[0][0], a[0][1], a[0][2], a[0][3], b[0], b[1]);
        mma<A>(y[n], a[1][0], a[1][1], a[1][2], a[1][3], b[2], b[3]);
      }
    }
  } else {
    constexpr int kPairs = 32 / L::kBits / 2;                        // of a word
#pragma unroll
    for (int i = 0; i < L::kPieces; ++i) {
      uint32_t wa[L::kWords], wb[L::kWords], pa[L::kChannels / 2], pb[L::kChannels / 2];
      const int byte = (int)bytes_of<F>(L::k_channel(i, c));
      shared_words(wa, stage + T::at(g, byte >> 4) + (byte & 15));
      shared_words(wb, stage + T::at(g + 8, byte >> 4) + (byte & 15));
#pragma unroll
      for (int w = 0; w < L::kWords; ++w) {
        uint32_t p[kPairs], r[kPairs];
        key_pairs<F>(wa[w], p);
        key_pairs<F>(wb[w], r);
#pragma unroll
        for (int j = 0; j < kPairs; ++j) { pa[w * kPairs + j] = p[j]; pb[w * kPairs + j] = r[j]; }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int e = 0; e < L::kChannels / 8; ++e) {                 // eight channels: two steps
          uint32_t b[4];
          if constexpr (kRegs) {
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = qr[((n * L::kPieces + i) * (L::kChannels / 8) + e) * 4 + j];
          } else {
            shared_words(b, q.sh + (n * 8 + g) * q.stride + (L::k_channel(i, c) + 8 * e) * 2);
          }
          mma<A>(x[n], pa[4 * e], pb[4 * e], pa[4 * e + 1], pb[4 * e + 1], b[0], b[1]);
          mma<A>(y[n], pa[4 * e + 2], pb[4 * e + 2], pa[4 * e + 3], pb[4 * e + 3], b[2], b[3]);
        }
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[n][i] += y[n][i];
}

// The tile's values as operands: for every m-tile use(t, four operand registers).
template <int F, int DP, class Use>
__device__ __forceinline__ void value_operands(uint32_t stage, int lane, Use&& use) {
  using L = Layout<F, DP>;
  using T = Stage<F, DP>;
  const uint32_t values = stage + T::kTileBytes;
  if constexpr (!kQuantized<F>) {
    const int key = (lane & 7) + (lane >> 4) * 8;
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) {
      uint32_t a[4];
      ldmatrix4<true>(a, values + T::at(key, 2 * t + (lane >> 3 & 1)));
      use(t, a[0], a[1], a[2], a[3]);
    }
  } else {
    constexpr int kPairs = 32 / L::kBits;
    const int g = lane >> 2, c = lane & 3;
#pragma unroll
    for (int i = 0; i < L::kVPieces; ++i) {
      uint32_t w[4][L::kVWords];
      const int byte = (int)bytes_of<F>(L::v_channel(i, g));
#pragma unroll
      for (int j = 0; j < 4; ++j) shared_words(w[j], values + T::at(2 * c + (j & 1) + (j >> 1) * 8, byte >> 4) + (byte & 15));
#pragma unroll
      for (int k = 0; k < L::kVWords; ++k) {
        uint32_t p[kPairs], r[kPairs];
        value_pairs<F>(w[0][k], w[1][k], p);
        value_pairs<F>(w[2][k], w[3][k], r);
#pragma unroll
        for (int j = 0; j < kPairs; j += 2) use(((i * L::kVWords + k) * kPairs + j) / 2, p[j], p[j + 1], r[j], r[j + 1]);
      }
    }
  }
}
// 16-bit values for an output in the layout of a quantised cache FO.
template <int F, int FO, int DP, class Use>
__device__ __forceinline__ void value_operands_like(uint32_t stage, int lane, Use&& use) {
  using T = Stage<F, DP>;
  const uint32_t values = stage + T::kTileBytes;
  const int g = lane >> 2, c = lane & 3;
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    uint32_t w[4][1];
    const int byte = Layout<FO, DP>::out_channel(t, g) * 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) shared_words(w[j], values + T::at(2 * c + (j & 1) + (j >> 1) * 8, byte >> 4) + (byte & 15));
    use(t, __byte_perm(w[0][0], w[1][0], 0x5410), __byte_perm(w[0][0], w[1][0], 0x7632), __byte_perm(w[2][0], w[3][0], 0x5410),
        __byte_perm(w[2][0], w[3][0], 0x7632));
  }
}

// Adds a tile to the running state.  x: logits (log2 domain), -inf where a key is not seen (then bit 4 n + i of `hidden` says
// so); F, A: the tile's type and the type it is multiplied in; FO: the cache's type, whose layout the output has.  Maxima
// start at the lowest finite number, so that a logit of -inf has weight 0 whatever came before.
template <int F, int FO, int A, int DP, int NB>
__device__ __forceinline__ void add_tile(uint32_t stage, const Halves& h, int D, float (&x)[NB][4], uint32_t hidden,
                                         Running<NB, DP, kQuantized<FO>>& run, int lane) {
  constexpr bool kScaled = kQuantized<FO>;
  using T = Stage<F, DP>;
  const int g = lane >> 2;
  // log2 of the value rows' scales
  float lv[2] = {0.f, 0.f}, vz[2] = {0.f, 0.f};
  if constexpr (kQuantized<F>) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 sc = T::scale(stage, true, g + 8 * j);
      lv[j] = __log2f(sc.x);
      if (F == KVCRUSH_INT4) vz[j] = fmaf(8.f, sc.x, sc.y);
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
  // Weights may exceed 1: what they are relative to moves only where a logit is kSlack above it (in the log2 domain; half
  // precision holds weights up to 2^15).  Most tiles after the first leave it alone.
  float most = 0.f;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    most = fmaxf(fmaxf(most, fmaxf(d[n][0], d[n][1])), fmaxf(d[n][2], d[n][3]));
    if (kScaled) most = fmaxf(fmaxf(most, fmaxf(d2[n][0], d2[n][1])), fmaxf(d2[n][2], d2[n][3]));
  }
  if (__any_sync(kAll, most > kSlack)) {
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
        if (kInteger<FO>) run.ones[n][i] *= f2;
      }
    differences();
  }
  const bool masked = __any_sync(kAll, hidden != 0u);
  if (kScaled && masked) {                             // a scale that is NaN stays with the rows that see it
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (hidden >> (4 * n + i) & 1u) d2[n][i] = neg_inf();
  }
  uint32_t b0[NB], b1[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = ex2(d[n][i]);
      run.l[n][i & 1] += p;
      w[i] = p;
      if constexpr (kScaled) {
        if (F == KVCRUSH_INT4 && p != 0.f) run.b[n][i & 1] = fmaf(p, vz[i >> 1], run.b[n][i & 1]);
        w[i] = ex2(d2[n][i]);
      }
    }
    x[n][0] = w[0]; x[n][1] = w[1]; x[n][2] = w[2]; x[n][3] = w[3];
    b0[n] = transpose8x8(A == KVCRUSH_BF16 ? pack_bf16(w[0], w[1]) : pack_fp16(w[0], w[1]));
    b1[n] = transpose8x8(A == KVCRUSH_BF16 ? pack_bf16(w[2], w[3]) : pack_fp16(w[2], w[3]));
  }
  if (!kInteger<F> && masked) {
    // A weight of 0 takes a value that is not finite along: where there is one, every row adds up the keys that it sees.
    bool bad = false;
    for (uint32_t e = lane * 16; e < (uint32_t)T::kTileBytes; e += 512) {
      uint32_t v[4];
      if (T::kPermuted || (int)(e % T::kPitch) < T::kRowBytes) {     // not the space between rows
        shared_words(v, stage + T::kTileBytes + e);
#pragma unroll
        for (int k = 0; k < 4; ++k) bad |= not_finite<F>(v[k]);
      }
    }
    if (__any_sync(kAll, bad)) {
      const int c = lane & 3;
#pragma unroll 1
      for (int key = 0; key < kTile; ++key) {
        if ((key & 7) >= h.n[key >> 3]) continue;
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
              const int ch = Layout<FO, DP>::out_channel(t, g) + (i >> 1) * Layout<FO, DP>::kPairStep;
              const bool unseen = hid >> (4 * n + (key < 8 ? 0 : 2) + (i & 1)) & 1u;
              if (ch < D && !unseen) run.o[n][t][i] = fmaf(w[i & 1], value_at<F, DP>(stage + T::kTileBytes, key, ch), run.o[n][t][i]);
            }
        }
      }
      return;
    }
  }
  auto multiply = [&](int t, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
    for (int n = 0; n < NB; ++n) mma<A>(run.o[n][t], a0, a1, a2, a3, b0[n], b1[n]);
  };
  if constexpr (F == FO && kInteger<F>) {
#pragma unroll
    for (int n = 0; n < NB; ++n) mma<A>(run.ones[n], kOnes, kOnes, kOnes, kOnes, b0[n], b1[n]);
  }
  if constexpr (F == FO) value_operands<F, DP>(stage, lane, multiply);
  else value_operands_like<F, FO, DP>(stage, lane, multiply);
}

// ---- the kernel ---------------------------------------------------------------------------------------------------

// Byte offsets in dynamic shared memory.  The warps' outputs take the place of the rings at the end.
template <int F, int FQ, int DP, int NB, int kWarps, bool kPages>
struct Mem {
  static constexpr int kRows = 8 * NB;
  static constexpr int kQStride = DP * 2 + 16, kOStride = DP + 4;
  static constexpr int kQ = 0;                                                    // queries in the cache's order
  static constexpr int kQNew = kQuantized<F> ? kQ + kRows * kQStride : kQ;        // queries as they are
  static constexpr int kRowScale = kQNew + kRows * kQStride;                      // [kRows] factor and sum of the queries
  static constexpr int kPart = kRowScale + kRows * 8;                             // [kWarps][kRows] Part
  static constexpr int kRecv = kPart + kWarps * kRows * (int)sizeof(Part);
  static constexpr int kRing = (kRecv + (int)sizeof(Received<kRows, DP>) + 127) / 128 * 128;
  static constexpr int kO = kRing;
  // Rings as large as two blocks an SM allow (the choice of pages needs room too): as many stages as that holds, two at least, and
  // room for a tile of 16-bit new tokens.
  static constexpr int kStageBytes = (Stage<F, DP>::kBytes + 127) / 128 * 128;
  static constexpr int kWarpBytes = (kPages ? 64 * 1024 : 113 * 1024 - kRing) / kWarps;
  static constexpr int kStages = kWarpBytes / kStageBytes < 2 ? 2 : kWarpBytes / kStageBytes > 6 ? 6 : kWarpBytes / kStageBytes;
  static constexpr int kNewBytes = kQuantized<F> ? Stage<FQ, DP>::kBytes : 0;
  static constexpr int kRingBytes = kStages * kStageBytes > kNewBytes ? kStages * kStageBytes : kNewBytes;
  static constexpr int kOBytes = kWarps * kRows * kOStride * 4;
  static constexpr int kEnd = kRing + (kWarps * kRingBytes > kOBytes ? kWarps * kRingBytes : kOBytes);
};

template <int F, int FQ, int DP, int NB, int kWarps, int kBlocks, bool kPages>
__global__ void __launch_bounds__(kWarps * 32, kBlocks)
attend_kernel(AttendArgs a) {
  using M = Mem<F, FQ, DP, NB, kWarps, kPages>;
  using L = Layout<F, DP>;
  constexpr bool kScaled = kQuantized<F>;
  constexpr int A = kArith<F, FQ>, kRows = M::kRows;
  constexpr bool kRegs = NB * DP <= 128;                       // queries in registers
  extern __shared__ __align__(128) unsigned char sh[];
  chain_wait();
  chain_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const int n_blk = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const Shape& s = a.s;
  Unit w;
  if (!unit_of<kPages>(a, kRows, w)) return;
  PageMem pages{};
  int n_chosen = 0;
  if constexpr (kPages) {
    pages = page_mem(sh + (M::kEnd + 15) / 16 * 16, a.pages.max_pages, a.pages.budget, s.D);
    n_chosen = choose_pages<FQ, kWarps * 32>(a, w, cluster, n_blk, rank, pages);
  }
  if (n_blk > 1) cluster_arrive_relaxed();
  float2* row_scale = reinterpret_cast<float2*>(sh + M::kRowScale);
  const Source src{static_cast<const unsigned char*>(a.K.ptr) + bytes_of<F>(w.layer * a.K.sl + w.hk * a.K.sh),
                   static_cast<const unsigned char*>(a.V.ptr) + bytes_of<F>(w.layer * a.V.sl + w.hk * a.V.sh),
                   (uint32_t)bytes_of<F>(a.K.st), (uint32_t)bytes_of<F>(a.V.st), a.K.scales + w.layer * a.K.scl + w.hk * a.K.sch,
                   a.V.scales + w.layer * a.V.scl + w.hk * a.V.sch, (uint32_t)a.K.sct, (uint32_t)a.V.sct};
  Source fresh{};
  if (!kPages && w.own)
    fresh = Source{static_cast<const unsigned char*>(a.K_new.ptr) + bytes_of<FQ>(w.layer * a.K_new.sl + w.hk * a.K_new.sh),
                   static_cast<const unsigned char*>(a.V_new.ptr) + bytes_of<FQ>(w.layer * a.V_new.sl + w.hk * a.V_new.sh),
                   (uint32_t)bytes_of<FQ>(a.K_new.st), (uint32_t)bytes_of<FQ>(a.V_new.st), nullptr, nullptr, 0, 0};
  const int halves_per_page = kPages ? a.pages.page_size / 8 : 1;
  const uint32_t page_magic = kPages && halves_per_page > 1 ? 0xFFFFFFFFu / (uint32_t)halves_per_page + 1u : 0u;
  const int cached = kPages ? (n_chosen * halves_per_page + 1) / 2 : (w.seen + kTile - 1) / kTile;
  const int n_tiles = cached + (w.own + kTile - 1) / kTile;
  const int per = (n_tiles + n_blk - 1) / n_blk, lo = min(n_tiles, rank * per), hi = min(n_tiles, lo + per);
  // tiles whose keys all exist and are seen by every query row; of the chosen pages only the last may be short
  int full;
  if (kPages) {
    const int last = n_chosen ? pages.chosen[n_chosen - 1] : 0;
    full = n_chosen ? ((n_chosen - 1) * a.pages.page_size + min(a.pages.page_size, w.seen - last * a.pages.page_size)) / kTile : 0;
  } else {
    full = (w.own ? w.seen : w.limit(0)) / kTile;
  }
  auto halves = [&](int t) {
    Halves h;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int pos = t * kTile + j * 8;
      bool there = true;
      if constexpr (kPages) {
        // page = hn / halves_per_page by a product: exact for hn below 2^32 / halves_per_page
        const int hn = 2 * t + j, page = halves_per_page == 1 ? hn : (int)__umulhi((uint32_t)hn, page_magic);
        there = page < n_chosen;
        pos = there ? pages.chosen[page] * a.pages.page_size + (hn - page * halves_per_page) * 8 : 0;
      }
      h.n[j] = there ? min(8, max(0, w.seen - pos)) : 0;
      h.row[j] = w.begin + pos;
    }
    return h;
  };
  auto new_halves = [&](int t) {
    Halves h;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int first = (t - cached) * kTile + j * 8;
      h.row[j] = w.first + first;
      h.n[j] = min(8, max(0, w.own - first));
    }
    return h;
  };
  // The ring: while a tile is multiplied the next kStages - 1 are under way, and its place is filled again behind it.  Tiles of new tokens go through it too where they are of
  // the cache's type.
  using T = Stage<F, DP>;
  const uint32_t ring = smem_addr(sh + M::kRing) + warp * M::kRingBytes;
  const int hi_ring = kScaled ? min(hi, cached) : hi;
  if (s.D < DP) {                                      // channels that the head does not have are never copied
    for (int e = lane * 16; e < M::kRingBytes; e += 512)
      *reinterpret_cast<uint4*>(sh + M::kRing + warp * M::kRingBytes + e) = make_uint4(0u, 0u, 0u, 0u);
    __syncwarp();
  }
  const typename T::Lane of_cache = T::lane_of(src, s.D, lane);
  auto fetch = [&](int t, int stage) {
    const uint32_t to = ring + stage * M::kStageBytes;
    if (t < min(full, hi_ring)) T::template fetch<true>(to, of_cache, halves(t), lane);
    else if (t < hi_ring) {
      if constexpr (kScaled) T::template fetch<false>(to, of_cache, halves(t), lane);
      else if (t < cached) T::template fetch<false>(to, of_cache, halves(t), lane);
      else T::template fetch<false>(to, T::lane_of(fresh, s.D, lane), new_halves(t), lane);
    }
    copies_commit();
  };
  // queries: DP / 8 lanes take a row, a lane eight channels; all rows are loaded before the first is used
  {
    constexpr int kLanes = DP / 8, kPerStep = kWarps * 32 / kLanes, kQSteps = (kRows + kPerStep - 1) / kPerStep;
    const int d = (tid % kLanes) * 8, r0 = tid / kLanes;
    Raw8<FQ> raw[kQSteps];
#pragma unroll
    for (int u = 0; u < kQSteps; ++u) {
      const int r = r0 + u * kPerStep;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[u].w[i] = 0u;
      if (r < w.rows && d < s.D)
        raw[u].load(static_cast<const unsigned char*>(a.Q.ptr) + bytes_of<FQ>(w.layer * a.Q.sl + (w.first + w.token(r)) * a.Q.st + (w.hk * s.G + w.head(r)) * a.Q.sh + d));
    }
    // the first tiles are under way while the queries arrive
#pragma unroll
    for (int i = 0; i < M::kStages; ++i) fetch(lo + warp + i * kWarps, i);
#pragma unroll
    for (int u = 0; u < kQSteps; ++u) {
      const int r = r0 + u * kPerStep;
      if (r < kRows) *reinterpret_cast<uint4*>(sh + M::kQNew + r * M::kQStride + d * 2) = make_uint4(raw[u].w[0], raw[u].w[1], raw[u].w[2], raw[u].w[3]);
      if constexpr (kScaled) {
        float v[8], big = 0.f, sum = 0.f, f = 1.f;
        raw[u].widen(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) { big = fmaxf(big, fabsf(v[i])); sum += v[i]; }
#pragma unroll
        for (int k = 1; k < kLanes; k <<= 1) { big = fmaxf(big, __shfl_xor_sync(kAll, big, k)); sum += __shfl_xor_sync(kAll, sum, k); }
        // Queries are multiplied as half precision: a power of two that brings the row's largest value just under 2^15 keeps all
        // their bits (those 2^-25 below the largest fade out).
        if (big > 0.f) {
          const int e = min((int)(__float_as_uint(big) >> 23), 254) - 127;
          f = __uint_as_float((uint32_t)(min(14 - e, 126) + 127) << 23);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= F == KVCRUSH_INT4 && i % 2 ? f * 0.0625f : f;
        // the 4-bit codes of a word pair up as 0 4, 1 5, 2 6, 3 7
        const uint4 x = F == KVCRUSH_INT4 ? make_uint4(pack_fp16(v[0], v[4]), pack_fp16(v[1], v[5]), pack_fp16(v[2], v[6]), pack_fp16(v[3], v[7]))
                                          : make_uint4(pack_fp16(v[0], v[1]), pack_fp16(v[2], v[3]), pack_fp16(v[4], v[5]), pack_fp16(v[6], v[7]));
        if (r < kRows) *reinterpret_cast<uint4*>(sh + M::kQ + r * M::kQStride + d * 2) = x;
        if (r < kRows && d == 0) row_scale[r] = make_float2((kInteger<F> ? 0x1p24f : 1.f) * a.scale_log2 / f, sum * a.scale_log2);
      }
    }
  }
  __syncthreads();
  const Queries q{smem_addr(sh + M::kQ), M::kQStride}, q_new{smem_addr(sh + M::kQNew), M::kQStride};
  constexpr int kQRegs = kRegs ? NB * DP / 8 : 1;
  uint32_t qr[kQRegs];
  if constexpr (kRegs) {
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      if constexpr (!kScaled) {
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
          uint32_t v[4];
          ldmatrix4<false>(v, q.sh + (n * 8 + (lane & 7)) * q.stride + (4 * i + (lane >> 3)) * 16);
#pragma unroll
          for (int j = 0; j < 4; ++j) qr[(n * (DP / 32) + i) * 4 + j] = v[j];
        }
      } else {
#pragma unroll
        for (int i = 0; i < L::kPieces; ++i)
#pragma unroll
          for (int e = 0; e < L::kChannels / 8; ++e) {
            uint32_t v[4];
            shared_words(v, q.sh + (n * 8 + g) * q.stride + (L::k_channel(i, c) + 8 * e) * 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) qr[((n * L::kPieces + i) * (L::kChannels / 8) + e) * 4 + j] = v[j];
          }
      }
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
#pragma unroll
    for (int i = 0; i < 4; ++i) run.ones[n][i] = 0.f;
  }
  // keys of the tile that row n * 8 + 2c + (i & 1) does not see
  auto hide = [&](float (&x)[NB][4], const Halves& h, auto&& sees) {
    uint32_t hidden = 0;
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (g >= h.n[i >> 1] || !sees(g + (i >> 1) * 8, min(n * 8 + 2 * c + (i & 1), w.rows - 1))) {
          x[n][i] = neg_inf();
          hidden |= 1u << (4 * n + i);
        }
    return hidden;
  };
  int stage = 0;
  for (int t = lo + warp; t < hi_ring; t += kWarps) {
    copies_wait<M::kStages - 1>();
    __syncwarp();
    const uint32_t at = ring + stage * M::kStageBytes;
    float x[NB][4];
    logits<F, A, DP, NB, kRegs>(at, q, qr, lane, x);
    if constexpr (kScaled) {
      const float2 k0 = T::scale(at, false, g), k1 = T::scale(at, false, g + 8);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 sc = i < 2 ? k0 : k1;
          const float f = rs[n][i & 1].x * sc.x;
          x[n][i] = F == KVCRUSH_E4M3 ? x[n][i] * f : fmaf(x[n][i], f, (F == KVCRUSH_INT8 ? -kOffset<F> * sc.x : sc.y) * rs[n][i & 1].y);
        }
    } else {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] *= a.scale_log2;
    }
    uint32_t hidden = 0;
    Halves h{};
    if (t >= full) {
      if (kScaled || t < cached) {
        h = halves(t);
        hidden = hide(x, h, [&](int key, int r) { return kPages || t * kTile + key < w.limit(r); });
      } else {
        h = new_halves(t);
        hidden = hide(x, h, [&](int key, int r) { return sees_new(a, w, w.token(r), (t - cached) * kTile + key); });
      }
    }
    add_tile<F, F, A, DP, NB>(at, h, s.D, x, hidden, run, lane);
    __syncwarp();
    fetch(t + M::kStages * kWarps, stage);
    stage = stage == M::kStages - 1 ? 0 : stage + 1;
  }
  if constexpr (kInteger<F>) {                         // from units of the integer products to values
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int t = 0; t < DP / 16; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) run.o[n][t][i] = fmaf(run.o[n][t][i], F == KVCRUSH_INT4 && i >= 2 ? 0x1p20f : 0x1p24f, -kOffset<F> * run.ones[n][i & 1]);
  }
  if constexpr (kScaled && !kPages) {                  // new tokens beside a quantised cache
    for (int t = max(lo, cached) + warp; t < hi; t += kWarps) {
      const Halves h = new_halves(t);
      copies_wait<0>();
      __syncwarp();
      using TN = Stage<FQ, DP>;
      if (s.D < DP) {
        for (int e = lane * 16; e < TN::kBytes; e += 512) *reinterpret_cast<uint4*>(sh + M::kRing + warp * M::kRingBytes + e) = make_uint4(0u, 0u, 0u, 0u);
        __syncwarp();
      }
      TN::template fetch<false>(ring, TN::lane_of(fresh, s.D, lane), h, lane);
      copies_commit();
      copies_wait<0>();
      __syncwarp();
      float x[NB][4];
      const uint32_t none[1] = {0u};
      logits<FQ, FQ, DP, NB, false>(ring, q_new, none, lane, x);
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[n][i] *= a.scale_log2;
      const uint32_t hidden = hide(x, h, [&](int key, int r) { return sees_new(a, w, w.token(r), (t - cached) * kTile + key); });
      add_tile<FQ, F, FQ, DP, NB>(ring, h, s.D, x, hidden, run, lane);
    }
  }
  copies_wait<0>();
  __syncthreads();                                     // the outputs go where the rings were

  // the block's warps
  Part* part = reinterpret_cast<Part*>(sh + M::kPart);
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
      if (g == 0) part[warp * kRows + n * 8 + 2 * c + i] = Part{run.m[n][i], run.l[n][i], kScaled ? run.m2[n][i] : run.m[n][i], run.b[n][i]};
#pragma unroll
      for (int t = 0; t < DP / 16; ++t) {
        float* at = o + (warp * kRows + n * 8 + 2 * c + i) * M::kOStride;
        const int ch = L::out_channel(t, g);
        if constexpr (L::kPairStep == 1) *reinterpret_cast<float2*>(at + ch) = make_float2(run.o[n][t][i], run.o[n][t][i + 2]);
        else { at[ch] = run.o[n][t][i]; at[ch + L::kPairStep] = run.o[n][t][i + 2]; }
      }
    }
  join_and_write<FQ, kWarps, kRows, DP>(a, w, cluster, n_blk, rank, o, M::kOStride, part, reinterpret_cast<Received<kRows, DP>*>(sh + M::kRecv));
}

// ---- host -----------------------------------------------------------------------------------------------------

template <int F, int FQ, int DP, int NB, bool kPages>
int launch_one(AttendArgs& a, cudaStream_t stream) {
  // Eight warps where the registers of two blocks an SM hold them (a chip has room for 14 clusters of 16 then, with one
  // block only for 7); two where 256 channels of 16 bits have to leave room for the choice of pages.
  constexpr bool kWide = DP == 256 && !kQuantized<F>;
  constexpr int kWarps = NB * DP <= 128 && (kQuantized<F> || DP == 64) ? 8 : kPages && kWide ? 2 : 4;
  constexpr int kBlocks = Mem<F, FQ, DP, NB, kWarps, kPages>::kEnd <= 113 * 1024 ? 2 : 1;
  auto kern = attend_kernel<F, FQ, DP, NB, kWarps, kBlocks, kPages>;
  using M = Mem<F, FQ, DP, NB, kWarps, kPages>;
  const Shape& s = a.s;
  constexpr int most = (M::kEnd + 15) / 16 * 16;
  const size_t dyn = most + (kPages ? page_mem_bytes(a.pages.max_pages, a.pages.budget, s.D) : 0);
  constexpr int bound = most + (kPages ? kMaxPagesPerSeq * 12 + 256 * 16 + 2048 : 0);
  static_assert(bound <= 227 * 1024, "shared memory of a block");
  // one table for launches that leave room for two blocks an SM, one for those with many pages
  static ClusterTable table, large;
  constexpr int two = bound < 113 * 1024 ? bound : 113 * 1024;
  const std::atomic<int>* resident = dyn <= (size_t)two ? table.resident(kern, kWarps * 32, two, bound) : large.resident(kern, kWarps * 32, bound, bound);
  if (!resident) return KVCRUSH_ERR_CUDA;
  // what a block does once takes as long as about three tiles of each of its warps
  const int n_blk = choose_cluster(resident, attend_units(a, M::kRows), attend_tiles(a), 3 * kWarps);
  dim3 grid;
  if (!attend_grid(a, M::kRows, n_blk, &grid)) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(kern, grid, dim3(kWarps * 32), dyn, stream, n_blk, a);
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
