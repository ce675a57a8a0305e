// What the attention kernels of new tokens share: the unit of work of a cluster, the choice of pages, and the sum over the
// cluster's blocks.
//
// A cluster of 1 to 16 blocks answers one unit: a block of query rows of one (layer, sequence, KV head), where the rows are
// the new tokens of the sequence times the query heads of the group (with pages: of one new token).  The keys are
// divided among the blocks, every warp keeps a running maximum, sum and output of its own keys, and the parts are added
// up through distributed shared memory, so that a call is one launch, needs no scratch memory and gives the same
// result every time.  Every block owns a share of the output and is sent the others' parts of it: stores that nobody waits for,
// one barrier, and what is left is done by each block alone (5500 to 12500 clocks where blocks read their peers' parts
// instead, 2800 to 6600 now, waiting for the slowest included).
#pragma once

#include <cooperative_groups.h>

#include <atomic>

#include "cache_format.cuh"

namespace kvc {
namespace att {

namespace cg = cooperative_groups;

constexpr int kTile = 16;                    // keys of a tile
constexpr int kMaxCluster = 16;
constexpr unsigned kAll = 0xFFFFFFFFu;

__device__ __forceinline__ float neg_inf() { return __uint_as_float(0xFF800000u); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

struct Unit {
  int layer, seq, hk;
  int first;                 // packed index of the first new token of the unit
  int n_tok;                 // new tokens of the unit's rows all together (row r: token r / G, head r % G)
  int row0, rows;            // this block of query rows
  int begin, seen;           // cached rows: the first one's number, and how many the block's last token sees
  int seen0;                 // how many the unit's token 0 would see (token j: seen0 + j), where own == 0
  int own;                   // keys among the new tokens
  int G;
  uint32_t magic;
  __device__ __forceinline__ int token(int r) const { return G == 1 ? row0 + r : (int)__umulhi((uint32_t)(row0 + r), magic); }
  __device__ __forceinline__ int head(int r) const { return row0 + r - token(r) * G; }
  // cached rows that the token of row r sees
  __device__ __forceinline__ int limit(int r) const { return own ? seen : min(max(seen0 + token(r), 0), seen); }
};

// The unit of this block's cluster; false: no rows (uniform over the cluster).  Grid: (clusters of a layer and sequence, or of a
// layer and new token; KV heads; blocks of query rows).
template <bool kPages>
__device__ __forceinline__ bool unit_of(const AttendArgs& a, int rows_per_block, Unit& w) {
  const Shape& s = a.s;
  unsigned u;
  asm("mov.u32 %0, %%clusterid.x;" : "=r"(u));
  w.hk = blockIdx.y;
  w.row0 = (int)blockIdx.z * rows_per_block;
  w.G = s.G; w.magic = a.group_magic;
  const unsigned per_layer = kPages ? a.fresh.total : s.n_seqs;
  w.layer = u < per_layer ? 0 : (int)(u / per_layer);
  u -= w.layer * per_layer;
  int count;
  if (kPages) {
    w.first = (int)u;
    w.seq = seq_of_token(a.fresh.cu, s.n_seqs, w.first);
    rows_of(s, a.row_begin, a.row_count, w.layer, w.seq, w.begin, count);
    w.seen0 = count - (__ldg(a.fresh.cu + w.seq + 1) - 1 - w.first);
    w.n_tok = 1;
  } else {
    w.seq = (int)u;
    w.first = __ldg(a.fresh.cu + w.seq);
    w.n_tok = __ldg(a.fresh.cu + w.seq + 1) - w.first;
    rows_of(s, a.row_begin, a.row_count, w.layer, w.seq, w.begin, count);
    w.seen0 = count - w.n_tok + 1;
  }
  w.rows = min(rows_per_block, w.n_tok * s.G - w.row0);
  if (w.rows <= 0) return false;
  const int j_last = w.token(w.rows - 1);
  if (!kPages && a.K_new.ptr) {
    w.seen = count;
    w.own = a.fresh.mask ? w.n_tok : j_last + 1;
  } else {
    w.seen = max(0, w.seen0 + j_last);
    w.own = 0;
  }
  return true;
}

// Does new token i (of the sequence) attend to new token j of the same sequence?
__device__ __forceinline__ bool sees_new(const AttendArgs& a, const Unit& w, int i, int j) {
  if (!a.fresh.mask) return j <= i;
  return (__ldg(a.fresh.mask + (long long)(w.first + i) * a.fresh.mask_words + (j >> 5)) >> (j & 31)) & 1u;
}

// ---- the choice of pages ----------------------------------------------------------------------------------

// Scores are sums of pairs of floats, good to 2^-45 of their terms' size: sums in float64 would convert every bound, and an
// SM converts 16 values a clock (it adds 63).  Pairs for float64 took 23.3 -> 22.1 us for 1024 pages, 38.8 -> 36.7 for 16 sequences.
struct Pair { float sum, rest; };
// a + x, and what the sum was rounded by
__device__ __forceinline__ void add_to(Pair& a, float x, float x_rest) {
  const float next = a.sum + x, back = next - a.sum;
  a.rest += ((a.sum - (next - back)) + (x - back)) + x_rest;
  a.sum = next;
}
// Larger score, larger key, every score below the pages that are read by decree: the bits of the score as a float64.
__device__ __forceinline__ unsigned long long bits_key(unsigned long long b) { return b & 0x8000000000000000ull ? ~b : b | 0x8000000000000000ull; }
__device__ __forceinline__ unsigned long long score_key(double x) {
  if (!(x == x)) return 0xFFF0000000000000ull;                      // counts as +inf
  return bits_key((unsigned long long)__double_as_longlong(x + 0.0));
}
// The same of a pair, 2^-60 <= |sum| < 2^100, by integers: the sum's bits, and the rest in units of the float64's last place.
__device__ __forceinline__ unsigned long long score_key(const Pair& p) {
  const float s = p.sum + p.rest, r = p.rest - (s - p.sum);
  const uint32_t b = __float_as_uint(s);
  const int e = (int)(b >> 23 & 255u) - 127;
  const int k = __float2int_rn(r * __uint_as_float((uint32_t)(52 - e + 127) << 23));
  const unsigned long long magnitude = ((unsigned long long)(b & 0x7FFFFFFFu) << 29) + (896ull << 52) + (unsigned long long)(long long)(b >> 31 ? -k : k);
  return bits_key(magnitude | (unsigned long long)(b >> 31) << 63);
}
constexpr unsigned long long kDecreed = ~0ull;

template <int FQ>
__device__ __forceinline__ float widen1(const void* p, long long i) {
  if constexpr (FQ == KVCRUSH_FP32) return static_cast<const float*>(p)[i];
  else if constexpr (FQ == KVCRUSH_BF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  else return __half2float(static_cast<const __half*>(p)[i]);
}

// Shared memory of the choice: keys of all pages, the chosen pages, and coefficients of the channels.
struct PageMem {
  unsigned long long* keys;                  // [max_pages]
  int* chosen;                               // [min(budget, max_pages)]
  float4* sums;                              // sums of the group's positive and of its negative query values (pairs), see sums_at
  int* count;                                // [256 + 64] counters
};
// The lanes that share a page read these sums 8 channels apart; 16 bytes between them keep them in different banks.
__host__ __device__ inline int sums_at(int c) { return c + (c >> 3); }
__host__ __device__ inline size_t page_mem_bytes(int max_pages, int budget, int D) {
  return ((size_t)max_pages + 1) / 2 * 16 + (size_t)sums_at(D) * 16 + (((size_t)(budget < max_pages ? budget : max_pages) + 3) / 4 * 4 + 320) * 4;
}
__device__ __forceinline__ PageMem page_mem(unsigned char* base, int max_pages, int budget, int D) {
  PageMem m;
  m.keys = reinterpret_cast<unsigned long long*>(base);
  m.sums = reinterpret_cast<float4*>(m.keys + (max_pages + 1) / 2 * 2);
  m.count = reinterpret_cast<int*>(m.sums + sums_at(D));
  m.chosen = m.count + 320;
  return m;
}

// Chooses the pages of the unit's token; all threads of the cluster.  Returns how many, in mem.chosen of every block.
// FQ: type of the bounds and queries.
template <int FQ, int kThreads>
__device__ __forceinline__ int choose_pages(const AttendArgs& a, const Unit& w, cg::cluster_group& cluster, int n_blk, int rank,
                                            const PageMem& mem) {
  using namespace fmt;
  const Shape& s = a.s;
  const PageChoice& p = a.pages;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kWarps = kThreads / 32;
  const int n_pages = (w.seen + p.page_size - 1) / p.page_size;
  const int want = min(p.budget, n_pages);
  if (n_pages > want) {
    if (n_blk > 1) cluster_arrive_relaxed();           // waited for before the first store to a peer: all blocks run then
    const unsigned char* q = static_cast<const unsigned char*>(a.Q.ptr) + bytes_of<FQ>(w.layer * a.Q.sl + w.first * a.Q.st + (long long)w.hk * s.G * a.Q.sh);
    for (int c = tid; c < s.D; c += kThreads) {
      Pair up{0.f, 0.f}, down{0.f, 0.f};
#pragma unroll 8
      for (int h = 0; h < s.G; ++h) {
        const float x = widen1<FQ>(q, h * a.Q.sh + c);
        add_to(up, x > 0.f || !(x == x) ? x : 0.f, 0.f);
        add_to(down, x < 0.f ? x : 0.f, 0.f);
      }
      mem.sums[sums_at(c)] = make_float4(up.sum, up.rest, down.sum, down.rest);
    }
    __syncthreads();
    if (n_blk > 1) cluster_wait();
    // scores of this block's pages; eight lanes a page
    const int per = (n_pages + n_blk - 1) / n_blk, p_lo = min(n_pages, rank * per), p_hi = min(n_pages, p_lo + per);
    // The bounds of two pages and up to 128 channels are loaded before the first is used.
    const int sub = lane & 7;
    constexpr int kPages2 = 2, kBlocks64 = 2;
    for (int base = p_lo + warp * 4; base < p_hi; base += kPages2 * kWarps * 4) {
      Pair score[kPages2];
      const unsigned char *lp[kPages2], *hp[kPages2];
#pragma unroll
      for (int g = 0; g < kPages2; ++g) {
        score[g] = Pair{0.f, 0.f};
        const long long row = (long long)w.seq * p.max_pages + min(base + g * kWarps * 4 + (lane >> 3), p_hi - 1);
        lp[g] = static_cast<const unsigned char*>(p.lo.ptr) + bytes_of<FQ>(w.layer * p.lo.sl + row * p.lo.st + w.hk * p.lo.sh);
        hp[g] = static_cast<const unsigned char*>(p.hi.ptr) + bytes_of<FQ>(w.layer * p.hi.sl + row * p.hi.st + w.hk * p.hi.sh);
      }
      for (int c0 = 0; c0 < s.D; c0 += 64 * kBlocks64) {
        Raw8<FQ> lo[kPages2][kBlocks64], hi[kPages2][kBlocks64];
#pragma unroll
        for (int g = 0; g < kPages2; ++g)
#pragma unroll
          for (int b = 0; b < kBlocks64; ++b) {
            const int c = min(c0 + b * 64 + sub * 8, s.D - 8);       // channels that there are; those beyond count as zeros below
            lo[g][b].load(lp[g] + bytes_of<FQ>(c));
            hi[g][b].load(hp[g] + bytes_of<FQ>(c));
          }
#pragma unroll
        for (int b = 0; b < kBlocks64; ++b) {
          const int c = c0 + b * 64 + sub * 8;
          if (c < s.D) {
            float x[kPages2][8], y[kPages2][8];
#pragma unroll
            for (int g = 0; g < kPages2; ++g) { lo[g][b].widen(x[g]); hi[g][b].widen(y[g]); }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 q = mem.sums[sums_at(c + i)];
#pragma unroll
              for (int g = 0; g < kPages2; ++g)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const float a = k ? q.z : q.x, a_rest = k ? q.w : q.y, v = a == 0.f ? 0.f : k ? x[g][i] : y[g][i];
                  const float t = a * v;
                  add_to(score[g], t, fmaf(a_rest, v, fmaf(a, v, -t)));
                }
            }
          }
        }
      }
#pragma unroll
      for (int g = 0; g < kPages2; ++g) {
        const int page = base + g * kWarps * 4 + (lane >> 3);
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) {
          const float o = __shfl_xor_sync(kAll, score[g].sum, d), o_rest = __shfl_xor_sync(kAll, score[g].rest, d);
          add_to(score[g], o, o_rest);
        }
        unsigned long long key = page < p.keep_initial || page >= n_pages - p.keep_recent ? kDecreed : score_key(score[g]);
        // a score that is out of float32's range, or near its end: by float64
        const bool out = key != kDecreed && (!(fabsf(score[g].sum) < 0x1p100f) || fabsf(score[g].sum) < 0x1p-60f);
        if (__any_sync(kAll, out)) {
          double exact = 0.;
#pragma unroll 1
          for (int c0 = sub * 8; out && c0 < s.D; c0 += 64)
#pragma unroll 1
            for (int c = c0; c < c0 + 8; ++c) {
              const float4 q = mem.sums[sums_at(c)];
              if (q.x != 0.f) exact = fma((double)widen1<FQ>(hp[g], c), (double)q.x + (double)q.y, exact);
              if (q.z != 0.f) exact = fma((double)widen1<FQ>(lp[g], c), (double)q.z + (double)q.w, exact);
            }
#pragma unroll
          for (int d = 1; d < 8; d <<= 1) exact += __shfl_xor_sync(kAll, exact, d);
          if (out) key = score_key(exact);
        }
        // To every block: the page's eight lanes share the work.  Which half of a sum a lane adds to which decides the last bits of
        // the rest, so the lanes' keys differ there; all blocks get that of the page's first lane.
        key = __shfl_sync(kAll, key, lane & ~7);
        if (page < p_hi)
          for (int b = sub; b < n_blk; b += 8) *(n_blk > 1 ? cluster.map_shared_rank(mem.keys + page, b) : mem.keys + page) = key;
      }
    }
    if (n_blk > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
    // The want-th largest key.  Scores differ little in their leading bits, so the search starts at the highest bit in which
    // any two keys differ (those read by decree apart) and goes on eight bits at a time until the keys that share the
    // bits found so far are all taken.
    unsigned long long both = ~0ull, any = 0ull;
    int decreed = 0;
    for (int i = tid; i < n_pages; i += kThreads) {
      const unsigned long long k = mem.keys[i];
      if (k == kDecreed) ++decreed; else { both &= k; any |= k; }
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      both &= __shfl_xor_sync(kAll, both, d);
      any |= __shfl_xor_sync(kAll, any, d);
      decreed += __shfl_xor_sync(kAll, decreed, d);
    }
    unsigned long long* bits = reinterpret_cast<unsigned long long*>(mem.count);   // [2][kWarps]
    if (lane == 0) { bits[warp] = both; bits[kWarps + warp] = any; mem.count[264 + warp] = decreed; }
    __syncthreads();
    both = ~0ull; any = 0ull; decreed = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) { both &= bits[i]; any |= bits[kWarps + i]; decreed += mem.count[264 + i]; }
    __syncthreads();
    unsigned long long prefix, mask;
    int left;
    if (decreed >= want) {                   // only pages by decree, the lowest ones
      prefix = kDecreed; mask = ~0ull; left = want;
    } else {
      const int top = 64 - __clzll(any & ~both);                     // bits below differ
      mask = top == 64 ? 0ull : ~0ull << top;
      prefix = both & mask;
      left = want - decreed;
      for (int high = top; high > 0;) {
        const int shift = max(0, high - 8);
        const unsigned digits = (1u << (high - shift)) - 1u;
        for (int i = tid; i < 256; i += kThreads) mem.count[i] = 0;
        __syncthreads();
        for (int i = tid; i < n_pages; i += kThreads) {
          const unsigned long long k = mem.keys[i];
          if (k != kDecreed && (k & mask) == prefix) atomicAdd(mem.count + ((unsigned)(k >> shift) & digits), 1);
        }
        __syncthreads();
        if (warp == 0) {                     // lane: eight digits, from the top
          int c[8], sum = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) { c[i] = mem.count[255 - (lane * 8 + i)]; sum += c[i]; }
          int before = sum;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(kAll, before, d); if (lane >= d) before += o; }
          before -= sum;
          if (before < left && before + sum >= left) {
            bool found = false;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if (!found && before + c[i] >= left) {
                mem.count[256] = 255 - (lane * 8 + i);
                mem.count[257] = left - before;
                mem.count[258] = c[i];
                found = true;
              }
              before += c[i];
            }
          }
        }
        __syncthreads();
        prefix |= (unsigned long long)mem.count[256] << shift;
        mask |= (unsigned long long)digits << shift;
        left = mem.count[257];
        if (mem.count[258] == left) break;
        high = shift;
      }
    }
    const bool by_decree = decreed < want;   // those come on top of what the search found
    // chosen pages in order: thread t looks at a run of pages; equals are taken from the front
    const int run = (n_pages + kThreads - 1) / kThreads, lo = min(n_pages, tid * run), hi = min(n_pages, lo + run);
    int above = 0, equal = 0;
    auto is_above = [&](unsigned long long k) { return k == kDecreed ? by_decree : (k & mask) > prefix; };
    auto is_equal = [&](unsigned long long k) { return k == kDecreed ? !by_decree : (k & mask) == prefix; };
    for (int i = lo; i < hi; ++i) { above += is_above(mem.keys[i]); equal += is_equal(mem.keys[i]); }
    int sa = above, se = equal;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int oa = __shfl_up_sync(kAll, sa, d), oe = __shfl_up_sync(kAll, se, d);
      if (lane >= d) { sa += oa; se += oe; }
    }
    if (lane == 31) { mem.count[264 + warp] = sa; mem.count[264 + 16 + warp] = se; }
    __syncthreads();
    sa -= above; se -= equal;
    for (int i = 0; i < warp; ++i) { sa += mem.count[264 + i]; se += mem.count[264 + 16 + i]; }
    int at = sa + min(se, left);
    for (int i = lo; i < hi; ++i) {
      const bool eq = is_equal(mem.keys[i]);
      if (is_above(mem.keys[i]) || (eq && se < left)) mem.chosen[at++] = i;
      se += eq;
    }
  } else {
    for (int i = tid; i < want; i += kThreads) mem.chosen[i] = i;
  }
  __syncthreads();
  if (rank == 0 && w.row0 == 0) {
    const long long out = ((long long)w.layer * a.fresh.total + w.first) * s.Hkv + w.hk;
    if (p.page_idx)
      for (int i = tid; i < p.budget; i += kThreads) p.page_idx[out * p.budget + i] = i < want ? mem.chosen[i] : -1;
    if (p.n_pages && tid == 0) p.n_pages[out] = want;
  }
  return want;
}

// ---- the sum over the cluster -----------------------------------------------------------------------------

// A part of a row: maximum and sum of the weights, what its output is relative to, and the sum of weights times zeros.
struct Part { float m, l, m2, b; };

// Where a block receives the parts of its share of the output: four channels of a row make an element.
template <int kRows, int kMaxD>
struct Received {
  float4 o[kRows * kMaxD / 4 + kMaxCluster];           // [block][element of the share]
  Part part[kMaxCluster * kRows];                      // [block][row]
};

// Adds up the warps' parts, then the blocks', and writes the unit's rows; all threads of the cluster.  o: [kWarps][kRows][stride]
// outputs, part: [kWarps][kRows], both of this block.  The caller has arrived at the cluster's barrier once (so that the
// peers are known to run) and not waited.
template <int FQ, int kWarps, int kRows, int kMaxD>
__device__ __forceinline__ void join_and_write(const AttendArgs& a, const Unit& w, cg::cluster_group& cluster, int n_blk, int rank,
                                               const float* o, int stride, const Part* part, Received<kRows, kMaxD>* recv) {
  using namespace fmt;
  constexpr int kThreads = kWarps * 32;
  const Shape& s = a.s;
  const int tid = threadIdx.x;
  const int vec = s.D / 4, total = w.rows * vec;
  const int per = n_blk == 1 ? total : (total + n_blk - 1) / n_blk;
  const uint32_t per_magic = 0xFFFFFFFFu / (uint32_t)per + 1u;                    // e / per for e < 2^16 (per > 1)
  if (n_blk > 1) cluster_wait();
  __syncthreads();
  for (int r = tid; r < w.rows * n_blk; r += kThreads) {                         // a row's part, to every block
    const int row = r % w.rows, to = r / w.rows;
    float m = -FLT_MAX, m2 = -FLT_MAX, l = 0.f, b = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) { m = fmaxf(m, part[k * kRows + row].m); m2 = fmaxf(m2, part[k * kRows + row].m2); }
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const Part p = part[k * kRows + row];
      const float f = ex2(p.m - m);
      l = fmaf(p.l, f, l);
      b = fmaf(p.b, f, b);
    }
    Part* dst = recv->part + rank * kRows + row;
    *(n_blk > 1 ? cluster.map_shared_rank(dst, to) : dst) = Part{m, l, m2, b};
  }
  for (int e = tid; e < total; e += kThreads) {                                 // an element, to its owner
    const int row = e / vec, d = (e - row * vec) * 4;
    float m2 = -FLT_MAX;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) m2 = fmaxf(m2, part[k * kRows + row].m2);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float f = ex2(part[k * kRows + row].m2 - m2);
      const float4 v = *reinterpret_cast<const float4*>(o + (k * kRows + row) * stride + d);
      sum.x = fmaf(v.x, f, sum.x); sum.y = fmaf(v.y, f, sum.y); sum.z = fmaf(v.z, f, sum.z); sum.w = fmaf(v.w, f, sum.w);
    }
    const int owner = per == 1 ? e : (int)__umulhi((uint32_t)e, per_magic);
    float4* dst = recv->o + rank * per + (n_blk == 1 ? e : e - owner * per);
    *(n_blk > 1 ? cluster.map_shared_rank(dst, owner) : dst) = sum;
  }
  if (n_blk > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
  const int mine = rank * per;
  for (int i = tid; i < min(per, total - mine); i += kThreads) {
    const int e = mine + i, row = e / vec, d = (e - row * vec) * 4;
    float M = neg_inf();
#pragma unroll 8
    for (int p = 0; p < n_blk; ++p) M = fmaxf(M, recv->part[p * kRows + row].m);
    float l = 0.f, b = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int p = 0; p < n_blk; ++p) {
      const Part q = recv->part[p * kRows + row];
      const float4 v = recv->o[p * per + i];
      const float f = ex2(q.m - M), f2 = ex2(q.m2 - M);
      l = fmaf(q.l, f, l);
      b = fmaf(q.b, f, b);
      // a block without weights has no output either, whatever its maximum
      sum.x += v.x == 0.f ? 0.f : v.x * f2; sum.y += v.y == 0.f ? 0.f : v.y * f2;
      sum.z += v.z == 0.f ? 0.f : v.z * f2; sum.w += v.w == 0.f ? 0.f : v.w * f2;
    }
    const bool none = l == 0.f;                        // no weight: zeros, whatever the values hold (0 times infinity)
    const float inv = 1.f / l;
    const float x[4] = {none ? 0.f : (sum.x + b) * inv, none ? 0.f : (sum.y + b) * inv, none ? 0.f : (sum.z + b) * inv, none ? 0.f : (sum.w + b) * inv};
    const int token = w.token(row), head = w.hk * w.G + row + w.row0 - token * w.G;
    unsigned char* op = static_cast<unsigned char*>(const_cast<void*>(a.O.ptr)) +
        bytes_of<FQ>(w.layer * a.O.sl + (w.first + token) * a.O.st + head * a.O.sh + d);
    if constexpr (FQ == KVCRUSH_FP32) *reinterpret_cast<float4*>(op) = make_float4(x[0], x[1], x[2], x[3]);
    else if constexpr (FQ == KVCRUSH_BF16) *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    else *reinterpret_cast<uint2*>(op) = make_uint2(pack_fp16(x[0], x[1]), pack_fp16(x[2], x[3]));
    if (d == 0 && a.lse)
      a.lse[((long long)w.layer * s.Hq + head) * a.fresh.total + w.first + token] = l == 0.f ? neg_inf() : (M + log2f(l)) * 0.6931471805599453f;
  }
}

// ---- host: the launch ------------------------------------------------------------------------------------------

constexpr int kMaxDevices = 64;

// How many clusters of 1 .. 16 blocks of a kernel a device runs at once (write-once cache per device; 16 are more than every
// device grants).
struct ClusterTable {
  std::atomic<int> held[kMaxDevices][kMaxCluster + 1];
  // The current device's row, for launches with `dyn` bytes of dynamic shared memory, after the kernel may be launched with up to
  // `bound`; NULL where something failed.
  template <class Kernel>
  const std::atomic<int>* resident(Kernel kern, int threads, int dyn, int bound) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) { cudaGetLastError(); return nullptr; }
    std::atomic<int>* row = held[dev];
    if (row[1].load(std::memory_order_acquire) > 0) return row;
    if (allow_dynamic_smem(kern, bound) != KVCRUSH_OK) return nullptr;
    const bool large = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    for (int c = kMaxCluster; c >= 1; --c) {
      cudaLaunchConfig_t cfg{};
      cfg.gridDim = dim3(c);
      cfg.blockDim = dim3(threads);
      cfg.dynamicSmemBytes = dyn;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = c; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      int n = 0;
      if ((c > 8 && !large) || cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 0) n = 0;
      if (c == 1 && n < 1) n = sm_count();
      row[c].store(n, std::memory_order_release);
    }
    cudaGetLastError();                              // of what could not be asked
    return row;
  }
};
// Blocks for each of `units` units of `tiles` tiles: the fewest rounds of resident clusters times what a block takes, its tiles and
// `fixed` tiles' worth of what it does once.  How many is of little account: from 0 to 20 tiles a warp (attend_tree.cu: a block) thirteen
// calls of one to 63 tokens over 1001 to 48000 rows, of all three kernels and over pages, took the same time to 1 %.
inline int choose_cluster(const std::atomic<int>* resident, long long units, int tiles, int fixed) {
  int best = 1;
  long long best_cost = -1;
  for (int c = 1; c <= kMaxCluster && (c == 1 || 2 * c <= tiles); ++c) {
    const int n = resident[c].load(std::memory_order_relaxed);
    if (n < 1) continue;
    const long long cost = (units + n - 1) / n * ((tiles + c - 1) / c + fixed);
    if (best_cost < 0 || cost < best_cost) { best = c; best_cost = cost; }
  }
  return best;
}

// The grid of clusters of n_blk blocks; false: too large.
inline bool attend_grid(const AttendArgs& a, int rows_per_block, int n_blk, dim3* grid) {
  const bool pages = a.pages.page_size > 0;
  const long long rows = (long long)(pages ? 1 : a.fresh.most) * a.s.G, x = (long long)a.s.n_layers * (pages ? a.fresh.total : a.s.n_seqs) * n_blk;
  *grid = dim3((unsigned)x, (unsigned)a.s.Hkv, (unsigned)((rows + rows_per_block - 1) / rows_per_block));
  return x <= 0x7FFFFFFFLL && grid->z <= 65535u;
}
inline long long attend_units(const AttendArgs& a, int rows_per_block) {
  dim3 g;
  attend_grid(a, rows_per_block, 1, &g);
  return (long long)a.s.n_layers * (a.pages.page_size > 0 ? a.fresh.total : a.s.n_seqs) * g.y * g.z;
}
inline int attend_tiles(const AttendArgs& a) {
  const PageChoice& p = a.pages;
  const long long keys = p.page_size > 0 ? (long long)(p.budget < p.max_pages ? p.budget : p.max_pages) * p.page_size
                                         : (long long)a.s.max_seqlen + (a.K_new.ptr ? a.fresh.most : 0);
  return (int)((keys + kTile - 1) / kTile);
}

}  // namespace att
}  // namespace kvc
