// What the attention kernels of new tokens share: the unit of work of a cluster, the choice of pages, and the sum over the
// cluster's blocks.
//
// A cluster of 1 to 16 blocks answers one unit: a block of query rows of one (layer, sequence, KV head), where the rows are
// the new tokens of the sequence times the query heads of the group (with pages: of one new token).  The keys are
// divided among the blocks, every warp keeps a running maximum, sum and output of its own keys, and the parts are added
// up through distributed shared memory, so that a call is one launch, needs no scratch memory and gives the same
// result every time.
#pragma once

#include <cooperative_groups.h>

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
// What exponentials are relative to; without a finite maximum all logits are -inf, which adds 0, or NaN, which stays.
__device__ __forceinline__ float reference(float maximum) { return maximum == neg_inf() ? 0.f : maximum; }

struct Unit {
  int layer, seq, hk;
  int first;                 // packed index of the first new token of the unit
  int n_tok;                 // new tokens of the unit's rows all together (row r: token r / G, head r % G)
  int row0, rows;            // this block of query rows
  int begin, seen;           // cached rows: the first one's number, and how many the block's last token sees
  int seen0;                 // how many the unit's token 0 would see (token j: seen0 + j), where own == 0
  int own;                   // keys among the new tokens
  __device__ __forceinline__ int token(int G, int r) const { return (row0 + r) / G; }
  __device__ __forceinline__ int head(int G, int r) const { return (row0 + r) % G; }
  // cached rows that the token of row r sees
  __device__ __forceinline__ int limit(int G, int r) const { return own ? seen : min(max(seen0 + token(G, r), 0), seen); }
};

// Unit number u; false: no rows (uniform over the cluster).
template <bool kPages>
__device__ __forceinline__ bool unit_of(const AttendArgs& a, unsigned u, int rows_per_block, Unit& w) {
  const Shape& s = a.s;
  const int rb = (int)(u % a.row_blocks); u /= a.row_blocks;
  w.hk = (int)(u % s.Hkv); u /= s.Hkv;
  int count, j_last;
  if (kPages) {
    w.first = (int)(u % a.fresh.total); w.layer = (int)(u / a.fresh.total);
    w.seq = seq_of_token(a.fresh.cu, s.n_seqs, w.first);
    rows_of(s, a.row_begin, a.row_count, w.layer, w.seq, w.begin, count);
    w.seen0 = count - (__ldg(a.fresh.cu + w.seq + 1) - 1 - w.first);
    w.n_tok = 1;
  } else {
    w.seq = (int)(u % s.n_seqs); w.layer = (int)(u / s.n_seqs);
    w.first = __ldg(a.fresh.cu + w.seq);
    w.n_tok = __ldg(a.fresh.cu + w.seq + 1) - w.first;
    rows_of(s, a.row_begin, a.row_count, w.layer, w.seq, w.begin, count);
    w.seen0 = count - w.n_tok + 1;
  }
  w.row0 = rb * rows_per_block;
  w.rows = min(rows_per_block, w.n_tok * s.G - w.row0);
  if (w.rows <= 0) return false;
  j_last = (w.row0 + w.rows - 1) / s.G;
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

// Larger score, larger key; every score below the pages that are read by decree.
__device__ __forceinline__ unsigned long long score_key(double x) {
  if (!(x == x)) return 0xFFF0000000000000ull;                      // counts as +inf
  const unsigned long long b = (unsigned long long)__double_as_longlong(x + 0.0);
  return b & 0x8000000000000000ull ? ~b : b | 0x8000000000000000ull;
}
constexpr unsigned long long kDecreed = ~0ull;

template <int FQ>
__device__ __forceinline__ double widen1(const void* p, long long i) {
  if constexpr (FQ == KVCRUSH_FP32) return (double)static_cast<const float*>(p)[i];
  else if constexpr (FQ == KVCRUSH_BF16) return (double)__bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  else return (double)__half2float(static_cast<const __half*>(p)[i]);
}

// Shared memory of the choice: keys of all pages, the chosen pages, and coefficients of the channels.
struct PageMem {
  unsigned long long* keys;                  // [max_pages]
  int* chosen;                               // [min(budget, max_pages)]
  double* up;                                // [D]: sum of the positive query values of the group's heads
  double* down;                              // [D]
  int* count;                                // [256 + 64] counters
};
__host__ __device__ inline size_t page_mem_bytes(int max_pages, int budget, int D) {
  return (size_t)max_pages * 8 + (size_t)D * 16 + (((size_t)(budget < max_pages ? budget : max_pages) + 3) / 4 * 4 + 320) * 4;
}
__device__ __forceinline__ PageMem page_mem(unsigned char* base, int max_pages, int budget, int D) {
  PageMem m;
  m.keys = reinterpret_cast<unsigned long long*>(base);
  m.up = reinterpret_cast<double*>(m.keys + max_pages);
  m.down = m.up + D;
  m.count = reinterpret_cast<int*>(m.down + D);
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
    const unsigned char* q = static_cast<const unsigned char*>(a.Q.ptr) + bytes_of<FQ>(w.layer * a.Q.sl + w.first * a.Q.st + (long long)w.hk * s.G * a.Q.sh);
    for (int c = tid; c < s.D; c += kThreads) {
      double up = 0., down = 0.;
      for (int h = 0; h < s.G; ++h) {
        const double x = widen1<FQ>(q, h * a.Q.sh + c);
        up += x > 0. || !(x == x) ? x : 0.;
        down += x < 0. ? x : 0.;
      }
      mem.up[c] = up; mem.down[c] = down;
    }
    __syncthreads();
    // scores of this block's pages; eight lanes a page
    const int per = (n_pages + n_blk - 1) / n_blk, p_lo = min(n_pages, rank * per), p_hi = min(n_pages, p_lo + per);
    const int sub = lane & 7;
    for (int base = p_lo + warp * 4; base < p_hi; base += kWarps * 4) {
      const int page = base + (lane >> 3);
      double score = 0.;
      if (page < p_hi) {
        const long long row = (long long)w.seq * p.max_pages + page;
        const unsigned char* lp = static_cast<const unsigned char*>(p.lo.ptr) + bytes_of<FQ>(w.layer * p.lo.sl + row * p.lo.st + w.hk * p.lo.sh);
        const unsigned char* hp = static_cast<const unsigned char*>(p.hi.ptr) + bytes_of<FQ>(w.layer * p.hi.sl + row * p.hi.st + w.hk * p.hi.sh);
        for (int c = sub * 8; c < s.D; c += 64) {
          Raw8<FQ> lo, hi;
          lo.load(lp + bytes_of<FQ>(c));
          hi.load(hp + bytes_of<FQ>(c));
          float x[8], y[8];
          lo.widen(x);
          hi.widen(y);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const double up = mem.up[c + i], down = mem.down[c + i];
            if (up != 0.) score = fma((double)y[i], up, score);
            if (down != 0.) score = fma((double)x[i], down, score);
          }
        }
      }
#pragma unroll
      for (int d = 1; d < 8; d <<= 1) score += __shfl_xor_sync(kAll, score, d);
      if (sub == 0 && page < p_hi)
        mem.keys[page] = page < p.keep_initial || page >= n_pages - p.keep_recent ? kDecreed : score_key(score);
    }
    // every block takes the other blocks' keys
    if (n_blk > 1) {
      cluster.sync();
      for (int i = tid; i < n_pages; i += kThreads) {
        const int owner = i / per;
        if (owner != rank) mem.keys[i] = *cluster.map_shared_rank(mem.keys + i, owner);
      }
    }
    __syncthreads();
    // the want-th largest key, eight bits at a time, and how many of its equals belong to the chosen ones
    unsigned long long prefix = 0, mask = 0;
    int left = want;
    for (int shift = 56; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kThreads) mem.count[i] = 0;
      __syncthreads();
      for (int i = tid; i < n_pages; i += kThreads)
        if ((mem.keys[i] & mask) == prefix) atomicAdd(mem.count + (int)(mem.keys[i] >> shift & 255u), 1);
      __syncthreads();
      if (warp == 0) {                       // lane: eight digits, from the top
        int c[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = mem.count[255 - (lane * 8 + i)]; sum += c[i]; }
        int before = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) { const int o = __shfl_up_sync(kAll, before, d); if (lane >= d) before += o; }
        before -= sum;
        if (before < left && before + sum >= left) {
          int i = 0;
          while (before + c[i] < left) before += c[i++];
          mem.count[256] = 255 - (lane * 8 + i);
          mem.count[257] = left - before;
        }
      }
      __syncthreads();
      prefix |= (unsigned long long)mem.count[256] << shift;
      mask |= 255ull << shift;
      left = mem.count[257];
    }
    // chosen pages in order: thread t looks at a run of pages; equals are taken from the front
    const int run = (n_pages + kThreads - 1) / kThreads, lo = min(n_pages, tid * run), hi = min(n_pages, lo + run);
    int above = 0, equal = 0;
    for (int i = lo; i < hi; ++i) { above += mem.keys[i] > prefix; equal += mem.keys[i] == prefix; }
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
      const bool eq = mem.keys[i] == prefix;
      if (mem.keys[i] > prefix || (eq && se < left)) mem.chosen[at++] = i;
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

// A block's part of a row: maximum and sum of the weights, what its output is relative to, and the sum of weights times zeros.
struct Part { float m, l, m2, b; };

// Adds up the blocks' parts and writes the unit's rows; all threads of the cluster.  o: [rows][stride] this block's output,
// part: [rows], factor: [rows][kMaxCluster + 1] scratch, all in shared memory at the same place in every block.
template <int FQ, int kThreads>
__device__ __forceinline__ void join_and_write(const AttendArgs& a, const Unit& w, cg::cluster_group& cluster, int n_blk, int rank,
                                               float* o, int stride, Part* part, float* factor) {
  using namespace fmt;
  const Shape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (n_blk > 1) cluster.sync(); else __syncthreads();
  for (int r = warp; r < w.rows; r += kThreads / 32) {
    Part p{neg_inf(), 0.f, neg_inf(), 0.f};
    if (lane < n_blk) p = n_blk > 1 ? *cluster.map_shared_rank(part + r, lane) : part[r];
    float M = p.m;
#pragma unroll
    for (int d = 1; d < kMaxCluster; d <<= 1) M = fmaxf(M, __shfl_xor_sync(kAll, M, d));
    const float ref = reference(M), f = exp2f(p.m - ref);
    float l = p.l == 0.f ? 0.f : p.l * f, b = p.l == 0.f ? 0.f : p.b * f;
#pragma unroll
    for (int d = 1; d < kMaxCluster; d <<= 1) { l += __shfl_xor_sync(kAll, l, d); b += __shfl_xor_sync(kAll, b, d); }
    if (lane < n_blk) factor[r * (kMaxCluster + 1) + lane] = l == 0.f ? 0.f : exp2f(p.m2 - ref) / l;
    if (lane == 0) {
      factor[r * (kMaxCluster + 1) + kMaxCluster] = l == 0.f ? 0.f : b / l;
      if (rank == 0 && a.lse)
        a.lse[((long long)w.layer * s.Hq + w.hk * s.G + w.head(s.G, r)) * a.fresh.total + w.first + w.token(s.G, r)] =
            l == 0.f ? neg_inf() : (M + log2f(l)) * 0.6931471805599453f;
    }
  }
  __syncthreads();
  // this block's share of the elements, eight channels a thread
  const int vec = s.D / 8, total = w.rows * vec, per = (total + n_blk - 1) / n_blk;
  for (int e = rank * per + tid; e < min(total, (rank + 1) * per); e += kThreads) {
    const int r = e / vec, c = (e - r * vec) * 8;
    const float* f = factor + r * (kMaxCluster + 1);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = f[kMaxCluster];
    for (int b = 0; b < n_blk; ++b) {
      const float* peer = n_blk > 1 ? cluster.map_shared_rank(o, b) : o;
      const float fb = f[b];
      const float4 u = *reinterpret_cast<const float4*>(peer + r * stride + c), v = *reinterpret_cast<const float4*>(peer + r * stride + c + 4);
      x[0] = fmaf(u.x, fb, x[0]); x[1] = fmaf(u.y, fb, x[1]); x[2] = fmaf(u.z, fb, x[2]); x[3] = fmaf(u.w, fb, x[3]);
      x[4] = fmaf(v.x, fb, x[4]); x[5] = fmaf(v.y, fb, x[5]); x[6] = fmaf(v.z, fb, x[6]); x[7] = fmaf(v.w, fb, x[7]);
    }
    Raw8<FQ> out;
    out.narrow(x);
    unsigned char* op = static_cast<unsigned char*>(const_cast<void*>(a.O.ptr)) +
        bytes_of<FQ>(w.layer * a.O.sl + (w.first + w.token(s.G, r)) * a.O.st + (w.hk * s.G + w.head(s.G, r)) * a.O.sh + c);
    out.store(op);
  }
  if (n_blk > 1) cluster.sync();             // peers may still read this block's part
}

// ---- host: the launch ------------------------------------------------------------------------------------------

// Blocks of a cluster: enough of them to fill the chip, none with fewer than a tile for each of its warps.
inline int cluster_size(long long units, int tiles, int warps, int largest, int blocks_wanted) {
  int n = 1;
  while (n < largest && units * n < blocks_wanted && tiles > n * warps) n *= 2;
  return n;
}

}  // namespace att
}  // namespace kvc
