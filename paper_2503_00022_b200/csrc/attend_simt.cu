// Attention of new tokens over a cache on the CUDA cores, in float32 throughout.
//
// A warp takes tiles of 16 keys against up to eight query rows: the four lanes of a quad share a key's row for the
// logits, the 32 lanes share the channels for the output, and the weights pass between the two through shared memory.
// Float32 queries only, over caches of any type.  Seven drafted tokens of 8 heads of 64 over 1001 float32 rows: 13 us; bound by the
// chain of a tile (one warp a scheduler, every key of a tile in turn for the output).
#include "attend_common.cuh"

namespace kvc {

namespace {

using namespace att;
using namespace fmt;

constexpr int kWarps = 4;
constexpr int kRows = 8;                     // query rows of a unit
constexpr int kMaxD = 256;
constexpr int FQ = KVCRUSH_FP32;            // queries, new tokens and bounds of pages
constexpr int kOBytes = kWarps * kRows * kMaxD * 4;

// Four consecutive channels: float32 values, or codes.
template <int F>
__device__ __forceinline__ void load4(const unsigned char* p, float (&x)[4]) {
  if constexpr (F == KVCRUSH_FP32) {
    const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
  } else if constexpr (F == KVCRUSH_INT4) {
    codes4<F>(__ldcs(reinterpret_cast<const unsigned short*>(p)), x);
  } else {
    codes4<F>(__ldcs(reinterpret_cast<const unsigned int*>(p)), x);
  }
}

struct Running {
  float m[kRows / 4], l[kRows / 4];          // rows 2c, 2c + 1 of the lane's quad position c
  float o[2][kRows][4];                      // channels 4 * lane and 128 + 4 * lane
};

// One tile: keys first .. first + n - 1 of `kv` (row numbers), and which of them row r may see.
template <int F, class Sees>
__device__ __forceinline__ void tile(const CacheView& K, const CacheView& V, long long k_base, long long v_base, long long ks_base,
                                     long long vs_base, const long long (&half)[2], const int (&n)[2], int D, int rows, float scale_log2,
                                     const float* q_sh, float* p_sh, Running& run, int lane, bool masked, Sees&& sees) {
  const int g = lane >> 2, c = lane & 3;
  float x[4];                                // key g: rows 2c, 2c + 1; key g + 8: the same
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float s[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) s[r] = 0.f;
    float scale = 1.f, zero = 0.f;
    const long long row = half[j] + g;
    if (g < n[j]) {
      const unsigned char* p = static_cast<const unsigned char*>(K.ptr) + bytes_of<F>(k_base + row * K.st);
      if constexpr (kQuantized<F>) {
        const float* sp = K.scales + ks_base + row * K.sct;
        scale = __ldg(sp);
        if (F == KVCRUSH_INT4) zero = __ldg(sp + 1);
      }
      for (int d = 4 * c; d < D; d += 16) {
        float v[4];
        load4<F>(p + bytes_of<F>(d), v);
        if (F == KVCRUSH_INT4) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], scale, zero);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
          const float4 q = *reinterpret_cast<const float4*>(q_sh + r * kMaxD + d);
          s[r] = fmaf(v[3], q.w, fmaf(v[2], q.z, fmaf(v[1], q.y, fmaf(v[0], q.x, s[r]))));
        }
      }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      s[r] += __shfl_xor_sync(kAll, s[r], 1);
      s[r] += __shfl_xor_sync(kAll, s[r], 2);
      if (kQuantized<F> && F != KVCRUSH_INT4) s[r] *= scale;
      if (r == 2 * c) x[2 * j] = s[r];
      if (r == 2 * c + 1) x[2 * j + 1] = s[r];
    }
  }
  // softmax of the tile; a key that a row does not see gets weight -1, which the second step leaves out
  bool seen[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = g + (i >> 1) * 8, r = 2 * c + (i & 1);
    seen[i] = (key & 7) < n[i >> 1] && r < rows && (!masked || sees(key, r));
    x[i] = seen[i] ? x[i] * scale_log2 : neg_inf();
  }
  float corr[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float big = fmaxf(x[i], x[i + 2]);
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) big = fmaxf(big, __shfl_xor_sync(kAll, big, d));
    const float m = fmaxf(run.m[i], big);                // from the lowest finite number on: logits of -inf have weight 0
    corr[i] = ex2(run.m[i] - m);
    run.m[i] = m;
    x[i] = seen[i] ? ex2(x[i] - m) : -1.f;
    x[i + 2] = seen[i + 2] ? ex2(x[i + 2] - m) : -1.f;
    run.l[i] = run.l[i] * corr[i] + (seen[i] ? x[i] : 0.f) + (seen[i + 2] ? x[i + 2] : 0.f);
  }
  __syncwarp();
  *reinterpret_cast<float2*>(p_sh + g * kRows + 2 * c) = make_float2(x[0], x[1]);
  *reinterpret_cast<float2*>(p_sh + (g + 8) * kRows + 2 * c) = make_float2(x[2], x[3]);
  __syncwarp();
#pragma unroll
  for (int r = 0; r < kRows; ++r) {
    const float f = __shfl_sync(kAll, corr[r & 1], r >> 1);
    if (f != 1.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) { run.o[0][r][i] *= f; run.o[1][r][i] *= f; }
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    for (int k = 0; k < n[j]; ++k) {
      const long long row = half[j] + k;
      const float4 pa = *reinterpret_cast<const float4*>(p_sh + (j * 8 + k) * kRows), pb = *reinterpret_cast<const float4*>(p_sh + (j * 8 + k) * kRows + 4);
      const float p[kRows] = {pa.x, pa.y, pa.z, pa.w, pb.x, pb.y, pb.z, pb.w};
      float scale = 1.f, zero = 0.f;
      if constexpr (kQuantized<F>) {
        const float* sp = V.scales + vs_base + row * V.sct;
        scale = __ldg(sp);
        if (F == KVCRUSH_INT4) zero = __ldg(sp + 1);
      }
      const unsigned char* vp = static_cast<const unsigned char*>(V.ptr) + bytes_of<F>(v_base + row * V.st);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int d = 128 * b + 4 * lane;
        if (d < D) {
          float v[4];
          load4<F>(vp + bytes_of<F>(d), v);
          if (kQuantized<F>) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = F == KVCRUSH_INT4 ? fmaf(v[i], scale, zero) : v[i] * scale;
          }
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            if (!(p[r] < 0.f)) {
#pragma unroll
              for (int i = 0; i < 4; ++i) run.o[b][r][i] = fmaf(p[r], v[i], run.o[b][r][i]);
            }
          }
        }
      }
    }
  }
}

template <int F, bool kPages>
__global__ void __launch_bounds__(kWarps * 32)
attend_simt_kernel(AttendArgs a) {
  extern __shared__ __align__(16) unsigned char dyn_sh[];            // outputs of the warps, then what the choice of pages needs
  __shared__ __align__(16) float q_sh[kRows * kMaxD];
  __shared__ __align__(16) float p_all[kWarps][kTile * kRows];
  __shared__ Part warp_part[kWarps][kRows];
  __shared__ __align__(16) Received<kRows, kMaxD> recv;
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
    pages = page_mem(dyn_sh + kOBytes, a.pages.max_pages, a.pages.budget, s.D);
    n_chosen = choose_pages<FQ, kWarps * 32>(a, w, cluster, n_blk, rank, pages);
  }
  if (n_blk > 1) cluster_arrive_relaxed();
  for (int e = tid; e < kRows * s.D; e += kWarps * 32) {
    const int r = e / s.D, d = e - r * s.D;
    q_sh[r * kMaxD + d] = r < w.rows ? widen1<FQ>(a.Q.ptr, w.layer * a.Q.sl + (w.first + w.token(r)) * a.Q.st +
                                                                     (w.hk * s.G + w.head(r)) * a.Q.sh + d) : 0.f;
  }
  __syncthreads();
  Running run;
#pragma unroll
  for (int i = 0; i < kRows / 4; ++i) { run.m[i] = -FLT_MAX; run.l[i] = 0.f; }
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
      for (int i = 0; i < 4; ++i) run.o[b][r][i] = 0.f;

  const int halves_per_page = kPages ? a.pages.page_size / 8 : 1;
  const int cached = kPages ? (n_chosen * halves_per_page + 1) / 2 : (w.seen + kTile - 1) / kTile;
  const int n_tiles = cached + (w.own + kTile - 1) / kTile;
  const int per = (n_tiles + n_blk - 1) / n_blk, lo = min(n_tiles, rank * per), hi = min(n_tiles, lo + per);
  const long long k_base = w.layer * a.K.sl + w.hk * a.K.sh, v_base = w.layer * a.V.sl + w.hk * a.V.sh;
  const long long ks_base = w.layer * a.K.scl + w.hk * a.K.sch, vs_base = w.layer * a.V.scl + w.hk * a.V.sch;
  for (int t = lo + warp; t < hi; t += kWarps) {
    long long half[2];
    int n[2];
    if (t < cached) {
      int pos[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        pos[j] = t * kTile + j * 8;
        bool there = true;
        if constexpr (kPages) {
          const int hn = 2 * t + j, page = hn / halves_per_page;
          there = page < n_chosen;
          pos[j] = there ? pages.chosen[page] * a.pages.page_size + (hn - page * halves_per_page) * 8 : 0;
        }
        n[j] = there ? min(8, max(0, w.seen - pos[j])) : 0;
        half[j] = (long long)w.begin + pos[j];
      }
      const bool masked = !kPages && w.own == 0 && t * kTile + kTile > w.limit(0);
      tile<F>(a.K, a.V, k_base, v_base, ks_base, vs_base, half, n, s.D, w.rows, a.scale_log2, q_sh, p_all[warp], run, lane, masked,
              [&](int key, int r) { return t * kTile + key < w.limit(r); });
    } else {
      const int first = (t - cached) * kTile;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        half[j] = w.first + first + j * 8;
        n[j] = min(8, max(0, w.own - first - j * 8));
      }
      const CacheView kn{a.K_new.ptr, a.K_new.dtype, a.K_new.sl, a.K_new.st, a.K_new.sh, nullptr, 0, 0, 0};
      const CacheView vn{a.V_new.ptr, a.V_new.dtype, a.V_new.sl, a.V_new.st, a.V_new.sh, nullptr, 0, 0, 0};
      tile<FQ>(kn, vn, w.layer * kn.sl + w.hk * kn.sh, w.layer * vn.sl + w.hk * vn.sh, 0, 0, half, n, s.D, w.rows, a.scale_log2, q_sh,
               p_all[warp], run, lane, true, [&](int key, int r) { return sees_new(a, w, w.token(r), first + key); });
    }
  }
  // the warps' parts, added up one warp after the other
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) run.l[i] += __shfl_xor_sync(kAll, run.l[i], d);
    if (g == 0) warp_part[warp][2 * c + i] = Part{run.m[i], run.l[i], run.m[i], 0.f};
  }
  float* o = reinterpret_cast<float*>(dyn_sh);
#pragma unroll
  for (int r = 0; r < kRows; ++r)
#pragma unroll
    for (int b = 0; b < 2; ++b)
      if (128 * b + 4 * lane < s.D)
        *reinterpret_cast<float4*>(o + (warp * kRows + r) * kMaxD + 128 * b + 4 * lane) = make_float4(run.o[b][r][0], run.o[b][r][1], run.o[b][r][2], run.o[b][r][3]);
  join_and_write<FQ, kWarps, kRows, kMaxD>(a, w, cluster, n_blk, rank, o, kMaxD, warp_part[0], &recv);
}

template <int F, bool kPages>
int launch_one(AttendArgs& a, cudaStream_t stream) {
  auto kern = attend_simt_kernel<F, kPages>;
  const Shape& s = a.s;
  const size_t dyn = kOBytes + (kPages ? page_mem_bytes(a.pages.max_pages, a.pages.budget, s.D) : 0);
  const int bound = kOBytes + (kPages ? (int)page_mem_bytes(kMaxPagesPerSeq, kMaxPagesPerSeq, kMaxD) : 0);
  // One table for launches that leave room for two blocks an SM, one for those with many pages.  64 pages of 32 out of 1024, 8 KV heads
  // of 128 with 4 query heads each: 57 us (96 with every launch planned as if it took the room of 8192 pages).
  static ClusterTable table, large;
  constexpr int kStatic = kRows * kMaxD * 4 + kWarps * kTile * kRows * 4 + kWarps * kRows * (int)sizeof(Part) + (int)sizeof(Received<kRows, kMaxD>);
  const int two = bound < 113 * 1024 - kStatic ? bound : 113 * 1024 - kStatic;
  const std::atomic<int>* resident = dyn <= (size_t)two ? table.resident(kern, kWarps * 32, two, bound) : large.resident(kern, kWarps * 32, bound, bound);
  if (!resident) return KVCRUSH_ERR_CUDA;
  const int n_blk = choose_cluster(resident, attend_units(a, kRows), attend_tiles(a), 2 * kWarps);
  dim3 grid;
  if (!attend_grid(a, kRows, n_blk, &grid)) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(kern, grid, dim3(kWarps * 32), dyn, stream, n_blk, a);
}

template <int F>
int launch_pages(AttendArgs& a, cudaStream_t stream) {
  return a.pages.page_size ? launch_one<F, true>(a, stream) : launch_one<F, false>(a, stream);
}

}  // namespace

int launch_attend_simt(AttendArgs a, cudaStream_t stream) {
  switch (a.K.dtype) {
    case KVCRUSH_INT8: return launch_pages<KVCRUSH_INT8>(a, stream);
    case KVCRUSH_E4M3: return launch_pages<KVCRUSH_E4M3>(a, stream);
    case KVCRUSH_INT4: return launch_pages<KVCRUSH_INT4>(a, stream);
    default: return launch_pages<KVCRUSH_FP32>(a, stream);
  }
}

}  // namespace kvc
