// Attention of many query rows over a cache of 16-bit values: trees of drafted tokens and grouped heads whose rows fill a tile of
// tcgen05.
//
// With 128 query rows a cached key costs 4 * 128 * D operations for its 4 D bytes, so that both the tensor cores and HBM have
// work.  A block takes 128 query rows (TMEM lane = row) of one (layer, sequence, KV head) and a share of the keys, in tiles of
// 64: S = Q K^T, the softmax in registers of the thread that owns the row, P back to TMEM as the left operand of O += P V, whose
// right operand V is read as it lies in memory (its channels are the fast axis).  The queries stay in shared memory, keys and
// values come by TMA into a ring.  Even and odd tiles are two streams with a softmax warpgroup, an output and two buffers of S
// each (P takes the first half of its own S; 512 columns in all), so that one stream's products and waits pass while the other
// takes its exponentials, which bound the kernel (16 a clock and SM).  Weights may exceed 1: the reference of a row moves only
// where a logit is 2^8 above it, and only then the output in TMEM is scaled.
// Tiles with keys that not every row sees (the tail of the cache, rows that only later tokens see, the new tokens with their
// mask) come last.  A weight of 0 would take a value that is not finite along, so a helper warp looks at the values of such
// a tile first: rows that do not exist or hold a value that is not finite are cleared, and in the second case the whole tile
// gets weight 0 and the threads of the rows add its keys one by one at the end.
// Trees over 32768 rows of 8 KV heads of 128, 4 query heads each (135 MB, 20.6 us at the measured copy bandwidth): 9 to 16 tokens
// 40 to 41 us, 63 tokens (34 GFLOP) 62 us, where attend_mma.cuh takes 82 to 89 and 151; 2048 rows, 63 tokens 15 against 20; 16 ragged
// sequences of 1192 to 4085 rows, 16 tokens 53 against 80.  In the 62 us tensor and special-function pipes are busy for 40 % on
// 96 SMs: two tiles of rows x 8 heads make 16 units, of which the chip holds clusters of six blocks (22, but 15 of seven).
#include "attend_common.cuh"
#include "tc_ptx.cuh"

namespace kvc {

namespace {

using namespace att;
using namespace fmt;

constexpr int kRows = 128;                   // query rows of a block
constexpr int kKeys = 64;                    // keys of a tile
constexpr int kThreads = 384;                // producer, an issuer for each stream, helper, two softmax warpgroups
constexpr int kExtra = 8;                    // keys added at a time by the rows' threads
constexpr float kSlackLog2 = 8.f;

template <int DP>
struct TreeMem {
  static constexpr int kBlocks = DP / 64;                               // of 64 channels: 128-byte rows
  static constexpr int kStages = DP == 128 ? 5 : 8;
  static constexpr int kQ = 0, kQBytes = kBlocks * kRows * 128;
  static constexpr int kTileBytes = kBlocks * kKeys * 128;              // keys or values of a stage
  static constexpr int kRing = kQ + kQBytes;
  static constexpr int kRecvO = kRing;                                  // outputs of the peers, when the ring is done with
  static constexpr int kRecvPart = kRing + 2 * kStages * kTileBytes + 256;
  static constexpr int kAux = kRecvPart + kMaxCluster * kRows * 8;
  static constexpr int kEnd = kAux + 3 * 1024;
  static_assert(kRows * DP * 4 + kMaxCluster * 16 <= 2 * kStages * kTileBytes + 256, "room for the peers' outputs");
  static_assert(kEnd <= 227 * 1024, "one block an SM");
};
struct TreeAux {
  // masked tiles have barriers of their own, since the helper warp does not follow the phases of the others
  unsigned long long k_full[8], k_empty[8], v_full[8], v_empty[8], masked_full[8], v_checked[8], s_full[2][2], p_ready[2][2], o_done[2], drain;
  float2 stats[2][kRows];                    // of the two streams, at the end
  uint32_t tmem;
  int abort_flag, slow;                      // slow: bit i, masked tile i of this block is added key by key
};
static_assert(sizeof(TreeAux) <= 3 * 1024, "auxiliary memory");

// Descriptor of 16 keys x 64 or 128 channels of values: rows of 64 channels (128 bytes, 128-byte swizzle), eight keys 1024 bytes
// apart, blocks of 64 channels kKeys rows apart.
__device__ __forceinline__ uint64_t values_desc(uint32_t addr) {
  return tc::smem_desc_sw128(addr) & ~(0x3FFFull << 16) | (uint64_t)(kKeys * 128 >> 4) << 16;
}
__device__ __forceinline__ void umma_p(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
        "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of the warp, the same each time; the code around stays uniform, so that descriptors are made in uniform registers
// (a thread by itself took 75 cycles for each product it issued).
__device__ __forceinline__ bool elect_one() {
  uint32_t ok;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
  return ok != 0;
}

template <int FQ>
__device__ __forceinline__ void widen8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = FQ == KVCRUSH_BF16 ? unpack_bf16(w[i]) : unpack_fp16(w[i]);
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}

template <int FQ, int DP>
__global__ void __launch_bounds__(kThreads, 1)
attend_tree_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_kn,
                   const __grid_constant__ CUtensorMap map_vn, AttendArgs a) {
  using M = TreeMem<DP>;
  using tc::mbar_wait;
  extern __shared__ __align__(1024) unsigned char sh[];
  chain_wait();
  chain_trigger();
  cg::cluster_group cluster = cg::this_cluster();
  const int n_blk = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Shape& s = a.s;
  Unit w;
  if (!unit_of<false>(a, kRows, w)) return;
  TreeAux* aux = reinterpret_cast<TreeAux*>(sh + M::kAux);
  const uint32_t base = tc::smem_u32(sh);
  if (tid == 0) {
    for (int i = 0; i < M::kStages; ++i) {
      tc::mbar_init(tc::smem_u32(&aux->k_full[i]), 1); tc::mbar_init(tc::smem_u32(&aux->k_empty[i]), 1);
      tc::mbar_init(tc::smem_u32(&aux->v_full[i]), 1); tc::mbar_init(tc::smem_u32(&aux->v_empty[i]), 1);
      tc::mbar_init(tc::smem_u32(&aux->masked_full[i]), 1); tc::mbar_init(tc::smem_u32(&aux->v_checked[i]), 32);
    }
    for (int x = 0; x < 2; ++x) {
      for (int i = 0; i < 2; ++i) { tc::mbar_init(tc::smem_u32(&aux->s_full[x][i]), 1); tc::mbar_init(tc::smem_u32(&aux->p_ready[x][i]), kRows); }
      tc::mbar_init(tc::smem_u32(&aux->o_done[x]), 1);
    }
    tc::mbar_init(tc::smem_u32(&aux->drain), 2);
    aux->abort_flag = 0;
    aux->slow = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tc::tmem_alloc(tc::smem_u32(&aux->tmem), 512);
    tc::tmem_relinquish();
  }
  // queries: rows of 128 bytes, 128-byte swizzle, as TMA would lay them out
  for (int e = tid; e < kRows * (DP / 8); e += kThreads) {
    const int r = e / (DP / 8), c = e % (DP / 8);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (r < w.rows && c * 8 < s.D)
      v = __ldg(reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(a.Q.ptr) +
              bytes_of<FQ>(w.layer * a.Q.sl + (w.first + w.token(r)) * a.Q.st + (w.hk * s.G + w.head(r)) * a.Q.sh + c * 8)));
    *reinterpret_cast<uint4*>(sh + M::kQ + (c >> 3) * kRows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = v;
  }
  proxy_fence();
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  volatile int* abort_flag = &aux->abort_flag;
  const uint32_t tmem = aux->tmem;                                    // stream x: S in columns 256 x, 256 x + 64, O from 256 x + 128 on

  const int full = (w.own ? w.seen : w.limit(0)) / kKeys;             // tiles that every row sees
  const int cached = (w.seen + kKeys - 1) / kKeys, total_tiles = cached + (w.own + kKeys - 1) / kKeys;
  const int per = (total_tiles + n_blk - 1) / n_blk, lo = min(total_tiles, rank * per), n = min(total_tiles, lo + per) - lo;
  const int n_full = max(0, min(n, full - lo));                       // of this block's tiles, those come first
  // keys of tile t of this block that exist
  auto keys_of = [&](int t) { return lo + t < cached ? min(kKeys, w.seen - (lo + t) * kKeys) : min(kKeys, w.own - (lo + t - cached) * kKeys); };

  if (warp == 0) {
    int issued = 0;
    if (lane == 0 && !a.withhold) {
      for (; issued < n; ++issued) {
        const int st = issued % M::kStages, round = issued / M::kStages;
        const bool is_new = lo + issued >= cached;
        const int row = is_new ? w.first + (lo + issued - cached) * kKeys : w.begin + (lo + issued) * kKeys;
        const uint32_t kb = tc::smem_u32(&aux->k_full[st]), vb = tc::smem_u32(issued < n_full ? &aux->v_full[st] : &aux->masked_full[st]);
        const uint32_t kd = base + M::kRing + st * 2 * M::kTileBytes, vd = kd + M::kTileBytes;
        if (round > 0 && !mbar_wait(tc::smem_u32(&aux->k_empty[st]), (round - 1) & 1, abort_flag, a.polls)) break;
        tc::mbar_expect_tx(kb, M::kTileBytes);
        for (int b = 0; b < M::kBlocks; ++b) tc::tma_load_4d(kd + b * kKeys * 128, is_new ? &map_kn : &map_k, kb, b * 64, row, w.hk, w.layer);
        if (round > 0 && !mbar_wait(tc::smem_u32(&aux->v_empty[st]), (round - 1) & 1, abort_flag, a.polls)) {
          for (uint32_t i = 0; i < tc::kDrainPolls && !tc::mbar_try_wait(kb, round & 1); ++i) {}
          break;
        }
        tc::mbar_expect_tx(vb, M::kTileBytes);
        for (int b = 0; b < M::kBlocks; ++b) tc::tma_load_4d(vd + b * kKeys * 128, is_new ? &map_vn : &map_v, vb, b * 64, row, w.hk, w.layer);
      }
      // nothing may be in flight when the block goes on: the last round's copies have landed (at once, but after a wait ran out)
      for (int t = max(0, issued - M::kStages); t < issued; ++t) {
        const int st = t % M::kStages, parity = (t / M::kStages) & 1;
        for (uint32_t i = 0; i < tc::kDrainPolls && !tc::mbar_try_wait(tc::smem_u32(&aux->k_full[st]), parity); ++i) {}
        const uint32_t vb = tc::smem_u32(t < n_full ? &aux->v_full[st] : &aux->masked_full[st]);
        const int v_parity = t < n_full ? parity : ((t - n_full) / M::kStages) & 1;
        for (uint32_t i = 0; i < tc::kDrainPolls && !tc::mbar_try_wait(vb, v_parity); ++i) {}
      }
    }
    __syncwarp();
  } else if (warp < 3) {
    // one issuer for each stream: a single one is bound by what it does between products (1800 cycles a tile)
    const int x = warp - 1;
    if (n > 0) {                                       // the whole warp follows, one lane issues
      constexpr uint32_t idesc_s = tc::make_idesc(kRows, kKeys, FQ == KVCRUSH_BF16);
      constexpr uint32_t idesc_o = tc::make_idesc(kRows, DP, FQ == KVCRUSH_BF16) | 1u << 16;      // right operand: channels are the fast axis
      const uint64_t desc_q = tc::smem_desc_sw128(base + M::kQ), desc_k = tc::smem_desc_sw128(base + M::kRing);
      const uint64_t desc_v = values_desc(base + M::kRing + M::kTileBytes);
      auto wait = [&](unsigned long long* bar, int parity) {
        return (bool)__all_sync(kAll, mbar_wait(tc::smem_u32(bar), parity, abort_flag, a.polls));
      };
      auto product_s = [&](int t, int st, int parity) {
        const int u = t >> 1;
        // S takes the place of the weights of two tiles before in its stream, which that tile's product has read
        if (u >= 2 && !wait(&aux->o_done[x], u & 1)) return false;
        if (!wait(&aux->k_full[st], parity)) return false;
        tc::tc_fence_after();
        const uint32_t d = tmem + x * 256 + (u & 1) * kKeys;
        const uint64_t dk = desc_k + (uint32_t)(st * (2 * M::kTileBytes >> 4));
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < DP / 16; ++k)
            tc::umma_bf16(d, desc_q + ((k >> 2) * kRows * 128 + (k & 3) * 32 >> 4), dk + ((k >> 2) * kKeys * 128 + (k & 3) * 32 >> 4), idesc_s, k > 0);
          tc::umma_commit(tc::smem_u32(&aux->k_empty[st]));
          tc::umma_commit(tc::smem_u32(&aux->s_full[x][u & 1]));
        }
        __syncwarp();
        return true;
      };
      auto product_o = [&](int t, int st, int parity) {
        const int u = t >> 1;
        if (t < n_full && !wait(&aux->v_full[st], parity)) return false;
        // (the weights of a masked tile come after its values)
        if (!wait(&aux->p_ready[x][u & 1], (u >> 1) & 1)) return false;
        tc::tc_fence_after();
        const uint32_t d = tmem + x * 256 + 128, p = tmem + x * 256 + (u & 1) * kKeys;
        const uint64_t dv = desc_v + (uint32_t)(st * (2 * M::kTileBytes >> 4));
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < kKeys / 16; ++k) umma_p(d, p + k * 8, dv + (k * 16 * 128 >> 4), idesc_o, u > 0 || k > 0);
          tc::umma_commit(tc::smem_u32(&aux->v_empty[st]));
          tc::umma_commit(tc::smem_u32(&aux->o_done[x]));
        }
        __syncwarp();
        return true;
      };
      bool ok = true;
      int st = x, parity = 0, st_o = x, parity_o = 0;   // ring positions of the two products
      for (int t = x; ok && t < n + 2; t += 2) {
        if (t < n) {
          ok = product_s(t, st, parity);
          if ((st += 2) >= M::kStages) { st -= M::kStages; parity ^= 1; }
        }
        if (ok && t >= 2) {
          ok = product_o(t - 2, st_o, parity_o);
          if ((st_o += 2) >= M::kStages) { st_o -= M::kStages; parity_o ^= 1; }
        }
      }
      // products in flight end before TMEM is freed
      if (elect_one()) tc::umma_commit(tc::smem_u32(&aux->drain));
      __syncwarp();
      for (uint32_t i = 0; i < tc::kDrainPolls && !tc::mbar_try_wait(tc::smem_u32(&aux->drain), 0); ++i) {}
    }
    __syncwarp();
  } else if (warp < 4) {
    // values of the masked tiles: a lane looks at rows lane and lane + 32
    for (int t = n_full; t < n; ++t) {
      const int st = t % M::kStages, keys = keys_of(t);
      if (!__all_sync(kAll, mbar_wait(tc::smem_u32(&aux->masked_full[st]), ((t - n_full) / M::kStages) & 1, abort_flag, a.polls))) break;
      for (int h = lane; h < kKeys; h += 32) {
        unsigned char* vd = sh + M::kRing + st * 2 * M::kTileBytes + M::kTileBytes + h * 128;    // row h of every block of channels
        bool bad = false;
        if (h < keys)
          for (int b = 0; b < M::kBlocks; ++b)
            for (int c = 0; c < 8; ++c) {
              const uint4 v = *reinterpret_cast<const uint4*>(vd + b * kKeys * 128 + c * 16);
              const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                constexpr uint32_t e = FQ == KVCRUSH_BF16 ? 0x7F80u : 0x7C00u;
                bad |= (x[i] & e) == e || (x[i] >> 16 & e) == e;
              }
            }
        if (bad) atomicOr(&aux->slow, 1 << (t - n_full));              // the whole tile then has weight 0, in its other rows too
        if (h >= keys || bad)
          for (int b = 0; b < M::kBlocks; ++b)
            for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(vd + b * kKeys * 128 + c * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      proxy_fence();
      tc::mbar_arrive(tc::smem_u32(&aux->v_checked[st]));
    }
  } else {
    const int x = (warp - 4) >> 2;                     // stream: tiles x, x + 2, ..
    const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16, tmem_o = tmem + x * 256 + 128;
    const int r = (warp & 3) * 32 + lane;
    const float scale = a.scale_log2;
    float m = -FLT_MAX, l = 0.f;
    const int tok = w.token(min(r, w.rows - 1)), limit = w.limit(min(r, w.rows - 1));
    // which keys of masked tile t this row sees
    auto seen_of = [&](int t) {
      const int keys = keys_of(t);
      unsigned long long see = keys >= 64 ? ~0ull : (1ull << keys) - 1ull;
      if (lo + t < cached) {
        const int left = max(0, limit - (lo + t) * kKeys);
        if (left < 64) see &= (1ull << left) - 1ull;
      } else {
        const int first = (lo + t - cached) * kKeys;
        if (!a.fresh.mask) {
          const int left = max(0, tok + 1 - first);
          if (left < 64) see &= (1ull << left) - 1ull;
        } else {
          const uint32_t* row = a.fresh.mask + (long long)(w.first + tok) * a.fresh.mask_words + first / 32;
          unsigned long long bits = __ldg(row);
          if (first / 32 + 1 < a.fresh.mask_words) bits |= (unsigned long long)__ldg(row + 1) << 32;
          see &= bits;
        }
      }
      return see;
    };
    bool ok = true;
    auto wait = [&](unsigned long long* bar, int parity) {             // one answer for the warp
      return (bool)__all_sync(kAll, mbar_wait(tc::smem_u32(bar), parity, abort_flag, a.polls));
    };
    // the output so far, times f (a factor for each row)
    auto scale_output = [&](float f) {
#pragma unroll 1
      for (int c = 0; c < DP; c += 16) {
        uint32_t v[16];
        tc::tmem_ld16(tmem_o + lanes + c, v);
        tc::tmem_wait16(v);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * f);
        tmem_st16(tmem_o + lanes + c, v);
      }
      tmem_wait_st();
    };
    for (int t = x; t < n; t += 2) {
      const int u = t >> 1;
      if (!wait(&aux->s_full[x][u & 1], (u >> 1) & 1)) { ok = false; break; }
      tc::tc_fence_after();
      const uint32_t at = tmem + x * 256 + lanes + (u & 1) * kKeys;
      uint32_t v[4][16];
#pragma unroll
      for (int i = 0; i < 4; ++i) tc::tmem_ld16(at + 16 * i, v[i]);
#pragma unroll
      for (int i = 0; i < 4; ++i) tc::tmem_wait16(v[i]);
      if (t >= n_full) {
        if (!wait(&aux->v_checked[t % M::kStages], ((t - n_full) / M::kStages) & 1)) { ok = false; break; }
        const unsigned long long see = *reinterpret_cast<volatile int*>(&aux->slow) >> (t - n_full) & 1 ? 0ull : seen_of(t);
#pragma unroll
        for (int i = 0; i < 64; ++i) v[i >> 4][i & 15] = see >> i & 1ull ? v[i >> 4][i & 15] : 0xFF800000u;
      }
      float top[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        top[i] = __uint_as_float(v[i][15]);
#pragma unroll
        for (int j = 0; j < 15; j += 3)
          top[i] = fmaxf(top[i], tc::max3(__uint_as_float(v[i][j]), __uint_as_float(v[i][j + 1]), __uint_as_float(v[i][j + 2])));
      }
      const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * scale;
      if (__any_sync(kAll, most - m > kSlackLog2)) {
        const float m_new = fmaxf(m, most), f = ex2(m - m_new);
        m = m_new;
        l *= f;
        if (u > 0) {                                   // the product of the tile before may still add to the output
          if (!wait(&aux->o_done[x], (u - 1) & 1)) { ok = false; break; }
          tc::tc_fence_after();
          scale_output(f);
        }
      }
      const tc::f32x2 scale2 = tc::splat2(scale), minus_m = tc::splat2(-m);
      tc::f32x2 sum[2] = {tc::splat2(0.f), tc::splat2(0.f)};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t p[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t* x = &v[2 * i + (j >> 3)][2 * (j & 7)];
          const tc::f32x2 e = tc::exp2_sfu2(tc::fma2(tc::pack2(x[0], x[1]), scale2, minus_m));
          sum[j & 1] = tc::add2(sum[j & 1], e);
          float e0, e1;
          tc::unpack2(e, e0, e1);
          p[j] = FQ == KVCRUSH_BF16 ? pack_bf16(e0, e1) : pack_fp16(e0, e1);
        }
        tmem_st16(at + 16 * i, p);
      }
      l += tc::sum4(sum);
      tmem_wait_st();
      tc::tc_fence_before();
      tc::mbar_arrive(tc::smem_u32(&aux->p_ready[x][u & 1]));
    }
    const int mine = (n - x + 1) >> 1;                 // tiles of this stream
    if (ok && mine > 0) ok = wait(&aux->o_done[x], (mine - 1) & 1);
    tc::tc_fence_after();
    // keys that are added one by one
    const int slow = ok ? *reinterpret_cast<volatile int*>(&aux->slow) : 0;
#pragma unroll 1
    for (int t = n_full; t < n; ++t) {
      if ((t & 1) != x || !(slow >> (t - n_full) & 1)) continue;
      const unsigned long long see = seen_of(t);
      const bool is_new = lo + t >= cached;
      const TensorView kv{a.K.ptr, a.K.dtype, a.K.sl, a.K.st, a.K.sh}, vv{a.V.ptr, a.V.dtype, a.V.sl, a.V.st, a.V.sh};
      const TensorView ks = is_new ? a.K_new : kv, vs = is_new ? a.V_new : vv;
      const long long row0 = is_new ? w.first + (lo + t - cached) * kKeys : w.begin + (lo + t) * kKeys;
      const unsigned char* kb = static_cast<const unsigned char*>(ks.ptr) + bytes_of<FQ>(w.layer * ks.sl + w.hk * ks.sh + row0 * ks.st);
      const unsigned char* vb = static_cast<const unsigned char*>(vs.ptr) + bytes_of<FQ>(w.layer * vs.sl + w.hk * vs.sh + row0 * vs.st);
      const int keys = keys_of(t);
#pragma unroll 1
      for (int e0 = 0; e0 < keys; e0 += kExtra) {
        const unsigned char *kp[kExtra], *vp[kExtra];
        float y[kExtra];
        bool sees[kExtra];
        float most = -FLT_MAX;
#pragma unroll
        for (int j = 0; j < kExtra; ++j) {
          const int e = min(e0 + j, keys - 1);
          kp[j] = kb + bytes_of<FQ>(e * ks.st); vp[j] = vb + bytes_of<FQ>(e * vs.st);
          sees[j] = e0 + j < keys && (see >> e & 1ull);
          y[j] = 0.f;
        }
#pragma unroll 1
        for (int c = 0; c < s.D / 8; ++c) {
          float q[8];
          widen8<FQ>(*reinterpret_cast<const uint4*>(sh + M::kQ + (c >> 3) * kRows * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)), q);
#pragma unroll
          for (int j = 0; j < kExtra; ++j) {
            float k[8];
            widen8<FQ>(__ldg(reinterpret_cast<const uint4*>(kp[j]) + c), k);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[j] = fmaf(q[i], k[i], y[j]);
          }
        }
#pragma unroll
        for (int j = 0; j < kExtra; ++j) {
          y[j] = sees[j] ? y[j] * scale : neg_inf();
          most = fmaxf(most, y[j]);
        }
        const float m_new = fmaxf(m, most), f = ex2(m - m_new);
        m = m_new;
        l *= f;
#pragma unroll
        for (int j = 0; j < kExtra; ++j) {
          y[j] = ex2(y[j] - m);
          l += sees[j] ? y[j] : 0.f;
        }
#pragma unroll 1
        for (int c = 0; c < DP; c += 16) {
          uint32_t o[16];
          tc::tmem_ld16(tmem_o + lanes + c, o);
          tc::tmem_wait16(o);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (c + 8 * h >= s.D) break;
#pragma unroll
            for (int j = 0; j < kExtra; ++j) {
              float v[8];
              widen8<FQ>(__ldg(reinterpret_cast<const uint4*>(vp[j]) + c / 8 + h), v);
              if (sees[j]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) o[8 * h + i] = __float_as_uint(fmaf(y[j], v[i], __uint_as_float(o[8 * h + i])));
              }
            }
          }
          tmem_st16(tmem_o + lanes + c, o);
        }
        tmem_wait_st();
      }
    }
    aux->stats[x][r] = make_float2(m, l);
    tc::tc_fence_before();
  }
  // The join: a row's thread sends its outputs to the owners of their shares.  The peers' rings are free when all have come here.
  __syncthreads();
  const int vec = s.D / 4, total = w.rows * vec, share = n_blk == 1 ? total : (total + n_blk - 1) / n_blk;
  const uint32_t share_magic = 0xFFFFFFFFu / (uint32_t)share + 1u;
  float4* recv_o = reinterpret_cast<float4*>(sh + M::kRecvO);
  float2* recv_part = reinterpret_cast<float2*>(sh + M::kRecvPart);
  if (n_blk > 1) { cluster_arrive(); cluster_wait(); }
  if (warp >= 4) {
    // either warpgroup joins the streams in half of the channels
    tc::tc_fence_after();
    const int half = (warp - 4) >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t at = tmem + ((uint32_t)(warp & 3) * 32u << 16) + 128;
    const float2 s0 = aux->stats[0][r], s1 = aux->stats[1][r];
    const float m = fmaxf(s0.x, s1.x), f0 = ex2(s0.x - m), f1 = ex2(s1.x - m);
    if (half == 0 && r < w.rows)
      for (int p = 0; p < n_blk; ++p) {
        float2* dst = recv_part + rank * kRows + r;
        *(n_blk > 1 ? cluster.map_shared_rank(dst, p) : dst) = make_float2(m, fmaf(s0.y, f0, s1.y * f1));
      }
#pragma unroll 1
    for (int c = half * DP / 2; c < (half + 1) * DP / 2; c += 16) {
      uint32_t o[16], o1[16];
      if (n > 0) { tc::tmem_ld16(at + c, o); tc::tmem_wait16(o); }
      if (n > 1) { tc::tmem_ld16(at + 256 + c, o1); tc::tmem_wait16(o1); }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = n > 0 ? __uint_as_float(o[i]) * f0 : 0.f;
        o[i] = __float_as_uint(n > 1 ? fmaf(__uint_as_float(o1[i]), f1, y) : y);
      }
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        if (r < w.rows && c + i < s.D) {
          const int e = r * vec + (c + i) / 4, owner = n_blk == 1 ? 0 : share == 1 ? e : (int)__umulhi((uint32_t)e, share_magic);
          float4* dst = recv_o + rank * share + (e - owner * share);
          *(n_blk > 1 ? cluster.map_shared_rank(dst, owner) : dst) =
              make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]), __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
        }
      }
    }
    tc::tc_fence_before();
  }
  if (n_blk > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
  if (warp == 1) {
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, 512);
  }
  const int mine = rank * share;
  for (int i = tid; i < min(share, total - mine); i += kThreads) {
    const int e = mine + i, row = e / vec, d = (e - row * vec) * 4;
    float top = neg_inf(), sum_l = 0.f;
    for (int p = 0; p < n_blk; ++p) top = fmaxf(top, recv_part[p * kRows + row].x);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int p = 0; p < n_blk; ++p) {
      const float2 q = recv_part[p * kRows + row];
      const float4 v = recv_o[p * share + i];
      const float f = ex2(q.x - top);
      sum_l = fmaf(q.y, f, sum_l);
      sum.x = fmaf(v.x, f, sum.x); sum.y = fmaf(v.y, f, sum.y); sum.z = fmaf(v.z, f, sum.z); sum.w = fmaf(v.w, f, sum.w);
    }
    const bool none = sum_l == 0.f;                    // no weight: zeros, whatever the values hold (0 times infinity)
    const float inv = 1.f / sum_l;
    const float x[4] = {none ? 0.f : sum.x * inv, none ? 0.f : sum.y * inv, none ? 0.f : sum.z * inv, none ? 0.f : sum.w * inv};
    const int token = w.token(row), head = w.hk * w.G + row + w.row0 - token * w.G;
    unsigned char* op = static_cast<unsigned char*>(const_cast<void*>(a.O.ptr)) +
        bytes_of<FQ>(w.layer * a.O.sl + (w.first + token) * a.O.st + head * a.O.sh + d);
    if constexpr (FQ == KVCRUSH_BF16) *reinterpret_cast<uint2*>(op) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    else *reinterpret_cast<uint2*>(op) = make_uint2(pack_fp16(x[0], x[1]), pack_fp16(x[2], x[3]));
    if (d == 0 && a.lse)
      a.lse[((long long)w.layer * s.Hq + head) * a.fresh.total + w.first + token] = sum_l == 0.f ? neg_inf() : (top + log2f(sum_l)) * 0.6931471805599453f;
  }
  if (tid == 0 && *abort_flag) report(a.status, KVCRUSH_DEV_TIMEOUT, KID_ATTEND_TREE, (int)blockIdx.x, 0);
}

template <int FQ, int DP>
int launch_one(const AttendArgs& a, const CUtensorMap (&maps)[4], cudaStream_t stream) {
  using M = TreeMem<DP>;
  auto kern = attend_tree_kernel<FQ, DP>;
  static ClusterTable table;
  const std::atomic<int>* resident = table.resident(kern, kThreads, M::kEnd, M::kEnd);
  if (!resident) return KVCRUSH_ERR_CUDA;
  // what a block does once takes as long as about ten tiles
  const int n_blk = choose_cluster(resident, attend_units(a, kRows), (a.s.max_seqlen + (a.K_new.ptr ? a.fresh.most : 0) + kKeys - 1) / kKeys, 10);
  dim3 grid;
  if (!attend_grid(a, kRows, n_blk, &grid)) return KVCRUSH_ERR_UNSUPPORTED;
  return launch_chained(kern, grid, dim3(kThreads), M::kEnd, stream, n_blk, maps[0], maps[1], maps[2], maps[3], a);
}

}  // namespace

// From more than 16 query rows on, and two tiles of keys; a negative scale would turn the maximum around.  us of this kernel / of
// attend_mma.cuh (whose blocks take 8, 16 or 32 rows), bf16, caches out of HBM:
//   KV heads x channels, cached rows      16 rows      20 rows      40 rows
//   8 x 128, 2048                        11.0 / 9.6   11.0 / 11.7  11.8 / 13.3
//   8 x 128, 32768                       40.4 / 33.0  40.5 / 45.3  41.0 / 53.6
//   8 x 64, 32768                        33.7 / 21.2  33.8 / 28.6  33.8 / 33.4
//   32 x 128, 32768                      92.9 / 82.4  92.0 / 87.2  93.9 / 157
//   32 x 64, 32768                       72.1 / 53.0  72.3 / 49.6  72.2 / 85.6
//   32 x 128, 16 sequences of 2048        124 / 91.0   125 / 100    133 / 210
// So up to 16 rows the other one is ahead everywhere and from 33 on nearly everywhere this one; between, this one is ahead for few
// heads of 128 over long caches only, and the rule, which does not look at heads and channels, costs the others up to a third.
bool attend_tree_fits(const AttendArgs& a) {
  const long long rows = (long long)a.fresh.most * a.s.G;
  return a.pages.page_size == 0 && (a.K.dtype == KVCRUSH_BF16 || a.K.dtype == KVCRUSH_FP16) && a.s.D <= 128 && rows > 16 &&
         a.s.max_seqlen >= 2 * kKeys && a.scale_log2 > 0.f;
}

int launch_attend_tree(const AttendArgs& a, bool* taken, cudaStream_t stream) {
  CUtensorMap maps[4];
  const TensorView cache[2] = {{a.K.ptr, a.K.dtype, a.K.sl, a.K.st, a.K.sh}, {a.V.ptr, a.V.dtype, a.V.sl, a.V.st, a.V.sh}};
  *taken = a.s.T > 0;
  for (int i = 0; i < 2 && *taken; ++i) {
    *taken = tc::make_map(&maps[i], cache[i], a.s.D, a.s.T, a.s.Hkv, a.s.n_layers, kKeys);
    if (*taken && a.K_new.ptr) *taken = tc::make_map(&maps[2 + i], i ? a.V_new : a.K_new, a.s.D, a.fresh.total, a.s.Hkv, a.s.n_layers, kKeys);
    else maps[2 + i] = maps[i];
  }
  if (!*taken) return KVCRUSH_OK;
  if (a.K.dtype == KVCRUSH_BF16) return a.s.D <= 64 ? launch_one<KVCRUSH_BF16, 64>(a, maps, stream) : launch_one<KVCRUSH_BF16, 128>(a, maps, stream);
  return a.s.D <= 64 ? launch_one<KVCRUSH_FP16, 64>(a, maps, stream) : launch_one<KVCRUSH_FP16, 128>(a, maps, stream);
}

}  // namespace kvc
