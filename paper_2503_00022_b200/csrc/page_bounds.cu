// Bounds of the keys of every page: least and largest value of each channel.
//
// Bound by reading K once.  A thread owns eight channels of one KV head of one page and walks down the page's rows, eight at a
// time; the heads of a row are neighbours, so a warp reads consecutive bytes.  Where there are few pages (the last one of each
// sequence, when a cache has grown) four threads share the rows and meet in shared memory, so that a page of 32 rows
// is under way as a whole.  8 heads of 128 in bf16, pages of 32, one thread -> four: the last page 4.0 -> 2.7 us, all of 8192 rows
// 8.6 -> 5.8; all of 32768 rows, which fill the chip anyway, 14.3 -> 17.6, so that many pages keep to one.
#include "cache_format.cuh"

namespace kvc {

namespace {

using namespace fmt;

constexpr int kUnroll = 8;

// kVectors: pieces of eight channels of a block; kGroups: threads for the same ones.
template <int F, int kVectors, int kGroups>
__global__ void __launch_bounds__(kVectors * kGroups)
page_bounds_kernel(Shape s, TensorView K, int page_size, int max_pages, int pages_per_seq, int recent, const int32_t* __restrict__ row_begin,
                   const int32_t* __restrict__ row_count, TensorView lo, TensorView hi) {
  chain_wait();
  chain_trigger();
  const int vec = s.D / 8, per_page = s.Hkv * vec;
  __shared__ float part[kGroups > 1 ? kGroups - 1 : 1][16][kGroups > 1 ? kVectors : 1];
  const int group = threadIdx.x / kVectors, at = threadIdx.x % kVectors, v = blockIdx.y * kVectors + at;
  const int page_of_seq = blockIdx.x % pages_per_seq, seg = blockIdx.x / pages_per_seq;
  const int layer = seg / s.n_seqs, seq = seg - layer * s.n_seqs;
  int begin, count;
  rows_of(s, row_begin, row_count, layer, seq, begin, count);
  const int pages = (int)(((long long)count + page_size - 1) / page_size);
  const int page = recent ? pages - pages_per_seq + page_of_seq : page_of_seq;
  if (page < 0 || page >= pages) return;
  const bool used = v < per_page;
  const int h = used ? v / vec : 0, c = used ? (v - h * vec) * 8 : 0;
  const long long first = (long long)page * page_size;
  const int rows = (int)min((long long)page_size, count - first);
  const unsigned char* p = static_cast<const unsigned char*>(K.ptr) + bytes_of<F>(layer * K.sl + (begin + first) * K.st + h * K.sh + c);
  const long long step = bytes_of<F>(K.st);
  float least[8], most[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { least[i] = __uint_as_float(0x7F800000u); most[i] = __uint_as_float(0xFF800000u); }
  for (int r = group * kUnroll; used && r < rows; r += kGroups * kUnroll) {
    Raw8<F> raw[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) raw[u].load(p + min(r + u, rows - 1) * step);       // the last row again: bounds do not change
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float x[8];
      raw[u].widen(x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // once NaN, both stay so
        asm("min.NaN.f32 %0, %0, %1;" : "+f"(least[i]) : "f"(x[i]));
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(most[i]) : "f"(x[i]));
      }
    }
  }
  if (kGroups > 1 && group) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { part[group - 1][i][at] = least[i]; part[group - 1][8 + i][at] = most[i]; }
  }
  if (kGroups > 1) __syncthreads();
  if (group || !used) return;
#pragma unroll
  for (int k = 0; k < kGroups - 1; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      asm("min.NaN.f32 %0, %0, %1;" : "+f"(least[i]) : "f"(part[k][i][at]));
      asm("max.NaN.f32 %0, %0, %1;" : "+f"(most[i]) : "f"(part[k][8 + i][at]));
    }
  const long long out_row = (long long)seq * max_pages + page;
  Raw8<F> out;
  out.narrow(least);
  out.store(static_cast<unsigned char*>(const_cast<void*>(lo.ptr)) + bytes_of<F>(layer * lo.sl + out_row * lo.st + h * lo.sh + c));
  out.narrow(most);
  out.store(static_cast<unsigned char*>(const_cast<void*>(hi.ptr)) + bytes_of<F>(layer * hi.sl + out_row * hi.st + h * hi.sh + c));
}

template <int F>
int launch_type(const Shape& s, const TensorView& K, int page_size, int max_pages, int per_seq, int recent, const int32_t* row_begin,
                const int32_t* row_count, const TensorView& lo, const TensorView& hi, cudaStream_t stream) {
  const long long blocks = (long long)s.n_layers * s.n_seqs * per_seq;
  if (blocks > 0x7FFFFFFFLL) return KVCRUSH_ERR_UNSUPPORTED;
  const int vectors = s.Hkv * (s.D / 8);
  const bool few = page_size > kUnroll && blocks * ((vectors + 127) / 128) < 2 * sm_count();
  auto launch = [&](auto kern, int per_block, int groups) {
    return launch_chained(kern, dim3((unsigned)blocks, (unsigned)((vectors + per_block - 1) / per_block)), dim3(per_block * groups), 0, stream, 1, s, K,
                          page_size, max_pages, per_seq, recent, row_begin, row_count, lo, hi);
  };
  return few ? launch(page_bounds_kernel<F, 64, 4>, 64, 4) : launch(page_bounds_kernel<F, 128, 1>, 128, 1);
}

}  // namespace

int launch_page_bounds(const Shape& s, const TensorView& K, int page_size, int recent_pages, const int32_t* row_begin,
                       const int32_t* row_count, const TensorView& lo, const TensorView& hi, cudaStream_t stream) {
  const int max_pages = (int)(((long long)s.max_seqlen + page_size - 1) / page_size);
  const int per_seq = recent_pages > 0 && recent_pages < max_pages ? recent_pages : max_pages, recent = recent_pages > 0;
  if (per_seq == 0) return KVCRUSH_OK;
  switch (K.dtype) {
    case KVCRUSH_BF16: return launch_type<KVCRUSH_BF16>(s, K, page_size, max_pages, per_seq, recent, row_begin, row_count, lo, hi, stream);
    case KVCRUSH_FP16: return launch_type<KVCRUSH_FP16>(s, K, page_size, max_pages, per_seq, recent, row_begin, row_count, lo, hi, stream);
    default: return launch_type<KVCRUSH_FP32>(s, K, page_size, max_pages, per_seq, recent, row_begin, row_count, lo, hi, stream);
  }
}

}  // namespace kvc
