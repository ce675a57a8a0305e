// Bounds of the keys of every page: least and largest value of each channel.
//
// Bound by reading K once.  A thread owns eight channels of one KV head of one page and walks down the page's rows; the heads
// of a row are neighbours, so a warp reads consecutive bytes.
#include "cache_format.cuh"

namespace kvc {

namespace {

using namespace fmt;

constexpr int kThreads = 128;

template <int F>
__global__ void __launch_bounds__(kThreads)
page_bounds_kernel(Shape s, TensorView K, int page_size, int max_pages, int pages_per_seq, int recent, const int32_t* __restrict__ row_begin,
                   const int32_t* __restrict__ row_count, TensorView lo, TensorView hi) {
  chain_wait();
  chain_trigger();
  const int vec = s.D / 8, per_page = s.Hkv * vec;
  const int v = blockIdx.y * kThreads + threadIdx.x;
  const int page_of_seq = blockIdx.x % pages_per_seq, seg = blockIdx.x / pages_per_seq;
  const int layer = seg / s.n_seqs, seq = seg - layer * s.n_seqs;
  int begin, count;
  rows_of(s, row_begin, row_count, layer, seq, begin, count);
  const int pages = (int)(((long long)count + page_size - 1) / page_size);
  const int page = recent ? pages - pages_per_seq + page_of_seq : page_of_seq;
  if (page < 0 || page >= pages || v >= per_page) return;
  const int h = v / vec, c = (v - h * vec) * 8;
  const long long first = (long long)page * page_size;
  const int rows = (int)min((long long)page_size, count - first);
  const unsigned char* p = static_cast<const unsigned char*>(K.ptr) + bytes_of<F>(layer * K.sl + (begin + first) * K.st + h * K.sh + c);
  const long long step = bytes_of<F>(K.st);
  float least[8], most[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { least[i] = __uint_as_float(0x7F800000u); most[i] = __uint_as_float(0xFF800000u); }
  constexpr int kUnroll = 8;
  for (int r = 0; r < rows; r += kUnroll) {
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
  const long long out_row = (long long)seq * max_pages + page;
  Raw8<F> out;
  out.narrow(least);
  out.store(static_cast<unsigned char*>(const_cast<void*>(lo.ptr)) + bytes_of<F>(layer * lo.sl + out_row * lo.st + h * lo.sh + c));
  out.narrow(most);
  out.store(static_cast<unsigned char*>(const_cast<void*>(hi.ptr)) + bytes_of<F>(layer * hi.sl + out_row * hi.st + h * hi.sh + c));
}

}  // namespace

int launch_page_bounds(const Shape& s, const TensorView& K, int page_size, int recent_pages, const int32_t* row_begin,
                       const int32_t* row_count, const TensorView& lo, const TensorView& hi, cudaStream_t stream) {
  const int max_pages = (int)(((long long)s.max_seqlen + page_size - 1) / page_size);
  const int per_seq = recent_pages > 0 && recent_pages < max_pages ? recent_pages : max_pages;
  const long long blocks = (long long)s.n_layers * s.n_seqs * per_seq;
  if (blocks == 0) return KVCRUSH_OK;
  const int groups = (s.Hkv * (s.D / 8) + kThreads - 1) / kThreads;
  if (blocks > 0x7FFFFFFFLL) return KVCRUSH_ERR_UNSUPPORTED;
  auto kern = K.dtype == KVCRUSH_BF16 ? page_bounds_kernel<KVCRUSH_BF16> : K.dtype == KVCRUSH_FP16 ? page_bounds_kernel<KVCRUSH_FP16> : page_bounds_kernel<KVCRUSH_FP32>;
  return launch_chained(kern, dim3((unsigned)blocks, (unsigned)groups), dim3(kThreads), 0, stream, 1, s, K, page_size, max_pages, per_seq,
                        recent_pages > 0 ? 1 : 0, row_begin, row_count, lo, hi);
}

}  // namespace kvc
