// Tokens into the pages of the 8-bit cache and out of them.
//
// All three kernels move bytes: a workgroup takes the keys or the values of one page, a page is one run of 8 or 16 KB.
// append reads 256 and writes 128 bytes per token and head (twice, for K and V), load the other way round, evict (the gather of
// the tokens that stay) reads and writes 128.
#include "cache_common.h"

namespace shplb {
namespace {

constexpr int kThreads = 256;

// The largest of a value over a workgroup of four waves.
__device__ __forceinline__ uint32_t workgroup_max(uint32_t x, uint32_t* lds) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x = max(x, uint32_t(__shfl_xor(int(x), d)));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
  __syncthreads();
  return max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}

__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Workgroup (pair of sequence and head, page of those that the step touches, K or V).  A thread has eight dims of every sixteenth token.
template <int BLOCK, int FMT>
__global__ __launch_bounds__(kThreads) void append_kernel(CacheArgs c, StepArgs t, const uint16_t* k, const uint16_t* v, int pages_each) {
  __shared__ uint32_t lds[4];
  const uint32_t x = blockIdx.x >> 1, which = blockIdx.x & 1;
  const int pair = x / uint32_t(pages_each), s = pair / c.n_kv_heads, h = pair - s * c.n_kv_heads;
  const int len = c.lens[pair];
  int row0, n;
  step_tokens(t, s, row0, n);
  if (n == 0 || len <= 0 || !good_length(c, len)) return;
  const int first = len - n, start = max(first, 0);              // position of row 0, of the first token written
  const int page_in_row = start / BLOCK + int(x - uint32_t(pair) * pages_each), at = page_in_row * BLOCK;
  if (at >= len) return;
  const int page = c.table[int64_t(pair) * c.max_pages + page_in_row];
  if (page < 0 || page >= c.n_pages) return;
  const int begin = max(start - at, 0), end = min(len - at, BLOCK);   // slots written
  uint8_t* codes = (which ? c.v : c.k) + int64_t(page) * (BLOCK * kHeadDim);
  float* scale = (which ? c.v_scale : c.k_scale) + page;
  const uint16_t* src = (which ? v : k) + (int64_t(row0) + (at - first)) * t.stride_t + h * t.stride_h;   // of slot 0
  const int r = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
  constexpr int kEach = BLOCK / 16;
  u32x4 in[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    in[u] = u32x4{0, 0, 0, 0};
    if (slot >= begin && slot < end) in[u] = *reinterpret_cast<const u32x4*>(src + slot * t.stride_t + d);
  }
  uint32_t before = begin > 0 ? __float_as_uint(*scale) : 0u;
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(in[u][e] << 16 & 0x7fff0000u, in[u][e] & 0x7fff0000u));
  asm volatile("" : "+v"(before));                              // here by now: thread 0 may write it behind the barrier
  top = workgroup_max(top, lds);
  const uint32_t bits = begin > 0 ? larger_scale(before, scale_bits<FMT>(top)) : scale_bits<FMT>(top);
  const float inv = inverse_scale(bits), limit = code_limit<FMT>(bits);
  const bool none = bits >= 0x7f800000u;                        // codes of a page without a scale are zeros
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    if (slot >= begin && slot < end) {
      const u32x4 w = none ? u32x4{0, 0, 0, 0} : in[u];
      u32x2 o;
      o.x = to_codes<FMT>(low_bf16(w.x) * inv, high_bf16(w.x) * inv, low_bf16(w.y) * inv, high_bf16(w.y) * inv, limit);
      o.y = to_codes<FMT>(low_bf16(w.z) * inv, high_bf16(w.z) * inv, low_bf16(w.w) * inv, high_bf16(w.w) * inv, limit);
      *reinterpret_cast<u32x2*>(codes + slot * kHeadDim + d) = o;
    }
  }
  if (threadIdx.x == 0 && (begin == 0 || bits != before)) *scale = __uint_as_float(bits);
  // the older tokens, where the scale has grown
  if (begin > 0 && bits != before) {
    const float ratio = __uint_as_float(before) * inv;          // a power of two below 1; it may underflow to 0, as the codes then do
    for (int slot = r; slot < begin; slot += 16) {
      u32x2 w = *reinterpret_cast<const u32x2*>(codes + slot * kHeadDim + d);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float y[4];
        from_codes<FMT>(w[e], y);
        w[e] = none ? 0 : to_codes<FMT>(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio, limit);
      }
      *reinterpret_cast<u32x2*>(codes + slot * kHeadDim + d) = w;
    }
  }
}

// The same tokens out of the pages, as bf16.
template <int BLOCK, int FMT>
__global__ __launch_bounds__(kThreads) void load_kernel(CacheArgs c, StepArgs t, uint16_t* k, uint16_t* v, int pages_each) {
  const uint32_t x = blockIdx.x >> 1, which = blockIdx.x & 1;
  const int pair = x / uint32_t(pages_each), s = pair / c.n_kv_heads, h = pair - s * c.n_kv_heads;
  const int len = c.lens[pair];
  int row0, n;
  step_tokens(t, s, row0, n);
  if (n == 0 || len <= 0 || !good_length(c, len)) return;
  const int first = len - n, start = max(first, 0);
  const int page_in_row = start / BLOCK + int(x - uint32_t(pair) * pages_each), at = page_in_row * BLOCK;
  if (at >= len) return;
  int page = c.table[int64_t(pair) * c.max_pages + page_in_row];
  const bool bad = page < 0 || page >= c.n_pages;
  page = bad ? 0 : page;
  const int begin = max(start - at, 0), end = min(len - at, BLOCK);
  const uint8_t* codes = (which ? c.v : c.k) + int64_t(page) * (BLOCK * kHeadDim);
  const float scale = bad ? __uint_as_float(kNanBits) : (which ? c.v_scale : c.k_scale)[page];
  uint16_t* dst = (which ? v : k) + (int64_t(row0) + (at - first)) * t.stride_t + h * t.stride_h;
  const int r = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
  constexpr int kEach = BLOCK / 16;
  u32x2 in[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    if (slot >= begin && slot < end) in[u] = *reinterpret_cast<const u32x2*>(codes + slot * kHeadDim + d);
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    if (slot < begin || slot >= end) continue;
    float a[4], b[4];
    from_codes<FMT>(in[u].x, a);
    from_codes<FMT>(in[u].y, b);
    const u32x4 o = {pack_bf16(a[0] * scale, a[1] * scale), pack_bf16(a[2] * scale, a[3] * scale),
                     pack_bf16(b[0] * scale, b[1] * scale), pack_bf16(b[2] * scale, b[3] * scale)};
    *reinterpret_cast<u32x4*>(dst + slot * t.stride_t + d) = o;
  }
}

// Key of a weight in the order of eviction: as unsigned numbers, the heaviest largest; +0 and -0 alike, NaN above all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w), mag = b & 0x7fffffffu;
  if (mag > 0x7f800000u) return 0xffffffffu;
  if (mag == 0) return 0x80000000u;
  return b >> 31 ? ~b : b | 0x80000000u;
}

constexpr int kSelectThreads = 1024, kBins = 2048;

// Which tokens of a head stay.  A workgroup per (sequence, head): the want-th largest key among the tokens that may go, eleven, eleven and
// ten bits at a time by counting, then every wave writes the tokens of its part of the positions, whose places follow from
// counts of keys above the threshold and at it.
__global__ __launch_bounds__(kSelectThreads) void evict_select_kernel(CacheArgs src, const float* weight, const int32_t* keep, int n_sink,
                                                                     int n_recent, CacheArgs dst, float* weight_out, int32_t* kept) {
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t wave_sum[2][16];
  __shared__ uint32_t found[2];
  const int pair = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = src.lens[pair], cap = dst.max_pages << dst.block_log2;
  if (!good_length(src, len)) {
    if (tid == 0) dst.lens[pair] = -1;
    return;
  }
  const int n = int(min(int64_t(min(len, cap)), max(int64_t(keep[pair]), int64_t(n_sink) + n_recent)));
  const int sink = min(n_sink, n), recent = min(n_recent, n - sink);
  const int from = sink, to = len - recent;                     // the tokens that may go
  const float* w = weight + (int64_t(pair) * src.max_pages << src.block_log2);
  if (tid == 0) dst.lens[pair] = n;
  uint32_t want = uint32_t(n - sink - recent);
  uint32_t threshold = 0, ties = 0;                             // keys above it stay, and the first `ties` at it
  if (n == len) {
    ties = 0xffffffffu;
  } else if (want == 0) {
    threshold = 0xffffffffu;
  } else {
    uint32_t mask = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, size = pass == 2 ? 1024 : 2048;
      for (int b = tid; b < kBins; b += kSelectThreads) bins[b] = 0;
      __syncthreads();
      for (int p = from + tid; p < to; p += kSelectThreads) {
        const uint32_t key = weight_key(w[p]);
        if ((key & mask) == threshold) atomicAdd(&bins[(key >> shift) & (size - 1)], 1u);
      }
      __syncthreads();
      // keys in the bins from a thread's two on, counted from the top
      const uint32_t high = bins[kBins - 1 - 2 * tid], low = bins[kBins - 2 - 2 * tid];
      uint32_t sum = high + low;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(int(sum), d);
        if (lane >= d) sum += up;
      }
      if (lane == 63) wave_sum[0][wave] = sum;
      __syncthreads();
      for (int x = 0; x < wave; ++x) sum += wave_sum[0][x];
      const uint32_t before = sum - high - low;
      if (before < want && sum >= want) {                       // one thread
        const bool upper = before + high >= want;
        found[0] = kBins - 1 - 2 * tid - (upper ? 0 : 1);
        found[1] = before + (upper ? 0 : high);
      }
      __syncthreads();
      threshold |= found[0] << shift;
      mask |= uint32_t(size - 1) << shift;
      want -= found[1];
      __syncthreads();
    }
    ties = want;
  }
  // every wave has a run of positions, a multiple of 64 of them
  const int run = ((len + kSelectThreads - 1) / kSelectThreads) * 64, begin = min(wave * run, len), end = min(begin + run, len);
  uint32_t above = 0, equal = 0;
  for (int p = begin + lane; p < end; p += 64) {
    const bool forced = p < from || p >= to;
    const uint32_t key = weight_key(w[p]);
    above += forced || key > threshold;
    equal += !forced && key == threshold;
  }
  if (n == len) {                                               // all of them stay
    above = 0;
    for (int p = begin + lane; p < end; p += 64) above += 1;
    equal = 0;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    above += __shfl_xor(int(above), d);
    equal += __shfl_xor(int(equal), d);
  }
  if (lane == 0) {
    wave_sum[0][wave] = above;
    wave_sum[1][wave] = equal;
  }
  __syncthreads();
  above = equal = 0;
  for (int x = 0; x < wave; ++x) {
    above += wave_sum[0][x];
    equal += wave_sum[1][x];
  }
  int32_t* kept_row = kept + int64_t(pair) * cap;
  float* out_row = weight_out + int64_t(pair) * cap;
  const uint64_t below = (uint64_t(1) << lane) - 1;
  for (int p0 = begin; p0 < end; p0 += 64) {
    const int p = p0 + lane;
    const bool there = p < end, forced = there && (p < from || p >= to || n == len);
    const float value = there ? w[p] : 0.0f;
    const uint32_t key = weight_key(value);
    const uint64_t a = __ballot(forced || (there && key > threshold)), e = __ballot(there && !forced && key == threshold);
    const uint32_t rank = equal + __popcll(e & below);
    if ((a >> lane & 1) || ((e >> lane & 1) && rank < ties)) {
      const uint32_t place = above + __popcll(a & below) + min(rank, ties);
      kept_row[place] = p;
      out_row[place] = value;
    }
    above += __popcll(a);
    equal += __popcll(e);
  }
}

// The codes of the tokens that stay, with the scales of the pages they come to.  A thread has sixteen dims of every 32nd token.
template <int FMT>
__global__ __launch_bounds__(kThreads) void evict_gather_kernel(CacheArgs src, CacheArgs dst, const int32_t* kept) {
  __shared__ uint32_t lds[4];
  const uint32_t x = blockIdx.x >> 1, which = blockIdx.x & 1;
  const int pair = x / uint32_t(dst.max_pages), i = int(x - uint32_t(pair) * dst.max_pages);
  const int n = dst.lens[pair], block = 1 << dst.block_log2, at = i * block;
  if (at >= n) return;
  const int page = dst.table[int64_t(pair) * dst.max_pages + i];
  if (page < 0 || page >= dst.n_pages) return;
  const int32_t* kept_row = kept + ((int64_t(pair) * dst.max_pages + i) << dst.block_log2);
  const uint8_t* from = which ? src.v : src.k;
  const float* from_scale = which ? src.v_scale : src.k_scale;
  uint8_t* to = (which ? dst.v : dst.k) + (int64_t(page) << dst.block_log2) * kHeadDim;
  const int r = threadIdx.x >> 3, d = (threadIdx.x & 7) * 16, end = min(n - at, block);
  u32x4 in[4];
  float scale[4];
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int slot = r + 32 * u;
    in[u] = u32x4{0, 0, 0, 0};
    scale[u] = 0.0f;
    if (slot >= end) continue;
    const int p = kept_row[slot];
    const int from_page = src.table[int64_t(pair) * src.max_pages + (p >> src.block_log2)];
    if (from_page < 0 || from_page >= src.n_pages) {
      top = kNanBits;
      continue;
    }
    scale[u] = from_scale[from_page];
    in[u] = *reinterpret_cast<const u32x4*>(from + ((int64_t(from_page) << src.block_log2) + (p & ((1 << src.block_log2) - 1))) * kHeadDim + d);
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[4];
      from_codes<FMT>(in[u][e], y);
#pragma unroll
      for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(y[j] * scale[u]) & 0x7fffffffu);
    }
  top = workgroup_max(top, lds);
  const uint32_t bits = scale_bits<FMT>(top);
  const float inv = inverse_scale(bits), limit = code_limit<FMT>(bits);
  const bool none = bits >= 0x7f800000u;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int slot = r + 32 * u;
    if (slot >= end) continue;
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[4];
      from_codes<FMT>(in[u][e], y);
      o[e] = none ? 0 : to_codes<FMT>(y[0] * scale[u] * inv, y[1] * scale[u] * inv, y[2] * scale[u] * inv, y[3] * scale[u] * inv, limit);
    }
    *reinterpret_cast<u32x4*>(to + slot * kHeadDim + d) = o;
  }
  if (threadIdx.x == 0) (which ? dst.v_scale : dst.k_scale)[page] = __uint_as_float(bits);
}

}  // namespace

static int32_t launched() { return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP; }

// Pages of a row that a step can touch at most, and the workgroups for all of them (0: more than a grid holds).
static int pages_touched(const CacheArgs& c, const StepArgs& t) {
  const int64_t block = int64_t(1) << c.block_log2, most = (int64_t(t.max_tokens) + block - 2) / block + 1;
  return int(most < c.max_pages ? most : c.max_pages);
}

int32_t launch_cache_append(const CacheArgs& c, const StepArgs& t, const void* k, const void* v, hipStream_t stream) {
  const int each = pages_touched(c, t);
  const int64_t grid = int64_t(c.n_seq) * c.n_kv_heads * each * 2;
  if (grid > INT32_MAX) return SHPLB_E_UNSUPPORTED;
  const auto run = c.block_log2 == 7 ? c.format == SHPLB_CACHE_E4M3 ? append_kernel<128, SHPLB_CACHE_E4M3> : append_kernel<128, SHPLB_CACHE_INT8>
                                     : c.format == SHPLB_CACHE_E4M3 ? append_kernel<64, SHPLB_CACHE_E4M3> : append_kernel<64, SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(c, t, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), each);
  return launched();
}

int32_t launch_cache_load(const CacheArgs& c, const StepArgs& t, void* k, void* v, hipStream_t stream) {
  const int each = pages_touched(c, t);
  const int64_t grid = int64_t(c.n_seq) * c.n_kv_heads * each * 2;
  if (grid > INT32_MAX) return SHPLB_E_UNSUPPORTED;
  const auto run = c.block_log2 == 7 ? c.format == SHPLB_CACHE_E4M3 ? load_kernel<128, SHPLB_CACHE_E4M3> : load_kernel<128, SHPLB_CACHE_INT8>
                                     : c.format == SHPLB_CACHE_E4M3 ? load_kernel<64, SHPLB_CACHE_E4M3> : load_kernel<64, SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(c, t, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), each);
  return launched();
}

int32_t launch_cache_evict(const CacheArgs& src, const float* weight, const int32_t* keep, int32_t n_sink, int32_t n_recent,
                           const CacheArgs& dst, float* weight_out, int32_t* kept, hipStream_t stream) {
  const int64_t pairs = int64_t(src.n_seq) * src.n_kv_heads, grid = pairs * dst.max_pages * 2;
  if (grid > INT32_MAX) return SHPLB_E_UNSUPPORTED;
  evict_select_kernel<<<dim3(uint32_t(pairs)), kSelectThreads, 0, stream>>>(src, weight, keep, n_sink, n_recent, dst, weight_out, kept);
  const auto run = src.format == SHPLB_CACHE_E4M3 ? evict_gather_kernel<SHPLB_CACHE_E4M3> : evict_gather_kernel<SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(src, dst, kept);
  return launched();
}

}  // namespace shplb
