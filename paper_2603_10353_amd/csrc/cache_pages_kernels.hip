// Tokens into the pages of the 8-bit cache and out of them.
//
// All three kernels move bytes: a workgroup takes the keys or the values of one page, a page is one run of 8 or 16 KB.  append
// reads 256 and writes 128 bytes per token and head (twice, for K and V), load the other way round, evict (the gather of the
// tokens that stay) reads and writes 128.  What is read or written once in a step, the 16-bit rows and what is evicted, leaves no
// trace in the caches (32768 x 8 heads written 54 -> 42 us, 65536 x 2 read back 23 -> 17, the gather of an eviction of 131072 x 8
// to a fifth 38 -> 32).
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

// Workgroup: of a sequence's pages that the step touches one, a head, K or V.  A thread has eight dims of every sixteenth token.
// SIDE_BY_SIDE: the heads of the same tokens, which lie side by side in the step's tensors, are neighbours (append, 32768 tokens
// x 8 heads of a fused projection 86 -> 51 us, this and fewer registers).  Neighbours are on different dies, so a head is then
// always on the same two; load, whose heads may have different lengths after an eviction, goes head after head (131072 tokens,
// one head whole, 62 -> 31 us).
struct PageOf {
  int pair, s, h, nth, which;      // nth page that the step touches
};
template <bool SIDE_BY_SIDE>
__device__ __forceinline__ PageOf page_of_block(const CacheArgs& c, int pages_each) {
  const uint32_t x = blockIdx.x >> 1;
  if (!SIDE_BY_SIDE) {
    const int pair = x / uint32_t(pages_each), s = pair / c.n_kv_heads;
    return {pair, s, pair - s * c.n_kv_heads, int(x) - pair * pages_each, int(blockIdx.x & 1)};
  }
  const uint32_t y = x / uint32_t(c.n_kv_heads);
  const int h = x - y * c.n_kv_heads, s = y / uint32_t(pages_each);
  return {s * c.n_kv_heads + h, s, h, int(y) - s * pages_each, int(blockIdx.x & 1)};
}

template <int BLOCK, int FMT>
__global__ __launch_bounds__(kThreads, 6) void append_kernel(CacheArgs c, StepArgs t, const uint16_t* k, const uint16_t* v, int pages_each) {
  __shared__ uint32_t lds[4];
  const PageOf x = page_of_block<true>(c, pages_each);
  const int h = x.h, which = x.which, len = c.lens[x.pair];
  int row0, n;
  step_tokens(t, x.s, row0, n);
  if (n == 0 || len <= 0 || !good_length(c, len)) return;
  const int first = len - n, start = max(first, 0);              // position of row 0, of the first token written
  const int page_in_row = start / BLOCK + x.nth, at = page_in_row * BLOCK;
  if (at >= len) return;
  const int page = c.table[int64_t(x.pair) * c.max_pages + page_in_row];
  const int begin = max(start - at, 0), end = min(len - at, BLOCK);   // slots written
  const uint16_t* src = (which ? v : k) + (int64_t(row0) + (at - first)) * t.stride_t + h * t.stride_h;   // of slot 0
  const int r = threadIdx.x >> 4, d = (threadIdx.x & 15) * 8;
  constexpr int kEach = BLOCK / 16;
  u32x4 in[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    in[u] = u32x4{0, 0, 0, 0};
    if (slot >= begin && slot < end) in[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + slot * t.stride_t + d));
  }
  if (page < 0 || page >= c.n_pages) return;
  uint8_t* codes = (which ? c.v : c.k) + int64_t(page) * (BLOCK * kHeadDim);
  float* scale = (which ? c.v_scale : c.k_scale) + page;
  uint32_t before = begin > 0 ? __float_as_uint(*scale) : 0u;
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < kEach; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(in[u][e] << 16 & 0x7fff0000u, in[u][e] & 0x7fff0000u));
  asm volatile("" : "+v"(before));                              // here by now: thread 0 may write it behind the barrier
  top = workgroup_max(top, lds);
  const uint32_t bits = begin > 0 ? larger_scale(before, scale_bits<FMT>(top)) : scale_bits<FMT>(top);
  const float inv = inverse_scale(bits);
  const bool last = last_scale<FMT>(bits);
  const bool none = bits >= 0x7f800000u;                        // codes of a page without a scale are zeros
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const int slot = r + 16 * u;
    if (slot >= begin && slot < end) {
      const u32x4 w = none ? u32x4{0, 0, 0, 0} : in[u];
      u32x2 o;
      o.x = to_codes<FMT>(low_bf16(w.x), high_bf16(w.x), low_bf16(w.y), high_bf16(w.y), inv, last);
      o.y = to_codes<FMT>(low_bf16(w.z), high_bf16(w.z), low_bf16(w.w), high_bf16(w.w), inv, last);
      *reinterpret_cast<u32x2*>(codes + slot * kHeadDim + d) = o;
    }
  }
  if (threadIdx.x == 0 && (begin == 0 || bits != before)) *scale = __uint_as_float(bits);
  // the older tokens, where the scale has grown
  if (begin > 0 && bits != before) {
    const float ratio = __uint_as_float(before) * inv;          // a power of two below 1; it may underflow to 0, as the codes then do
#pragma unroll 1
    for (int slot = r; slot < begin; slot += 16) {
      u32x2 w = *reinterpret_cast<const u32x2*>(codes + slot * kHeadDim + d);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float y[4];
        from_codes<FMT>(w[e], y);
        w[e] = none ? 0 : to_codes<FMT>(y[0], y[1], y[2], y[3], ratio, last);
      }
      *reinterpret_cast<u32x2*>(codes + slot * kHeadDim + d) = w;
    }
  }
}

// The same tokens out of the pages, as bf16.
template <int BLOCK, int FMT>
__global__ __launch_bounds__(kThreads) void load_kernel(CacheArgs c, StepArgs t, uint16_t* k, uint16_t* v, int pages_each) {
  const PageOf x = page_of_block<false>(c, pages_each);
  const int h = x.h, which = x.which, len = c.lens[x.pair];
  int row0, n;
  step_tokens(t, x.s, row0, n);
  if (n == 0 || len <= 0 || !good_length(c, len)) return;
  const int first = len - n, start = max(first, 0);
  const int page_in_row = start / BLOCK + x.nth, at = page_in_row * BLOCK;
  if (at >= len) return;
  int page = c.table[int64_t(x.pair) * c.max_pages + page_in_row];
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
    __builtin_nontemporal_store(o, reinterpret_cast<u32x4*>(dst + slot * t.stride_t + d));
  }
}

// Key of a weight in the order of eviction: as unsigned numbers, the heaviest largest; +0 and -0 alike, NaN above all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t b = __float_as_uint(w), mag = b & 0x7fffffffu;
  if (mag > 0x7f800000u) return 0xffffffffu;
  if (mag == 0) return 0x80000000u;
  return b >> 31 ? ~b : b | 0x80000000u;
}

// Which tokens of a head stay: the want-th largest key among the tokens that may go is found eleven, eleven and ten bits at a
// time by counting keys in bins; the tokens' places follow from how many keys in front of them lie above it or at it.
//
// Of caches of up to 2 kRun positions a head is one workgroup's, from the first count to the last token written.  Longer heads
// are cut into parts of up to kRun positions, and counting, counting, counting and writing are launches of their own: each begins
// by adding up what the parts of its head counted in the launch before.  (8 heads of 13269 tokens: 15 us by one workgroup each,
// 25 and what lies between launches in two parts; of 32525 53, with more weights than registers, and 26 in four; of 131072 28.)
constexpr int kBins = 2048, kEach = 8;                           // bins of a count, weights that a thread holds (of one workgroup's heads up to kMostEach)
constexpr int kSelectThreads = 1024, kFewThreads = 256, kMostEach = 16, kRun = kSelectThreads * kEach;
static_assert((int64_t(SHPLB_MAX_BLOCKS) * 128 + kRun - 1) / kRun * SHPLB_MAX_SEQ_HEADS * kSelectThreads <= int64_t(UINT32_MAX), "a grid for all parts");

struct SelectArgs {
  CacheArgs src, dst;
  const float* weight;
  const int32_t* keep;
  int32_t n_sink, n_recent, parts;
  float* weight_out;
  int32_t* kept;
  uint32_t* bins;                  // workspace: [pairs][parts][3][kBins]
  uint32_t* found;                 // workspace: [pairs][parts][4]: threshold so far, keys still wanted at it, keys above it in the parts in front
};

// What eviction does to a head.
struct Plan {
  int len, n, from, to;            // tokens held and kept, those that may go
  uint32_t want;                   // how many of those stay
  bool good;
};
__device__ __forceinline__ Plan plan_of(const SelectArgs& a, int pair) {
  Plan p;
  p.len = a.src.lens[pair];
  p.good = good_length(a.src, p.len);
  if (!p.good) p.len = 0;
  const int cap = a.dst.max_pages << a.dst.block_log2;
  p.n = int(min(int64_t(min(p.len, cap)), max(int64_t(a.keep[pair]), int64_t(a.n_sink) + a.n_recent)));
  const int sink = min(a.n_sink, p.n), recent = min(a.n_recent, p.n - sink);
  p.from = sink;
  p.to = p.len - recent;
  p.want = uint32_t(p.n - sink - recent);
  return p;
}

struct SelectLds {
  alignas(16) uint32_t bins[kBins];
  int sums[2][kSelectThreads / 64];
  uint32_t picked[4];
};

// Of sums that every wave has left in LDS, those of the waves in front of one's own, added up.
__device__ __forceinline__ int waves_in_front(const int (&sums)[kSelectThreads / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  return __builtin_amdgcn_readlane(lane_sums(lane < wave ? sums[lane] : 0), 63);
}

__device__ __forceinline__ int pass_shift(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t pass_mask(int pass) { return pass == 0 ? 0u : pass == 1 ? 0xffe00000u : 0xfffffc00u; }

// Counts the keys that agree with the threshold in the bits settled so far, by the next bits.  A thread's keys are those of positions
// p + 64 i, of which those in [first, last) count.
template <int THREADS, int EACH>
__device__ __forceinline__ void count_keys(const float (&x)[EACH], int p, int first, int last, int pass, uint32_t threshold, SelectLds& lds) {
  for (int b = threadIdx.x; b < kBins / 4; b += THREADS) reinterpret_cast<u32x4*>(lds.bins)[b] = u32x4{0, 0, 0, 0};
  __syncthreads();
  const uint32_t mask = pass_mask(pass), low = pass == 2 ? 1023 : 2047;
  const int shift = pass_shift(pass);
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const uint32_t key = weight_key(x[i]);
    if (p + 64 * i >= first && p + 64 * i < last && (key & mask) == threshold) atomicAdd(&lds.bins[(key >> shift) & low], 1u);
  }
  __syncthreads();
}

// Finds the bin of the want-th key from the top: `all` are the keys of all parts in the thread's bins, `front` those of the parts in front.
// Writes the bin, how many keys lie above it, how many of those in the parts in front, and how many of these at it.
template <bool FRONT, int PER>
__device__ __forceinline__ void pick_bin(const uint32_t (&all)[PER], const uint32_t (&front)[PER], uint32_t want, SelectLds& lds) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine = 0, mine_front = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    mine += all[i];
    mine_front += front[i];
  }
  int sum = lane_sums(mine), sum_front = FRONT ? lane_sums(mine_front) : 0;
  if (lane == 63) {
    lds.sums[0][wave] = sum;
    if (FRONT) lds.sums[1][wave] = sum_front;
  }
  __syncthreads();
  sum += waves_in_front(lds.sums[0]);
  if (FRONT) sum_front += waves_in_front(lds.sums[1]);
  uint32_t above = sum - mine, above_front = sum_front - mine_front;
  if (above < want && uint32_t(sum) >= want) {                   // one thread; its bins from the top
    bool search = true;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (search && above + all[i] >= want) {
        lds.picked[0] = kBins - 1 - (PER * tid + i);
        lds.picked[1] = above;
        lds.picked[2] = above_front;
        lds.picked[3] = front[i];
        search = false;
      }
      above += all[i];
      above_front += front[i];
    }
  }
  __syncthreads();
}

// STAGE 0, 1, 2 count, 3 writes; -1: all of it.
template <int STAGE, int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(SelectArgs a) {
  constexpr bool kAll = STAGE < 0;
  constexpr int kPer = kBins / THREADS;
  __shared__ SelectLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int parts = kAll ? 1 : a.parts, pair = blockIdx.x / uint32_t(parts), part = blockIdx.x - pair * parts;
  const Plan plan = plan_of(a, pair);
  if ((kAll || STAGE == 3) && part == 0 && tid == 0) a.dst.lens[pair] = plan.good ? plan.n : -1;
  const int len = plan.len;
  const bool all = plan.n == len, counted = !all && plan.want > 0;
  if (len == 0 || (!kAll && STAGE < 3 && !counted)) return;
  const int per = (len + parts * 64 - 1) / (parts * 64) * 64, begin = min(part * per, len), end = min(begin + per, len);
  const float* w = a.weight + (int64_t(pair) * a.src.max_pages << a.src.block_log2);
  // every wave has a run of positions, all of whose weights it keeps in registers
  const int run = (end - begin + THREADS - 1) / THREADS * 64, run_begin = min(begin + wave * run, end), run_end = min(run_begin + run, end);
  const int first = plan.from, last = min(run_end, plan.to), mine = run_begin + lane;
  float x[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) x[i] = mine + 64 * i < run_end ? w[mine + 64 * i] : 0.0f;
  uint32_t* bins = kAll ? nullptr : a.bins + int64_t(blockIdx.x) * 3 * kBins;
  uint32_t* found = kAll ? nullptr : a.found + int64_t(blockIdx.x) * 4;

  uint32_t threshold = all ? 0u : 0xffffffffu, ties = 0, above_front = 0, equal_front = 0;
  if (counted) {
    threshold = 0;
    uint32_t want = plan.want;
    if (!kAll && STAGE > 1) {
      threshold = found[0];
      want = found[1];
      above_front = found[2];
    }
#pragma unroll
    for (int pass = kAll ? 0 : max(STAGE - 1, 0); pass < (kAll ? 3 : STAGE); ++pass) {
      uint32_t n[kPer] = {}, front[kPer] = {};
      if (kAll) {
        count_keys<THREADS, EACH>(x, mine, first, last, pass, threshold, lds);
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
          const u32x2 two = *reinterpret_cast<const u32x2*>(lds.bins + (kBins - kPer - kPer * tid) + (kPer - 2 - i));
          n[i] = two.y;
          n[i + 1] = two.x;
        }
      } else {
        static_assert(kAll || kPer == 2, "eight bytes of each part");
        const uint32_t* from = a.bins + (int64_t(pair) * parts * 3 + pass) * kBins + (kBins - kPer - kPer * tid);
        for (int p0 = 0; p0 < parts; p0 += 32) {                 // all of them in flight
          u32x2 y[32];
#pragma unroll
          for (int p = 0; p < 32; ++p) y[p] = p0 + p < parts ? *reinterpret_cast<const u32x2*>(from + int64_t(p0 + p) * 3 * kBins) : u32x2{0, 0};
#pragma unroll
          for (int p = 0; p < 32; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              n[i] += y[p][1 - i];
              front[i] += p0 + p < part ? y[p][1 - i] : 0;
            }
        }
      }
      pick_bin<!kAll>(n, front, want, lds);
      threshold |= lds.picked[0] << pass_shift(pass);
      want -= lds.picked[1];
      above_front += lds.picked[2];
      equal_front = lds.picked[3];
    }
    ties = want;
    if (!kAll && STAGE < 3) {
      count_keys<THREADS, EACH>(x, mine, first, last, STAGE, threshold, lds);
      for (int b = tid; b < kBins / 4; b += THREADS) reinterpret_cast<u32x4*>(bins + STAGE * kBins)[b] = reinterpret_cast<const u32x4*>(lds.bins)[b];
      if (tid == 0 && STAGE > 0) {
        found[0] = threshold;
        found[1] = want;
        found[2] = above_front;
      }
      return;
    }
  }
  // tokens that stay in any case count as above; those of the parts in front of this one are known
  uint32_t above = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = mine + 64 * i;
    const uint32_t key = weight_key(x[i]);
    const bool there = p < run_end, forced = all || p < plan.from || p >= plan.to;
    above += there && (forced || key > threshold);
    equal += there && !forced && key == threshold;
  }
  // (a wave has up to 64 EACH of both)
  static_assert(64 * EACH < 0x10000, "both in 32 bits");
  const int both = lane_sums(int(equal << 16 | above));
  if (lane == 63) {
    lds.sums[0][wave] = both & 0xffff;
    lds.sums[1][wave] = int(uint32_t(both) >> 16);
  }
  __syncthreads();
  above = above_front + (all ? begin : min(begin, plan.from) + max(begin - plan.to, 0)) + waves_in_front(lds.sums[0]);
  equal = equal_front + waves_in_front(lds.sums[1]);
  const int64_t row = int64_t(pair) * a.dst.max_pages << a.dst.block_log2;
  const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int p = mine + 64 * i;
    const uint32_t key = weight_key(x[i]);
    if (run_begin + 64 * i >= run_end) break;
    const bool there = p < run_end, forced = there && (all || p < plan.from || p >= plan.to);
    const uint64_t over = __ballot(forced || (there && key > threshold)), at = __ballot(there && !forced && key == threshold);
    const uint32_t rank = equal + __popcll(at & below);
    if ((over >> lane & 1) || ((at >> lane & 1) && rank < ties)) {
      const uint32_t place = above + __popcll(over & below) + min(rank, ties);
      a.kept[row + place] = p;
      a.weight_out[row + place] = x[i];
    }
    above += __popcll(over);
    equal += __popcll(at);
  }
}

// The codes of the tokens that stay, with the scales of the pages they come to.  A thread has sixteen dims of every 32nd token.
template <int FMT>
__global__ __launch_bounds__(kThreads) void evict_gather_kernel(CacheArgs src, CacheArgs dst, const int32_t* kept) {
  __shared__ uint32_t lds[4];
  const uint32_t x = blockIdx.x >> 1, which = blockIdx.x & 1;
  const int pair = x / uint32_t(dst.max_pages), i = int(x - uint32_t(pair) * dst.max_pages);
  // what does not wait for anything else is asked for together; places behind the last token hold anything
  const int block = 1 << dst.block_log2, at = i * block, r = threadIdx.x >> 3, d = (threadIdx.x & 7) * 16;
  const int32_t* kept_row = kept + ((int64_t(pair) * dst.max_pages + i) << dst.block_log2);
  int p[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) p[u] = r + 32 * u < block ? kept_row[r + 32 * u] : 0;
  const int n = dst.lens[pair], page = dst.table[int64_t(pair) * dst.max_pages + i];
  if (at >= n || page < 0 || page >= dst.n_pages) return;
  const uint8_t* from = which ? src.v : src.k;
  const float* from_scale = which ? src.v_scale : src.k_scale;
  uint8_t* to = (which ? dst.v : dst.k) + (int64_t(page) << dst.block_log2) * kHeadDim;
  const int end = min(n - at, block);
  u32x4 in[4];
  float scale[4];
  int from_page[4];
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    from_page[u] = r + 32 * u < end ? src.table[int64_t(pair) * src.max_pages + (p[u] >> src.block_log2)] : -1;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    in[u] = u32x4{0, 0, 0, 0};
    scale[u] = 0.0f;
    if (from_page[u] >= 0 && from_page[u] < src.n_pages) {
      scale[u] = from_scale[from_page[u]];
      in[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(from + ((int64_t(from_page[u]) << src.block_log2) + (p[u] & ((1 << src.block_log2) - 1))) * kHeadDim + d));
    } else if (r + 32 * u < end) {
      top = kNanBits;
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) top = max(top, __float_as_uint(largest_code<FMT>(in[u]) * scale[u]) & 0x7fffffffu);
  top = workgroup_max(top, lds);
  const uint32_t bits = scale_bits<FMT>(top);
  const float inv = inverse_scale(bits);
  const bool last = last_scale<FMT>(bits);
  const bool none = bits >= 0x7f800000u;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int slot = r + 32 * u;
    if (slot >= end) continue;
    // A token of zeros may come from a scale 2^128 times the new one, or more: an infinite ratio would make NaN of it.  (Codes other
    // than zero come from at most 448 * 2^9 times the new scale.)
    const float ratio = fminf(scale[u] * inv, 0x1p127f);
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float y[4];
      from_codes<FMT>(in[u][e], y);
      o[e] = none ? 0 : to_codes<FMT>(y[0], y[1], y[2], y[3], ratio, last);
    }
    *reinterpret_cast<u32x4*>(to + slot * kHeadDim + d) = o;
  }
  if (threadIdx.x == 0) (which ? dst.v_scale : dst.k_scale)[page] = __uint_as_float(bits);
}

}  // namespace

static int32_t launched() { return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP; }

// Whether a grid holds so many workgroups: its threads are counted in 32 bits.  (Those of 1024 that select are at most 65535 heads
// x 64 parts.)
static bool grid_holds(int64_t workgroups) { return workgroups * kThreads <= int64_t(UINT32_MAX); }

// Pages of a row that a step can touch at most.
static int pages_touched(const CacheArgs& c, const StepArgs& t) {
  const int64_t block = int64_t(1) << c.block_log2, most = (int64_t(t.max_tokens) + block - 2) / block + 1;
  return int(most < c.max_pages ? most : c.max_pages);
}

int32_t launch_cache_append(const CacheArgs& c, const StepArgs& t, const void* k, const void* v, hipStream_t stream) {
  const int each = pages_touched(c, t);
  const int64_t grid = int64_t(c.n_seq) * c.n_kv_heads * each * 2;
  if (!grid_holds(grid)) return SHPLB_E_UNSUPPORTED;
  const auto run = c.block_log2 == 7 ? c.format == SHPLB_CACHE_E4M3 ? append_kernel<128, SHPLB_CACHE_E4M3> : append_kernel<128, SHPLB_CACHE_INT8>
                                     : c.format == SHPLB_CACHE_E4M3 ? append_kernel<64, SHPLB_CACHE_E4M3> : append_kernel<64, SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(c, t, static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), each);
  return launched();
}

int32_t launch_cache_load(const CacheArgs& c, const StepArgs& t, void* k, void* v, hipStream_t stream) {
  const int each = pages_touched(c, t);
  const int64_t grid = int64_t(c.n_seq) * c.n_kv_heads * each * 2;
  if (!grid_holds(grid)) return SHPLB_E_UNSUPPORTED;
  const auto run = c.block_log2 == 7 ? c.format == SHPLB_CACHE_E4M3 ? load_kernel<128, SHPLB_CACHE_E4M3> : load_kernel<128, SHPLB_CACHE_INT8>
                                     : c.format == SHPLB_CACHE_E4M3 ? load_kernel<64, SHPLB_CACHE_E4M3> : load_kernel<64, SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(c, t, static_cast<uint16_t*>(k), static_cast<uint16_t*>(v), each);
  return launched();
}

static int evict_parts(const CacheArgs& c) {
  const int64_t capacity = int64_t(c.max_pages) << c.block_log2;
  return capacity <= kSelectThreads * kMostEach ? 1 : int((capacity + kRun - 1) / kRun);
}
int64_t cache_evict_workspace(const CacheArgs& c) {
  const int64_t parts = evict_parts(c);
  return parts == 1 ? 256 : (int64_t(c.n_seq) * c.n_kv_heads * parts * (3 * kBins + 4) * 4 + 255) & ~int64_t(255);
}

int32_t launch_cache_evict(const CacheArgs& src, const float* weight, const int32_t* keep, int32_t n_sink, int32_t n_recent,
                           const CacheArgs& dst, float* weight_out, int32_t* kept, void* workspace, hipStream_t stream) {
  const int parts = evict_parts(src);
  const int64_t pairs = int64_t(src.n_seq) * src.n_kv_heads, grid = pairs * dst.max_pages * 2;    // (the entry point sees to it that a grid holds them)
  uint32_t* bins = static_cast<uint32_t*>(workspace);
  const SelectArgs a{src, dst, weight, keep, n_sink, n_recent, parts, weight_out, kept, bins, bins + pairs * parts * 3 * kBins};
  const dim3 all(uint32_t(pairs * parts));
  if (parts == 1) {
    // as few threads and weights of each as there can be (48 sequences x 4 heads of up to 2000 tokens: 7.8 us with 1024 threads,
    // 7.3 with 256)
    const int64_t capacity = int64_t(src.max_pages) << src.block_log2;
    if (capacity <= kFewThreads * kEach) evict_select_kernel<-1, kFewThreads, kEach><<<all, kFewThreads, 0, stream>>>(a);
    else if (capacity <= kRun) evict_select_kernel<-1, kSelectThreads, kEach><<<all, kSelectThreads, 0, stream>>>(a);
    else evict_select_kernel<-1, kSelectThreads, kMostEach><<<all, kSelectThreads, 0, stream>>>(a);
  } else {
    evict_select_kernel<0, kSelectThreads, kEach><<<all, kSelectThreads, 0, stream>>>(a);
    evict_select_kernel<1, kSelectThreads, kEach><<<all, kSelectThreads, 0, stream>>>(a);
    evict_select_kernel<2, kSelectThreads, kEach><<<all, kSelectThreads, 0, stream>>>(a);
    evict_select_kernel<3, kSelectThreads, kEach><<<all, kSelectThreads, 0, stream>>>(a);
  }
  const auto run = src.format == SHPLB_CACHE_E4M3 ? evict_gather_kernel<SHPLB_CACHE_E4M3> : evict_gather_kernel<SHPLB_CACHE_INT8>;
  run<<<dim3(uint32_t(grid)), kThreads, 0, stream>>>(src, dst, kept);
  return launched();
}

}  // namespace shplb
