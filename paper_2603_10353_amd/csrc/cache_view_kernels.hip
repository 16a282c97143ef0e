// Attention over the 8-bit cache that sees part of it, or more than it: windows with first tokens that stay visible, and prefixes that
// sequences share.  The kernels that attend are in cache_attn.h; here are their launches, and the join of what a row has from its
// prefix and from its own tokens.
#include "cache_attn.h"

namespace shplb {
namespace {

// ---- windows.  A step's work does not grow with the context: a head has the units of its window and of its first tokens, and how the
// work is divided follows from them like that of cache_attn_kernel.hip from a table's room.
template <int FMT>
int32_t launch_window(const CacheAttnArgs& a, int rows, int most_rows, int compute_units, hipStream_t stream) {
  const int grid = min(kCacheMaxWorkers / kWaves, compute_units * 2), pairs = a.c.n_seq * a.c.n_kv_heads;
  const int64_t most = min(int64_t(a.c.max_pages) << a.c.block_log2, int64_t(a.view.most_units) * kUnit);
  constexpr int kShort = kWholeWaves * kWholeUnits * kUnit;
  if (rows == 16 && pairs <= 2 * compute_units && most <= kShort) {
    cache_whole_kernel<false, FMT, kWindow><<<pairs, 64 * kWholeWaves, 0, stream>>>(a);
  } else if (rows > 16 && (most <= kShort || (most <= 2 * kShort && int64_t(pairs) * a.tiles >= 2 * compute_units))) {
    cache_attn_kernel<2, kWaves, true, FMT, kWindow><<<uint32_t(pairs) * a.tiles, kThreads, 0, stream>>>(a, 0);
  } else {
    if (rows == 16) cache_attn_kernel<1, 1, false, FMT, kWindow><<<grid, kThreads, 0, stream>>>(a, 3);
    else cache_attn_kernel<2, kWaves, false, FMT, kWindow><<<grid, kThreads, 0, stream>>>(a, kWaves);
    launch_join(a, rows, most_rows, stream);
  }
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

// ---- shared prefixes.  The rows of all sequences that share a prefix are rows of one item: its keys are read once for 32 of
// them (16 where there are no more).  A second launch attends to the sequences' own tokens; both leave partial results.
template <int FMT>
void launch_prefix(const CacheAttnArgs& a, int grid, int rows, hipStream_t stream) {
  if (rows == 16) cache_attn_kernel<1, 1, false, FMT, kGroups, true><<<grid, kThreads, 0, stream>>>(a, 3);
  else cache_attn_kernel<2, kWaves, false, FMT, kGroups, true><<<grid, kThreads, 0, stream>>>(a, kWaves);
}
template <int FMT>
void launch_own(const CacheAttnArgs& a, int grid, int rows, hipStream_t stream) {
  if (rows == 16) cache_attn_kernel<1, 1, false, FMT, kAll, true><<<grid, kThreads, 0, stream>>>(a, 3);
  else cache_attn_kernel<2, kWaves, false, FMT, kAll, true><<<grid, kThreads, 0, stream>>>(a, kWaves);
}

// Joins a row's pieces, those of its prefix and those of its own tokens: with M the largest m, out = sum 2^(m - M) O / sum 2^(m -
// M) l.  A wave a row; its halves take turns at the pieces, a lane four dims.
__global__ __launch_bounds__(kThreads) void shared_join_kernel(CacheAttnArgs a, CacheAttnArgs pre, int rows_own, int rows_pre) {
  const int lane = threadIdx.x & 63, d4 = lane & 31, half = lane >> 5;
  const int pair = blockIdx.x / uint32_t(a.tiles), tile = blockIdx.x - pair * a.tiles;
  const int in_tile = int(blockIdx.y) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = tile * rows_own + in_tile;
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, group = group_size(a.groups, h);
  int row0, n;
  step_tokens<true>(a.t, s, row0, n);
  if (in_tile >= rows_own || row >= n * group) return;
  const int j = row / group, i = row - j * group, head = group_head(a.groups, h, i), len = scalar_load(a.c.lens + pair);
  const int2 own = *reinterpret_cast<const int2*>(a.begun + 2 * int64_t(blockIdx.x));
  // the prefix: the first one whose run of sequences holds this one
  int g = -1;
  for (int g0 = 0; g0 < pre.c.n_seq && g < 0; g0 += 64) {
    const int at = min(g0 + lane, pre.c.n_seq - 1);
    const uint64_t here = __ballot(g0 + lane < pre.c.n_seq && pre.view.groups[at] <= s && s < pre.view.groups[at + 1]);
    if (here) g = g0 + int(__builtin_ctzll(here));
  }
  int2 front = {0, 0};
  int front_row = 0, prefix_len = 0;
  bool good = good_length(a.c, len);
  if (g >= 0) {
    int first, tokens;
    view_tokens<kGroups, true>(pre, g, first, tokens);
    prefix_len = scalar_load(pre.c.lens + int64_t(g) * pre.c.n_kv_heads + h);
    const int t = row0 + j - first;
    good = good && good_length(pre.c, prefix_len) && t >= 0 && t < tokens;      // (offsets that go backwards: rows outside of their prefix's)
    if (good) {
      const int at = t * group + i, tile_row = at / rows_pre * rows_pre;
      front = *reinterpret_cast<const int2*>(pre.begun + 2 * begun_row(pre, first, tile_row, h, group));
      front_row = at - tile_row;
    }
  }
  // what was whole lies by rows, the pieces of the others in their shares' slots
  const int64_t by_row = begun_row(a, row0, row, h, group);
  const int n_own = good ? max(own.y, 1) : 0, pieces = n_own + (good && g >= 0 ? max(front.y, 1) : 0);
  const auto stats = [&](int x) {
    const int y = x - n_own;
    const float* at = y < 0 ? (own.y == 0 ? a.view.whole_ml + 2 * by_row : a.part_ml + 2 * ((2 * int64_t(own.x + x) + (x == 0)) * rows_own + in_tile))
                            : (front.y == 0 ? pre.view.whole_ml + 2 * by_row : pre.part_ml + 2 * ((2 * int64_t(front.x + y) + (y == 0)) * rows_pre + front_row));
    return *reinterpret_cast<const f32x2*>(at);
  };
  const auto values = [&](int x) {
    const int y = x - n_own;
    const float* at = y < 0 ? (own.y == 0 ? a.view.whole_o + by_row * kHeadDim : a.part_o + ((2 * int64_t(own.x + x) + (x == 0)) * rows_own + in_tile) * kHeadDim)
                            : (front.y == 0 ? pre.view.whole_o + by_row * kHeadDim : pre.part_o + ((2 * int64_t(front.x + y) + (y == 0)) * rows_pre + front_row) * kHeadDim);
    return *reinterpret_cast<const f32x4*>(at + d4 * 4);
  };
  constexpr int kEarly = 4;
  f32x4 early[kEarly];
  float early_m[kEarly];
#pragma unroll
  for (int x = 0; x < kEarly; ++x) {
    early[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    early_m[x] = -INFINITY;
    if (half + 2 * x < pieces) {
      early[x] = values(half + 2 * x);
      early_m[x] = stats(half + 2 * x).x;
    }
  }
  f32x2 mine = {-INFINITY, 0.0f};
  if (lane < pieces) mine = stats(lane);
  float top = mine.x;
  for (int x = lane + 64; x < pieces; x += 64) top = fmaxf(top, stats(x).x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = __builtin_amdgcn_exp2f(mine.x - ref) * mine.y;
  for (int x = lane + 64; x < pieces; x += 64) sum += __builtin_amdgcn_exp2f(stats(x).x - ref) * stats(x).y;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < kEarly; ++x)
    if (half + 2 * x < pieces) o += __builtin_amdgcn_exp2f(early_m[x] - ref) * early[x];
#pragma unroll 8
  for (int x = half + 2 * kEarly; x < pieces; x += 2) o += __builtin_amdgcn_exp2f(stats(x).x - ref) * values(x);
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
  if (half) return;
  const float inv = row_inverse(good, max(len - n + 1 + j, 0) + prefix_len, sum);
  *reinterpret_cast<u32x2*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d4 * 4) =
      u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
  if (lane == 0 && a.lse != nullptr) a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = row_lse(top, sum, inv);
}

}  // namespace

int32_t launch_cache_attn_window(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream) {
  const int rows = cache_attn_rows(most_rows);
  return a.c.format == SHPLB_CACHE_E4M3 ? launch_window<SHPLB_CACHE_E4M3>(a, rows, most_rows, compute_units, stream)
                                        : launch_window<SHPLB_CACHE_INT8>(a, rows, most_rows, compute_units, stream);
}

int32_t prefix_attn_rows(int64_t rows) { return rows <= 16 ? 16 : 32; }
int64_t prefix_slot_rows(int32_t) { return kCacheSlotRows; }

int32_t launch_cache_attn_shared(const CacheAttnArgs& own, const CacheAttnArgs& pre, int32_t most_rows, int32_t rows_pre, int32_t compute_units, hipStream_t stream) {
  const int grid = min(kCacheMaxWorkers / kWaves, compute_units * 2), rows = cache_attn_rows(most_rows);
  if (pre.c.format == SHPLB_CACHE_E4M3) launch_prefix<SHPLB_CACHE_E4M3>(pre, grid, rows_pre, stream);
  else launch_prefix<SHPLB_CACHE_INT8>(pre, grid, rows_pre, stream);
  if (own.c.format == SHPLB_CACHE_E4M3) launch_own<SHPLB_CACHE_E4M3>(own, grid, rows, stream);
  else launch_own<SHPLB_CACHE_INT8>(own, grid, rows, stream);
  const dim3 all(uint32_t(own.c.n_seq * own.c.n_kv_heads) * own.tiles, (min(rows, most_rows) + kWaves - 1) / kWaves);
  shared_join_kernel<<<all, kThreads, 0, stream>>>(own, pre, rows, rows_pre);
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace shplb
