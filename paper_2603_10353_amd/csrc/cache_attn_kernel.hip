// Attention over the 8-bit cache, every token of it: the weights that tokens are given, and the launches.  The kernels that attend are in
// cache_attn.h.
#include "cache_attn.h"

namespace shplb {
namespace {

// What rows need of their attention to say which weights they gave.
template <int NT>
struct Statistics {
  float to_log2[NT], m[NT], inv[NT];           // inv: 1 / denominator
  int seen[NT];
};

// The probabilities that the rows, of which there is one at least, put on each key of a unit, added up: a lane is left with those
// of key key_of_lane() of the unit.  (A key whose product is NaN is one that a row sees, or masked: rows that are not there add
// nothing to others.)  The keys of the next one are asked for on the way.
template <int NT, int FMT>
__device__ __forceinline__ float weigh_unit(const CacheAttnArgs& a, int key0, const Page& ahead, bool more, int seen_first,
                                            const f16x8 (*lds_q)[4][64], int lane, Flight& f, const Statistics<NT>& r) {
  const int g = lane >> 4;
  const float k_scale = f.here.bad ? __uint_as_float(kNanBits) : f.here.k_scale;
  f32x4 sc[NT][4];
  scores<NT, FMT>(f.k, lds_q, lane, sc);
  load_keys<false>(a, ahead, more, (lane & 15) * kHeadDim + g * 16, f.k);
  __builtin_amdgcn_sched_barrier(0);
  f.here = ahead;
  float w[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) w[x] = 0.0f;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    float c = r.to_log2[nt] * k_scale;
    if (key0 + kUnit > seen_first) {
      if (seen_first == kFar) {
        const bool far = c == INFINITY;
        const float first = far ? r.to_log2[nt] : c;
#pragma unroll
        for (int x = 0; x < 4; ++x) sc[nt][x] *= first;
        c = far ? k_scale : 1.0f;
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const float p = __builtin_amdgcn_exp2f(sc[nt][x >> 2][x & 3] * c - r.m[nt]) * r.inv[nt];
        w[x] += key0 + (x >> 2) * 16 + g * 4 + (x & 3) < r.seen[nt] ? p : 0.0f;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x) w[x] += __builtin_amdgcn_exp2f(sc[nt][x >> 2][x & 3] * c - r.m[nt]) * r.inv[nt];
    }
  }
  return sums_of_rows(w, lane);
}

// weight_out = before + those of units first .. end - 1.
template <int FMT>
__device__ __forceinline__ void weigh(const CacheAttnArgs& a, int pair, int len, int first, int end, int last, int seen_first,
                                      const f16x8 (*lds_q)[4][64], const float* before, int lane, Flight& f, const Statistics<1>& r) {
  const int64_t row_of_weights = int64_t(pair) * a.c.max_pages << a.c.block_log2;
  for (int u = first; u < end; ++u) {
    const Page ahead = page_at(a.c, f.page_next, min(u + 1, last));
    f.page_next = page_number(a.c, pair, min(u + 2, last));
    const int key = u * kUnit + key_of_lane(lane);
    float old = 0.0f;
    if (before != nullptr && key < len) old = before[row_of_weights + key];
    const float sum = weigh_unit<1, FMT>(a, u * kUnit, ahead, u + 1 < end, seen_first, lds_q, lane, f, r);
    if (key < len) a.weight_out[row_of_weights + key] = old + sum;
  }
}

// What a wave begins to weigh with: rows first_row on and the unit `first`, if it is below end.  Returns whether there is a far_row().
template <int NT>
__device__ __forceinline__ bool begin_weights(const CacheAttnArgs& a, int pair, int h, int group, int row0, int n, int first_row, int len, int first, int step,
                                              int end, int last, int lane, f16x8 (*lds_q)[4][64], Flight& f, Statistics<NT>& r) {
  const int rows = n * group, page = page_number(a.c, pair, min(first, last));
  f.page_next = page_number(a.c, pair, min(first + step, last));
  Query q[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = first_row + nt * 16 + (lane & 15);
    r.m[nt] = r.inv[nt] = 0.0f;
    r.seen[nt] = 0;
    ask_query(a, row0, n, h, group, row, lane, q[nt]);
    if (row < rows) {
      const int j = row / group, head = group_head(a.groups, h, row - j * group);
      const f32x2 st = *reinterpret_cast<const f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head));
      r.seen[nt] = len - n + 1 + j;
      r.m[nt] = st.x;
      r.inv[nt] = st.y;
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  ask_unit<false>(a, page, min(first, last), first < end ? end : 0, lane, false, f);
  bool far = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    f16x8 operand[4];
    const float to_log2 = query_operands(a, q[nt], operand);
    far |= far_row(to_log2) || far_reference(r.m[nt]);
    r.to_log2[nt] = first_row + nt * 16 + (lane & 15) < rows ? to_log2 : 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) lds_q[nt][e][lane] = operand[e];
  }
  return __ballot(far) != 0;
}

// Weights of keys first .. end - 1 of a head that has no rows in this step: what they were.
__device__ __forceinline__ void copy_weights(const CacheAttnArgs& a, int64_t row_of_weights, int first, int end, int me, int threads) {
  if (a.weight_in == a.weight_out) return;
#pragma unroll 4
  for (int key = first + me; key < end; key += threads) a.weight_out[row_of_weights + key] = a.weight_in != nullptr ? a.weight_in[row_of_weights + key] : 0.0f;
}

// The weights of the step by themselves, taken again from the keys and the rows' statistics: every key belongs to one share, so
// nothing is added up between workgroups.  Up to 16 rows every wave has a share.
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void cache_weight_kernel(CacheAttnArgs a) {
  constexpr int kStart = start_units(1);
  __shared__ f16x8 lds_q[kWaves][1][4][64];
  __shared__ int lds_i[kWaves + kThreads];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int at, end;
  Shares<false> shares;
  Item it = locate<true, 1, kStart>(a, int(blockIdx.x) + wave * int(gridDim.x), int(gridDim.x) * kWaves, 1, 1, lds_i, at, end, shares);
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens<true>(a.t, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h), rows = n * group;
    pair_units<true, 1>(a, rows, len, tiles, units);
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at)), last = max(u1 - 1, 0);
    if (rows == 0) {
      copy_weights(a, int64_t(pair) * a.c.max_pages << a.c.block_log2, u0 * kUnit, min(u1 * kUnit, len), lane, 64);
    } else {
      Flight f;
      Statistics<1> r;
      const bool far = begin_weights<1>(a, pair, h, group, row0, n, 0, len, u0, 1, u1, last, lane, lds_q[wave], f, r);
      weigh<FMT>(a, pair, len, u0, u1, last, far ? kFar : len - n + 1, lds_q[wave], a.weight_in, lane, f, r);
    }
    at += units - it.unit;
    it = next_pair<kStart>(a, pair);
  }
}

// More rows: a workgroup has the share, and its waves 32 rows each, up to 128 at a time.  Where there are fewer, 64 or 32, two or
// all waves take turns at the units.  What the slices of rows put on the keys of kSteps units each meets in LDS.  (128 rows x 8
// heads x 32768 int8 tokens: 30 us with a share for every wave and 64 rows at a time, of which beginning was the half, 26 so;
// VALU work, turning the codes into fp16 for every 32 rows and the exponentials.)
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void cache_weight_rows_kernel(CacheAttnArgs a) {
  constexpr int kStart = start_units(kWaves), kSteps = 8, kSlice = 32;
  __shared__ f16x8 lds_q[kWaves][2][4][64];
  __shared__ float lds_w[kSteps][kWaves][kUnit];
  __shared__ int lds_i[kWaves + kThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int at, end;
  Shares<true> shares;
  Item it = locate<true, 1, kStart>(a, int(blockIdx.x), int(gridDim.x), 1, 1, lds_i, at, end, shares);
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens<true>(a.t, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h), rows = n * group;
    pair_units<true, 1>(a, rows, len, tiles, units);
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at));
    const int64_t row_of_weights = int64_t(pair) * a.c.max_pages << a.c.block_log2;
    if (rows == 0) copy_weights(a, row_of_weights, u0 * kUnit, min(u1 * kUnit, len), tid, kThreads);
    for (int first_row = 0; u0 < u1 && first_row < rows; first_row += kWaves * kSlice) {
      const int left = rows - first_row, log2 = left > 2 * kSlice ? 2 : left > kSlice ? 1 : 0, slices = 1 << log2, step = kWaves >> log2;
      const int phase = wave >> log2, my_row = first_row + (wave & (slices - 1)) * kSlice;
      const int seen_last = my_row < rows ? len - n + 1 + (min(my_row + kSlice, rows) - 1) / group : 0;
      const float* before = first_row == 0 ? a.weight_in : a.weight_out;
      Flight f;
      Statistics<2> r;
      const bool far = begin_weights<2>(a, pair, h, group, row0, n, my_row, len, u0 + phase, step, u1, u1 - 1, lane, lds_q[wave], f, r);
      const int seen_first = far ? kFar : len - n + 1 + my_row / group;
      for (int c = u0; c < u1; c += kSteps * step) {
        // a thread's keys of all these units: kThreads apart
        const int key = c * kUnit + tid, key_end = min(len, min(u1, c + kSteps * step) * kUnit);
        float old[kSteps];
#pragma unroll
        for (int x = 0; x < kSteps; ++x) {
          old[x] = 0.0f;
          if (before != nullptr && key + x * kThreads < key_end) old[x] = before[row_of_weights + key + x * kThreads];
        }
#pragma unroll 1
        for (int i = 0; i < kSteps; ++i) {
          const int u = c + i * step + phase;
          if (u >= u1) break;
          const Page ahead = page_at(a.c, f.page_next, min(u + step, u1 - 1));
          f.page_next = page_number(a.c, pair, min(u + 2 * step, u1 - 1));
          float sum = 0.0f;
          if (u * kUnit < seen_last) sum = weigh_unit<2, FMT>(a, u * kUnit, ahead, u + step < u1, seen_first, lds_q[wave], lane, f, r);
          lds_w[i][wave][key_of_lane(lane)] = sum;
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kSteps; ++x) {
          if (key + x * kThreads >= key_end) break;
          const int nth = (tid + x * kThreads) >> 6, i = nth >> (2 - log2), p = nth & (step - 1);        // of these units; phase p's i-th
          float sum = 0.0f;
          for (int sl = 0; sl < slices; ++sl) sum += lds_w[i][(p << log2) + sl][lane];
          a.weight_out[row_of_weights + key + x * kThreads] = old[x] + sum;
        }
        __syncthreads();
      }
    }
    at += units - it.unit;
    it = next_pair<kStart>(a, pair);
  }
}

template <int FMT>
int32_t launch_format(const CacheAttnArgs& a, int rows, int most_rows, int compute_units, hipStream_t stream) {
  const int grid = min(kCacheMaxWorkers / kWaves, compute_units * 2), pairs = a.c.n_seq * a.c.n_kv_heads;
  const int64_t capacity = int64_t(a.c.max_pages) << a.c.block_log2;
  constexpr int kShort = kWholeWaves * kWholeUnits * kUnit;
  if (rows == 16 && pairs <= 2 * compute_units && capacity <= kShort) {
    // (twice as many heads as compute units: 100 sequences x 4 heads of up to 1492 tokens with weights 18 us, and 13, 4 and 7 by
    // shares; three times: 100 x 8 of up to 719 21, and 14 and 4)
    if (a.weight_out != nullptr) cache_whole_kernel<true, FMT><<<pairs, 64 * kWholeWaves, 0, stream>>>(a);
    else cache_whole_kernel<false, FMT><<<pairs, 64 * kWholeWaves, 0, stream>>>(a);
    return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
  }
  if (a.t.n_tokens > 0 && rows > 16 && (capacity <= kShort || (capacity <= 2 * kShort && int64_t(pairs) * a.tiles >= 2 * compute_units))) {
    // item by item (48 sequences x 8 heads of up to 1498 tokens, 32 rows, 23 us, and 24 and 6 to join by shares; 100 x 8 of up to
    // 615, 160 rows, 46, and 51 and 20; one of 900 x 8 heads, 128 rows, 14, and 11 and 4), also twice as long if there are items
    // for all compute units (100 x 2 of up to 2861, 128 rows, 35, and 34 and 7): one that is much longer than the others keeps a
    // compute unit for 30 us
    cache_attn_kernel<2, kWaves, true, FMT><<<uint32_t(pairs) * a.tiles, kThreads, 0, stream>>>(a, 0);
  } else if (a.t.n_tokens > 0) {
    // (three units at least where there is more than one share for every workgroup: waves that share a compute unit wait for one
    // another's beginnings, and pieces are joined; five sequences of up to 39284 tokens x 2 heads 15 and 9 us with one unit, 13
    // and 5 with three, 12 and 5 with four; 16 up to 8000 13 and 7, 11 and 5, 12 and 4; one of 2048 x 8 heads, 272 units, 7 and 4
    // with one, 10 and 4 with three)
    if (rows == 16) cache_attn_kernel<1, 1, false, FMT><<<grid, kThreads, 0, stream>>>(a, 3);
    else cache_attn_kernel<2, kWaves, false, FMT><<<grid, kThreads, 0, stream>>>(a, kWaves);
    launch_join(a, rows, most_rows, stream);
  }
  if (a.weight_out != nullptr) {
    if (rows == 16) cache_weight_kernel<FMT><<<grid, kThreads, 0, stream>>>(a);
    else cache_weight_rows_kernel<FMT><<<grid, kThreads, 0, stream>>>(a);
  }
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace

int32_t cache_attn_rows(int64_t most_rows) { return most_rows <= 16 ? 16 : 32; }

int32_t launch_cache_attn(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream) {
  const int rows = cache_attn_rows(most_rows);
  return a.c.format == SHPLB_CACHE_E4M3 ? launch_format<SHPLB_CACHE_E4M3>(a, rows, most_rows, compute_units, stream)
                                        : launch_format<SHPLB_CACHE_INT8>(a, rows, most_rows, compute_units, stream);
}

}  // namespace shplb
