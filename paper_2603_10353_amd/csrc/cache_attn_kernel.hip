// Attention of a step's queries over the 8-bit cache (gfx950).
//
// For every query row (a token of the step and a head of the KV head's group) with key codes k_t and value codes v_t of pages with
// scales a, b:
//
//   y_t = (q . k_t) * scale * log2(e) * a,   m = max y,   l = sum 2^(y_t - m),   out = sum 2^(y_t - m) b v_t / l,   lse = (m + log2 l) ln 2,
//
// in one pass over the keys with a running m (rescaling l and the output when it grows).  Bound by reading the codes once: a
// token of a KV head is 256 bytes and, for a group of four heads, 4 KFLOP.  So the matrix instructions are used for what they save in
// registers and lanes, with most of their rows empty in a plain decoding step.
//
// Split.  All heads' keys together are one list of units of 64 keys, of which every workgroup takes an equal, contiguous share
// whatever the heads' lengths are: lengths differ between sequences, and between heads after an eviction.  The lengths are on the
// device (they change while a captured launch stays), so each workgroup adds them up by itself.  A (sequence, KV head, tile of rows)
// whose units lie in several workgroups has partial results (m, l, unnormalised output), which a second kernel joins in order.
//
// Tile.  A wave works on units of its own: keys are the rows of the first product (S^T = K Q^T), so a lane has scores of one query
// and four adjacent keys of each 16; the second one is O^T = V^T P^T, whose operand P^T needs exactly those (the order of the keys
// inside a product is free, as long as V's are taken alike).  Codes come straight from global memory into registers, are turned to fp16
// there (exact in both formats), V's after a byte transposition of key pairs; nothing goes through LDS.
// Q is brought to fp16 by a power of two per row, so that its largest magnitude lies in [2^13, 2^14): exact down to 2^-27 of it.
// Probabilities are rounded to fp16 at 2^15 times their size: eleven bits down to 2^-29 of the largest.  All sums are fp32.
#include "cache_common.h"

namespace shplb {
namespace {

constexpr int kThreads = 256, kWaves = 4, kUnit = 64;
// What beginning with an item costs, in units of the list of all units (where it is that many empty ones in front of the item's own):
// the queries, the first keys, the results, all of them waited for.  For a batch of 128 sequences x 8 heads of lengths between 100 and
// 16000, where a wave has one to five items, 121 us without, 112 with three.
constexpr int kStart = 3;
constexpr float kLift = 15.0f;                 // log2 of what probabilities are multiplied by
constexpr int kLdsRow = kHeadDim + 4;          // floats of a row in LDS: rows four banks apart

struct Item {                                  // a place in the list of units
  int pair, len;                               // the head, and its length
  int tile, unit;                              // tile of rows, unit inside it; from -kStart on, where there are none yet
};
// How the list is divided: the first `more` shares have one unit more than the others.
struct Shares {
  int each, more;
  __device__ int begin(int w) const { return w * each + min(w, more); }
  __device__ int of(int at) const { return at < more * (each + 1) ? at / (each + 1) : more + (at - more * (each + 1)) / each; }
};

__device__ __forceinline__ int group_size(const HeadGroups& g, int h) { return g.mapped ? g.begin[h + 1] - g.begin[h] : g.group; }
__device__ __forceinline__ int group_head(const HeadGroups& g, int h, int x) { return g.mapped ? g.head[g.begin[h] + x] : h * g.group + x; }

// Rows of a pair in this step (query tokens times heads of the group).
template <bool SCALAR>
__device__ __forceinline__ int pair_rows(const CacheAttnArgs& a, int pair) {
  if (a.t.cu == nullptr && !a.groups.mapped) return a.t.max_tokens * a.groups.group;    // the same for all: no division
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
  int row0, n;
  step_tokens<SCALAR>(a.t, s, row0, n);
  return n * group_size(a.groups, h);
}
// Tiles of rows of a pair and units of each.
template <bool WEIGHTS, int ROWS>
__device__ __forceinline__ void pair_units(const CacheAttnArgs& a, int rows, int len, int& tiles, int& units) {
  units = good_length(a.c, len) ? (len + kUnit - 1) / kUnit : 0;
  if (WEIGHTS) {
    tiles = 1;                                 // all rows together, and keys no row looks at are copied
  } else {
    tiles = (rows + ROWS - 1) / ROWS;
    units = max(units, 1);                     // a head without keys has an output, too
  }
}

// Sums over the lanes up to and with one's own.
__device__ __forceinline__ int lane_sums(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);      // from 1, 2, 4, 8 lanes below in the row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);     // the last lane of a row to the next one, of 32 to the others
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// The place where a worker's share [begin, end) of all units begins.  Up to 512 pairs every wave adds them up by itself, a lane a run of
// them; beyond, the four waves do it together, and each looks for its place in the run where it lies, 64 pairs at a time.  (All
// units are below 2^30: the entry point sees to that.)
template <bool WEIGHTS, int ROWS>
__device__ __forceinline__ Item locate(const CacheAttnArgs& a, int worker, int workers, int least, int* lds, int& begin, int& end, Shares& shares) {
  const int pairs = a.c.n_seq * a.c.n_kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool together = pairs > 512;
  const int me = together ? threadIdx.x : lane, each = together ? (pairs + kThreads - 1) / kThreads : (pairs + 63) / 64;
  const int first = min(me * each, pairs), last = min(first + each, pairs);
  int mine = 0, len = 0, tiles = 0, units = 1;
#pragma unroll 4
  for (int p = first; p < last; ++p) {
    len = a.c.lens[p];
    pair_units<WEIGHTS, ROWS>(a, pair_rows<false>(a, p), len, tiles, units);
    mine += tiles * (units + kStart);
  }
  int sum = lane_sums(mine);
  int total = __builtin_amdgcn_readlane(sum, 63);
  if (together) {
    if (lane == 63) lds[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) sum += lds[w];
      total += lds[w];
    }
    lds[kWaves + threadIdx.x] = sum;
    __syncthreads();
  }
  if (total < workers * least) workers = max((total + least - 1) / least, 1);
  shares.each = total / workers;
  shares.more = total - shares.each * workers;
  begin = worker < workers ? shares.begin(worker) : total;
  end = worker < workers ? shares.begin(worker + 1) : total;
  if (begin >= end) return {0, 0, 0, 0};
  int p = first, left = begin - (sum - mine);
  bool here = left >= 0 && left < mine;                          // one lane
  if (!together) {
    if (here && each > 1)
      for (;; ++p) {
        len = a.c.lens[p];
        pair_units<WEIGHTS, ROWS>(a, pair_rows<false>(a, p), len, tiles, units);
        if (left < tiles * (units + kStart)) break;
        left -= tiles * (units + kStart);
      }
  } else {
    int run = 0;                                                 // runs that end before the share begins
    for (int w = 0; w < kWaves; ++w) run += __popcll(__ballot(lds[kWaves + w * 64 + lane] <= begin));
    int before = run > 0 ? lds[kWaves + run - 1] : 0;
    for (int p0 = run * each;; p0 += 64) {                       // (it is found before the run ends)
      p = p0 + lane;
      len = p < pairs ? a.c.lens[p] : 0;
      tiles = units = 0;
      if (p < pairs) pair_units<WEIGHTS, ROWS>(a, pair_rows<false>(a, p), len, tiles, units);
      mine = tiles * (units + kStart);
      sum = before + lane_sums(mine);
      left = begin - (sum - mine);
      here = left >= 0 && left < mine;
      if (__ballot(here) || p0 + 64 >= pairs) break;
      before = __builtin_amdgcn_readlane(sum, 63);
    }
  }
  const int tile = tiles <= 1 ? 0 : left / (units + kStart), unit = left - tile * (units + kStart) - kStart;
  const uint64_t who = __ballot(here);
  const int from = who ? __builtin_ctzll(who) : 0;
  return {__builtin_amdgcn_readlane(p, from), __builtin_amdgcn_readlane(len, from), __builtin_amdgcn_readlane(tile, from),
          __builtin_amdgcn_readlane(unit, from)};
}
// The beginning of the next pair (which may be none: the caller's share has ended then).
__device__ __forceinline__ Item next_pair(const CacheAttnArgs& a, int pair) {
  return {pair + 1, scalar_load(a.c.lens + min(pair + 1, a.c.n_seq * a.c.n_kv_heads - 1)), 0, -kStart};
}

// Sixteen query rows as operand: lane n + 16 g holds of row n dims 64 x + 16 g .. + 15, x = 0, 1, eight to a product.  Returns what the products
// are to be multiplied by (softmax scale * log2(e), less the power of two), and 0 for rows that are not there.
__device__ __forceinline__ float load_queries(const CacheAttnArgs& a, int row0, int n, int h, int group, int row, f16x8 (&q)[4]) {
  const int g = (threadIdx.x & 63) >> 4;
  u32x4 in[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) in[x] = u32x4{0, 0, 0, 0};
  const bool there = row < n * group;
  if (there) {
    const int j = row / group, head = group_head(a.groups, h, row - j * group);
    const uint16_t* src = a.q + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h;
#pragma unroll
    for (int x = 0; x < 4; ++x) in[x] = *reinterpret_cast<const u32x4*>(src + (x >> 1) * 64 + g * 16 + (x & 1) * 8);
  }
  uint32_t top = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(in[x][e] << 16 & 0x7fff0000u, in[x][e] & 0x7fff0000u));
  top = max(top, uint32_t(__shfl_xor(int(top), 16)));
  top = max(top, uint32_t(__shfl_xor(int(top), 32)));
  const int up = top == 0 ? 0 : min(max(13 - (int(top >> 23) - 127), -120), 100);
  const float f = __uint_as_float(uint32_t(up + 127) << 23);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f16x2 two = {(_Float16)(__uint_as_float(in[x][e] << 16) * f), (_Float16)(__uint_as_float(in[x][e] & 0xffff0000u) * f)};
      o[e] = __builtin_bit_cast(uint32_t, two);
    }
    q[x] = __builtin_bit_cast(f16x8, o);
  }
  return there ? a.scale_log2 * __uint_as_float(uint32_t(127 - up) << 23) : 0.0f;
}

// Sixteen bytes of a K row: two operands of eight dims.
template <int FMT>
__device__ __forceinline__ void key_operands(u32x4 w, f16x8& a, f16x8& b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = turned<FMT>(w[e]);
  a = __builtin_bit_cast(f16x8, u32x4{half_codes<FMT, false>(w.x), half_codes<FMT, true>(w.x), half_codes<FMT, false>(w.y), half_codes<FMT, true>(w.y)});
  b = __builtin_bit_cast(f16x8, u32x4{half_codes<FMT, false>(w.z), half_codes<FMT, true>(w.z), half_codes<FMT, false>(w.w), half_codes<FMT, true>(w.w)});
}

// The page of a unit of a head: its number in the table, not looked at yet.
__device__ __forceinline__ int page_number(const CacheArgs& c, int pair, int unit) {
  return scalar_load(c.table + int64_t(pair) * c.max_pages + (unit * kUnit >> c.block_log2));
}
// Where a unit's codes are: of a page that is not in the pool those of the first one, with scales of NaN.  (The scales
// come later than the codes are asked for, and are looked at when they are used.)
struct Page {
  int64_t byte;
  bool bad;
  float k_scale, v_scale;
};
__device__ __forceinline__ Page page_at(const CacheArgs& c, int page, int unit) {
  const bool bad = page < 0 || page >= c.n_pages;
  page = bad ? 0 : page;
  return {((int64_t(page) << c.block_log2) + (unit * kUnit & ((1 << c.block_log2) - 1))) * kHeadDim, bad, scalar_load(c.k_scale + page),
          scalar_load(c.v_scale + page)};
}

// Codes of a unit as a lane holds them: of K row 16 t + n16 bytes 64 x + 16 g and on, of V rows 32 kk + 16 half + 4 g + i dims 8 n16 and on.
struct Keys {
  u32x4 code[4][2];
};
struct Values {
  u32x2 code[2][2][4];
};
// `there`: whether the unit is to be loaded at all.  Loads of one that is not return zeros and touch no memory, but they are in the
// program all the same: behind loads that are only sometimes made, every wait would have to be one for all that is in flight.
__device__ __forceinline__ SlotBuffer unit_buffer(const uint8_t* base, int64_t byte, bool there) {
  const uint64_t x = reinterpret_cast<uint64_t>(base) + byte;
  const uint64_t at = uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x)))) | uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x >> 32)))) << 32;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(at), 0, __builtin_amdgcn_readfirstlane(there ? kUnit * kHeadDim : 0), 0x00020000);
}
// (kOnce: the codes are read by no other tile of rows, and stay in no cache: for the batch of 128 above 121 -> 104 us, for one
// sequence of 131072 tokens 52 -> 46)
template <bool kOnce>
__device__ __forceinline__ void load_keys(const CacheAttnArgs& a, const Page& page, bool there, int n16, int g, Keys& x) {
  const SlotBuffer k = unit_buffer(a.c.k, page.byte, there);
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x.code[t][e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k, n16 * kHeadDim + g * 16 + (t & 1) * 16 * kHeadDim + e * 64, (t >> 1) * 32 * kHeadDim, kOnce ? 2 : 0));
}
template <bool kOnce>
__device__ __forceinline__ void load_values(const CacheAttnArgs& a, const Page& page, bool there, int n16, int g, Values& x) {
  const SlotBuffer v = unit_buffer(a.c.v, page.byte, there);
#pragma unroll
  for (int kk = 0; kk < 2; ++kk)
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x.code[kk][half][i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(v, g * 4 * kHeadDim + n16 * 8 + (half * 16 + i) * kHeadDim, kk * 32 * kHeadDim, kOnce ? 2 : 0));
}

template <int NT, int WAVES, int FMT>
__global__ __launch_bounds__(kThreads, NT == 1 ? 2 : 1) void cache_attn_kernel(CacheAttnArgs a, int least) {
  constexpr int kRows = 16 * NT, kShare = WAVES;                 // waves that work on one share
  constexpr int kJoined = kShare == 1 ? 1 : kWaves;              // waves whose results meet in LDS
  __shared__ float lds_o[kJoined][16][kLdsRow];
  __shared__ float lds_m[kJoined][kRows], lds_l[kJoined][kRows];
  __shared__ int lds_i[kWaves + kThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
  int at, end;
  Shares shares;
  // neighbouring shares in different workgroups, on different compute units
  const int worker = kShare == 1 ? int(blockIdx.x) + wave * int(gridDim.x) : int(blockIdx.x);
  Item it = locate<false, kRows>(a, worker, int(gridDim.x) * (kWaves / kShare), least, lds_i, at, end, shares);
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens<true>(a.t, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h);
    pair_units<false, kRows>(a, n * group, len, tiles, units);
    if (tiles == 0) {
      it = next_pair(a, pair);
      continue;
    }
    const bool good = good_length(a.c, len);
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at));
    if (u1 <= u0) break;                                         // the share ends before the item's first unit
    // the first unit is asked for before the queries, every other one while the one before it is worked on, its place in
    // the page table one more ahead
    const int u_first = u0 + (kShare == 1 ? 0 : wave), u_end = good && len > 0 ? u1 : 0;
    // With 64 rows there are registers for the keys of two units but the values of one, which then come while the scores are worked on.
    constexpr bool kAhead = NT < 4;
    Keys k_even, k_odd;
    Values v_even, v_odd;
    Page here = page_at(a.c, page_number(a.c, pair, min(u_first, u1 - 1)), min(u_first, u1 - 1));
    int page_next = page_number(a.c, pair, min(u_first + kShare, u1 - 1));
    load_keys<NT == 1>(a, here, u_first < u_end, n16, g, k_even);
    if (kAhead) load_values<NT == 1>(a, here, u_first < u_end, n16, g, v_even);
    __builtin_amdgcn_sched_barrier(0);

    f16x8 q[NT][4];
    float to_log2[NT], m[NT], l[NT];
    int seen[NT];                                                // keys that the lane's row sees
    f32x4 acc[NT][8];
    const int seen_first = len - n + 1 + it.tile * kRows / group;     // by the tile's first row: the fewest
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = it.tile * kRows + nt * 16 + n16;
      to_log2[nt] = load_queries(a, row0, n, h, group, row, q[nt]);
      seen[nt] = row < n * group && good ? len - n + 1 + row / group : 0;
      m[nt] = -INFINITY;
      l[nt] = 0.0f;
#pragma unroll
      for (int t = 0; t < 8; ++t) acc[nt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    const auto work = [&](int u, Keys& kc, Values& vc, Keys& k_next, Values& v_next) __attribute__((always_inline)) {
      const float k_scale = here.bad ? __uint_as_float(kNanBits) : here.k_scale, v_scale_here = here.bad ? k_scale : here.v_scale;
      const Page ahead = page_at(a.c, page_next, min(u + kShare, u1 - 1));
      const bool more = u + kShare < u_end;
      if (!kAhead) load_values<NT == 1>(a, here, true, n16, g, vc);
      load_keys<NT == 1>(a, ahead, more, n16, g, k_next);
      if (kAhead) load_values<NT == 1>(a, ahead, more, n16, g, v_next);
      here = ahead;
      page_next = page_number(a.c, pair, min(u + 2 * kShare, u1 - 1));
      __builtin_amdgcn_sched_barrier(0);
      const int key0 = u * kUnit;
      f32x4 sc[NT][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f16x8 k0, k1, k2, k3;
        key_operands<FMT>(kc.code[t][0], k0, k1);
        key_operands<FMT>(kc.code[t][1], k2, k3);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
          x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[nt][0], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[nt][1], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k2, q[nt][2], x, 0, 0, 0);
          sc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k3, q[nt][3], x, 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);                       // operands of one tile at a time, or the registers do not suffice
      }
      f16x8 p[NT][2];
      float alpha[NT], v_scale[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float c = to_log2[nt] * k_scale;
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) sc[nt][t][i] *= c;
        if (key0 + kUnit > seen_first) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + t * 16 + g * 4 + i >= seen[nt]) sc[nt][t][i] = -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[nt][t][i]);
        const float m_new = fmaxf(m[nt], quad_max(top));
        const float ref = m_new == -INFINITY ? 0.0f : m_new;
        alpha[nt] = __builtin_amdgcn_exp2f(m[nt] - ref);
        m[nt] = m_new;
        float sum = 0.0f;
        f16x2 two[8];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            e[i] = __builtin_amdgcn_exp2f(sc[nt][t][i] - ref + kLift);
            sum += e[i];
          }
          two[2 * t] = f16x2{(_Float16)e[0], (_Float16)e[1]};
          two[2 * t + 1] = f16x2{(_Float16)e[2], (_Float16)e[3]};
        }
        l[nt] = l[nt] * alpha[nt] + sum;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, two[4 * kk + e]);
          p[nt][kk] = __builtin_bit_cast(f16x8, w);
        }
        v_scale[nt] = key0 < seen[nt] ? v_scale_here : 0.0f;      // a scale of NaN does not reach rows that see none of the page
      }
      if (key0 + kUnit > len) {
        // codes behind the last token may be anything, NaN among them
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (key0 + kk * 32 + half * 16 + g * 4 + i >= len) vc.code[kk][half][i] = u32x2{0, 0};
      }
      // V^T: dim 8 n16 + t of key pairs; two bytes of a pair lie side by side after one permutation
#pragma unroll
      for (int t2 = 0; t2 < 4; ++t2) {                           // dims 2 t2 and 2 t2 + 1
        f16x8 lo[2], hi[2];
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          u32x4 wl, wh;
#pragma unroll
          for (int e = 0; e < 4; ++e) {                          // pairs of keys
            const uint32_t x = vc.code[kk][e >> 1][2 * (e & 1)][t2 >> 1], y = vc.code[kk][e >> 1][2 * (e & 1) + 1][t2 >> 1];
            const uint32_t w = turned<FMT>(__builtin_amdgcn_perm(y, x, t2 & 1 ? 0x07030602u : 0x05010400u));
            wl[e] = half_codes<FMT, false>(w);
            wh[e] = half_codes<FMT, true>(w);
          }
          lo[kk] = __builtin_bit_cast(f16x8, wl);
          hi[kk] = __builtin_bit_cast(f16x8, wh);
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = {0.0f, 0.0f, 0.0f, 0.0f};
          x = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[0], p[nt][0], x, 0, 0, 0);
          x = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[1], p[nt][1], x, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[0], p[nt][0], y, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[1], p[nt][1], y, 0, 0, 0);
          acc[nt][2 * t2] = acc[nt][2 * t2] * alpha[nt] + x * v_scale[nt];
          acc[nt][2 * t2 + 1] = acc[nt][2 * t2 + 1] * alpha[nt] + y * v_scale[nt];
        }
        if (t2 & 1) __builtin_amdgcn_sched_barrier(0);
      }
    };
    for (int u = u_first; u < u_end; u += 2 * kShare) {
      work(u, k_even, v_even, k_odd, v_odd);
      if (u + kShare >= u_end) break;
      work(u + kShare, k_odd, v_odd, k_even, v_even);
    }

    // the four waves' results become one; dims 8 (4 g + i) + t of row n16 are the lane's
    const bool whole = u0 == 0 && u1 == units;
    const int slot = 2 * worker + (u0 == 0 ? 1 : 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) l[nt] = quad_sum(l[nt]);
    if constexpr (kShare == 1) {
      // one wave's own: a lane has 32 dims of a row
      const int row = it.tile * kRows + n16;
      if (row < n * group) {
        const float sum = l[0], ref = m[0] == -INFINITY ? 0.0f : m[0];
        if (whole) {
          const int j = row / group, head = group_head(a.groups, h, row - j * group);
          float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
          if (!good) inv = __uint_as_float(kNanBits);            // a length that cannot be
          uint16_t* dst = a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + g * 32;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x4*>(dst + i * 8) = u32x4{pack_bf16(acc[0][0][i] * inv, acc[0][1][i] * inv), pack_bf16(acc[0][2][i] * inv, acc[0][3][i] * inv),
                                                           pack_bf16(acc[0][4][i] * inv, acc[0][5][i] * inv), pack_bf16(acc[0][6][i] * inv, acc[0][7][i] * inv)};
          if (g == 0) {
            if (a.lse != nullptr)
              a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = good ? (m[0] + __builtin_amdgcn_logf(sum) - kLift) * 0.6931471805599453f : inv;
            if (a.weight_out != nullptr)
              *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{ref - kLift, inv};
          }
        } else {
          float* dst = a.part_o + (int64_t(slot) * kRows + n16) * kHeadDim + g * 32;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<f32x4*>(dst + i * 8) = f32x4{acc[0][0][i], acc[0][1][i], acc[0][2][i], acc[0][3][i]};
            *reinterpret_cast<f32x4*>(dst + i * 8 + 4) = f32x4{acc[0][4][i], acc[0][5][i], acc[0][6][i], acc[0][7][i]};
          }
          if (g == 0) {
            a.part_ml[int64_t(slot) * 2 * kRows + n16] = m[0];
            a.part_ml[int64_t(slot) * 2 * kRows + kRows + n16] = sum;
          }
        }
      }
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (g == 0) {
          lds_m[wave][nt * 16 + n16] = m[nt];
          lds_l[wave][nt * 16 + n16] = l[nt];
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* dst = &lds_o[wave][n16][(g * 4 + i) * 8];
          *reinterpret_cast<f32x4*>(dst) = f32x4{acc[nt][0][i], acc[nt][1][i], acc[nt][2][i], acc[nt][3][i]};
          *reinterpret_cast<f32x4*>(dst + 4) = f32x4{acc[nt][4][i], acc[nt][5][i], acc[nt][6][i], acc[nt][7][i]};
        }
        __syncthreads();
        const int r = tid >> 4, d = (tid & 15) * 8, in_tile = nt * 16 + r, row = it.tile * kRows + in_tile;
        if (row < n * group) {
          float top = -INFINITY, sum = 0.0f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds_m[w][in_tile]);
          const float ref = top == -INFINITY ? 0.0f : top;
          f32x4 o0 = {0.0f, 0.0f, 0.0f, 0.0f}, o1 = o0;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_m[w][in_tile] - ref);
            sum += f * lds_l[w][in_tile];
            o0 += f * *reinterpret_cast<const f32x4*>(&lds_o[w][r][d]);
            o1 += f * *reinterpret_cast<const f32x4*>(&lds_o[w][r][d + 4]);
          }
          if (whole) {
            const int j = row / group, head = group_head(a.groups, h, row - j * group);
            float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            if (!good) inv = __uint_as_float(kNanBits);            // a length that cannot be
            const u32x4 o = {pack_bf16(o0.x * inv, o0.y * inv), pack_bf16(o0.z * inv, o0.w * inv),
                             pack_bf16(o1.x * inv, o1.y * inv), pack_bf16(o1.z * inv, o1.w * inv)};
            *reinterpret_cast<u32x4*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d) = o;
            if (d == 0) {
              if (a.lse != nullptr)
                a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = good ? (top + __builtin_amdgcn_logf(sum) - kLift) * 0.6931471805599453f : inv;
              if (a.weight_out != nullptr)
                *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{ref - kLift, inv};
            }
          } else {
            float* dst = a.part_o + (int64_t(slot) * kRows + in_tile) * kHeadDim + d;
            *reinterpret_cast<f32x4*>(dst) = o0;
            *reinterpret_cast<f32x4*>(dst + 4) = o1;
            if (d == 0) {
              a.part_ml[int64_t(slot) * 2 * kRows + in_tile] = top;
              a.part_ml[int64_t(slot) * 2 * kRows + kRows + in_tile] = sum;
            }
          }
        }
      }
      __syncthreads();
    }
    if (u0 == 0 && (kShare == 1 ? lane == 0 : tid == 0))         // for the joining kernel: pieces of the item, if it ends in another share
      *reinterpret_cast<int2*>(a.begun + 2 * (int64_t(pair) * a.tiles + it.tile)) = int2{worker, whole ? 0 : shares.of(at - it.unit + units - 1) - worker + 1};
    at += u1 - it.unit;
    it.unit = -kStart;
    if (++it.tile == tiles) it = next_pair(a, pair);
  }
}

// Joins the pieces of one row of an item: with M the largest m, out = sum 2^(m - M) O / sum 2^(m - M) l.  A workgroup a row (y) of an
// item (x).  The first piece lies in slot 2 w + 1 of the share w it begins in, the others in 2 (w + 1), 2 (w + 2) ...; eight groups of
// 32 lanes take every eighth piece, a lane four dims, and what they have is added up in order.  What the first pieces hold is asked for
// together with the statistics.
__global__ __launch_bounds__(kThreads) void cache_join_kernel(CacheAttnArgs a, int rows_per_tile) {
  __shared__ f32x4 lds_o[8][32];
  const int tid = threadIdx.x, lane = tid & 63, d4 = tid & 31, part = tid >> 5;
  const int pair = blockIdx.x / uint32_t(a.tiles), tile = blockIdx.x - pair * a.tiles, in_tile = blockIdx.y, row = tile * rows_per_tile + in_tile;
  const int2 begun = *reinterpret_cast<const int2*>(a.begun + 2 * int64_t(blockIdx.x));
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, group = group_size(a.groups, h);
  int row0, n;
  step_tokens(a.t, s, row0, n);
  if (row >= n * group) return;                                  // (the item may not be one: nothing was written for it then)
  const int w = begun.x, pieces = begun.y;
  if (pieces == 0) return;                                       // it was whole
  const auto slot = [&](int x) { return 2 * int64_t(w + x) + (x == 0); };
  const auto stats = [&](int x) { return a.part_ml + slot(x) * 2 * rows_per_tile + in_tile; };
  const auto values = [&](int x) { return *reinterpret_cast<const f32x4*>(a.part_o + (slot(x) * rows_per_tile + in_tile) * kHeadDim + d4 * 4); };
  constexpr int kEarly = 4;
  f32x4 early[kEarly];
  float early_m[kEarly];
#pragma unroll
  for (int x = 0; x < kEarly; ++x) {
    early[x] = part + 8 * x < pieces ? values(part + 8 * x) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    early_m[x] = part + 8 * x < pieces ? *stats(part + 8 * x) : -INFINITY;
  }
  // every wave by itself, in the same order
  float m = -INFINITY, l = 0.0f;
  if (lane < pieces) {
    m = stats(lane)[0];
    l = stats(lane)[rows_per_tile];
  }
  float top = m;
  for (int x = lane + 64; x < pieces; x += 64) top = fmaxf(top, *stats(x));
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = __builtin_amdgcn_exp2f(m - ref) * l;
  for (int x = lane + 64; x < pieces; x += 64) sum += __builtin_amdgcn_exp2f(*stats(x) - ref) * stats(x)[rows_per_tile];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < kEarly; ++x) o += __builtin_amdgcn_exp2f(early_m[x] - ref) * early[x];
#pragma unroll 8
  for (int x = part + 8 * kEarly; x < pieces; x += 8) o += __builtin_amdgcn_exp2f(*stats(x) - ref) * values(x);
  lds_o[part][d4] = o;
  __syncthreads();
  if (tid >= 32) return;
#pragma unroll
  for (int x = 1; x < 8; ++x) o += lds_o[x][d4];
  const int j = row / group, head = group_head(a.groups, h, row - j * group);
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  *reinterpret_cast<u32x2*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d4 * 4) =
      u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
  if (tid == 0) {
    if (a.lse != nullptr) a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = (top + __builtin_amdgcn_logf(sum) - kLift) * 0.6931471805599453f;
    if (a.weight_out != nullptr)
      *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{ref - kLift, inv};
  }
}

// weight_out = weight_in + the probabilities that the step's rows put on each key, taken again from the keys and the rows' statistics: every
// key belongs to one wave, so nothing is added up between workgroups.
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void cache_weight_kernel(CacheAttnArgs a) {
  __shared__ int lds_i[kWaves + kThreads];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  int at, end;
  Shares shares;
  Item it = locate<true, 1>(a, int(blockIdx.x) + wave * int(gridDim.x), int(gridDim.x) * kWaves, 1, lds_i, at, end, shares);
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens<true>(a.t, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h), rows = n * group;
    pair_units<true, 1>(a, rows, len, tiles, units);
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at));
    const int64_t row_of_weights = int64_t(pair) * a.c.max_pages << a.c.block_log2;
    for (int u = u0; u < u1; ++u) {
      const Page page = page_at(a.c, page_number(a.c, pair, u), u);
      const float k_scale = page.bad ? __uint_as_float(kNanBits) : page.k_scale;
      const int key0 = u * kUnit;
      f16x8 k[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        u32x4 kc[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) kc[x] = *reinterpret_cast<const u32x4*>(a.c.k + page.byte + (t * 16 + n16) * kHeadDim + g * 16 + x * 64);
        key_operands<FMT>(kc[0], k[t][0], k[t][1]);
        key_operands<FMT>(kc[1], k[t][2], k[t][3]);
      }
      f32x4 w[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      for (int r0 = 0; r0 < rows; r0 += 16) {
        f16x8 q[4];
        const int row = r0 + n16;
        const float c = load_queries(a, row0, n, h, group, row, q) * k_scale;
        int seen = 0;
        float m = 0.0f, inv = 0.0f;
        if (row < rows) {
          const int j = row / group, head = group_head(a.groups, h, row - j * group);
          const f32x2 st = *reinterpret_cast<const f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head));
          seen = len - n + 1 + j;
          m = st.x;
          inv = st.y;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[t][e], q[e], x, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(x[i] * c - m) * inv;
            w[t][i] += key0 + t * 16 + g * 4 + i < seen ? p : 0.0f;
          }
        }
      }
      // over the sixteen rows; lane n16 == 0 of each group of keys writes
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int d = 1; d < 16; d <<= 1) w[t][i] += __shfl_xor(w[t][i], d);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if (n16 != t) continue;
        const int key = key0 + t * 16 + g * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (key + i < len) {
            const int64_t x = row_of_weights + key + i;
            a.weight_out[x] = (a.weight_in != nullptr ? a.weight_in[x] : 0.0f) + w[t][i];
          }
      }
    }
    at += units - it.unit;
    it = next_pair(a, pair);
  }
}

template <int FMT>
int32_t launch_format(const CacheAttnArgs& a, int rows, int most_rows, int compute_units, hipStream_t stream) {
  static_assert(kCacheMaxWorkers % kWaves == 0, "");
  const int two = min(kCacheMaxWorkers / kWaves, compute_units * 2), one = min(two, compute_units);
  if (a.t.n_tokens > 0) {
    if (rows == 16) cache_attn_kernel<1, 1, FMT><<<two, kThreads, 0, stream>>>(a, 1);
    else if (rows == 32) cache_attn_kernel<2, kWaves, FMT><<<one, kThreads, 0, stream>>>(a, kWaves);
    else cache_attn_kernel<4, kWaves, FMT><<<one, kThreads, 0, stream>>>(a, kWaves);
    cache_join_kernel<<<dim3(a.c.n_seq * a.c.n_kv_heads * a.tiles, min(rows, most_rows)), kThreads, 0, stream>>>(a, rows);
  }
  if (a.weight_out != nullptr) cache_weight_kernel<FMT><<<two, kThreads, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace

int32_t cache_attn_rows(int64_t most_rows) { return most_rows <= 16 ? 16 : most_rows <= 32 ? 32 : 64; }

int32_t launch_cache_attn(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream) {
  const int rows = cache_attn_rows(most_rows);
  return a.c.format == SHPLB_CACHE_E4M3 ? launch_format<SHPLB_CACHE_E4M3>(a, rows, most_rows, compute_units, stream)
                                        : launch_format<SHPLB_CACHE_INT8>(a, rows, most_rows, compute_units, stream);
}

}  // namespace shplb
