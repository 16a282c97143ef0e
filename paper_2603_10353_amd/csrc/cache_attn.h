// Attention of a step's queries over the 8-bit cache (gfx950).
//
// For every query row (a token of the step and a head of the KV head's group) with key codes k_t and value codes v_t of pages with
// scales a, b:
//
//   y_t = (q . k_t) * scale * log2(e) * a,   m = max y,   l = sum 2^(y_t - m),   out = sum 2^(y_t - m) b v_t / l,   lse = (m + log2 l) ln 2,
//
// in one pass over the keys with a running m: a reference exponent, raised to the largest y (and l and the output scaled down)
// only where a y is more than 8 above it, which after the first keys is hardly ever.  Bound by reading the codes once: a token of
// a KV head is 256 bytes and, for a group of four heads, 4 KFLOP.  So the matrix instructions are used for what they save in
// registers and lanes, with most of their rows empty in a plain decoding step.
//
// Split.  All heads' keys together are one list of units of 64 keys, which is cut into equal, contiguous shares whatever the heads'
// lengths are: lengths differ between sequences, and between heads after an eviction.  A share is a wave's where a head has up to 16
// rows, and a workgroup's where it has more (tiles of 32 rows).  The lengths are on the device (they change while a captured
// launch stays), so each wave adds them up by itself.  A (sequence, KV head, tile of rows) whose units lie in several shares has
// partial results (m, l, unnormalised output), which a second kernel joins in order.  Short caches are worked on head by head or
// item by item, without partial results.
//
// Tile.  A wave works on a unit at a time: keys are the rows of the first product (S^T = K Q^T), so a lane has scores of one
// query and four adjacent keys of each 16; the second one is O^T = V^T P^T, whose operand P^T needs exactly those (the order of
// the keys inside a product is free, as long as V's are taken alike).  Codes come straight from global memory into registers and
// are turned to fp16 there (exact in both formats), V's after a byte transposition of key pairs; queries wait in LDS as operands.
// Q is brought to fp16 by a power of two per row, so that its largest magnitude lies in [2^13, 2^14), or as far up as 2^120 takes
// it: exact down to 2^-27 of it.  Probabilities are rounded to fp16 at 2^7 times their size: eleven bits down to 2^-21 of the
// reference, steps of 2^-31 of it below.  Values are fp16 numbers, too, scale and all, where the scale lies between 2^-15 and 2^7
// (int8 2^-14 and 2^5).  All sums are fp32.
//
// Measured: 128 sequences x 8 heads of 100 to 16000 tokens (570 MB) 98 us, 5.8 TB/s; one sequence of 131072 tokens x 8 heads 47 us, and
// 6 to join; a sequence of 777 tokens 10 us, of which the launch and three reads that wait for one another are eight.
#pragma once
#include "cache_common.h"

namespace shplb {
namespace {

constexpr int kThreads = 256, kWaves = 4;
// What beginning with an item costs, in units of the list of all units (where it is that many empty ones in front of the item's own):
// the queries, the first keys, the results, all of them waited for.  A wave by itself: for a batch of 128 sequences x 8 heads of lengths
// between 100 and 16000, where it has one to five items, 102 us without, 97 with two, 100 with five.  Four waves together, which
// have a unit's work done in a quarter of the time: for 100 sequences x 2 heads of 128 rows and up to a few hundred tokens 44 us with
// two, 34 with eight, 42 with sixteen; for 128 rows x 8 heads x 32768 tokens 53 with two, 51 from four on.
constexpr int start_units(int waves) { return waves == 1 ? 2 : kCacheMostStart; }
constexpr float kLift = 7.0f;                  // log2 of what probabilities are multiplied by, beside their reference ...
constexpr float kHeadroom = 8.0f;              // ... and how far, in the exponent, they may be above it: 2^15 in fp16
constexpr int kLdsRow = kHeadDim + 4;          // floats of a row in LDS: rows four banks apart

// What rows see.
//  - kAll: their head's tokens up to their own.
//  - kWindow: of those the last `window` and the first n_sink.  A tile of rows goes through the units that any of its rows
//    sees: those of the first tokens, then those of the windows (cache_span.h).  As many units are reckoned with for every tile as one has at most.
//  - kGroups: all of the tokens of a cache whose sequence s is shared by the rows of the step's sequences groups[s] ..
//    groups[s + 1] - 1.
enum { kAll, kWindow, kGroups };

struct Item {                                  // a place in the list of units
  int pair, len;                               // the head, and its length
  int tile, unit;                              // tile of rows, unit inside it; below 0 the beginning
};
// How the list is divided: `each` units a share, and `more` of the shares one more.  Those of waves by themselves: the first
// ones.  Those of workgroups: evenly among the others, or shares and items of equal lengths drift apart, and more shares have the
// end of one item and the beginning of another (128 rows x 8 heads x 32768 tokens, eight units a beginning: 51 us, 56 with the
// first ones, before other changes; the larger number of shares of waves has less of it, and some power of two apart the longer
// ones meet on one compute unit: weights of those rows 31 us, 33 evenly).
template <bool EVENLY>
struct Shares {
  int each, more, n;                           // n: of shares, at most kCacheMaxWorkers; more is less
  __device__ int begin(int w) const { return w * each + (EVENLY ? int(uint32_t(w * more) / uint32_t(n)) : min(w, more)); }
  // the share that unit `at` of the list is in
  __device__ int of(int at) const {
    if (!EVENLY) return at < more * (each + 1) ? at / (each + 1) : more + (at - more * (each + 1)) / each;
    int w = min(int(float(at) / (float(each) + float(more) / float(n))), n - 1);       // a near guess: less than one off
    while (begin(w) > at) --w;
    while (begin(w + 1) <= at) ++w;
    return w;
  }
};

__device__ __forceinline__ int group_size(const HeadGroups& g, int h) { return g.mapped ? g.begin[h + 1] - g.begin[h] : g.group; }
__device__ __forceinline__ int group_head(const HeadGroups& g, int h, int x) { return g.mapped ? g.head[g.begin[h] + x] : h * g.group + x; }

// The rows of sequence s of the cache.
template <int VIEW, bool SCALAR = false>
__device__ __forceinline__ void view_tokens(const CacheAttnArgs& a, int s, int& row0, int& n) {
  if constexpr (VIEW == kGroups) {
    int first = SCALAR ? scalar_load(a.view.groups + s) : a.view.groups[s], end = SCALAR ? scalar_load(a.view.groups + s + 1) : a.view.groups[s + 1];
    first = min(max(first, 0), a.view.members);
    end = min(max(end, first), a.view.members);
    if (a.t.cu == nullptr) {
      row0 = first * a.t.max_tokens;
      n = (end - first) * a.t.max_tokens;
    } else {
      row0 = min(max(SCALAR ? scalar_load(a.t.cu + first) : a.t.cu[first], 0), a.t.n_tokens);
      n = min(max(SCALAR ? scalar_load(a.t.cu + end) : a.t.cu[end], row0), a.t.n_tokens) - row0;
    }
  } else {
    step_tokens<SCALAR>(a.t, s, row0, n);
  }
}
// Rows of a pair in this step (query tokens times heads of the group).
template <bool SCALAR, int VIEW = kAll>
__device__ __forceinline__ int pair_rows(const CacheAttnArgs& a, int pair) {
  if (VIEW != kGroups && a.t.cu == nullptr && !a.groups.mapped) return a.t.max_tokens * a.groups.group;    // the same for all: no division
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
  int row0, n;
  view_tokens<VIEW, SCALAR>(a, s, row0, n);
  return n * group_size(a.groups, h);
}
// Tiles of rows of a pair and units of each.
template <bool WEIGHTS, int ROWS, int VIEW = kAll>
__device__ __forceinline__ void pair_units(const CacheAttnArgs& a, int rows, int len, int& tiles, int& units) {
  units = good_length(a.c, len) ? (len + kUnit - 1) / kUnit : 0;
  if (VIEW == kWindow) units = min(units, a.view.most_units);
  if (WEIGHTS) {
    tiles = 1;                                 // all rows together, and keys no row looks at are copied
  } else {
    tiles = (rows + ROWS - 1) / ROWS;
    units = max(units, 1);                     // a head without keys has an output, too
  }
}

// What the rows first_row .. first_row + ROWS - 1 of n tokens see with windows.
template <int VIEW, int ROWS>
__device__ __forceinline__ Span span_of(const CacheAttnArgs& a, int first_row, int n, int group, bool good, int len) {
  if constexpr (VIEW != kWindow) return {};
  else return window_span(a.view.window, a.view.n_sink, first_row, ROWS, n, group, good ? len : 0);
}

// The place where a worker's share [begin, end) of all units begins.  Shares are of `least` units at least, if there are more
// than `few` of them.  Up to 512 pairs every wave adds them up by itself, a lane a run of them; beyond, the four waves do it
// together, and each looks for its place in the run where it lies, 64 pairs at a time.  (All units, beginnings and all, are below
// 2^30: the entry point sees to that.  Groups that overlap, as offsets that go backwards have them, may have more between them: their sums
// end at what groups have that do not, the place that is found is one of some pair all the same, and as much of the list lies behind it as
// behind the place in the sums.)
template <bool WEIGHTS, int ROWS, int START, int VIEW = kAll, class SHARES>
__device__ __forceinline__ Item locate(const CacheAttnArgs& a, int worker, int workers, int least, int few, int* lds, int& begin, int& end, SHARES& shares) {
  const int pairs = a.c.n_seq * a.c.n_kv_heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const auto add = [&]() {
    if constexpr (VIEW == kGroups) return UnitSums{a.view.most_listed};
    else return PlainSums{};
  }();
  const bool together = pairs > 512;
  const int me = together ? threadIdx.x : lane, each = together ? (pairs + kThreads - 1) / kThreads : (pairs + 63) / 64;
  const int first = min(me * each, pairs), last = min(first + each, pairs);
  int mine = 0, len = 0, tiles = 0, units = 1;
#pragma unroll 4
  for (int p = first; p < last; ++p) {
    len = a.c.lens[p];
    pair_units<WEIGHTS, ROWS, VIEW>(a, pair_rows<false, VIEW>(a, p), len, tiles, units);
    mine = add(mine, tiles * (units + START));
  }
  int sum = lane_sums(mine, add);
  int total = __builtin_amdgcn_readlane(sum, 63);
  if (together) {
    if (lane == 63) lds[wave] = total;
    __syncthreads();
    total = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) sum = add(sum, lds[w]);
      total = add(total, lds[w]);
    }
    lds[kWaves + threadIdx.x] = sum;
    __syncthreads();
  }
  if (total < workers * least) workers = max((total + least - 1) / least, max(min(total, few), 1));
  shares.each = total / workers;
  shares.more = total - shares.each * workers;
  shares.n = workers;
  begin = worker < workers ? shares.begin(worker) : total;
  end = worker < workers ? shares.begin(worker + 1) : total;
  if (begin >= end) return {0, 0, 0, 0};
  int p = first, left = begin - (sum - mine);
  bool here = left >= 0 && left < mine;                          // one lane
  if (!together) {
    if (here && each > 1)
      for (;; ++p) {
        len = a.c.lens[p];
        pair_units<WEIGHTS, ROWS, VIEW>(a, pair_rows<false, VIEW>(a, p), len, tiles, units);
        if (left < tiles * (units + START)) break;
        left -= tiles * (units + START);
      }
  } else {
    int run = 0;                                                 // runs that end before the share begins
    for (int w = 0; w < kWaves; ++w) run += __popcll(__ballot(lds[kWaves + w * 64 + lane] <= begin));
    int before = run > 0 ? lds[kWaves + run - 1] : 0;
    for (int p0 = run * each;; p0 += 64) {                       // (it is found before the run ends)
      p = p0 + lane;
      len = p < pairs ? a.c.lens[p] : 0;
      tiles = units = 0;
      if (p < pairs) pair_units<WEIGHTS, ROWS, VIEW>(a, pair_rows<false, VIEW>(a, p), len, tiles, units);
      mine = tiles * (units + START);
      sum = add(before, lane_sums(mine, add));
      left = begin - (sum - mine);
      here = left >= 0 && left < mine;
      if (__ballot(here) || p0 + 64 >= pairs) break;
      before = __builtin_amdgcn_readlane(sum, 63);
    }
  }
  const int tile = tiles <= 1 ? 0 : left / (units + START), unit = left - tile * (units + START) - START;
  const uint64_t who = __ballot(here);
  const int from = who ? __builtin_ctzll(who) : 0;
  return {__builtin_amdgcn_readlane(p, from), __builtin_amdgcn_readlane(len, from), __builtin_amdgcn_readlane(tile, from),
          __builtin_amdgcn_readlane(unit, from)};
}
// The beginning of the next pair (the last one's again where there is none: the caller's share has ended then).
template <int START>
__device__ __forceinline__ Item next_pair(const CacheAttnArgs& a, int pair) {
  const int next = min(pair + 1, a.c.n_seq * a.c.n_kv_heads - 1);
  return {next, scalar_load(a.c.lens + next), 0, -START};
}
// The beginning of the next sequence after s that has tokens in this step, 64 looked at together: a batch may have many that have none.
template <int START, int VIEW = kAll>
__device__ __forceinline__ bool next_sequence(const CacheAttnArgs& a, int s, int lane, Item& it) {
  for (int s0 = s + 1; s0 < a.c.n_seq; s0 += 64) {
    int row0, n;
    view_tokens<VIEW>(a, min(s0 + lane, a.c.n_seq - 1), row0, n);
    const uint64_t found = __ballot(n > 0);
    if (found == 0) continue;
    const int pair = min(s0 + int(__builtin_ctzll(found)), a.c.n_seq - 1) * a.c.n_kv_heads;
    it = {pair, scalar_load(a.c.lens + pair), 0, -START};
    return true;
  }
  return false;
}

// A query row as a lane has it on the way: lane n + 16 g of row n dims 64 x + 16 g .. + 15, x = 0, 1.
struct Query {
  u32x4 part[4];
};
// Asks for it; of rows that are not there it is zeros.
__device__ __forceinline__ void ask_query(const CacheAttnArgs& a, int row0, int n, int h, int group, int row, int lane, Query& q) {
#pragma unroll
  for (int x = 0; x < 4; ++x) q.part[x] = u32x4{0, 0, 0, 0};
  if (row >= n * group) return;
  const int j = row / group, head = group_head(a.groups, h, row - j * group);
  const uint16_t* src = a.q + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + (lane >> 4) * 16;
#pragma unroll
  for (int x = 0; x < 4; ++x) q.part[x] = *reinterpret_cast<const u32x4*>(src + (x >> 1) * 64 + (x & 1) * 8);
}
// ... and makes it four operands, eight dims to a product each.  Returns what the products are to be multiplied by: softmax scale *
// log2(e), less the power of two that brings the row to fp16.
__device__ __forceinline__ float query_operands(const CacheAttnArgs& a, const Query& in, f16x8 (&q)[4]) {
  uint32_t top = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(in.part[x][e] << 16 & 0x7fff0000u, in.part[x][e] & 0x7fff0000u));
  top = max(top, uint32_t(__shfl_xor(int(top), 16)));
  top = max(top, uint32_t(__shfl_xor(int(top), 32)));
  // (at most 2^120: 2^-133, which all bf16 numbers are multiples of, becomes 2^-13, and a softmax scale of about 1 over it is no subnormal)
  const int up = top == 0 ? 0 : min(max(13 - (int(top >> 23) - 127), -120), 120);
  const float f = __uint_as_float(uint32_t(up + 127) << 23);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f16x2 two = {(_Float16)(__uint_as_float(in.part[x][e] << 16) * f), (_Float16)(__uint_as_float(in.part[x][e] & 0xffff0000u) * f)};
      o[e] = __builtin_bit_cast(uint32_t, two);
    }
    q[x] = __builtin_bit_cast(f16x8, o);
  }
  return a.scale_log2 * __uint_as_float(uint32_t(127 - up) << 23);
}

// What lies far outside of what a model computes with, and is right all the same.
//  - Rows whose products' factor, times the scale of some page, may be infinite (their queries are in the hundreds of thousands): the products
//    themselves may be small, or 0 where a query and a key have no dim in common.  They are multiplied by one after the other.
//  - Rows whose reference is 2^22 or more: a product that is rounded, as the reference was, and one inside of a multiply-add differ by
//    so much there that a probability may be above all that fp16 holds.  Their products are rounded.
// A wave with such a row takes every unit for one that not all rows see all of: its "fewest keys that a row sees" are kFar.
constexpr int kFar = INT32_MIN;
__device__ __forceinline__ bool far_row(float to_log2) { return to_log2 >= 2.0f; }
__device__ __forceinline__ bool far_reference(float m) { return fabsf(m) >= 0x1p22f && fabsf(m) < INFINITY; }

// Eight bytes of a K row as operand.
template <int FMT>
__device__ __forceinline__ f16x8 key_operand(uint32_t x, uint32_t y) {
  x = turned<FMT>(x);
  y = turned<FMT>(y);
  return __builtin_bit_cast(f16x8, u32x4{half_codes<FMT, false>(x), half_codes<FMT, true>(x), half_codes<FMT, false>(y), half_codes<FMT, true>(y)});
}

// The page of a unit of a head: its number in the table, not looked at yet.
__device__ __forceinline__ int page_number(const CacheArgs& c, int pair, int unit) {
  return scalar_load(c.table + int64_t(pair) * c.max_pages + (unit * kUnit >> c.block_log2));
}
// Where a unit's codes are.  Those of a page that is not in the pool are not loaded, zeros with scales of NaN: codes that are NaN
// themselves would reach rows that see none of them.  (The scales come later than the codes are asked for, and are looked at when
// they are used.)
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

// Codes of a unit as a lane holds them: of K row 16 t + n16 bytes 64 x + 16 g and on, of V rows 32 kk + 16 half + 4 g + i dims 8
// n16 and on.
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
__device__ __forceinline__ void load_keys(const CacheAttnArgs& a, const Page& page, bool there, int lane_byte, Keys& x) {
  const SlotBuffer k = unit_buffer(a.c.k, page.byte, there && !page.bad);
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e)
      x.code[t][e] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(k, lane_byte, t * 16 * kHeadDim + e * 64, kOnce ? 2 : 0));
}
template <bool kOnce>
__device__ __forceinline__ void load_values(const CacheAttnArgs& a, const Page& page, bool there, int lane_byte, Values& x) {
  const SlotBuffer v = unit_buffer(a.c.v, page.byte, there && !page.bad);
#pragma unroll
  for (int kk = 0; kk < 2; ++kk)
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        x.code[kk][half][i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(v, lane_byte, (kk * 32 + half * 16 + i) * kHeadDim, kOnce ? 2 : 0));
}

// The rows of a wave: the reference exponent, the denominator and the output of row 16 nt + lane % 16, of which a lane has dims
// 8 (4 (lane / 16) + i) + t.
template <int NT>
struct Rows {
  float m[NT], l[NT];
  f32x4 acc[NT][8];
};
// ... and what does not change, which would cost registers: the queries as operands, what products are multiplied by and the keys
// seen.  What a lane reads it wrote itself.
template <int NT>
struct RowsLds {
  f16x8 q[NT][4][64];
  f32x2 row[NT][64];
  __device__ __forceinline__ float to_log2(int nt, int lane) const { return row[nt][lane].x; }
  __device__ __forceinline__ int seen(int nt, int lane) const { return __float_as_int(row[nt][lane].y); }
};
// What is on its way to a wave: the codes of a unit, where they come from, and the place of the next one in the page table.  Keys are
// asked for as soon as those of the unit before are operands, values when those are: either come while the other half of the work
// is done, and one set of registers is enough.  A place in the page table is read one unit more ahead.
struct Flight {
  Keys k;
  Values v;
  Page here;
  int page_next;
};

// Asks for unit `first`, if it is below end, whose page's number is `page`.
template <bool ONCE>
__device__ __forceinline__ void ask_unit(const CacheAttnArgs& a, int page, int first, int end, int lane, bool values, Flight& f) {
  const int n16 = lane & 15, g = lane >> 4;
  f.here = page_at(a.c, page, first);
  load_keys<ONCE>(a, f.here, first < end, n16 * kHeadDim + g * 16, f.k);
  if (values) load_values<ONCE>(a, f.here, first < end, g * 4 * kHeadDim + n16 * 8, f.v);
  __builtin_amdgcn_sched_barrier(0);
}

// What a wave begins with: the rows from first_row on and the first unit of first, first + STEP .. below end (last: a unit whose
// place in the page table can be read in any case).  Queries are on their way while the page is looked up, and are worked on
// while its codes are.  They go into LDS, as each lane needs them: what it reads it wrote itself, and they cost no registers.
// Returns whether there is a far_row().
template <int NT, int STEP, bool ONCE, int VIEW = kAll>
__device__ __forceinline__ bool begin_rows(const CacheAttnArgs& a, int pair, int h, int group, int row0, int n, int first_row, int seen_before, int first,
                                           int end, int last, int lane, RowsLds<NT>& lds, Flight& f, Rows<NT>& r, const Span& span = {}) {
  const auto unit = [&](int u) { return VIEW == kWindow ? span.unit(u) : u; };
  const int page = page_number(a.c, pair, unit(min(first, last)));
  f.page_next = page_number(a.c, pair, unit(min(first + STEP, last)));
  Query q[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) ask_query(a, row0, n, h, group, first_row + nt * 16 + (lane & 15), lane, q[nt]);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (VIEW == kWindow) ask_unit<ONCE>(a, page, unit(min(first, last)), first < end ? INT32_MAX : 0, lane, true, f);
  else ask_unit<ONCE>(a, page, min(first, last), first < end ? end : 0, lane, true, f);
  bool far = false;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int row = first_row + nt * 16 + (lane & 15);
    f16x8 operand[4];
    const float to_log2 = query_operands(a, q[nt], operand);
    far |= far_row(to_log2);
#pragma unroll
    for (int e = 0; e < 4; ++e) lds.q[nt][e][lane] = operand[e];
    const bool there = row < n * group;
    lds.row[nt][lane] = f32x2{there ? to_log2 : 0.0f, __int_as_float(there ? VIEW == kGroups ? seen_before : seen_before + row / group : 0)};
    r.m[nt] = -INFINITY;
    r.l[nt] = 0.0f;
#pragma unroll
    for (int t = 0; t < 8; ++t) r.acc[nt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  return __ballot(far) != 0;
}

// Scores of a unit, S^T.
template <int NT, int FMT>
__device__ __forceinline__ void scores(const Keys& keys, const f16x8 (*lds_q)[4][64], int lane, f32x4 (&sc)[NT][4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f16x8 k[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) k[t] = key_operand<FMT>(keys.code[t][e >> 1][2 * (e & 1)], keys.code[t][e >> 1][2 * (e & 1) + 1]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const f16x8 q = lds_q[nt][e][lane];
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[t], q, e == 0 ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sc[nt][t], 0, 0, 0);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Goes through the units first, first + STEP ..; seen_first: the fewest keys that a row sees (or kFar).  KEEP > 0: there are no
// more than that, and y of each (-inf where it is masked) stays in `kept`.
template <int NT, int STEP, bool ONCE, int FMT, int KEEP = 0, int VIEW = kAll>
__device__ __forceinline__ void attend(const CacheAttnArgs& a, int pair, int len, int first, int end, int last, int seen_first,
                                       const RowsLds<NT>& lds, int lane, Flight& f, Rows<NT>& r, f32x4 (*kept)[4] = nullptr, const Span& span = {}) {
  const auto unit = [&](int u) { return VIEW == kWindow ? span.unit(u) : u; };
  const int n16 = lane & 15, g = lane >> 4, k_byte = n16 * kHeadDim + g * 16, v_byte = g * 4 * kHeadDim + n16 * 8;
  const auto attend_unit = [&](int u, f32x4* keep) {
    const float k_scale = f.here.bad ? __uint_as_float(kNanBits) : f.here.k_scale, v_scale = f.here.bad ? k_scale : f.here.v_scale;
    const bool more = u + STEP < end;
    const Page ahead = page_at(a.c, f.page_next, unit(min(u + STEP, last)));
    f.page_next = page_number(a.c, pair, unit(min(u + 2 * STEP, last)));
    const int key0 = unit(u) * kUnit;
    // whether the unit begins in front of some row's window, and is not all first tokens
    const bool cut = VIEW == kWindow && key0 < span.low_last && key0 + kUnit > a.view.n_sink;
    f32x4 sc[NT][4];
    scores<NT, FMT>(f.k, lds.q, lane, sc);
    load_keys<ONCE>(a, ahead, more, k_byte, f.k);
    __builtin_amdgcn_sched_barrier(0);
    // the reference exponent, raised where a score is more than 2^kHeadroom above it
    float to[NT], top[NT];
    bool raise = false;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      to[nt] = lds.to_log2(nt, lane) * k_scale;
      if (key0 + kUnit > seen_first || cut) {
        if (seen_first == kFar) {
          const bool far = to[nt] == INFINITY;
          const float first = far ? lds.to_log2(nt, lane) : to[nt];
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[nt][t] *= first;
          to[nt] = far ? k_scale : 1.0f;
        }
        const int seen = lds.seen(nt, lane);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + t * 16 + g * 4 + i;
            bool sees = key < seen;
            if constexpr (VIEW == kWindow) sees = sees & ((key >= seen - a.view.window) | (key < a.view.n_sink));
            sc[nt][t][i] = sees ? sc[nt][t][i] * to[nt] : -INFINITY;
          }
        to[nt] = 1.0f;
      } else if (KEEP > 0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) sc[nt][t] *= to[nt];
        to[nt] = 1.0f;
      }
      top[nt] = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[nt] = fmaxf(top[nt], sc[nt][t][i]);
      top[nt] *= to[nt];
      raise |= top[nt] > r.m[nt] + kHeadroom;
    }
    if constexpr (KEEP > 0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) keep[t] = sc[0][t];
    }
    if (__ballot(raise)) {
      // The outputs are scaled in place: as other values, every register would be moved where nothing is raised (and spilled: 51 -> 41 us
      // for 128 rows x 8 heads x 32768 tokens).  The compiler does not look into these lines and puts no wait states between them and the
      // products that write and read the outputs: here they are, 20 on either side, which no product needs more of.
      asm volatile("s_nop 15\n\ts_nop 3");
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        top[nt] = quad_max(top[nt]);
        const float m_new = top[nt] > r.m[nt] + kHeadroom ? top[nt] : r.m[nt];
        const float alpha = m_new == r.m[nt] ? 1.0f : __builtin_amdgcn_exp2f(r.m[nt] - m_new);
        r.m[nt] = m_new;
        r.l[nt] *= alpha;
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x = r.acc[nt][t][i];
            asm volatile("v_mul_f32 %0, %1, %0" : "+v"(x) : "v"(alpha));
            r.acc[nt][t][i] = x;
          }
      }
      asm volatile("s_nop 15\n\ts_nop 3");
      bool far = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) far |= far_reference(r.m[nt]);
      if (__ballot(far) && seen_first != kFar) {
        seen_first = kFar;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[nt][t] *= to[nt];
          to[nt] = 1.0f;
        }
      }
    }
    f16x8 p[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float off = kLift - (r.m[nt] == -INFINITY ? 0.0f : r.m[nt]);
      f16x2 two[8];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float e[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          e[i] = __builtin_amdgcn_exp2f(sc[nt][t][i] * to[nt] + off);
          r.l[nt] += e[i];
        }
        two[2 * t] = f16x2{(_Float16)e[0], (_Float16)e[1]};
        two[2 * t + 1] = f16x2{(_Float16)e[2], (_Float16)e[3]};
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __builtin_bit_cast(uint32_t, two[4 * kk + e]);
        p[nt][kk] = __builtin_bit_cast(f16x8, w);
      }
      asm volatile("" : "+v"(r.l[nt]));                         // here and now: added up later, all the addends would have to be kept
    }
    if (key0 + kUnit > len) {
      // codes behind the last token may be anything, NaN among them
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + kk * 32 + half * 16 + g * 4 + i >= len) f.v.code[kk][half][i] = u32x2{0, 0};
    }
    if constexpr (VIEW == kWindow) {
      if (key0 < span.low_first && key0 + kUnit > a.view.n_sink) {
        // ... and so may those in front of all rows' windows
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = key0 + kk * 32 + half * 16 + g * 4 + i;
              if ((key < span.low_first) & (key >= a.view.n_sink)) f.v.code[kk][half][i] = u32x2{0, 0};
            }
      }
    }
    // V^T: dim 8 n16 + t of key pairs; two bytes of a pair lie side by side after one permutation.  With a scale that leaves
    // them fp16 numbers the values themselves are multiplied, and the sums go on where they are; else the codes, and the products
    // are scaled (a scale of NaN does not reach rows that see none of the page).
    const bool fp16 = fp16_scale<FMT>(v_scale);
    const float factor = fp16 ? v_scale : 1.0f;
#pragma unroll
    for (int t2 = 0; t2 < 4; ++t2) {                           // dims 2 t2 and 2 t2 + 1
      __builtin_amdgcn_sched_barrier(0);
      f16x8 lo[2], hi[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        u32x4 wl, wh;
#pragma unroll
        for (int e = 0; e < 4; ++e) {                          // pairs of keys
          const uint32_t x = f.v.code[kk][e >> 1][2 * (e & 1)][t2 >> 1], y = f.v.code[kk][e >> 1][2 * (e & 1) + 1][t2 >> 1];
          const uint32_t w = turned<FMT>(__builtin_amdgcn_perm(y, x, t2 & 1 ? 0x07030602u : 0x05010400u));
          wl[e] = half_codes<FMT, false>(w, factor);
          wh[e] = half_codes<FMT, true>(w, factor);
        }
        lo[kk] = __builtin_bit_cast(f16x8, wl);
        hi[kk] = __builtin_bit_cast(f16x8, wh);
      }
      if (fp16) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            r.acc[nt][2 * t2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[kk], p[nt][kk], r.acc[nt][2 * t2], 0, 0, 0);
            r.acc[nt][2 * t2 + 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[kk], p[nt][kk], r.acc[nt][2 * t2 + 1], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f}, y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            x = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo[kk], p[nt][kk], x, 0, 0, 0);
            y = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi[kk], p[nt][kk], y, 0, 0, 0);
          }
          const int seen = lds.seen(nt, lane);
          const bool sees = key0 < seen && (VIEW != kWindow || key0 + kUnit > seen - a.view.window || key0 < a.view.n_sink);
          const float scale = sees ? v_scale : 0.0f;
          r.acc[nt][2 * t2] += x * scale;
          r.acc[nt][2 * t2 + 1] += y * scale;
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_values<ONCE>(a, ahead, more, v_byte, f.v);
    f.here = ahead;
  };
  if constexpr (KEEP == 0) {
    for (int u = first; u < end; u += STEP) attend_unit(u, nullptr);
  } else {
    static_assert(NT == 1, "of one group of rows");
#pragma unroll
    for (int x = 0; x < KEEP; ++x)
      if (first + x * STEP < end) attend_unit(first + x * STEP, kept[x]);
  }
}

// The place of a row among all rows (query tokens times query heads), of rows row0 and on that read KV head h.
__device__ __forceinline__ int64_t begun_row(const CacheAttnArgs& a, int row0, int row, int h, int group) {
  const int j = row / group;
  return (int64_t(row0) + j) * a.n_q_heads + group_head(a.groups, h, row - j * group);
}

// Where a group's rows first_row .. first_row + rows - 1, a tile of it, have their results: for each of them the share that the tile begins in,
// its pieces (0: it is whole) times 256, and the row's place in the tile.
__device__ __forceinline__ void note_rows(const CacheAttnArgs& a, int row0, int n, int h, int group, int first_row, int rows, int me, int worker, int pieces) {
  if (me < rows && first_row + me < n * group)
    *reinterpret_cast<int2*>(a.begun + 2 * begun_row(a, row0, first_row + me, h, group)) = int2{worker, pieces << 8 | me};
}

// 1 / denominator of a row: 0 of one that sees nothing, so that its output is; of a head whose length cannot be, NaN.  A row that
// sees tokens and whose products are all -inf (a query that is not finite) has 1 / 0, which makes NaN of its output, its weights
// and its logarithm.
__device__ __forceinline__ float row_inverse(bool good, int sees, float sum) {
  return !good ? __uint_as_float(kNanBits) : sees > 0 ? 1.0f / sum : 0.0f;
}
__device__ __forceinline__ float row_lse(float top, float sum, float inv) {
  return (top + __builtin_amdgcn_logf(sum) - kLift) * 0.6931471805599453f + 0.0f * inv;
}

// What a workgroup of it has in LDS.
template <int NT, int WAVES>
struct AttnLds {
  RowsLds<NT> rows[WAVES == 1 ? kWaves : 1];
  float o[WAVES][16][kLdsRow];
  float m[WAVES][16 * NT], l[WAVES][16 * NT];
  int i[kWaves + kThreads];
};
// Up to 16 rows (WAVES = 1) every wave has a share of its own.  More rows are worked on 32 at a time, by all WAVES = 4 of a
// workgroup, which take turns at its share's units; their results meet in LDS, or there would be four times as many partial ones.
// (For 128 rows x 8 heads x 32768 int8 tokens 41 us, VALU work for the most part: turning the codes into fp16 for every 32 rows.
// Tiles side by side in a workgroup, to read the codes from memory once, bring nothing.)  ITEMS: no shares, a workgroup an item,
// for short caches.  PARTS: results are partial ones in any case, for a join with others.
template <int NT, int WAVES, bool ITEMS, int FMT, int VIEW = kAll, bool PARTS = false>
__device__ __forceinline__ void attend_shares(const CacheAttnArgs& a, int least, int block, int blocks, AttnLds<NT, WAVES>& lds) {
  static_assert(VIEW != kGroups || (PARTS && !ITEMS), "a row of a group has tokens of its own, too");
  constexpr bool kOwn = WAVES == 1;
  constexpr int kRows = 16 * NT, kStart = start_units(WAVES);
  static_assert(kOwn || WAVES == kWaves, "one, or all of a workgroup");
  auto& lds_rows = lds.rows;
  auto& lds_o = lds.o;
  auto &lds_m = lds.m, &lds_l = lds.l;
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  int at = 0, end = 1 << 30;
  Shares<!kOwn> shares;
  // neighbouring shares in different workgroups, on different compute units
  const int worker = kOwn ? block + wave * blocks : block;
  Item it;
  if constexpr (ITEMS) {
    const int pair = worker / uint32_t(a.tiles);
    it = {pair, scalar_load(a.c.lens + pair), worker - pair * a.tiles, 0};
  } else {
    it = locate<false, kRows, kStart, VIEW>(a, worker, blocks * (kOwn ? kWaves : 1), least, kOwn ? blocks : 1, lds.i, at, end, shares);
  }
  while (at < end) {
    // (the lane as a number of which the compiler knows nothing: what follows from it is worked out here and again at the item's end, and
    // takes no registers in between)
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    view_tokens<VIEW, true>(a, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h);
    pair_units<false, kRows, VIEW>(a, n * group, len, tiles, units);
    if (ITEMS && it.tile >= tiles) break;
    if (tiles == 0) {
      if (n > 0) it = next_pair<kStart>(a, pair);               // no query heads of this KV head
      else if (!next_sequence<kStart, VIEW>(a, s, lane, it)) break;
      continue;
    }
    const bool good = good_length(a.c, len);
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at));
    if (u1 <= u0) break;                                         // the share ends before the item's first unit
    const int first_row = it.tile * kRows, u_first = u0 + (kOwn ? 0 : wave);
    int u_end = good && len > 0 ? u1 : 0;
    // units behind what the tile's last row sees are none (a step that is a whole prompt: half of them)
    if (!kOwn && VIEW == kAll) u_end = min(u_end, (max(len - n + 1 + (min(first_row + kRows, n * group) - 1) / group, 0) + kUnit - 1) / kUnit);
    const Span span = span_of<VIEW, kRows>(a, first_row, n, group, good, len);
    int u_last = u1 - 1;
    if (VIEW == kWindow) {
      u_end = min(u_end, span.count);
      u_last = span.last(u1);
    }
    const int seen_before = VIEW == kGroups ? len : len - n + 1, seen_first = VIEW == kGroups ? len : len - n + 1 + first_row / group;
    RowsLds<NT>& rows_lds = lds_rows[kOwn ? wave : 0];           // (waves of one share write the same)
    Flight f;
    Rows<NT> r;
    const bool far = begin_rows<NT, WAVES, kOwn, VIEW>(a, pair, h, group, row0, n, first_row, seen_before, u_first, u_end, u_last, lane, rows_lds, f, r, span);
    attend<NT, WAVES, kOwn, FMT, 0, VIEW>(a, pair, len, u_first, u_end, u_last, far ? kFar : seen_first, rows_lds, lane, f, r, nullptr, span);

    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int col = tid & 15, quad = (tid & 63) >> 4;
    // a lane has dims 8 (4 quad + i) + t of rows 16 nt + col
    const bool whole = ITEMS || (u0 == 0 && u1 == units), out_row = whole && !PARTS;
    const int64_t slot_row = (2 * int64_t(worker) + (u0 == 0 ? 1 : 0)) * kRows;
    // where a partial result goes: a share's slots have room for one item that begins in it, so (PARTS) those that are whole lie by rows
    const auto part = [&](int row, int in_tile, float*& o, float*& ml) {
      const int64_t at = PARTS && whole ? begun_row(a, row0, row, h, group) : slot_row + in_tile;
      o = (PARTS && whole ? a.view.whole_o : a.part_o) + at * kHeadDim;
      ml = (PARTS && whole ? a.view.whole_ml : a.part_ml) + 2 * at;
    };
    // what a whole row has beside its output; of a length that cannot be all is NaN
    const auto row_done = [&](int j, int head, float top, float sum, float inv) {
      if (a.lse != nullptr)
        a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = row_lse(top, sum, inv);
      if (a.weight_out != nullptr)
        *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{(top == -INFINITY ? 0.0f : top) - kLift, inv};
    };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) r.l[nt] = quad_sum(r.l[nt]);
    if constexpr (kOwn) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int in_tile = nt * 16 + col, row = first_row + in_tile;
        if (row >= n * group) continue;
        if (out_row) {
          const int j = row / group, head = group_head(a.groups, h, row - j * group);
          const float inv = row_inverse(good, len - n + 1 + j, r.l[nt]);
          uint16_t* dst = a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + quad * 32;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<u32x4*>(dst + i * 8) = u32x4{pack_bf16(r.acc[nt][0][i] * inv, r.acc[nt][1][i] * inv), pack_bf16(r.acc[nt][2][i] * inv, r.acc[nt][3][i] * inv),
                                                           pack_bf16(r.acc[nt][4][i] * inv, r.acc[nt][5][i] * inv), pack_bf16(r.acc[nt][6][i] * inv, r.acc[nt][7][i] * inv)};
          if (quad == 0) row_done(j, head, r.m[nt], r.l[nt], inv);
        } else {
          float *dst, *ml;
          part(row, in_tile, dst, ml);
          dst += quad * 32;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<f32x4*>(dst + i * 8) = f32x4{r.acc[nt][0][i], r.acc[nt][1][i], r.acc[nt][2][i], r.acc[nt][3][i]};
            *reinterpret_cast<f32x4*>(dst + i * 8 + 4) = f32x4{r.acc[nt][4][i], r.acc[nt][5][i], r.acc[nt][6][i], r.acc[nt][7][i]};
          }
          if (quad == 0) *reinterpret_cast<f32x2*>(ml) = f32x2{r.m[nt], r.l[nt]};
        }
      }
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if (quad == 0) {
          lds_m[wave][nt * 16 + col] = r.m[nt];
          lds_l[wave][nt * 16 + col] = r.l[nt];
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* dst = &lds_o[wave][col][(quad * 4 + i) * 8];
          *reinterpret_cast<f32x4*>(dst) = f32x4{r.acc[nt][0][i], r.acc[nt][1][i], r.acc[nt][2][i], r.acc[nt][3][i]};
          *reinterpret_cast<f32x4*>(dst + 4) = f32x4{r.acc[nt][4][i], r.acc[nt][5][i], r.acc[nt][6][i], r.acc[nt][7][i]};
        }
        __syncthreads();
        const int in_group = tid >> 4, d = (tid & 15) * 8, in_tile = nt * 16 + in_group, row = first_row + in_tile;
        if (row < n * group) {
          float top = -INFINITY, sum = 0.0f;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) top = fmaxf(top, lds_m[w][in_tile]);
          const float ref = top == -INFINITY ? 0.0f : top;
          f32x4 o0 = {0.0f, 0.0f, 0.0f, 0.0f}, o1 = o0;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(lds_m[w][in_tile] - ref);
            sum += f * lds_l[w][in_tile];
            o0 += f * *reinterpret_cast<const f32x4*>(&lds_o[w][in_group][d]);
            o1 += f * *reinterpret_cast<const f32x4*>(&lds_o[w][in_group][d + 4]);
          }
          if (out_row) {
            const int j = row / group, head = group_head(a.groups, h, row - j * group);
            const float inv = row_inverse(good, len - n + 1 + j, sum);
            *reinterpret_cast<u32x4*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d) =
                u32x4{pack_bf16(o0.x * inv, o0.y * inv), pack_bf16(o0.z * inv, o0.w * inv), pack_bf16(o1.x * inv, o1.y * inv), pack_bf16(o1.z * inv, o1.w * inv)};
            if (d == 0) row_done(j, head, top, sum, inv);
          } else {
            float *dst, *ml;
            part(row, in_tile, dst, ml);
            dst += d;
            *reinterpret_cast<f32x4*>(dst) = o0;
            *reinterpret_cast<f32x4*>(dst + 4) = o1;
            if (d == 0) *reinterpret_cast<f32x2*>(ml) = f32x2{top, sum};
          }
        }
      }
      __syncthreads();
    }
    if (ITEMS) {
      if (PARTS && tid == 0) *reinterpret_cast<int2*>(a.begun + 2 * (int64_t(pair) * a.tiles + it.tile)) = int2{0, 0};       // whole
      break;
    }
    // for the joining kernel: pieces of the item, if it ends in another share
    if (VIEW == kGroups) {
      if (u0 == 0) note_rows(a, row0, n, h, group, first_row, kRows, kOwn ? tid & 63 : tid, worker, whole ? 0 : shares.of(at - it.unit + units - 1) - worker + 1);
    } else if (u0 == 0 && (kOwn ? (tid & 63) == 0 : tid == 0)) {
      *reinterpret_cast<int2*>(a.begun + 2 * (int64_t(pair) * a.tiles + it.tile)) = int2{worker, whole ? 0 : shares.of(at - it.unit + units - 1) - worker + 1};
    }
    at += u1 - it.unit;
    it.unit = -kStart;
    if (++it.tile == tiles) it = next_pair<kStart>(a, pair);
  }
}

template <int NT, int WAVES, bool ITEMS, int FMT, int VIEW = kAll, bool PARTS = false>
__global__ __launch_bounds__(kThreads, 2) void cache_attn_kernel(CacheAttnArgs a, int least) {
  __shared__ AttnLds<NT, WAVES> lds;
  attend_shares<NT, WAVES, ITEMS, FMT, VIEW, PARTS>(a, least, int(blockIdx.x), int(gridDim.x), lds);
}

// Joins the pieces of one row of an item: with M the largest m, out = sum 2^(m - M) O / sum 2^(m - M) l.  A workgroup a row (y)
// of an item (x), or, where there are many of few pieces, a wave (THREADS = 64, four of them in a workgroup: a grid of 32768
// rows, of which most have nothing to join, takes 8 us, 10 with a workgroup each).  The first piece lies in slot 2 w + 1 of the
// share w it begins in, the others in 2 (w + 1), 2 (w + 2) ...; groups of 32 lanes take turns at the pieces, a lane four dims,
// and what they have is added up in order.  What the first pieces hold is asked for together with the statistics.
constexpr int join_threads(int threads) { return threads > 64 ? threads : kThreads; }

template <int THREADS>
__global__ __launch_bounds__(join_threads(THREADS)) void cache_join_kernel(CacheAttnArgs a, int rows_per_tile) {
  constexpr int kGroups = THREADS / 32;
  constexpr bool kShared = THREADS > 64;       // each piece's statistics are read by one thread and shared
  __shared__ float lds_m[kShared ? kCacheMaxWorkers : 1], lds_l[kShared ? kCacheMaxWorkers : 1];
  __shared__ f32x4 lds_o[kShared ? kGroups : 1][32];
  const int tid = kShared ? threadIdx.x : threadIdx.x & 63, lane = tid & 63, d4 = tid & 31, part = tid >> 5;
  const int pair = blockIdx.x / uint32_t(a.tiles), tile = blockIdx.x - pair * a.tiles;
  const int in_tile = kShared ? int(blockIdx.y) : int(blockIdx.y) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = tile * rows_per_tile + in_tile;
  const int2 begun = *reinterpret_cast<const int2*>(a.begun + 2 * int64_t(blockIdx.x));
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, group = group_size(a.groups, h);
  int row0, n;
  step_tokens(a.t, s, row0, n);
  if (row >= n * group) return;                                  // (the item may not be one: nothing was written for it then)
  const int w = begun.x, pieces = begun.y;
  if (pieces == 0) return;                                       // it was whole
  const auto slot = [&](int x) { return 2 * int64_t(w + x) + (x == 0); };
  const auto stats = [&](int x) { return *reinterpret_cast<const f32x2*>(a.part_ml + 2 * (slot(x) * rows_per_tile + in_tile)); };
  const auto values = [&](int x) { return *reinterpret_cast<const f32x4*>(a.part_o + (slot(x) * rows_per_tile + in_tile) * kHeadDim + d4 * 4); };
  constexpr int kEarly = 4;
  f32x4 early[kEarly];
#pragma unroll
  for (int x = 0; x < kEarly; ++x) early[x] = part + kGroups * x < pieces ? values(part + kGroups * x) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float early_m[kEarly];
  f32x2 mine = {-INFINITY, 0.0f};
  if (!kShared) {
#pragma unroll
    for (int x = 0; x < kEarly; ++x) early_m[x] = part + kGroups * x < pieces ? stats(part + kGroups * x).x : -INFINITY;
    if (lane < pieces) mine = stats(lane);
  } else {
    for (int x = tid; x < pieces; x += THREADS) {
      const f32x2 ml = stats(x);
      lds_m[x] = ml.x;
      lds_l[x] = ml.y;
    }
    __syncthreads();
  }
  const auto m = [&](int x) { return kShared ? lds_m[x] : stats(x).x; };
  // every wave by itself, in the same order
  if (kShared && lane < pieces) mine = f32x2{lds_m[lane], lds_l[lane]};
  float top = mine.x;
  for (int x = lane + 64; x < pieces; x += 64) top = fmaxf(top, m(x));
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = __builtin_amdgcn_exp2f(mine.x - ref) * mine.y;
  for (int x = lane + 64; x < pieces; x += 64) sum += __builtin_amdgcn_exp2f(m(x) - ref) * (kShared ? lds_l[x] : stats(x).y);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < kEarly; ++x)
    if (part + kGroups * x < pieces) o += __builtin_amdgcn_exp2f((kShared ? lds_m[part + kGroups * x] : early_m[x]) - ref) * early[x];
#pragma unroll 8
  for (int x = part + kGroups * kEarly; x < pieces; x += kGroups) o += __builtin_amdgcn_exp2f(m(x) - ref) * values(x);
  if constexpr (!kShared) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
  } else {
    lds_o[part][d4] = o;
    __syncthreads();
  }
  if constexpr (kGroups > 8) {
    if (part < 4) {
#pragma unroll
      for (int x = 1; x < kGroups / 4; ++x) o += lds_o[part + 4 * x][d4];
    }
    __syncthreads();
    if (part < 4) lds_o[part][d4] = o;
    __syncthreads();
  }
  if (tid >= 32) return;
  if constexpr (kShared) {
#pragma unroll
    for (int x = 1; x < min(kGroups, kGroups > 8 ? 4 : 8); ++x) o += lds_o[x][d4];
  }
  const int j = row / group, head = group_head(a.groups, h, row - j * group);
  const float inv = row_inverse(true, a.c.lens[pair] - n + 1 + j, sum);     // (of a length that cannot be there are no pieces)
  *reinterpret_cast<u32x2*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d4 * 4) =
      u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
  if (tid == 0) {
    if (a.lse != nullptr) a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = row_lse(top, sum, inv);
    if (a.weight_out != nullptr)
      *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{ref - kLift, inv};
  }
}

inline void launch_join(const CacheAttnArgs& a, int rows, int most_rows, hipStream_t stream) {
  // few rows are of many pieces, many of few: 32 rows of 256 pieces (131072 tokens x 8 heads) take 6.6 us with 1024 threads
  // each, 9 with 256; 4096 rows of one to four 5.4 with 64, 7 with 256
  const dim3 all(a.c.n_seq * a.c.n_kv_heads * a.tiles, min(rows, most_rows));
  if (int64_t(all.x) * all.y <= 256) cache_join_kernel<1024><<<all, 1024, 0, stream>>>(a, rows);
  else if (int64_t(all.x) * all.y < 2048) cache_join_kernel<256><<<all, 256, 0, stream>>>(a, rows);
  else cache_join_kernel<64><<<dim3(all.x, (all.y + kThreads / 64 - 1) / (kThreads / 64)), kThreads, 0, stream>>>(a, rows);
}

// Sums over the sixteen lanes of a row of lanes, of which lane j is left with that of x[j]: every step halves the values a lane
// looks after.
__device__ __forceinline__ float sums_of_rows(float (&x)[16], int lane) {
  const auto halve = [&](auto dpp, int n, bool upper) {
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float keep = upper ? x[j + n] : x[j], give = upper ? x[j] : x[j + n];
      x[j] = keep + __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(give), decltype(dpp)::value, 0xf, 0xf, true));
    }
  };
  halve(std::integral_constant<int, 0x128>{}, 8, lane & 8);     // from lane ^ 8
  halve(std::integral_constant<int, 0x141>{}, 4, lane & 4);     // from lane ^ 7
  halve(std::integral_constant<int, 0x4e>{}, 2, lane & 2);      // from lane ^ 2
  halve(std::integral_constant<int, 0xb1>{}, 1, lane & 1);      // from lane ^ 1
  return x[0];
}

__device__ __forceinline__ int key_of_lane(int lane) { return ((lane & 15) >> 2) * 16 + (lane >> 4) * 4 + (lane & 3); }

// A head a workgroup, eight waves taking turns at its units: output, denominators and weights in one launch, without partial
// results.  For up to 16 rows and twice as many heads as there are compute units, in caches that leave a wave no more than
// kWholeUnits units, whose products stay in registers until the weights can be told (48 sequences x 4 heads of up to 2000 tokens,
// 7 rows: 21 us with the keys gone through again, 15 so).
constexpr int kWholeWaves = 8, kWholeUnits = 4;

template <bool WEIGHTS, int FMT, int VIEW = kAll>
__global__ __launch_bounds__(64 * kWholeWaves, 2) void cache_whole_kernel(CacheAttnArgs a) {
  static_assert(VIEW == kAll || (VIEW == kWindow && !WEIGHTS), "weights are those of all tokens");
  __shared__ RowsLds<1> lds;
  __shared__ float lds_o[kWholeWaves][16][kLdsRow];
  __shared__ float lds_m[kWholeWaves][16], lds_l[kWholeWaves][16], lds_ref[16], lds_inv[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, quad = lane >> 4;
  const int pair = blockIdx.x, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, len = scalar_load(a.c.lens + pair);
  const int group = group_size(a.groups, h);
  int row0, n;
  step_tokens<true>(a.t, s, row0, n);
  const bool good = good_length(a.c, len);
  // (the page table is read up to its end: what is looked up does not wait for the length)
  const int rows = n * group, seen_before = len - n + 1;
  if (rows == 0 && !WEIGHTS) return;
  const Span span = span_of<VIEW, 16>(a, 0, n, max(group, 1), good, len);
  const int units = !good ? 0 : VIEW == kWindow ? span.count : (len + kUnit - 1) / kUnit;
  const int last = VIEW == kWindow ? span.last(units) : ((a.c.max_pages << a.c.block_log2) / kUnit) - 1;
  Flight f;
  Rows<1> r;
  f32x4 kept[kWholeUnits][4];
  const int key = wave * kUnit + key_of_lane(lane);              // of the first unit, whose probabilities' sum comes to this lane
  const int64_t row_of_weights = int64_t(pair) * a.c.max_pages << a.c.block_log2;
  float old[kWholeUnits];
  // (a KV head without query heads has no rows to ask for)
  const bool far = begin_rows<1, kWholeWaves, false, VIEW>(a, pair, h, max(group, 1), row0, group > 0 ? n : 0, 0, seen_before, wave, units, last, lane, lds, f, r, span);
  if (rows > 0) {
    attend<1, kWholeWaves, false, FMT, WEIGHTS ? kWholeUnits : 0, VIEW>(a, pair, len, wave, units, last, far ? kFar : seen_before, lds, lane, f, r, kept, span);
    r.l[0] = quad_sum(r.l[0]);
    if (quad == 0) {
      lds_m[wave][n16] = r.m[0];
      lds_l[wave][n16] = r.l[0];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* dst = &lds_o[wave][n16][(quad * 4 + i) * 8];
      *reinterpret_cast<f32x4*>(dst) = f32x4{r.acc[0][0][i], r.acc[0][1][i], r.acc[0][2][i], r.acc[0][3][i]};
      *reinterpret_cast<f32x4*>(dst + 4) = f32x4{r.acc[0][4][i], r.acc[0][5][i], r.acc[0][6][i], r.acc[0][7][i]};
    }
  }
  if constexpr (WEIGHTS) {
#pragma unroll
    for (int x = 0; x < kWholeUnits; ++x) {
      const int at = key + x * kWholeWaves * kUnit;
      old[x] = a.weight_in != nullptr && at < len && good ? a.weight_in[row_of_weights + at] : 0.0f;
    }
  }
  __syncthreads();
  const int row = tid >> 5, d = (tid & 31) * 4;
  if (row < rows) {
    float top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWholeWaves; ++w) top = fmaxf(top, lds_m[w][row]);
    const float ref = top == -INFINITY ? 0.0f : top;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWholeWaves; ++w) {
      const float x = __builtin_amdgcn_exp2f(lds_m[w][row] - ref);
      sum += x * lds_l[w][row];
      o += x * *reinterpret_cast<const f32x4*>(&lds_o[w][row][d]);
    }
    const int j = row / group, head = group_head(a.groups, h, row - j * group);
    const float inv = row_inverse(good, seen_before + j, sum);
    *reinterpret_cast<u32x2*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d) =
        u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
    if (d == 0) {
      if (a.lse != nullptr)
        a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = row_lse(top, sum, inv);
      lds_ref[row] = ref - kLift;
      lds_inv[row] = inv;
    }
  }
  if constexpr (WEIGHTS) {
    __syncthreads();
    const float m = n16 < rows ? lds_ref[n16] : 0.0f, inv = n16 < rows ? lds_inv[n16] : 0.0f;
#pragma unroll
    for (int x = 0; x < kWholeUnits; ++x) {
      if (wave + x * kWholeWaves >= units) break;
      float sum = 0.0f;
      if (rows > 0) {
        float p[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(kept[x][e >> 2][e & 3] - m) * inv;
        const int key0 = (wave + x * kWholeWaves) * kUnit;
        if (key0 + kUnit > seen_before) {                        // (1 / denominator may be NaN: keys that a row does not see are none of its business)
          const int seen = lds.seen(0, lane);
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = key0 + (e >> 2) * 16 + quad * 4 + (e & 3) < seen ? p[e] : 0.0f;
        }
        sum = sums_of_rows(p, lane);
      }
      const int at = key + x * kWholeWaves * kUnit;
      if (at < len) a.weight_out[row_of_weights + at] = old[x] + sum;
    }
  }
}

}  // namespace
}  // namespace shplb
