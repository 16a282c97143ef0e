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
constexpr float kLift = 15.0f;                 // log2 of what probabilities are multiplied by
constexpr int kLdsRow = kHeadDim + 4;          // floats of a row in LDS: rows four banks apart

struct Item {                                  // a place in the list of units
  int pair, tile;
  int unit;                                    // inside the item
};

__device__ __forceinline__ int group_size(const HeadGroups& g, int h) { return g.mapped ? g.begin[h + 1] - g.begin[h] : g.group; }
__device__ __forceinline__ int group_head(const HeadGroups& g, int h, int x) { return g.mapped ? g.head[g.begin[h] + x] : h * g.group + x; }

// Tiles of rows of a pair and units of each.
template <bool WEIGHTS>
__device__ __forceinline__ void pair_units(const CacheAttnArgs& a, int pair, int rows_per_tile, int& tiles, int& units) {
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
  int row0, n;
  step_tokens(a.t, s, row0, n);
  const int len = a.c.lens[pair], rows = n * group_size(a.groups, h);
  units = good_length(a.c, len) ? (len + kUnit - 1) / kUnit : 0;
  if (WEIGHTS) {
    tiles = 1;                                 // all rows together, and keys no row looks at are copied
  } else {
    tiles = (rows + rows_per_tile - 1) / rows_per_tile;
    units = max(units, 1);                     // a head without keys has an output, too
  }
}

// The workgroup's share [begin, end) of all units, and where it begins.  Every thread adds up a run of pairs.
template <bool WEIGHTS>
__device__ __forceinline__ Item locate(const CacheAttnArgs& a, int rows_per_tile, int least, int64_t* sums, int* place,
                                       int64_t& begin, int64_t& end, int64_t& share) {
  const int pairs = a.c.n_seq * a.c.n_kv_heads, each = (pairs + kThreads - 1) / kThreads;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int first = min(tid * each, pairs), last = min(first + each, pairs);
  int64_t sum = 0;
  for (int p = first; p < last; ++p) {
    int tiles, units;
    pair_units<WEIGHTS>(a, p, rows_per_tile, tiles, units);
    sum += int64_t(tiles) * units;
  }
  const int64_t mine = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  if (lane == 63) sums[wave] = sum;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) sum += sums[w];
    total += sums[w];
  }
  share = max(int64_t(least), (total + gridDim.x - 1) / gridDim.x);
  begin = min(int64_t(blockIdx.x) * share, total);
  end = min(begin + share, total);
  int64_t left = begin - (sum - mine);
  if (begin < end && left >= 0 && left < mine) {                 // one thread
    int p = first, tiles, units;
    for (;; ++p) {
      pair_units<WEIGHTS>(a, p, rows_per_tile, tiles, units);
      if (left < int64_t(tiles) * units) break;
      left -= int64_t(tiles) * units;
    }
    place[0] = p;
    place[1] = int(left / units);
    place[2] = int(left % units);
  }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(place[0]), __builtin_amdgcn_readfirstlane(place[1]), __builtin_amdgcn_readfirstlane(place[2])};
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

// Where a unit's codes are: the page and its scales; of a page that is not in the pool the first one, with scales of NaN.
struct Page {
  const uint8_t *k, *v;
  float k_scale, v_scale;
};
__device__ __forceinline__ Page page_of(const CacheArgs& c, int pair, int unit) {
  const int at = unit * kUnit, i = at >> c.block_log2;
  int page = __builtin_amdgcn_readfirstlane(c.table[int64_t(pair) * c.max_pages + i]);
  const bool bad = page < 0 || page >= c.n_pages;
  page = bad ? 0 : page;
  const int64_t byte = ((int64_t(page) << c.block_log2) + (at & ((1 << c.block_log2) - 1))) * kHeadDim;
  const float nan = __uint_as_float(kNanBits);
  return {c.k + byte, c.v + byte, bad ? nan : c.k_scale[page], bad ? nan : c.v_scale[page]};
}

template <int NT, int FMT>
__global__ __launch_bounds__(kThreads, NT == 4 ? 1 : 2) void cache_attn_kernel(CacheAttnArgs a, int least) {
  constexpr int kRows = 16 * NT;
  __shared__ float lds_o[kWaves][16][kLdsRow];
  __shared__ float lds_m[kWaves][kRows], lds_l[kWaves][kRows];
  __shared__ int64_t sums[kWaves];
  __shared__ int place[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
  int64_t at, end, share;
  Item it = locate<false>(a, kRows, least, sums, place, at, end, share);
  int pieces = 0, begun_pair = 0, begun_tile = 0;                // the item that begins here and ends elsewhere
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens(a.t, s, row0, n);
    pair_units<false>(a, pair, kRows, tiles, units);
    if (tiles == 0) {
      it = {pair + 1, 0, 0};
      continue;
    }
    const int len = a.c.lens[pair], group = group_size(a.groups, h);
    const bool good = good_length(a.c, len);
    const int u0 = it.unit, u1 = int(min(int64_t(units), u0 + (end - at)));

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

    if (good && len > 0)
      for (int u = u0 + wave; u < u1; u += kWaves) {
        const Page page = page_of(a.c, pair, u);
        const int key0 = u * kUnit;
        u32x4 kc[4][2];
        u32x2 vc[2][2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) kc[t][x] = *reinterpret_cast<const u32x4*>(page.k + (t * 16 + n16) * kHeadDim + g * 16 + x * 64);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
          for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              vc[kk][half][i] = *reinterpret_cast<const u32x2*>(page.v + (kk * 32 + half * 16 + g * 4 + i) * kHeadDim + n16 * 8);
        if (key0 + kUnit > len) {
          // codes behind the last token may be anything, NaN among them
#pragma unroll
          for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (key0 + kk * 32 + half * 16 + g * 4 + i >= len) vc[kk][half][i] = u32x2{0, 0};
        }
        f32x4 sc[NT][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          f16x8 k0, k1, k2, k3;
          key_operands<FMT>(kc[t][0], k0, k1);
          key_operands<FMT>(kc[t][1], k2, k3);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
            x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, q[nt][0], x, 0, 0, 0);
            x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, q[nt][1], x, 0, 0, 0);
            x = __builtin_amdgcn_mfma_f32_16x16x32_f16(k2, q[nt][2], x, 0, 0, 0);
            sc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k3, q[nt][3], x, 0, 0, 0);
          }
        }
        f16x8 p[NT][2];
        float alpha[NT], v_scale[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float c = to_log2[nt] * page.k_scale;
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
          v_scale[nt] = key0 < seen[nt] ? page.v_scale : 0.0f;   // a scale of NaN does not reach rows that see none of the page
        }
        // V^T: dim 8 n16 + t of key pairs; two bytes of a pair lie side by side after one permutation
#pragma unroll
        for (int t2 = 0; t2 < 4; ++t2) {                         // dims 2 t2 and 2 t2 + 1
          f16x8 lo[2], hi[2];
#pragma unroll
          for (int kk = 0; kk < 2; ++kk) {
            u32x4 wl, wh;
#pragma unroll
            for (int e = 0; e < 4; ++e) {                        // pairs of keys
              const uint32_t x = vc[kk][e >> 1][2 * (e & 1)][t2 >> 1], y = vc[kk][e >> 1][2 * (e & 1) + 1][t2 >> 1];
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
        }
      }

    // the four waves' results become one; dims 8 (4 g + i) + t of row n16 are the lane's
    const bool whole = u0 == 0 && u1 == units;
    const int slot = 2 * int(blockIdx.x) + (u0 == 0 ? 1 : 0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] = quad_sum(l[nt]);
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
    if (!whole && u0 == 0) {
      begun_pair = pair;
      begun_tile = it.tile;
      pieces = int((at + units - 1) / share) - int(blockIdx.x) + 1;
    }
    at += u1 - u0;
    it.unit = 0;
    if (++it.tile == tiles) it = {pair + 1, 0, 0};
  }
  if (tid == 0) *reinterpret_cast<int4*>(a.pieces + 4 * blockIdx.x) = int4{pieces, begun_pair, begun_tile, 0};
}

// Joins the pieces of the item that began in workgroup blockIdx.x of the launch before: with M the largest m,
// out = sum 2^(m - M) O / sum 2^(m - M) l over them, in order.  The first one's slot is 2 w + 1, the others' 2 (w + 1), 2 (w + 2) ...
template <int NT>
__global__ __launch_bounds__(kThreads) void cache_join_kernel(CacheAttnArgs a) {
  constexpr int kRows = 16 * NT;
  const int4 begun = *reinterpret_cast<const int4*>(a.pieces + 4 * blockIdx.x);
  const int pieces = begun.x, pair = begun.y, tile = begun.z, w = blockIdx.x;
  if (pieces == 0) return;
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, group = group_size(a.groups, h);
  int row0, n;
  step_tokens(a.t, s, row0, n);
  const int d = (threadIdx.x & 15) * 8;
  for (int in_tile = threadIdx.x >> 4; in_tile < kRows; in_tile += 16) {
    const int row = tile * kRows + in_tile;
    if (row >= n * group) break;
    float top = -INFINITY, sum = 0.0f;
    for (int x = 0; x < pieces; ++x) top = fmaxf(top, a.part_ml[int64_t(2 * (w + x) + (x == 0)) * 2 * kRows + in_tile]);
    const float ref = top == -INFINITY ? 0.0f : top;
    f32x4 o0 = {0.0f, 0.0f, 0.0f, 0.0f}, o1 = o0;
    for (int x = 0; x < pieces; ++x) {
      const int64_t slot = 2 * (w + x) + (x == 0);
      const float f = __builtin_amdgcn_exp2f(a.part_ml[slot * 2 * kRows + in_tile] - ref);
      sum += f * a.part_ml[slot * 2 * kRows + kRows + in_tile];
      const float* src = a.part_o + (slot * kRows + in_tile) * kHeadDim + d;
      o0 += f * *reinterpret_cast<const f32x4*>(src);
      o1 += f * *reinterpret_cast<const f32x4*>(src + 4);
    }
    const int j = row / group, head = group_head(a.groups, h, row - j * group);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const u32x4 o = {pack_bf16(o0.x * inv, o0.y * inv), pack_bf16(o0.z * inv, o0.w * inv),
                     pack_bf16(o1.x * inv, o1.y * inv), pack_bf16(o1.z * inv, o1.w * inv)};
    *reinterpret_cast<u32x4*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d) = o;
    if (d == 0) {
      if (a.lse != nullptr) a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = (top + __builtin_amdgcn_logf(sum) - kLift) * 0.6931471805599453f;
      if (a.weight_out != nullptr)
        *reinterpret_cast<f32x2*>(a.stats + 2 * ((int64_t(row0) + j) * a.n_q_heads + head)) = f32x2{ref - kLift, inv};
    }
  }
}

// weight_out = weight_in + the probabilities that the step's rows put on each key, taken again from the keys and the rows' statistics: every
// key belongs to one wave, so nothing is added up between workgroups.
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void cache_weight_kernel(CacheAttnArgs a, int least) {
  __shared__ int64_t sums[kWaves];
  __shared__ int place[3];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
  int64_t at, end, share;
  Item it = locate<true>(a, 1, least, sums, place, at, end, share);
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    step_tokens(a.t, s, row0, n);
    pair_units<true>(a, pair, 1, tiles, units);
    if (units == 0) {
      it = {pair + 1, 0, 0};
      continue;
    }
    const int len = a.c.lens[pair], group = group_size(a.groups, h), rows = n * group;
    const int u0 = it.unit, u1 = int(min(int64_t(units), u0 + (end - at)));
    const int64_t row_of_weights = int64_t(pair) * a.c.max_pages << a.c.block_log2;
    for (int u = u0 + wave; u < u1; u += kWaves) {
      const Page page = page_of(a.c, pair, u);
      const int key0 = u * kUnit;
      f16x8 k[4][4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        u32x4 kc[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) kc[x] = *reinterpret_cast<const u32x4*>(page.k + (t * 16 + n16) * kHeadDim + g * 16 + x * 64);
        key_operands<FMT>(kc[0], k[t][0], k[t][1]);
        key_operands<FMT>(kc[1], k[t][2], k[t][3]);
      }
      f32x4 w[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) w[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      for (int r0 = 0; r0 < rows; r0 += 16) {
        f16x8 q[4];
        const int row = r0 + n16;
        const float c = load_queries(a, row0, n, h, group, row, q) * page.k_scale;
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
    at += u1 - u0;
    it = {pair + 1, 0, 0};
  }
}

template <int FMT>
int32_t launch_format(const CacheAttnArgs& a, int rows, int grid, hipStream_t stream) {
  const int least = kWaves;                    // a unit for every wave
  if (a.t.n_tokens > 0) {
    if (rows == 16) cache_attn_kernel<1, FMT><<<grid, kThreads, 0, stream>>>(a, least);
    else if (rows == 32) cache_attn_kernel<2, FMT><<<grid, kThreads, 0, stream>>>(a, least);
    else cache_attn_kernel<4, FMT><<<grid, kThreads, 0, stream>>>(a, least);
    if (rows == 16) cache_join_kernel<1><<<grid, kThreads, 0, stream>>>(a);
    else if (rows == 32) cache_join_kernel<2><<<grid, kThreads, 0, stream>>>(a);
    else cache_join_kernel<4><<<grid, kThreads, 0, stream>>>(a);
  }
  if (a.weight_out != nullptr) cache_weight_kernel<FMT><<<grid, kThreads, 0, stream>>>(a, least);
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace

int32_t cache_attn_rows(int64_t most_rows) { return most_rows <= 16 ? 16 : most_rows <= 32 ? 32 : 64; }

int32_t launch_cache_attn(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream) {
  const int rows = cache_attn_rows(most_rows);
  const int grid = min(kCacheMaxWg, compute_units * (rows == 64 ? 1 : 2));
  return a.c.format == SHPLB_CACHE_E4M3 ? launch_format<SHPLB_CACHE_E4M3>(a, rows, grid, stream)
                                        : launch_format<SHPLB_CACHE_INT8>(a, rows, grid, stream);
}

}  // namespace shplb
