// Attention over the 8-bit cache that sees part of it, or more than it: windows with first tokens that stay visible, and prefixes that
// sequences share.  The kernels that attend are in cache_attn.h; here are their launches, and the join of what a row has from its
// prefix and from its own tokens.
#include "cache_attn.h"

namespace shplb {
namespace {

// ---- windows.  A step's work does not grow with the context: a head has the units of its window and of its first tokens, and how the
// work is divided follows from them like that of cache_attn_kernel.hip from a table's room.  Bound by reading with few rows (128 sequences
// x 8 heads, a window of 4096: 148 us, 5.7 TB/s of what is seen), by VALU work with many (codes to fp16 for every 32 rows: 8 sequences x 32 tokens x 28/4
// int8 heads, a window of 2000: 27 to 30 us).  128 rows at a time, as prefixes below have them, are 40 there, and 15 to 70% slower in smaller
// calls: windows are short, and an item of 128 rows has too few of their units to pay for its beginning.
template <int FMT>
int32_t launch_window(const CacheAttnArgs& a, int rows, int most_rows, int compute_units, hipStream_t stream) {
  const int grid = min(kCacheMaxWorkers / kWaves, compute_units * 2), pairs = a.c.n_seq * a.c.n_kv_heads;
  const int64_t most = min(int64_t(a.c.max_pages) << a.c.block_log2, int64_t(a.view.most_units) * kUnit);
  constexpr int kShort = kWholeWaves * kWholeUnits * kUnit;
  // More rows: a workgroup a tile of them, without shares and joining, where a tile's chain of units costs less than that: always up to 2048 tokens; up to
  // 2560 from a tile for every other compute unit on (a window of 2000, 32 new tokens of a sequence: 256 tiles 28 us, 39 in shares, 128 24 and 26, 32 of
  // them 23 and 20); up to 4608 from two for every compute unit on (a window of 4000: 512 tiles 84 and 92, 1024 160 and 174; 256 46 and 57, but 38 and 34
  // if lengths are from 100 on); beyond, shares (of 8000: 512 tiles 165 and 169, 320 128 and 110).
  const int64_t items = int64_t(pairs) * a.tiles;
  const bool whole_tiles = most <= kShort || (most <= kShort * 5 / 4 && items >= compute_units / 2) || (most <= kShort * 9 / 4 && items >= 2 * compute_units);
  if (rows == 16 && pairs <= 2 * compute_units && most <= kShort) {
    cache_whole_kernel<false, FMT, kWindow><<<pairs, 64 * kWholeWaves, 0, stream>>>(a);
  } else if (rows > 16 && whole_tiles) {
    cache_attn_kernel<2, kWaves, true, FMT, kWindow><<<uint32_t(items), kThreads, 0, stream>>>(a, 0);
  } else {
    if (rows == 16) cache_attn_kernel<1, 1, false, FMT, kWindow><<<grid, kThreads, 0, stream>>>(a, 3);
    else cache_attn_kernel<2, kWaves, false, FMT, kWindow><<<grid, kThreads, 0, stream>>>(a, kWaves);
    launch_join(a, rows, most_rows, stream);
  }
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

// ---- shared prefixes.  The rows of all sequences that share a prefix are rows of one item: its keys are read once for many of them.
// Prefixes and own tokens are attended to in one launch or two, either divided like the cache of cache_attn_kernel.hip; all results are
// partial ones, which a last launch joins.  Prefixes are bound by the products and what feeds them (of 512 rows x 8 heads x 32768 tokens
// the units take 65 us, 1.05 PFLOP/s, and 22 go to beginnings, results and the last shares' wait), own tokens by reading.

// Rows of a prefix's item.  Up to 48 of them are worked on like those of a cache, 16 or 32 at a time: codes come from memory
// into registers, and are turned to fp16 for each tile by itself.  More rows: 128 at a time, 32 of each wave, whose workgroup turns the
// codes of 64 keys to fp16 once, in LDS, while the products of the last ones are done; the tile is that of window_attn_kernel.hip, in
// fp16.  (Its 256 registers are not enough for an item's beginning and end: 33 are spilled there, none in the loop over units.)
constexpr int kPrefixRows = 128, kPrefixStart = 4;

struct PrefixLds {
  char k[2][kUnit * kRowBytes], v[2][kUnit * kRowBytes];        // keys and values of two units in fp16: chunk c of row r in slot c ^ swz(r)
  int i[kWaves + kThreads];
};

template <int FMT>
__device__ __forceinline__ void prefix_shares(const CacheAttnArgs& a, int least, int block, int blocks, PrefixLds& lds) {
  constexpr int NT = 2, MT = kUnit / 16, kQK = 4 * MT, kPV = 8 * (kUnit / 32), kLook = 8;
  // a lane has sixteen probabilities of a row and unit: with this sum none is more than fp16 holds
  constexpr float kSumLimit = 60000.0f;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, hi = lane >> 4;
  int at, end;
  Shares<true> shares;
  Item it = locate<false, kPrefixRows, kPrefixStart, kGroups>(a, block, blocks, least, 1, lds.i, at, end, shares);
  // operands in LDS, as in window_attn_kernel.hip; a thread brings eight codes of rows tid / 16 + 16 x, one chunk each
  const int k_rd0 = n16 * kRowBytes + ((hi ^ swz(n16)) << 4);
  const int tr_row = 4 * hi + ((lane >> 2) & 3), tr_a = lane & 3;
  const int v_rd0 = tr_row * kRowBytes + (((tr_a >> 1) ^ swz(tr_row)) << 4) + 8 * (tr_a & 1);
  const int wr = (tid >> 4) * kRowBytes + (((tid & 15) ^ swz(tid >> 4)) << 4);
  struct Codes {
    u32x2 x[4];
  };
  while (at < end) {
    const int pair = it.pair, s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads;
    int row0, n, tiles, units;
    view_tokens<kGroups, true>(a, s, row0, n);
    const int len = it.len, group = group_size(a.groups, h), rows = n * group;
    pair_units<false, kPrefixRows, kGroups>(a, rows, len, tiles, units);
    if (tiles == 0) {
      if (n > 0) it = next_pair<kPrefixStart>(a, pair);
      else if (!next_sequence<kPrefixStart, kGroups>(a, s, lane, it)) break;
      continue;
    }
    const int u0 = max(it.unit, 0), u1 = min(units, it.unit + (end - at));
    if (u1 <= u0) break;
    const int u_end = good_length(a.c, len) && len > 0 ? u1 : u0, first_row = it.tile * kPrefixRows, my_row = first_row + wave * 32;
    const bool mine = my_row < rows;                             // whether the wave has rows

    // The queries are on their way while pages are looked up.
    Query q[2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int row = my_row + nt * 16 + n16;
#pragma unroll
      for (int x = 0; x < 4; ++x) q[nt].part[x] = u32x4{0, 0, 0, 0};
      if (row < rows) {
        const int j = row / group, head = group_head(a.groups, h, row - j * group);
        const uint16_t* src = a.q + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + 8 * hi;
#pragma unroll
        for (int x = 0; x < 4; ++x) q[nt].part[x] = *reinterpret_cast<const u32x4*>(src + 32 * x);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    // The pages of 64 places of the table on, a lane each.  (One by one by scalar loads the waits for LDS operands would be waits for them, too.)
    int looked_up = 0, page_here = 0;
    float k_here = 0.0f, v_here = 0.0f;
    const auto look_up = [&](int first) {
      looked_up = first;
      const int place = min(first + lane, (u1 - 1) * kUnit >> a.c.block_log2);
      const int page = a.c.table[int64_t(pair) * a.c.max_pages + place];
      const bool bad = page < 0 || page >= a.c.n_pages;
      page_here = bad ? -1 : page;
      k_here = a.c.k_scale[max(page_here, 0)];
      v_here = a.c.v_scale[max(page_here, 0)];
    };
    const auto place_of = [&](int u) { return (min(u, u1 - 1) * kUnit >> a.c.block_log2) - looked_up; };
    // where a unit's codes are; its scales are asked for while it is on its way, and are there later
    struct Codes8 {
      int64_t byte;
      bool bad;
    };
    const auto page_of = [&](int u) {
      if (place_of(u) >= 64) look_up(looked_up + place_of(u));
      const int page = __builtin_amdgcn_readlane(page_here, place_of(u));
      return Codes8{((int64_t(max(page, 0)) << a.c.block_log2) + (min(u, u1 - 1) * kUnit & ((1 << a.c.block_log2) - 1))) * kHeadDim, page < 0};
    };
    struct Scales {
      float k, v;
    };
    const auto scales_of = [&](int u, bool bad) {                // (of a unit whose page was the last one asked for, or one before it)
      const auto lane_value = [&](float y) { return bad ? __uint_as_float(kNanBits) : __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(y), place_of(u))); };
      return Scales{lane_value(k_here), lane_value(v_here)};
    };
    look_up(u0 * kUnit >> a.c.block_log2);
    const auto ask = [&](const uint8_t* base, const Codes8& page, bool there, Codes& c) {
      const SlotBuffer b = unit_buffer(base, page.byte, there && !page.bad);
#pragma unroll
      for (int x = 0; x < 4; ++x) c.x[x] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, tid * 8, x * 16 * kHeadDim, 0));
    };
    const auto put_keys = [&](const Codes& c, int stage) {
#pragma unroll
      for (int x = 0; x < 4; ++x) *reinterpret_cast<f16x8*>(lds.k[stage] + wr + x * 16 * kRowBytes) = key_operand<FMT>(c.x[x][0], c.x[x][1]);
    };
    // values with their scale, where that leaves fp16 numbers of them
    const auto put_values = [&](Codes& c, int key0, float scale, int stage) {
      if (key0 + kUnit > len) {                                  // codes behind the last token may be anything
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (key0 + (tid >> 4) + 16 * x >= len) c.x[x] = u32x2{0, 0};
      }
      const float f = fp16_scale<FMT>(scale) ? scale : 1.0f;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const uint32_t p = turned<FMT>(c.x[x][0]), q = turned<FMT>(c.x[x][1]);
        *reinterpret_cast<u32x4*>(lds.v[stage] + wr + x * 16 * kRowBytes) =
            u32x4{half_codes<FMT, false>(p, f), half_codes<FMT, true>(p, f), half_codes<FMT, false>(q, f), half_codes<FMT, true>(q, f)};
      }
    };

    // ---- the first units
    const Codes8 p0 = page_of(u0);
    Codes8 p1 = page_of(u0 + 1), p2 = page_of(u0 + 2);           // of units u + 1 and u + 2
    Codes kc, vc, k_first;
    ask(a.c.k, p0, u0 < u_end, k_first);
    ask(a.c.k, p1, u0 + 1 < u_end, kc);
    ask(a.c.v, p0, u0 < u_end, vc);
    f16x8 qf[NT][4];
    float to_log2[NT], m[NT], l[NT];
    f32x4 acc[NT][8], sc[NT][MT];
    bool far_lane = false;
    {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        to_log2[nt] = query_operands(a, q[nt], qf[nt]);
        far_lane |= far_row(to_log2[nt]);
        m[nt] = -INFINITY;
        l[nt] = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[nt][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    bool far = __ballot(far_lane) != 0;

    const auto read_k = [&](const char* kt, int gi) {
      const int ks = gi / MT, mt = gi % MT;
      return *reinterpret_cast<const f16x8*>(kt + (k_rd0 ^ (ks << 6)) + mt * 16 * kRowBytes);
    };
    const auto read_v = [&](const char* vt, int gi) {
      const int gq = gi >> 3, dt = gi & 7;
      const char* from = vt + (v_rd0 ^ (dt << 5)) + gq * 32 * kRowBytes;
      const s16x4 lo = lds_read_tr16(from), up = lds_read_tr16(from + 16 * kRowBytes);
      return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto next_scores = [&](const char* kt) {
      f16x8 kf[kQK];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sc[nt][mt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int gi = 0; gi < kLook; ++gi) kf[gi] = read_k(kt, gi);
#pragma unroll
      for (int gi = 0; gi < kQK; ++gi) {
        if (gi + kLook < kQK) kf[gi + kLook] = read_k(kt, gi + kLook);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[nt][gi % MT] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[gi], qf[nt][gi / MT], sc[nt][gi % MT], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    };

    __syncthreads();                                             // the stages are free
    put_keys(k_first, 0);
    __syncthreads();
    if (mine && u0 < u_end) next_scores(lds.k[0]);
    put_keys(kc, 1);
    Scales s0 = scales_of(u0, p0.bad), s1 = scales_of(u0 + 1, p1.bad);         // of units u and u + 1
    put_values(vc, u0 * kUnit, s0.v, 0);
    ask(a.c.k, p2, u0 + 2 < u_end, kc);
    ask(a.c.v, p1, u0 + 1 < u_end, vc);
    int stage = 0;                                               // of unit u
    int u = u0;
    // One unit.  scaled: its values are codes, and what they add is multiplied by the page's scale.
    const auto step = [&](auto scaled_c) __attribute__((always_inline)) {
      constexpr bool kScaled = decltype(scaled_c)::value;
      const int key0 = u * kUnit;
      const float k_scale = s0.k, v_scale = s0.v;
      const Scales s2 = scales_of(u + 2, p2.bad);
      const Codes8 p3 = page_of(u + 3);
      __builtin_amdgcn_s_setprio(0);
      __syncthreads();                       // keys of u + 1 and values of u are there; the stages of keys of u and values of u - 1 are free
      f16x2 pk[NT][MT][2];
      if (mine) {
        float to[NT], rs[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) to[nt] = to_log2[nt] * k_scale;
        if (far || key0 + kUnit > len) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const bool apart = far && to[nt] == INFINITY;
            const float first = apart ? to_log2[nt] : to[nt], second = apart ? k_scale : 1.0f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
              for (int r = 0; r < 4; ++r) sc[nt][mt][r] = key0 + 16 * mt + 4 * hi + r < len ? sc[nt][mt][r] * first * second : -INFINITY;
            to[nt] = 1.0f;
          }
        }
        const auto probabilities = [&]() {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const float off = kLift - (m[nt] == -INFINITY ? 0.0f : m[nt]);
            float sum[2] = {0.0f, 0.0f};
#pragma unroll
            for (int x = 0; x < 2 * MT; ++x) {
              const int mt = x >> 1, c = x & 1;
              const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][mt][2 * c], to[nt], off));
              const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[nt][mt][2 * c + 1], to[nt], off));
              pk[nt][mt][c] = f16x2{(_Float16)e0, (_Float16)e1};
              sum[0] += e0;
              sum[1] += e1;
            }
            rs[nt] = sum[0] + sum[1];
          }
        };
        probabilities();
        // the reference is raised where a probability may be too large, or where there is none yet
        const auto too_low = [&](int nt) { return !(rs[nt] <= kSumLimit) || m[nt] == -INFINITY; };
        if (__any(too_low(0) || too_low(NT - 1))) {
          bool raised_far = false;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float top = sc[nt][0][0];
#pragma unroll
            for (int x = 1; x < 4 * MT; ++x) top = fmaxf(top, sc[nt][x >> 2][x & 3]);
            top = quad_max(top * to[nt]);
            const float m_new = fmaxf(m[nt], top), alpha = m_new == m[nt] ? 1.0f : __builtin_amdgcn_exp2f(m[nt] - m_new);
            m[nt] = m_new;
            l[nt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) acc[nt][dt] *= alpha;
            raised_far |= far_reference(m_new);
          }
          if (!far && __ballot(raised_far)) {
            far = true;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) sc[nt][mt] *= to[nt];
              to[nt] = 1.0f;
            }
          }
          probabilities();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) l[nt] += rs[nt];
      }
      __builtin_amdgcn_sched_barrier(0);
      // the codes that are there go into the free stages, and the next ones are asked for
      put_keys(kc, stage);
      put_values(vc, key0 + kUnit, s1.v, stage ^ 1);
      ask(a.c.k, p3, u + 3 < u_end, kc);
      ask(a.c.v, p2, u + 2 < u_end, vc);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
      if (mine) {
        if (u + 1 < u_end) next_scores(lds.k[stage ^ 1]);
        const char* const vt = lds.v[stage];
        const auto p_of = [&](int nt, int gq) {
          return __builtin_bit_cast(f16x8, u32x4{__builtin_bit_cast(uint32_t, pk[nt][2 * gq][0]), __builtin_bit_cast(uint32_t, pk[nt][2 * gq][1]),
                                                 __builtin_bit_cast(uint32_t, pk[nt][2 * gq + 1][0]), __builtin_bit_cast(uint32_t, pk[nt][2 * gq + 1][1])});
        };
        if constexpr (!kScaled) {
          f16x8 vf[kPV];
#pragma unroll
          for (int gi = 0; gi < kLook; ++gi) vf[gi] = read_v(vt, gi);
#pragma unroll
          for (int gi = 0; gi < kPV; ++gi) {
            if (gi + kLook < kPV) vf[gi + kLook] = read_v(vt, gi + kLook);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][gi & 7] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[gi], p_of(nt, gi >> 3), acc[nt][gi & 7], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        } else {
          const float scale = fp16_scale<FMT>(v_scale) ? 1.0f : v_scale;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int gq = 0; gq < 2; ++gq) x = __builtin_amdgcn_mfma_f32_16x16x32_f16(read_v(vt, 8 * gq + dt), p_of(nt, gq), x, 0, 0, 0);
              acc[nt][dt] += x * scale;
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      stage ^= 1;
      s0 = s1;
      s1 = s2;
      p1 = p2;
      p2 = p3;
      ++u;
    };
    // From the first page on whose scale does not leave fp16 numbers of its values, units go by a loop of their own: in one with the other's
    // products the output's registers would be moved.
    while (u < u_end && fp16_scale<FMT>(s0.v)) step(std::false_type{});
#pragma unroll 1
    while (u < u_end) step(std::true_type{});
    __builtin_amdgcn_s_setprio(0);

    // ---- partial results: a lane has dims 16 dt + 4 hi and on of its rows
    const bool whole = u0 == 0 && u1 == units;
    if (mine) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int row = my_row + nt * 16 + n16;
        const float sum = quad_sum(l[nt]);
        if (row >= rows) continue;
        const int64_t slot = whole ? begun_row(a, row0, row, h, group) : (2 * int64_t(block) + (u0 == 0)) * kPrefixRows + (row - first_row);
        float* o = (whole ? a.view.whole_o : a.part_o) + slot * kHeadDim + 4 * hi;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<f32x4*>(o + 16 * dt) = acc[nt][dt];
        if (hi == 0) *reinterpret_cast<f32x2*>((whole ? a.view.whole_ml : a.part_ml) + 2 * slot) = f32x2{m[nt], sum};
      }
    }
    if (u0 == 0) note_rows(a, row0, n, h, group, first_row, kPrefixRows, tid, block, whole ? 0 : shares.of(at - it.unit + units - 1) - block + 1);
    at += u1 - it.unit;
    it.unit = -kPrefixStart;
    if (++it.tile == tiles) it = next_pair<kPrefixStart>(a, pair);
  }
}

template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void prefix_kernel(CacheAttnArgs a) {
  __shared__ __attribute__((aligned(1024))) PrefixLds lds;
  prefix_shares<FMT>(a, 4, int(blockIdx.x), int(gridDim.x), lds);
}

// Both in one launch: every other workgroup of a die attends to the prefixes.  Workgroup b goes to die b % 8, there to shader engine
// (b / 8) % 4 in turn, whether it is free or not, and there to the eight compute units in turn: of two neighbours on a die there is one of
// either kind, every engine has the kinds in turn, and so has every compute unit.
template <int ROWS, int FMT, int VIEW>
__device__ __forceinline__ void attend_rows(const CacheAttnArgs& a, int block, int blocks, AttnLds<ROWS / 16, ROWS == 16 ? 1 : kWaves>& lds) {
  attend_shares<ROWS / 16, ROWS == 16 ? 1 : kWaves, false, FMT, VIEW, true>(a, ROWS == 16 ? 3 : kWaves, block, blocks, lds);
}
template <int ROWS, int OWN, int FMT>
__global__ __launch_bounds__(kThreads, 2) void shared_attn_kernel(CacheAttnArgs a, CacheAttnArgs pre) {
  __shared__ union {
    AttnLds<OWN / 16, OWN == 16 ? 1 : kWaves> own;
    AttnLds<ROWS / 16, ROWS == 16 ? 1 : kWaves> pre;
  } lds;
  const int b = int(blockIdx.x), blocks = int(gridDim.x) / 2, block = b / (2 * kXcds) * kXcds + b % kXcds, on_die = b / kXcds;
  if ((on_die + on_die / 4 + on_die / 32) % 2 == 0) attend_rows<ROWS, FMT, kGroups>(pre, block, blocks, lds.pre);
  else attend_rows<OWN, FMT, kAll>(a, block, blocks, lds.own);
}

// Prefixes 128 rows at a time, and behind them, where a workgroup has ended, own tokens of drafts: neither waits for the other's last shares.
template <int FMT>
__global__ __launch_bounds__(kThreads, 2) void shared_wide_kernel(CacheAttnArgs a, CacheAttnArgs pre) {
  __shared__ __attribute__((aligned(1024))) union Lds {
    AttnLds<2, kWaves> own;
    PrefixLds pre;
  } lds;
  const int b = int(blockIdx.x), blocks = int(gridDim.x) / 2;
  if (b < blocks) prefix_shares<FMT>(pre, 4, b, blocks, lds.pre);
  else attend_rows<32, FMT, kAll>(a, b - blocks, blocks, lds.own);
}

// Joins a row's pieces, those of its prefix and those of its own tokens: with M the largest m, out = sum 2^(m - M) O / sum 2^(m -
// M) l.  A workgroup a row (y) of an item (x) of own tokens, or, where there are many, a wave (THREADS = 64, four of them in a
// workgroup); groups of 32 lanes take turns at the pieces, a lane four dims, and what they have is added up in order.  Where the
// pieces are is noted by rows, so that all that has to be known of them comes in one go.
template <int THREADS>
__global__ __launch_bounds__(join_threads(THREADS)) void shared_join_kernel(CacheAttnArgs a, CacheAttnArgs pre, int rows_own, int rows_pre, int shares_pre) {
  constexpr int kParts = THREADS / 32, kMost = 2 * kCacheMaxWorkers;
  constexpr bool kShared = THREADS > 64;       // each piece's statistics are read by one thread and shared
  __shared__ float lds_m[kShared ? kMost : 1], lds_l[kShared ? kMost : 1];
  __shared__ f32x4 lds_o[kShared ? kParts : 1][32];
  const int tid = kShared ? threadIdx.x : threadIdx.x & 63, lane = tid & 63, d4 = tid & 31, part = tid >> 5;
  const int pair = blockIdx.x / uint32_t(a.tiles), tile = blockIdx.x - pair * a.tiles;
  const int in_tile = kShared ? int(blockIdx.y) : int(blockIdx.y) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = tile * rows_own + in_tile;
  const int s = pair / a.c.n_kv_heads, h = pair - s * a.c.n_kv_heads, group = group_size(a.groups, h);
  int row0, n;
  step_tokens<true>(a.t, s, row0, n);
  const int2 own = *reinterpret_cast<const int2*>(a.begun + 2 * int64_t(blockIdx.x));
  const int len = scalar_load(a.c.lens + pair);
  const auto holds = [&](int x) { return x < pre.c.n_seq && pre.view.groups[min(x, pre.c.n_seq - 1)] <= s && s < pre.view.groups[min(x, pre.c.n_seq - 1) + 1]; };
  const bool some = holds(lane);
  if (in_tile >= rows_own || row >= n * group) return;           // (the item may not be one: nothing was written for it then)
  const int j = row / group, i = row - j * group, head = group_head(a.groups, h, i);
  const int64_t by_row = (int64_t(row0) + j) * a.n_q_heads + head;
  const int2 front = *reinterpret_cast<const int2*>(pre.begun + 2 * by_row);
  // the prefix: the first one whose run of sequences holds this one
  uint64_t here = __ballot(some);
  int g = here ? int(__builtin_ctzll(here)) : -1;
  for (int g0 = 64; g0 < pre.c.n_seq && g < 0; g0 += 64) {
    here = __ballot(holds(g0 + lane));
    if (here) g = g0 + int(__builtin_ctzll(here));
  }
  // (What a row notes that is outside of its prefix's rows, as offsets that go backwards have it, is nothing that was written for it: it
  // is not followed out of the slots, and the row is NaN.)
  const int front_pieces = min(max(front.y >> 8, 0), shares_pre), front_begin = min(max(front.x, 0), shares_pre - front_pieces);
  const int64_t front_row = min(front.y & 255, rows_pre - 1);
  const int n_own = max(own.y, 1), pieces = n_own + (g >= 0 ? max(front_pieces, 1) : 0);
  const auto place = [&](int x, const float*& o, const float*& ml) {
    const int y = x - n_own;
    const bool mine = y < 0, whole = mine ? own.y == 0 : front_pieces == 0;
    const int64_t slot = mine ? (2 * int64_t(own.x + x) + (x == 0)) * rows_own + in_tile : (2 * int64_t(front_begin + y) + (y == 0)) * rows_pre + front_row;
    const int64_t at = whole ? by_row : slot;
    o = (mine ? whole ? a.view.whole_o : a.part_o : whole ? pre.view.whole_o : pre.part_o) + at * kHeadDim;
    ml = (mine ? whole ? a.view.whole_ml : a.part_ml : whole ? pre.view.whole_ml : pre.part_ml) + 2 * at;
  };
  const auto stats = [&](int x) {
    const float *o, *ml;
    place(x, o, ml);
    return *reinterpret_cast<const f32x2*>(ml);
  };
  const auto values = [&](int x) {
    const float *o, *ml;
    place(x, o, ml);
    return *reinterpret_cast<const f32x4*>(o + d4 * 4);
  };
  // (a wave that has a row for itself asks for 32 pieces at once: prefixes of 8192 tokens that 64 sequences share, 20 pieces a row, 73 us, 76 with sixteen)
  constexpr int kEarly = kShared ? 4 : 16;
  f32x4 early[kEarly];
#pragma unroll
  for (int x = 0; x < kEarly; ++x) early[x] = part + kParts * x < pieces ? values(part + kParts * x) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  f32x2 mine = {-INFINITY, 0.0f};
  if (!kShared) {
    if (lane < pieces) mine = stats(lane);
  } else {
    for (int x = tid; x < pieces; x += THREADS) {
      const f32x2 ml = stats(x);
      lds_m[x] = ml.x;
      lds_l[x] = ml.y;
    }
  }
  bool good = good_length(a.c, len);
  int prefix_len = 0;
  if (g >= 0) {
    int first, tokens;
    view_tokens<kGroups, true>(pre, g, first, tokens);
    prefix_len = scalar_load(pre.c.lens + int64_t(g) * pre.c.n_kv_heads + h);
    const int t = row0 + j - first;
    good = good && good_length(pre.c, prefix_len) && t >= 0 && t < tokens;
  }
  // every wave by itself, in the same order
  if (kShared) {
    __syncthreads();
    if (lane < pieces) mine = f32x2{lds_m[lane], lds_l[lane]};
  }
  const auto again = [&](int x) { return kShared ? f32x2{lds_m[x], lds_l[x]} : stats(x); };
  float top = mine.x;
  for (int x = lane + 64; x < pieces; x += 64) top = fmaxf(top, again(x).x);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float ref = top == -INFINITY ? 0.0f : top;
  const float my_factor = __builtin_amdgcn_exp2f(mine.x - ref);
  float sum = my_factor * mine.y;
  for (int x = lane + 64; x < pieces; x += 64) {
    const f32x2 ml = again(x);
    sum += __builtin_amdgcn_exp2f(ml.x - ref) * ml.y;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int x = 0; x < kEarly; ++x) {
    const int at = part + kParts * x;
    const float f = kShared ? __builtin_amdgcn_exp2f(lds_m[at] - ref) : __shfl(my_factor, at);
    if (at < pieces) o += f * early[x];
  }
#pragma unroll 8
  for (int x = part + kParts * kEarly; x < pieces; x += kParts) o += __builtin_amdgcn_exp2f(again(x).x - ref) * values(x);
  if constexpr (!kShared) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
  } else {
    lds_o[part][d4] = o;
    __syncthreads();
  }
  if constexpr (kParts > 8) {
    if (part < 4) {
#pragma unroll
      for (int x = 1; x < kParts / 4; ++x) o += lds_o[part + 4 * x][d4];
    }
    __syncthreads();
    if (part < 4) lds_o[part][d4] = o;
    __syncthreads();
  }
  if (tid >= 32) return;
  if constexpr (kShared) {
#pragma unroll
    for (int x = 1; x < min(kParts, kParts > 8 ? 4 : 8); ++x) o += lds_o[x][d4];
  }
  const float inv = row_inverse(good, max(len - n + 1 + j, 0) + prefix_len, sum);
  *reinterpret_cast<u32x2*>(a.out + (int64_t(row0) + j) * a.t.stride_t + head * a.t.stride_h + d4 * 4) =
      u32x2{pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv)};
  if (tid == 0 && a.lse != nullptr) a.lse[int64_t(head) * a.t.n_tokens + row0 + j] = row_lse(top, sum, inv);
}

}  // namespace

int32_t launch_cache_attn_window(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream) {
  const int rows = cache_attn_rows(most_rows);
  return a.c.format == SHPLB_CACHE_E4M3 ? launch_window<SHPLB_CACHE_E4M3>(a, rows, most_rows, compute_units, stream)
                                        : launch_window<SHPLB_CACHE_INT8>(a, rows, most_rows, compute_units, stream);
}

int32_t prefix_attn_rows(int64_t rows, int64_t pairs, int64_t room) {
  // 128 at a time from more than 48 rows and 6144 units on, reckoned in tiles of 32 rows: 128 rows x 8 heads of 16000 tokens 44 us either way, of 4000
  // 36 and 31 with 32 at a time; 256 rows 55 and 62, 44 and 38; 64 rows of 16000 37.6 and 35.5, of 32768 44 and 56
  if (rows <= 16) return 16;
  return rows <= 48 || pairs * ((rows + 31) / 32) * ((room + kUnit - 1) / kUnit) < 6144 ? 32 : kPrefixRows;
}
int64_t prefix_slot_rows(int32_t rows) { return rows == kPrefixRows ? int64_t(2) * (kCacheMaxWorkers / kWaves) * kPrefixRows : kCacheSlotRows; }

int32_t launch_cache_attn_shared(const CacheAttnArgs& own, const CacheAttnArgs& pre, int32_t most_rows, int32_t rows_pre, int32_t compute_units, hipStream_t stream) {
  const int grid = min(kCacheMaxWorkers / kWaves, compute_units * 2), rows = cache_attn_rows(most_rows);
  // Small calls, by what the tables have room for, go in one launch: four sequences behind 2048 tokens x 8 heads 15 us, 23 in two launches (14 and 20
  // later, the second with a table that has room for 131072 tokens, be it the prefix's or the sequences'),
  // 8 prefixes of 8192 tokens with four of 1500 each 70 and 71, 32 of 4096 154 and 138.
  const auto units = [](const CacheAttnArgs& a, int64_t tiles) { return a.c.n_kv_heads * tiles * (((int64_t(a.c.max_pages) << a.c.block_log2) + kUnit - 1) / kUnit); };
  const int64_t most_heads = own.t.max_tokens > 0 ? most_rows / own.t.max_tokens : 1;
  const bool apart = units(pre, int64_t(own.t.n_tokens) * most_heads / rows_pre + pre.c.n_seq) + units(own, int64_t(own.c.n_seq) * own.tiles) >= 16384;
  // Own tokens of more than 16 rows: a workgroup a tile of rows where tables have room for 1024 tokens (64 sequences x 5 new tokens, up to 700 held, behind
  // 8000 91 us, 98 in shares; 16 with room for 2048 57 and 54); else, behind prefixes of 128 rows, in one launch with these (64 with room for 2048 97 us,
  // 101 in two, 32 of them 62 and 71; with up to 16 rows, one token each, 75 and 73).
  const bool own_items = rows > 16 && int64_t(own.c.max_pages) << own.c.block_log2 <= kWholeWaves * kWholeUnits * kUnit / 2;
  const auto launch_own = [&](auto fmt_c) {
    constexpr int FMT = decltype(fmt_c)::value;
    if (rows == 16) cache_attn_kernel<1, 1, false, FMT, kAll, true><<<grid, kThreads, 0, stream>>>(own, 3);
    else if (own_items)
      cache_attn_kernel<2, kWaves, true, FMT, kAll, true><<<uint32_t(own.c.n_seq * own.c.n_kv_heads) * own.tiles, kThreads, 0, stream>>>(own, 0);
    else cache_attn_kernel<2, kWaves, false, FMT, kAll, true><<<grid, kThreads, 0, stream>>>(own, kWaves);
  };
  const auto launch = [&](auto fmt_c) {
    constexpr int FMT = decltype(fmt_c)::value;
    if (rows_pre == kPrefixRows) {
      if (rows > 16 && !own_items) {
        shared_wide_kernel<FMT><<<2 * grid, kThreads, 0, stream>>>(own, pre);
        return;
      }
      prefix_kernel<FMT><<<grid, kThreads, 0, stream>>>(pre);
      launch_own(std::integral_constant<int, FMT>{});
    } else if (apart) {
      if (rows_pre == 16) cache_attn_kernel<1, 1, false, FMT, kGroups, true><<<grid, kThreads, 0, stream>>>(pre, 3);
      else cache_attn_kernel<2, kWaves, false, FMT, kGroups, true><<<grid, kThreads, 0, stream>>>(pre, kWaves);
      launch_own(std::integral_constant<int, FMT>{});
    } else if (rows_pre == 16) {
      if (rows == 16) shared_attn_kernel<16, 16, FMT><<<2 * grid, kThreads, 0, stream>>>(own, pre);
      else shared_attn_kernel<16, 32, FMT><<<2 * grid, kThreads, 0, stream>>>(own, pre);
    } else {
      if (rows == 16) shared_attn_kernel<32, 16, FMT><<<2 * grid, kThreads, 0, stream>>>(own, pre);
      else shared_attn_kernel<32, 32, FMT><<<2 * grid, kThreads, 0, stream>>>(own, pre);
    }
  };
  if (own.c.format == SHPLB_CACHE_E4M3) launch(std::integral_constant<int, SHPLB_CACHE_E4M3>{});
  else launch(std::integral_constant<int, SHPLB_CACHE_INT8>{});
  const int shares_pre = int(prefix_slot_rows(rows_pre) / (2 * rows_pre));      // that there are slots for
  const dim3 all(uint32_t(own.c.n_seq * own.c.n_kv_heads) * own.tiles, min(rows, most_rows));
  if (int64_t(all.x) * all.y <= 256) shared_join_kernel<1024><<<all, 1024, 0, stream>>>(own, pre, rows, rows_pre, shares_pre);
  else if (int64_t(all.x) * all.y < 2048) shared_join_kernel<256><<<all, 256, 0, stream>>>(own, pre, rows, rows_pre, shares_pre);
  else shared_join_kernel<64><<<dim3(all.x, (all.y + kWaves - 1) / kWaves), kThreads, 0, stream>>>(own, pre, rows, rows_pre, shares_pre);
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace shplb
