// Causal attention with a sliding window and first tokens that stay visible (gfx950).
//
// For a query at position p of its sequence, over the positions t <= p with t > p - window or t < n_sink:
//
//   s_t = (q . k_t) * scale * log2(e),  m a reference near max s,  l = sum 2^(s_t - m),  out = sum 2^(s_t - m) v_t / l,  lse = (m + log2 l) ln 2,
//
// in one pass over the keys.  Bound by the products: 512 FLOP for every query head and visible pair, window / (1 + 1 / G) of them for
// every byte of Q, K, V and the output.  32768 tokens x 32/8 heads with a window of 4096 take 1.87 to 2.00 ms on several cards, 1.06 to 1.13
// PFLOP/s of visible pairs, 1.09 to 1.17 of all that is multiplied (the tile loop of attn_pipe_kernel.hip reaches 1.29 at this length); 131072 with one
// of 1024 2.5 to 2.7 ms, 0.97 to 1.04 of all (18.9 key tiles an item, of which 5 have masks for some wave).  Short calls are bound by an item's chain of
// tiles: 777 tokens x 32 heads, a window of 256, 12 us.
//
// Split.  A work item is a tile of 64 QG queries of one head; it goes through the 64-key tiles that any of its queries sees: those
// of the first tokens, then those of the window (tile u of the item is key tile u below `sinks`, u + skip from there on).  Items cost
// about the same, so there are no queues: an item is a workgroup, longer sequences first.  Of every lap of two workgroups a compute
// unit a die (workgroup b is on die b % 8) has a run of neighbouring items, which share heads and most of a window in its L2.  (Workgroups that
// stay and take an item of every lap, the next one's first tiles on their way behind the last one's results: 2720 us for 131072 tokens x
// 32 heads with a window of 1024, 2630 so; 48 sequences of up to 2000 tokens 151 and 139: their times differ by 12 to 44%.)
//
// Tile.  That of attn_pipe_kernel.hip: four waves of 16 QG queries, S^T = K Q^T and O^T = V^T P^T in 16x16x32 products, K and V copied
// from memory to two LDS stages each, softmax of a tile in front of the next tile's first product and its own second one.  Beside it:
//  - tiles that all queries of a wave see whole have no masks (a wave that leaves out the products of those of which its queries see
//    nothing: 1 to 3% slower, the tile lasts as long as the other waves' part);
//  - a query may see nothing of the first tiles: its reference is -infinity until it does, and is then raised at once;
//  - denominators are sums of the fp32 probabilities (products use them rounded to bf16, as V is), so that lse keeps fp32's precision:
//    sums of the rounded ones, two at a time, are 2 to 3% faster, and 2^-9 off;
//  - a value that is infinite or NaN must not reach queries that do not see it, to which a product would carry it as 0 * NaN.  Tiles
//    with masks are looked through for such values, and where there are some, they are counted apart, but only once an item has come out
//    with a sum that is not finite, as it does whenever there are some; it is then worked on again.  (Looked through at once: 777 tokens
//    13.7 us, 13.1 so, 48 sequences 132 and 127.)
//  - a reference is a rounded product, a probability's exponent a multiply-add: from references of 2^31 on the two can differ by 128, and
//    probabilities be infinite or all 0.  An item with a reference of 2^22 or more is worked on again, too, with products rounded alike.
#include <algorithm>

#include "attn_common.h"

namespace shplb {
namespace {

struct WindowArgs {
  const uint16_t *q, *k, *v;
  uint16_t* out;
  float* lse;                                // or null
  Strides st;
  int64_t total_tokens;
  float scale_log2;
  int32_t window, n_sink;                    // at most 2^30 each
  int32_t n_seq, n_q_heads, items;
  int32_t group;                             // query heads per KV head; 0: kv_of names them
  int32_t lap;                               // workgroups that are on the device together
  int32_t tok_begin[SHPLB_MAX_SEQ], len[SHPLB_MAX_SEQ];         // of the sequences, longer ones first
  int32_t tile_begin[SHPLB_MAX_SEQ + 1];     // tiles of queries in front of each sequence
  uint32_t kv_of[SHPLB_MAX_MAPPED_HEADS / 4];
};

constexpr int kKeys = 64, kTileBytes = kKeys * kRowBytes, kWaves = 4, kThreads = 64 * kWaves;

struct WindowItem {                          // all the same in all lanes
  int head, kv_head, seq_begin, len, q0;
  int sinks, skip, tiles;                    // key tiles: see above; at least two (one behind all that is visible does no harm)
  __device__ __forceinline__ int key0(int u) const { return kKeys * (u < sinks ? u : u + skip); }
};

template <int BQ>
__device__ __forceinline__ WindowItem window_item(const WindowArgs& a, int place) {
  WindowItem it;
  const auto scalar = [](int x) { return int(__builtin_amdgcn_readfirstlane(x)); };
  int t0 = 0, t1 = a.tile_begin[1];
  it.seq_begin = a.tok_begin[0];
  it.len = a.len[0];
  if (a.n_seq > 1) {
    const int lane = threadIdx.x & 63, s = __builtin_popcountll(__ballot(lane < a.n_seq - 1 && place >= a.tile_begin[lane + 1] * a.n_q_heads));
    t0 = scalar(a.tile_begin[s]);
    t1 = scalar(a.tile_begin[s + 1]);
    it.seq_begin = scalar(a.tok_begin[s]);
    it.len = scalar(a.len[s]);
  }
  const int nt = t1 - t0, local = place - t0 * a.n_q_heads;
  const int group = a.group > 0 ? a.group : 1;
  const int run = scalar(uint32_t(local) / uint32_t(nt * group)), rest = local - run * nt * group;     // heads that share keys, tile by tile
  const int nth = scalar(uint32_t(rest) / uint32_t(group)), tile = nt - 1 - nth;
  it.head = run * group + rest - nth * group;
  it.kv_head = a.group > 0 ? run : scalar(int(a.kv_of[it.head >> 2] >> (8 * (it.head & 3)) & 0xff));
  it.q0 = tile * BQ;
  const int hi = min(it.q0 + BQ, it.len), lo = max(it.q0 - a.window + 1, 0);
  const int end = (hi + kKeys - 1) / kKeys, first = lo / kKeys;
  it.sinks = min((min(a.n_sink, hi) + kKeys - 1) / kKeys, end);
  it.skip = max(first - it.sinks, 0);
  it.tiles = max(end - it.skip, 2);
  return it;
}

// A pointer that is the same in all lanes, said explicitly: in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char*>(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x)))) |
                                       uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x >> 32)))) << 32);
}

// One item; whether it is to be worked on again, CAREFUL: a sum came out that is not finite, or a reference that is far out.  Then values that
// are not finite are told apart from zeros by what sees them, and scores are rounded as references are.
// lds: two stages of K, two of V; s_bad: -1.
template <int QG, bool CAREFUL>
__device__ __forceinline__ bool attend_item(const WindowArgs& a, const WindowItem& it, char* lds, int& s_bad) {
  constexpr int BQ = 64 * QG, MT = kKeys / 16, kQK = 4 * MT, kPV = 8 * (kKeys / 32);
  constexpr int kLook = 8;                   // LDS operands are fetched so far ahead
  // a lane's 16 probabilities of a query and tile can only sum to more if one of them exceeds 2^8
  constexpr float kSumLimit = 4.0f * MT * 256.0f;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, hi = lane >> 4, q_wave = 16 * QG * wave;
  const int64_t row_bytes = a.st.kv_t * 2;

  // copies: a wave moves four rows at a time, row 16 r + cp_row of the tile in round r, 16-byte chunk c of it to slot c ^ swz(row)
  const int cp_row = 4 * wave + (lane >> 4);
  const uint32_t cp_chunk = ((lane & 15) ^ swz(cp_row)) << 4, cp_off = uint32_t(cp_row) * uint32_t(row_bytes) + cp_chunk;
  // K operands: lane (n, hi) reads row 16 mt + n, chunk 4 ks + hi; V's by transpose reads (see attn_pipe_kernel.hip)
  const int k_rd0 = n * kRowBytes + ((hi ^ swz(n)) << 4);
  const int tr_row = 4 * hi + ((lane >> 2) & 3), tr_a = lane & 3;
  const int v_rd0 = tr_row * kRowBytes + (((tr_a >> 1) ^ swz(tr_row)) << 4) + 8 * (tr_a & 1);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_offset_of(lds) + 4 * wave * kRowBytes);

  const auto copy_tile = [&](const uint16_t* base, int u, uint32_t dst) {
    const int at = min(it.key0(u), it.len - 1), last = it.len - 1 - at;
    const char* tile = uniform(reinterpret_cast<const char*>(base + int64_t(it.kv_head) * a.st.kv_h) + (int64_t(it.seq_begin) + at) * row_bytes);
    dst = __builtin_amdgcn_readfirstlane(dst);
    if (last >= kKeys - 1) {
#pragma unroll
      for (int r = 0; r < 4; ++r) copy_g2l_16(tile + int64_t(16 * r) * row_bytes, cp_off, dst + 16 * r * kRowBytes);
    } else {                                 // rows behind the end: the last token again (masked)
#pragma unroll
      for (int r = 0; r < 4; ++r) copy_g2l_16(tile, uint32_t(min(16 * r + cp_row, last)) * uint32_t(row_bytes) + cp_chunk, dst + 16 * r * kRowBytes);
    }
  };
  const auto copy_k = [&](int u, int stage) { copy_tile(a.k, u, lds0 + stage * kTileBytes); };
  const auto copy_v = [&](int u, int stage) { copy_tile(a.v, u, lds0 + (2 + stage) * kTileBytes); };
  // the first tiles and the queries (operand B: dims 32 ks + 8 hi and on of query 16 qg + n)
  copy_k(0, 0);
  bf16x8 qf[QG][4];
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int tok = it.seq_begin + min(it.q0 + q_wave + 16 * qg + n, it.len - 1);
    const uint16_t* src = a.q + int64_t(tok) * a.st.q_t + int64_t(it.head) * a.st.q_h + 8 * hi;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) qf[qg][ks] = *reinterpret_cast<const bf16x8*>(src + 32 * ks);
  }
  __builtin_amdgcn_sched_barrier(0);
  copy_v(0, 0);
  copy_k(1, 1);
  __builtin_amdgcn_sched_barrier(0);

  int u = 0;                                 // the tile; tile u is in stage u mod 2
  f32x4 sc[QG][MT], acc[QG][8];
  float m_ref[QG], l_run[QG];
  const float to_log2 = CAREFUL ? 1.0f : a.scale_log2;           // what scores are multiplied by beside their reference
  int q_pos[QG];                           // (queries behind the end of the sequence: the last one again)
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    q_pos[qg] = min(it.q0 + q_wave + 16 * qg + n, it.len - 1);
    m_ref[qg] = -INFINITY;
    l_run[qg] = 0.0f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) acc[qg][dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // positions of the tile's first and last query, and of the wave's
  const int first = it.q0, last = min(it.q0 + BQ, it.len) - 1;
  const int w_first = min(first + q_wave, last), w_last = min(first + q_wave + 16 * QG - 1, last);
  const auto masked = [&](int key0, int lo, int up) { return key0 + kKeys - 1 > lo || (key0 <= up - a.window && key0 + kKeys > a.n_sink); };
  const auto hidden = [&](int key0) { return key0 > w_last || (key0 + kKeys - 1 <= w_first - a.window && key0 >= a.n_sink); };

  const auto read_k = [&](const char* kt, int gi) {
    const int ks = gi / MT, mt = gi % MT;
    return *reinterpret_cast<const bf16x8*>(kt + (k_rd0 ^ (ks << 6)) + mt * 16 * kRowBytes);
  };
  const auto read_v = [&](const char* vt, int gi) {
    const int gq = gi >> 3, dt = gi & 7;
    const char* at = vt + (v_rd0 ^ (dt << 5)) + gq * 32 * kRowBytes;
    const s16x4 lo = lds_read_tr16(at), up = lds_read_tr16(at + 16 * kRowBytes);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const auto tile_max = [&](int qg) {
    float mx = sc[qg][0][0];
#pragma unroll
    for (int x = 1; x < 4 * MT; ++x) mx = fmaxf(mx, sc[qg][x >> 2][x & 3]);
    return mx;
  };
  typedef bf16x8 Operands[kQK];
  static_assert(kPV == kQK, "as many for either product");
  const auto first_k = [&](const char* kt, Operands& kf) {
#pragma unroll
    for (int gi = 0; gi < kLook; ++gi) kf[gi] = read_k(kt, gi);
  };
  const auto first_v = [&](const char* vt, Operands& vf) {
#pragma unroll
    for (int gi = 0; gi < kLook; ++gi) vf[gi] = read_v(vt, gi);
  };
  // scores of a tile, the first operands being there; vt: the first ones of its values are fetched behind the last, into vf
  const auto products_k = [&](const char* kt, Operands& kf, const char* vt, Operands* vf) {
#pragma unroll
    for (int gi = 0; gi < kQK; ++gi) {
      if (gi + kLook < kQK) kf[gi + kLook] = read_k(kt, gi + kLook);
      else if (vf != nullptr) (*vf)[gi + kLook - kQK] = read_v(vt, gi + kLook - kQK);
#pragma unroll
      for (int qg = 0; qg < QG; ++qg)
        sc[qg][gi % MT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[gi], qf[qg][gi / MT], gi < MT ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : sc[qg][gi % MT], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto mask_scores = [&](int key0) {
    const auto mask = [&](auto sinks_c) {
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) {
        int back = q_pos[qg] - key0 - 4 * hi, left = a.n_sink - key0 - 4 * hi;       // how far back a key lies; first tokens from it on
        asm volatile("" : "+v"(back), "+v"(left));
#pragma unroll
        for (int x = 0; x < 4 * MT; ++x) {
          const int at = 16 * (x >> 2) + (x & 3);
          bool sees = uint32_t(back - at) < uint32_t(a.window);
          if constexpr (decltype(sinks_c)::value) sees = sees | ((back >= at) & (left > at));
          sc[qg][x >> 2][x & 3] = sees ? sc[qg][x >> 2][x & 3] : -INFINITY;
          if ((x & 3) == 3) asm volatile("" : "+v"(sc[qg][x >> 2]));
        }
      }
    };
    if (key0 < a.n_sink) mask(std::true_type{});
    else mask(std::false_type{});
  };
  const auto scores = [&](const char* kt, int key0) {
    Operands kf;
    first_k(kt, kf);
    products_k(kt, kf, nullptr, nullptr);
    if (masked(key0, w_first, w_last)) mask_scores(key0);
  };

  // ---- S(0)
  wait_vmem_but(std::integral_constant<int, 8>{});             // K(0) and the queries; V(0) and K(1) are under way
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) asm volatile("" : "+v"(qf[qg][0]), "+v"(qf[qg][1]), "+v"(qf[qg][2]), "+v"(qf[qg][3]));
  __syncthreads();
  if (!CAREFUL || !hidden(it.key0(0))) scores(lds, it.key0(0));

  // One tile.  plain: it is not the last one, and (CAREFUL) all queries see all of it.
  const auto step = [&](auto plain_c) __attribute__((always_inline)) {
    constexpr bool kPlain = decltype(plain_c)::value;
    const int key0 = it.key0(u), key1 = it.key0(u + 1);
    const bool ends = !kPlain && u + 1 == it.tiles, mine = kPlain || !hidden(key0), checked = CAREFUL && !kPlain && masked(key0, first, last);
    const int stage = u & 1;
    const char* const vt = lds + (2 + stage) * kTileBytes;
    const char* const kt = lds + (stage ^ 1) * kTileBytes;
    Operands kf, vf;
    __builtin_amdgcn_s_setprio(0);
    wait_vmem_all();                       // own copies of K(u + 1), V(u) have landed ...
    __syncthreads();                       // ... and everyone's; the stages of K(u) and V(u - 1) are free
    if constexpr (kPlain) {
      first_k(kt, kf);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!ends) {
      copy_v(u + 1, stage ^ 1);
      if (u + 2 < it.tiles) copy_k(u + 2, stage);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (checked) {
      // whether all values are finite, a quarter of them looked at by each wave
      typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
      u16x2 top[4] = {};
#pragma unroll
      for (int x = 0; x < kTileBytes / (16 * kThreads); ++x) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(vt + (x * kThreads + tid) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) top[e] = __builtin_elementwise_max(top[e], __builtin_bit_cast(u16x2, w[e] & 0x7fff7fffu));
      }
      const u16x2 most = __builtin_elementwise_max(__builtin_elementwise_max(top[0], top[1]), __builtin_elementwise_max(top[2], top[3]));
      if (__ballot(max(most.x, most.y) >= 0x7f80) != 0 && lane == 0) s_bad = u;
    }

    // ---- probabilities of tile u
    uint32_t pk[QG][MT][2];
    float rs[QG];
    const auto probabilities = [&]() {
      float sum[QG][2];
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) sum[qg][0] = sum[qg][1] = 0.0f;
#pragma unroll
      for (int x = 0; x < 2 * QG * MT; ++x) {       // two probabilities of a query group, the groups in turn
        const int qg = x % QG, mt = x / (2 * QG), c = x / QG % 2;
        const float m_use = m_ref[qg] == -INFINITY ? 0.0f : m_ref[qg];
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qg][mt][2 * c], to_log2, -m_use));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[qg][mt][2 * c + 1], to_log2, -m_use));
        pk[qg][mt][c] = pack_bf16(p0, p1);
        sum[qg][0] += p0;
        sum[qg][1] += p1;
      }
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) rs[qg] = sum[qg][0] + sum[qg][1];
    };
    if (mine) {
      if constexpr (CAREFUL) {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            sc[qg][mt] *= a.scale_log2;
            asm volatile("" : "+v"(sc[qg][mt]));               // rounded: not part of a multiply-add
          }
      }
      probabilities();
      // The reference was fixed by earlier tiles: it is too low for this one where a probability, and with it the sum, came out
      // large, or where there was none.  Then it is raised to the tile's maximum.
      const auto too_low = [&](int qg) { return !(rs[qg] <= kSumLimit) || m_ref[qg] == -INFINITY; };
      if (__any(too_low(0) || too_low(QG - 1))) {
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) {
          const float m_tile = quad_max(tile_max(qg)) * to_log2;
          const float m_new = fmaxf(m_ref[qg], m_tile);
          const float alpha = m_new == m_ref[qg] ? 1.0f : __builtin_amdgcn_exp2f(m_ref[qg] - m_new);
          m_ref[qg] = m_new;
          l_run[qg] *= alpha;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) acc[qg][dt] *= alpha;
        }
        probabilities();
      }
#pragma unroll
      for (int qg = 0; qg < QG; ++qg) l_run[qg] += rs[qg];
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- S(u + 1)
    __builtin_amdgcn_s_setprio(1);
    if constexpr (kPlain) {
      products_k(kt, kf, vt, &vf);
      if (masked(key1, w_first, w_last)) mask_scores(key1);
    } else if (!ends && !hidden(key1)) scores(kt, key1);

    // ---- O^T += V(u)^T P(u)^T
    if (checked) {
      __syncthreads();
      if (s_bad == u) {
        // Values that are not finite are counted for each query among the keys that it sees, those that are +infinity or NaN and those
        // that are -infinity or NaN, and are zeros for the products.
        if (mine) {
          u32x4 seen[QG][2];
#pragma unroll
          for (int qg = 0; qg < QG; ++qg) {
            int d = key0 + 4 * hi - q_pos[qg], e = key0 + 4 * hi - a.n_sink;
            asm volatile("" : "+v"(d), "+v"(e));
#pragma unroll
            for (int x = 0; x < 2 * MT; ++x) {
              const auto one = [&](int key) { return (d + key <= 0) & ((d + key > -a.window) | (e + key < 0)) ? 0x3f80u : 0u; };
              const int key = 16 * (x >> 1) + 2 * (x & 1);
              seen[qg][x >> 2][x & 3] = one(key) | one(key + 1) << 16;
            }
          }
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) {
            f32x4 up[QG], down[QG];
#pragma unroll
            for (int qg = 0; qg < QG; ++qg) up[qg] = down[qg] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int gq = 0; gq < 2; ++gq) {
              const u32x4 w = __builtin_bit_cast(u32x4, read_v(vt, 8 * gq + dt));
              u32x4 pos, neg;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t lo = w[e] & 0xffffu, hi16 = w[e] >> 16;
                const bool lo_bad = (lo & 0x7f80u) == 0x7f80u, hi_bad = (hi16 & 0x7f80u) == 0x7f80u;
                pos[e] = (lo_bad & (lo != 0xff80u) ? 0x3f80u : 0u) | (hi_bad & (hi16 != 0xff80u) ? 0x3f800000u : 0u);
                neg[e] = (lo_bad & (lo != 0x7f80u) ? 0x3f80u : 0u) | (hi_bad & (hi16 != 0x7f80u) ? 0x3f800000u : 0u);
              }
#pragma unroll
              for (int qg = 0; qg < QG; ++qg) {
                up[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, pos), __builtin_bit_cast(bf16x8, seen[qg][gq]), up[qg], 0, 0, 0);
                down[qg] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, neg), __builtin_bit_cast(bf16x8, seen[qg][gq]), down[qg], 0, 0, 0);
              }
            }
#pragma unroll
            for (int qg = 0; qg < QG; ++qg)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const float x = up[qg][r] > 0.0f ? INFINITY : 0.0f;
                acc[qg][dt][r] += down[qg][r] > 0.0f ? x - INFINITY : x;
              }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kTileBytes / (4 * kThreads); ++x) {
          uint32_t* const at = reinterpret_cast<uint32_t*>(lds + (2 + stage) * kTileBytes) + x * kThreads + threadIdx.x;
          const uint32_t w = *at, lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu, up = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
          *at = lo | up;
        }
        __syncthreads();
      }
    }
    if (mine) {
      if constexpr (!kPlain) first_v(vt, vf);
#pragma unroll
      for (int gi = 0; gi < kPV; ++gi) {
        if (gi + kLook < kPV) vf[gi + kLook] = read_v(vt, gi + kLook);
        const int gq = gi >> 3, dt = gi & 7;
#pragma unroll
        for (int qg = 0; qg < QG; ++qg) {
          const u32x4 w = {pk[qg][2 * gq][0], pk[qg][2 * gq][1], pk[qg][2 * gq + 1][0], pk[qg][2 * gq + 1][1]};
          acc[qg][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[gi], __builtin_bit_cast(bf16x8, w), acc[qg][dt], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    ++u;
  };
  const auto plain = [&]() { return u + 1 < it.tiles && (!CAREFUL || !masked(it.key0(u), first, last)); };
#pragma unroll 1
  while (u < it.tiles) {
#pragma unroll 1
    while (plain()) step(std::true_type{});
    step(std::false_type{});               // (the last tile is never plain)
  }
  __builtin_amdgcn_s_setprio(0);
  bool again = false;
  if constexpr (!CAREFUL) {
    float odd = 0.0f;                        // NaN if there is such a sum
#pragma unroll
    for (int x = 0; x < 32 * QG; ++x) odd = __builtin_fmaf(acc[x >> 5][x >> 2 & 7][x & 3], 0.0f, odd);
    again = odd != 0.0f;
#pragma unroll
    for (int qg = 0; qg < QG; ++qg) again |= fabsf(m_ref[qg]) >= 0x1p22f;
  }

  // ---- out: a lane has dims 16 dt + 4 hi + r of its queries; neighbours trade, and a lane stores eight dims at a time
  const int n_valid = it.len - it.q0;
#pragma unroll
  for (int qg = 0; qg < QG; ++qg) {
    const int q_at = q_wave + 16 * qg + n;
    const bool valid = q_at < n_valid;
    const float l = quad_sum(l_run[qg]), inv = 1.0f / l;
    const int64_t tok = int64_t(it.seq_begin) + it.q0 + min(q_at, n_valid - 1);
    if (a.lse != nullptr && hi == 0 && valid) a.lse[int64_t(it.head) * a.total_tokens + tok] = (m_ref[qg] + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
    uint16_t* dst = a.out + tok * a.st.q_t + int64_t(it.head) * a.st.q_h + 16 * (hi & 1) + 8 * (hi >> 1);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const f32x4 &x = acc[qg][2 * p], &y = acc[qg][2 * p + 1];
      uint32_t e0 = pack_bf16(x[0] * inv, x[1] * inv), e1 = pack_bf16(x[2] * inv, x[3] * inv);
      uint32_t o0 = pack_bf16(y[0] * inv, y[1] * inv), o1 = pack_bf16(y[2] * inv, y[3] * inv);
      swap_rows(e0, o0);
      swap_rows(e1, o1);
      if (valid) *reinterpret_cast<u32x4*>(dst + 32 * p) = u32x4{e0, e1, o0, o1};
    }
  }
  return __ballot(again) != 0;
}

// QG: groups of 16 queries of a wave.
template <int QG>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void window_attn_kernel(WindowArgs a) {
  __shared__ __attribute__((aligned(1024))) char lds[4 * kTileBytes];
  __shared__ int s_bad, s_again;             // the last step whose values are not all finite; whether the item is worked on again
  if (threadIdx.x == 0) {
    s_bad = -1;
    s_again = 0;
  }
  const int in_lap = int(uint32_t(blockIdx.x) % uint32_t(a.lap)), place = int(blockIdx.x) - in_lap + in_lap % kXcds * (a.lap / kXcds) + in_lap / kXcds;
  if (place >= a.items) return;
  const WindowItem it = window_item<64 * QG>(a, place);
  if (attend_item<QG, false>(a, it, lds, s_bad) && threadIdx.x % 64 == 0) s_again = 1;
  __syncthreads();
  if (s_again != 0) attend_item<QG, true>(a, it, lds, s_bad);      // (and writes the outputs again)
}

}  // namespace

int32_t launch_window_attn(const Geometry& g, int32_t n_sink, int32_t window, const void* q, const void* k, const void* v, void* out, float* lse, int32_t compute_units,
                           hipStream_t stream) {
  WindowArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.st = g.st;
  a.total_tokens = g.total_tokens;
  a.scale_log2 = g.scale * 1.4426950408889634f;
  a.window = window < 1 << 30 ? window : 1 << 30;
  a.n_sink = n_sink < 1 << 30 ? n_sink : 1 << 30;
  a.n_seq = g.meta.n_seq;
  a.n_q_heads = g.meta.n_q_heads;
  a.group = g.meta.kv_map ? 0 : g.meta.n_q_heads / g.meta.n_kv_heads;
  for (int x = 0; x < SHPLB_MAX_MAPPED_HEADS / 4; ++x) a.kv_of[x] = g.meta.kv_of[x];
  int order[SHPLB_MAX_SEQ];
  const auto length = [&](int s) { return g.meta.tok_begin[s + 1] - g.meta.tok_begin[s]; };
  for (int s = 0; s < a.n_seq; ++s) order[s] = s;
  std::stable_sort(order, order + a.n_seq, [&](int x, int y) { return length(x) > length(y); });
  const auto deal = [&](int rows) {
    int64_t tiles = 0;
    for (int s = 0; s < a.n_seq; ++s) {
      a.tok_begin[s] = g.meta.tok_begin[order[s]];
      a.len[s] = length(order[s]);
      a.tile_begin[s] = int32_t(tiles);
      tiles += (int64_t(a.len[s]) + rows - 1) / rows;
    }
    a.tile_begin[a.n_seq] = int32_t(tiles);
    return tiles * a.n_q_heads;
  };
  int64_t items = deal(128);
  const bool half = items <= compute_units;
  if (half) items = deal(64);
  a.items = int32_t(items);                                      // (at most 2^30: make_geometry())
  const int64_t most = int64_t(2) * compute_units / kXcds * kXcds;
  a.lap = int32_t(items < most ? (items + kXcds - 1) / kXcds * kXcds : most);
  const uint32_t grid = uint32_t((items + a.lap - 1) / a.lap * a.lap);
  if (half) window_attn_kernel<1><<<grid, kThreads, 0, stream>>>(a);
  else window_attn_kernel<2><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError() == hipSuccess ? SHPLB_OK : SHPLB_E_HIP;
}

}  // namespace shplb
