// Shared by the kernels of the 8-bit key/value cache (gfx950): what the launchers take, and the two formats.
//
// A page is `block` tokens x 128 dims of one KV head, a byte a value.  Its scale is the smallest power of two 2^e, e >= -126,
// with which the largest magnitude of the page fits the format (448 in e4m3, 127 in int8).  A power of two makes value /
// scale and code * scale exact, so a code is one rounding of its value, the same whoever computes it; it costs e4m3 nothing and
// int8 at most one bit against a scale of largest / 127.  A value that is not finite has no such scale: its page's becomes NaN, and
// so does everything read from the page.
#pragma once
#include "attn_common.h"
#include "cache_span.h"

namespace shplb {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct CacheArgs {
  int32_t n_seq, n_kv_heads, max_pages, n_pages;
  int32_t block_log2;              // 6 or 7
  int32_t format;
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  const int32_t* table;
  int32_t* lens;
};

// The step's tokens: rows of Q, K, V and the output.
struct StepArgs {
  int32_t n_tokens, max_tokens;
  const int32_t* cu;
  int64_t stride_t, stride_h;
};

// The query heads of every KV head: groups of equal size, or listed head after head.
struct HeadGroups {
  int32_t mapped, group;                              // mapped = 0: KV head h has heads h * group .. + group - 1
  uint16_t begin[SHPLB_MAX_MAPPED_HEADS + 1];
  uint8_t head[SHPLB_MAX_MAPPED_HEADS];
};

// Which tokens rows see, where that is not all up to their own (see cache_attn.h).
struct CacheView {
  int32_t window, n_sink;          // at most 2^30 each
  int32_t most_units;              // of 64 tokens, that a tile of rows sees at most, and one more
  const int32_t* groups;           // [sequences of the cache + 1]
  int32_t members;                 // sequences of the step
  int32_t most_listed;             // units of all groups, beginnings and all, where no two of them overlap; below 2^30
  float *whole_o, *whole_ml;       // workspace: partial results of rows, [n_tokens][n_q_heads][128] and [2]
};

struct CacheAttnArgs {
  CacheArgs c;
  StepArgs t;                      // strides of Q and the output
  HeadGroups groups;
  int32_t n_q_heads;
  int32_t tiles;                   // of rows, of a KV head at most
  float scale_log2;                // softmax scale * log2(e)
  const uint16_t* q;
  uint16_t* out;
  float* lse;                      // or null
  const float* weight_in;          // or null
  float* weight_out;               // or null
  // workspace
  float *part_o, *part_ml;         // partial results: [2 shares][rows][128], [2 shares][rows][2]
  int32_t* begun;                  // [sequences x KV heads][tiles][2]: the share that a tile of rows begins in, its pieces (0: it is whole)
  float* stats;                    // [n_tokens][n_q_heads][2]: reference exponent and 1 / denominator, for the weights
  CacheView view;
};

// Shares of an attention launch at most: of up to 16 rows every wave's own, of more a workgroup's; and rows of partial results,
// two tiles a share.
constexpr int kCacheMaxWorkers = 2048;
constexpr int64_t kCacheSlotRows = int64_t(2) * kCacheMaxWorkers * 16;
static_assert(kCacheSlotRows >= int64_t(2) * (kCacheMaxWorkers / 4) * 32, "those of 32 rows, too");

// Units that the beginning of an item counts as at most, beside its own.
constexpr int kCacheMostStart = 8;

int32_t launch_cache_append(const CacheArgs& c, const StepArgs& t, const void* k, const void* v, hipStream_t stream);
int32_t launch_cache_load(const CacheArgs& c, const StepArgs& t, void* k, void* v, hipStream_t stream);
int32_t launch_cache_evict(const CacheArgs& src, const float* weight, const int32_t* keep, int32_t n_sink, int32_t n_recent,
                           const CacheArgs& dst, float* weight_out, int32_t* kept, void* workspace, hipStream_t stream);
int64_t cache_evict_workspace(const CacheArgs& c);
// Rows (query token, head of the group) of an item of the list that the work is divided from.
int32_t cache_attn_rows(int64_t most_rows);
int32_t launch_cache_attn_window(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream);
// Rows of an item of the list that the work on prefixes is divided from: of `pairs` prefixes and KV heads with so many rows on average and
// room for so many tokens.
int32_t prefix_attn_rows(int64_t rows, int64_t pairs, int64_t room);
// ... and rows of partial results of such items.
int64_t prefix_slot_rows(int32_t rows);
int32_t launch_cache_attn_shared(const CacheAttnArgs& own, const CacheAttnArgs& pre, int32_t most_rows, int32_t rows_pre, int32_t compute_units, hipStream_t stream);
int32_t launch_cache_attn(const CacheAttnArgs& a, int32_t most_rows, int32_t compute_units, hipStream_t stream);

// A load of what no kernel of the launch writes, at an address that is the same in all lanes: by way of the scalar cache, which leaves
// the vector loads in flight alone.
template <typename T>
__device__ __forceinline__ T scalar_load(const T* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) T*>(reinterpret_cast<uintptr_t>(p));
}

// Sums over the lanes up to and with one's own.
struct PlainSums {
  constexpr int operator()(int x, int y) const { return x + y; }
};
template <class ADD = PlainSums>
__device__ __forceinline__ int lane_sums(int x, ADD add = {}) {
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));      // from 1, 2, 4, 8 lanes below in the row of 16
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));     // the last lane of a row to the next one, of 32 to the others
  x = add(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
  return x;
}

// The rows of sequence s in this step (SCALAR: s is the same in all lanes).
template <bool SCALAR = false>
__device__ __forceinline__ void step_tokens(const StepArgs& t, int s, int& row0, int& n) {
  if (t.cu == nullptr) {
    row0 = s * t.max_tokens;
    n = t.max_tokens;
  } else {
    // (offsets that go backwards or lie outside the rows: none of a difference's operands is negative, whatever they are)
    row0 = min(max(SCALAR ? scalar_load(t.cu + s) : t.cu[s], 0), t.n_tokens);
    n = min(max(min(SCALAR ? scalar_load(t.cu + s + 1) : t.cu[s + 1], t.n_tokens), row0) - row0, t.max_tokens);
  }
}

// Whether a head's length is one that its page table row can hold.
__device__ __forceinline__ bool good_length(const CacheArgs& c, int len) { return length_fits(len, c.max_pages << c.block_log2); }

constexpr uint32_t kNanBits = 0x7fc00000u;

// Scale for a page whose largest magnitude is the float of these bits (sign clear): its bits.
template <int FMT>
__device__ __forceinline__ uint32_t scale_bits(uint32_t amax) {
  if (amax >= 0x7f800000u) return kNanBits;
  // amax = 1.m * 2^e: 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6
  const int below = FMT == SHPLB_CACHE_E4M3 ? 8 : 6;
  const uint32_t m = FMT == SHPLB_CACHE_E4M3 ? 0x600000u : 0x7e0000u;
  const int e = int(amax >> 23) - below + ((amax & 0x7fffffu) > m ? 1 : 0);
  return uint32_t(max(e, 1)) << 23;
}
// 1 / scale, exact; of NaN: 0 (codes of such a page are zeros)
__device__ __forceinline__ float inverse_scale(uint32_t bits) {
  return __uint_as_float(bits >= 0x7f800000u ? 0u : 0x7f000000u - bits);
}
// The larger of two scales; NaN stays.
__device__ __forceinline__ uint32_t larger_scale(uint32_t a, uint32_t b) {
  if ((a & 0x7fffffffu) > 0x7f800000u) return kNanBits;
  return max(int32_t(a), int32_t(b));
}

// The codes of four values times f, the inverse of their page's scale, to nearest, ties to even: the product is exact, the one
// rounding is that of the conversion, in int8 that of adding 1.5 * 2^23.  `last`: the page has the largest scale there is, at
// which codes stay at those whose values are finite (240 * 2^120 and 63 * 2^122; one step more is 2^128).
template <int FMT>
__device__ __forceinline__ bool last_scale(uint32_t scale) { return scale >= (FMT == SHPLB_CACHE_E4M3 ? 247u : 249u) << 23; }
template <int FMT>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d, float f, bool last) {
  if (last) {
    const float limit = (FMT == SHPLB_CACHE_E4M3 ? 240.0f : 63.0f) / f;
    a = __builtin_amdgcn_fmed3f(a, -limit, limit);
    b = __builtin_amdgcn_fmed3f(b, -limit, limit);
    c = __builtin_amdgcn_fmed3f(c, -limit, limit);
    d = __builtin_amdgcn_fmed3f(d, -limit, limit);
  }
  if constexpr (FMT == SHPLB_CACHE_E4M3) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c * f, d * f, __builtin_amdgcn_cvt_pk_fp8_f32(a * f, b * f, 0, false), true);
  } else {
    constexpr float kMagic = 12582912.0f;
    const uint32_t x = __float_as_uint(__builtin_fmaf(a, f, kMagic)), y = __float_as_uint(__builtin_fmaf(b, f, kMagic));
    const uint32_t z = __float_as_uint(__builtin_fmaf(c, f, kMagic)), w = __float_as_uint(__builtin_fmaf(d, f, kMagic));
    return __builtin_amdgcn_perm(y, x, 0x0c0c0400u) | __builtin_amdgcn_perm(w, z, 0x04000c0cu);
  }
}
// The largest magnitude of sixteen codes, as a number.
template <int FMT>
__device__ __forceinline__ float largest_code(u32x4 w) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  if constexpr (FMT == SHPLB_CACHE_E4M3) {
    // magnitudes are in the order of their bits
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
      const u16x2 even = __builtin_bit_cast(u16x2, w[e] & 0x007f007fu), odd = __builtin_bit_cast(u16x2, w[e] >> 8 & 0x007f007fu);
      top = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_elementwise_max(even, odd)));
    }
    const f32x2 x = __builtin_amdgcn_cvt_pk_f32_fp8(max(top & 0xffff, top >> 16), false);
    return x.x;
  } else {
    // every code in the upper byte of sixteen bits
    i16x2 most = {0, 0}, least = {0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const i16x2 odd = __builtin_bit_cast(i16x2, w[e] & 0xff00ff00u), even = __builtin_bit_cast(i16x2, w[e] << 8 & 0xff00ff00u);
      most = __builtin_elementwise_max(most, __builtin_elementwise_max(odd, even));
      least = __builtin_elementwise_min(least, __builtin_elementwise_min(odd, even));
    }
    return float(max(max(int(most.x), int(most.y)), -min(int(least.x), int(least.y))) >> 8);
  }
}
// Four codes as numbers.
template <int FMT>
__device__ __forceinline__ void from_codes(uint32_t w, float (&x)[4]) {
  if constexpr (FMT == SHPLB_CACHE_E4M3) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  } else {
    x[0] = float(int(w << 24) >> 24); x[1] = float(int(w << 16) >> 24); x[2] = float(int(w << 8) >> 24); x[3] = float(int(w) >> 24);
  }
}
// Two codes, the low or the high half of w, as fp16, times a scale that is a power of two.  Exact wherever the results are fp16 numbers
// (fp16_scale(); with 1 always).  int8 codes come with their sign bits turned (turned()): code + 128.
template <int FMT, bool HIGH>
__device__ __forceinline__ uint32_t half_codes(uint32_t w, float scale = 1.0f) {
  if constexpr (FMT == SHPLB_CACHE_E4M3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HIGH));
  } else {
    // 0x6400 | u is 1024 + u in fp16
    const uint32_t u = __builtin_amdgcn_perm(0x64646464u, w, HIGH ? 0x04030402u : 0x04010400u);
    const _Float16 f = (_Float16)scale, bias = (_Float16)(-1152.0f * scale);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, u), f16x2{f, f}, f16x2{bias, bias}));
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t turned(uint32_t w) { return FMT == SHPLB_CACHE_E4M3 ? w : w ^ 0x80808080u; }
// Whether all codes times this scale are fp16 numbers (in e4m3 448 * 2^7 and 2^-9 * 2^-15; in int8 so that the scale and 1152
// times it are, too).
template <int FMT>
__device__ __forceinline__ bool fp16_scale(float scale) {
  const uint32_t b = __float_as_uint(scale), lowest = FMT == SHPLB_CACHE_E4M3 ? 127 - 15 : 127 - 14, most = FMT == SHPLB_CACHE_E4M3 ? 127 + 7 : 127 + 5;
  return (b & 0x7fffffu) == 0 && (b >> 23) - lowest <= most - lowest;
}

}  // namespace shplb
