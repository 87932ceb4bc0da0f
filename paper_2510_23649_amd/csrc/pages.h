// Device helpers of the paged K/V cache: where a position lies, and rows held in 8 bits.
#pragma once

#include <type_traits>

#include "lrqk_device.h"
#include "lrqk_internal.h"

namespace lrqk {

int check_pages(const lrqk_pages_shape* s);
// K, V, the scales that the type needs, table, start and kv_len: given and aligned.
bool pages_given(const lrqk_pages_shape& s, const lrqk_pages* p);

namespace pages {

constexpr int kScaleBlock = 32;               // elements of a row that share a scale
constexpr int kScales = kD / kScaleBlock;     // scale bytes of a row
constexpr int kMinExp = -110;                 // smallest scale 2^e (include/lrqk.h)

__host__ __device__ constexpr bool is8(int page_dtype) {
  return page_dtype == LRQK_PAGE_E4M3 || page_dtype == LRQK_PAGE_I8;
}
__host__ __device__ constexpr int page_elem_bytes(int page_dtype) {
  return page_dtype == LRQK_PAGE_F32 ? 4 : page_dtype == LRQK_PAGE_BF16 ? 2 : 1;
}

// The shape and the tables as the kernels take them.
struct Map {
  const int32_t* table;
  const int32_t* start;
  const int32_t* kv_len;
  int B, Hkv, T, l_max, n_pages, max_pages, page_log2;
};
inline Map make_map(const lrqk_pages_shape& s, const lrqk_pages& p) {
  return Map{p.table, p.start, p.kv_len, s.B,         s.Hkv,
             s.T,     s.l_max, s.n_pages, s.max_pages, __builtin_ctz((unsigned)s.page)};
}

// Sequence b: its packed rows [first, first + n) and its length; position of row first + i: len - n + i.
struct Seq {
  int first, n, len;
};
__device__ __forceinline__ Seq sequence(const Map& m, int b) {
  Seq q;
  q.first = min(max(m.start[b], 0), m.T);
  q.n = min(max(m.start[b + 1], q.first), m.T) - q.first;
  q.len = max(m.kv_len[b], 0);
  return q;
}

// Row (of d elements) of position p in [0, l_max) of sequence b for KV head kvh, or -1: no page.
__device__ __forceinline__ int64_t row_of(const Map& m, int b, int kvh, int p) {
  const int pg = m.table[(size_t)b * m.max_pages + (p >> m.page_log2)];
  if ((unsigned)pg >= (unsigned)m.n_pages) return -1;
  return ((((int64_t)pg * m.Hkv + kvh) << m.page_log2) + (p & ((1 << m.page_log2) - 1)));
}

// 2^(byte - 127); 255: NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  const uint32_t x = max(byte << 23, 0x00400000u);
  return __uint_as_float(byte == 255u ? 0x7fc00000u : x);
}

// Eight codes (two dwords) times their scale, in fp32 (exact).
template <int PAGE>
__device__ __forceinline__ void decode8(uint2 c, float s, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t w = i ? c.y : c.x;
    if constexpr (PAGE == LRQK_PAGE_E4M3) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
      x[4 * i] = lo[0] * s;
      x[4 * i + 1] = lo[1] * s;
      x[4 * i + 2] = hi[0] * s;
      x[4 * i + 3] = hi[1] * s;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = (float)(int8_t)(w >> (8 * j)) * s;
    }
  }
}

// The same as four packed bf16 pairs: exact too (a code has at most seven bits, and with scales as they are written the product
// is a normal number of bf16 or 0; with larger ones, in a pool from elsewhere, it may be an infinity).
template <int PAGE>
__device__ __forceinline__ uint4 decode8_bf16(uint2 c, float s) {
  if constexpr (PAGE == LRQK_PAGE_E4M3) {
    auto pair = [&](uint32_t w, auto high) {
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, high.value));
    };
    using std::false_type;
    using std::true_type;
    return make_uint4(pair(c.x, false_type{}), pair(c.x, true_type{}), pair(c.y, false_type{}), pair(c.y, true_type{}));
  } else {
    float f[8];
    decode8<PAGE>(c, s, f);
    return make_uint4(dev::pack_bf16(f[0], f[1]), dev::pack_bf16(f[2], f[3]), dev::pack_bf16(f[4], f[5]),
                      dev::pack_bf16(f[6], f[7]));
  }
}

// The scale byte of a block whose largest magnitude has the bits `top` (compared as integers, so that
// infinity and NaN win): the smallest e >= kMinExp with max <= 448 2^e or 127 2^e.  448 = 1.75 * 2^8,
// 127 = 1.984375 * 2^6: one more where the mantissa is above theirs.
template <int PAGE>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  constexpr int kTopExp = PAGE == LRQK_PAGE_E4M3 ? 8 : 6;
  constexpr uint32_t kTopMant = PAGE == LRQK_PAGE_E4M3 ? 0x600000u : 0x7e0000u;
  const int ex = (int)(top >> 23);
  if (ex == 255) return 255u;
  const int e = ex - 127 - kTopExp + ((top & 0x7fffffu) > kTopMant ? 1 : 0);
  return (uint32_t)(max(e, kMinExp) + 127);
}

// Eight elements as codes of a block with that scale byte.  With the largest scale (that of a block whose largest magnitude is
// above 448 2^119 or 127 2^121) a number may lie nearest to 256 2^120 or 64 2^122, which is 2^128: it takes the code below, so
// that what is finite is read back finite.
template <int PAGE>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], uint32_t byte) {
  if (byte == 255u) return make_uint2(0u, 0u);
  const float inv = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte), a normal number
  constexpr bool kE4m3 = PAGE == LRQK_PAGE_E4M3;
  const float most = byte >= (kE4m3 ? 247u : 249u) ? (kE4m3 ? 240.0f : 63.0f) : (kE4m3 ? 448.0f : 127.0f);
  auto scaled = [&](int i) { return __builtin_amdgcn_fmed3f(x[i] * inv, -most, most); };
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if constexpr (PAGE == LRQK_PAGE_E4M3) {
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(4 * i), scaled(4 * i + 1), 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(scaled(4 * i + 2), scaled(4 * i + 3), v, true);
      w[i] = (uint32_t)v;
    } else {
      uint32_t v = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        v |= ((uint32_t)(int)__builtin_rintf(scaled(4 * i + j)) & 0xffu) << (8 * j);
      w[i] = v;
    }
  }
  return make_uint2(w[0], w[1]);
}

// Sequence that each packed row t belongs to, or -1; the whole wavefront asks, each lane for its own rows: the starts are
// read once, 64 at a time, without a chain of dependent loads.
template <int N>
__device__ __forceinline__ void sequences_of(const Map& m, const int (&t)[N], int (&b)[N]) {
  const int lane = threadIdx.x & 63;
  const int first = m.start[0];
#pragma unroll
  for (int j = 0; j < N; ++j) b[j] = 0;
  for (int i0 = 0; i0 < m.B; i0 += 64) {
    const int todo = min(64, m.B - i0);
    const int e = m.start[i0 + min(lane, todo - 1) + 1];
    for (int i = 0; i < todo; ++i) {
      const int end = __builtin_amdgcn_readlane(e, i);
#pragma unroll
      for (int j = 0; j < N; ++j) b[j] += end <= t[j] ? 1 : 0;
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) b[j] = b[j] < m.B && t[j] >= first && t[j] < m.T ? b[j] : -1;
}
__device__ __forceinline__ int sequence_of(const Map& m, int t) {
  int b[1];
  sequences_of(m, {t}, b);
  return b[0];
}

// f(bf16 dense rows, page type) for the five combinations that check_pages lets through
template <typename F>
void by_type(const lrqk_pages_shape& s, F f) {
  using std::integral_constant;
  const bool bf16 = s.kv_dtype == LRQK_KV_BF16;
  auto with = [&](auto page) {
    if constexpr (page.value == LRQK_PAGE_BF16) f(std::true_type{}, page);
    else if constexpr (page.value == LRQK_PAGE_F32) f(std::false_type{}, page);
    else if (bf16) f(std::true_type{}, page);
    else f(std::false_type{}, page);
  };
  switch (s.page_dtype) {
    case LRQK_PAGE_BF16: with(integral_constant<int, LRQK_PAGE_BF16>{}); break;
    case LRQK_PAGE_F32: with(integral_constant<int, LRQK_PAGE_F32>{}); break;
    case LRQK_PAGE_E4M3: with(integral_constant<int, LRQK_PAGE_E4M3>{}); break;
    default: with(integral_constant<int, LRQK_PAGE_I8>{}); break;
  }
}

}  // namespace pages
}  // namespace lrqk
