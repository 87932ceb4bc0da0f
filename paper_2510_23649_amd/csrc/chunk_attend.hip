// g3 -- exact causal attention of new tokens over the paged cache (include/lrqk.h).
//
// The query heads of a KV head attend to the same rows, so the n G (token, query head) pairs of a
// sequence are the rows of one problem per KV head.  A wavefront holds 32 of them and makes
//   S^T = K Q^T    (positions x rows)        O^T += V^T P^T    (elements x rows)
// on the matrix cores.  With the positions as rows of the product, a lane has 16 scores of one row of
// the problem in a register tile and lane + 32 the other 16: a row's maximum and sum are in-lane
// operations and one exchange, and the exponentials are, register for register, the operand that the second
// product takes, as long as it takes the positions in the order in which they lie there (register v, half h:
// position 8 (v / 4) + 4 h + v % 4), which is how V is read from LDS, four positions at a time through the
// transposing read.
// One pass over the positions with a running maximum and sum.  The maximum is raised, and the accumulators
// rescaled, only when a score exceeds it by more than kLag powers of two (or, in the tiles' steps, when 16 weights exceed
// kHeavy); until then it is one of an earlier block, which is exact up to the rounding that the weights have anyway.
//
// Four shapes of workgroup, all of four wavefronts:
//   tile  the wavefronts take 32 rows of the problem each and share the positions, 64 at a time (32
//         in fp32) through two buffers in LDS: K and V are read once for 128 rows
//   pair  at most 64 rows (bf16): two wavefronts take 32 rows each at one half of every block of 64
//         positions, the other two the same rows at the other half
//   thin  at most 32 rows: each wavefront takes every fourth block of 32 positions through an LDS
//         area of its own, without a barrier
//   few   pages of 4 bits, at most 64 rows in bf16 and any number in fp32: as thin, with tiles of 16
//         rows and blocks of 64 positions, and K from its load into the product, not through LDS; in
//         fp32 q and the weights as three bf16 terms each
// The states of wavefronts that have the same rows, and of the pieces that a long context is cut into, are joined at the
// end.  Rows of the pool's own type go straight to LDS (thin: through registers), codes are decoded on the way into
// it, exactly: a code times its scale is a bf16 number.
//
// V rows that a token does not see meet its weights as 0 * V, which is not 0 if V is not finite.
// Positions that nobody sees are cleared; in blocks that some rows of the problem see and others do not,
// elements that are not finite are cleared as well and added to the rows that see them at the end.
#include <cmath>
#include <algorithm>

#include "pages.h"

namespace lrqk {
namespace {

using namespace pages;

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLag = 8.0f;
constexpr float kHeavy = 4096.0f;
constexpr float kFar = 1073741824.0f;  // see Rows::weigh
constexpr int kPartial = kPartialStride;  // floats of a partial state: max, sum, 2 unused, acc[128]

struct Args {
  Map m;
  const void *K, *V;
  const uint8_t *K_scale, *V_scale;
  const void* q;
  void* out;
  float* partials;  // [T*Hq][pieces][kPartial], or null: one piece, straight to out
  int G, rows_log2;                    // rows of the problem a workgroup takes
  int pieces, prefer, want, least;     // pieces: of a sequence at most, and places in partials; see piece_of
  uint32_t page16;               // 16-byte chunks of a page (of all KV heads)
  float scale;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
using dev::bf16x8;
using dev::f32x16;

// Row r of the problem of a sequence: token and query head within the group.
struct Problem {
  Seq s;
  int b, step, piece, r0, rows;  // positions of a piece; piece and first row of this workgroup; rows of the sequence
};

__device__ __forceinline__ int wave_max(int v) {  // of numbers that are not negative
  v = max(v, (int)dev::dpp_zero_fill<0x111, 0xf>((uint32_t)v));
  v = max(v, (int)dev::dpp_zero_fill<0x112, 0xf>((uint32_t)v));
  v = max(v, (int)dev::dpp_zero_fill<0x114, 0xf>((uint32_t)v));
  v = max(v, (int)dev::dpp_zero_fill<0x118, 0xf>((uint32_t)v));
  v = max(v, (int)dev::dpp_zero_fill<0x142, 0xa>((uint32_t)v));
  v = max(v, (int)dev::dpp_zero_fill<0x143, 0xc>((uint32_t)v));
  return __builtin_amdgcn_readlane(v, 63);
}

// Sequence i0 + lane (behind the last one: that again).
__device__ __forceinline__ Seq lane_sequence(const Args& a, int i0) {
  int lane = threadIdx.x & 63;
  asm volatile("" : "+v"(lane));  // (addresses made anew, and not kept in registers over all units)
  const int i = min(i0 + lane, a.m.B - 1);
  const int len = a.m.kv_len[i], first = a.m.start[i], end = a.m.start[i + 1];  // together, not one after the other
  Seq s;
  s.first = min(max(first, 0), a.m.T);
  s.n = min(max(end, s.first), a.m.T) - s.first;
  s.len = max(len, 0);
  return s;
}
__device__ __forceinline__ int tiles_of(const Args& a, int n) { return (n * a.G + (1 << a.rows_log2) - 1) >> a.rows_log2; }

// The same in all lanes: of numbers that are not negative.
__device__ __forceinline__ uint32_t wave_sum(uint32_t v) {
  return __builtin_amdgcn_readlane(dev::wave_inclusive_scan(v), 63);
}

// Positions of a piece in this call: the lengths say, not l_max, which a captured call has for all its replays.  The whole
// wavefront asks, with the first 64 sequences.
//   want > 0   few rows a sequence: as short as it can be without there being more than `want` units of work a KV head.  With
//              t_b tiles of sequence b, t = sum_b t_b and x = sum_b t_b len_b, at least x / want, and surely enough x / (want - t + 1),
//              as sum_b t_b ceil(len_b / p) <= ceil(x / p) + t - 1; up to 64 sequences' units are counted for some between
//   want == 0  many: a `prefer`th of the longest sequence, but no more than 16384
// and no less than `least` or than there is room for states.  EVEN: want may be > 0.
template <bool EVEN>
__device__ __forceinline__ int piece_of(const Args& a, Seq s) {
  const int lane = threadIdx.x & 63;
  int longest = 0, p;
  if (EVEN && a.want > 0) {
    uint32_t x = 0, t = 0, len, mine;  // lengths in 128 positions; 32 bits hold x: want > 0 only if B <= 4096, or 2048 with 16 rows a tile
    for (int i0 = 0;;) {
      mine = i0 + lane < a.m.B ? (uint32_t)tiles_of(a, s.n) : 0;
      len = mine > 0 ? ((uint32_t)min(s.len, a.m.l_max) + 127) >> 7 : 0;
      longest = max(longest, (int)len);
      x += mine * len;
      t += mine;
      i0 += 64;
      if (i0 >= a.m.B) break;
      s = lane_sequence(a, i0);
    }
    longest = wave_max(longest) * 128;
    x = wave_sum(x);
    t = wave_sum(t);
    const uint32_t parts = (uint32_t)max(a.want - (int)t + 1, 1), enough = (x + parts - 1) / parts;
    uint32_t q = (x + a.want - 1) / a.want;
    const uint32_t by = (enough - q + 3) / 4;
    if (a.m.B > 64) q = enough;
    while (q < enough && wave_sum(mine * max((len + q - 1) / q, 1u)) > (uint32_t)a.want) q = min(q + by, enough);
    p = (int)q * 128;
  } else {
    for (int i0 = 0;;) {
      longest = max(longest, min(s.len, a.m.l_max));
      i0 += 64;
      if (i0 >= a.m.B) break;
      s = lane_sequence(a, i0);
    }
    longest = wave_max(longest);
    p = min((longest + a.prefer - 1) / a.prefer, 16384);
  }
  p = max(max(p, (longest + a.pieces - 1) / a.pieces), a.least);
  return (p + 127) / 128 * 128;
}

// Unit `unit` of the work of a KV head: a sequence's units are its pieces, last one first, a piece's its tiles (M rows
// each).  False if there are not that many.  Every wavefront finds it for itself, 64 sequences at a time; p.step is given.
// q: sequences from.i0 + lane.  Where the unit was found is left in `from`, for a later one to begin there.
struct Cursor {
  int i0, before;  // first of 64 sequences; units of those before them
};
template <int M>
__device__ __forceinline__ bool find_from(const Args& a, int unit, Problem& p, Seq q, Cursor& from) {
  const int lane = threadIdx.x & 63;
  int before = from.before;
  const int first = from.i0;
  for (int i0 = first; i0 < a.m.B; i0 += 64) {
    if (i0 > first) q = lane_sequence(a, i0);
    const int tiles = (q.n * a.G + M - 1) / M, pieces = max(1, (min(q.len, a.m.l_max) + p.step - 1) / p.step);
    const int units = i0 + lane < a.m.B ? tiles * pieces : 0;
    const int upto = before + (int)dev::wave_inclusive_scan((uint32_t)units);
    const uint64_t past = __ballot(upto > unit);
    if (past) {
      const int j = __builtin_ctzll(past);
      const int mine = unit - (__builtin_amdgcn_readlane(upto, j) - __builtin_amdgcn_readlane(units, j));
      const int t = __builtin_amdgcn_readlane(tiles, j);
      p.b = i0 + j;
      p.s.first = __builtin_amdgcn_readlane(q.first, j);
      p.s.n = __builtin_amdgcn_readlane(q.n, j);
      p.s.len = __builtin_amdgcn_readlane(q.len, j);
      p.rows = p.s.n * a.G;
      if (mine < 0) return false;  // (no start may send a workgroup anywhere)
      // the last tiles of a sequence see most: they come first
      const int back = __builtin_amdgcn_readlane(units, j) - 1 - mine;
      p.piece = back / t;
      p.r0 = (back - p.piece * t) * M;
      from = Cursor{i0, before};
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}
template <int M, bool EVEN>
__device__ __forceinline__ bool find_unit(const Args& a, int unit, Problem& p) {
  const Seq q = lane_sequence(a, 0);
  p.step = piece_of<EVEN>(a, q);
  Cursor from{0, 0};
  return find_from<M>(a, unit, p, q, from);
}

// Positions that a row of the problem sees: [0, result).
__device__ __forceinline__ int sees(const Args& a, const Problem& p, int row) {
  return min(max(p.s.len - p.s.n + row / a.G + 1, 0), a.m.l_max);
}

// |scale| in units of log2 (its sign goes into q).  Never 0: a masked score is -infinity before it is scaled.
__device__ __forceinline__ float log2_scale(const Args& a) { return fmaxf(fabsf(a.scale) * kLog2e, 1.17549435e-38f); }

__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A dword of V (two bf16 or one fp32): an infinity or a NaN in it; the same without them.
template <bool BF16>
__device__ __forceinline__ bool odd(uint32_t w) {
  return (w & 0x7f800000u) == 0x7f800000u || (BF16 && (w & 0x7f80u) == 0x7f80u);
}
template <bool BF16>
__device__ __forceinline__ uint32_t clear(uint32_t w) {
  if ((w & 0x7f800000u) == 0x7f800000u) w &= BF16 ? 0xffffu : 0u;
  if (BF16 && (w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  return w;
}

// ---- a block of rows on its way from the pages through registers into LDS ------------------------------
// ROWS rows by NW wavefronts; wavefront w takes rows w ROWS / NW and on.  LDS rows of kRowB bytes in 16-byte chunks, their
// order within a row turned by a mask that depends on the row, so that neither the reads of K (32 rows, one chunk each) nor
// those of V (8 rows, 32 bytes each) fall on the same banks; and in bf16 turned once more in the row's second half, because a
// lane that decodes 16 codes stores two chunks: eight lanes' first ones would meet in the four even chunks of 128 bytes
// (1024 tokens at 128K of e4m3: 2560 us, and 2460 without those conflicts).
template <bool BF16>
constexpr int kRowB = kD * (BF16 ? 2 : 4);
__device__ __forceinline__ int half_turn(int c) { return c ^ (c >> 3); }  // (of 16; its own inverse)
template <bool BF16>
__device__ __forceinline__ int k_chunk(int row, int c) {
  return row * kRowB<BF16> + (((BF16 ? half_turn(c) : c) ^ (row & 15)) << 4);
}
__device__ __forceinline__ int v_turn(int row) { return ((row & 3) << 2) ^ (((row >> 2) & 1) << 1); }
__device__ __forceinline__ int v_chunk(int row, int c) { return row * kRowB<true> + ((half_turn(c) ^ v_turn(row)) << 4); }

// Blocks and a wavefront's share of them begin at multiples of 16 positions (8 in fp32), so with pages of 16 positions
// and more up to 16 rows at a time lie one behind the other in one page: their place is one number for the wavefront,
// and a lane's part of an address does not change from block to block.  SMALL: smaller pages, a table entry for every row.
template <bool BF16, int PAGE, int ROWS, int NW, bool SMALL = false>
struct Block {
  static constexpr int kRow16 = row_bytes(PAGE) / 16;                     // 16-byte chunks of a row in the pool
  using Raw = std::conditional_t<PAGE == LRQK_PAGE_E2M1 && !BF16, uint2, uint4>;  // what a lane loads of a row
  static constexpr int kLanes = row_bytes(PAGE) / (int)sizeof(Raw);       // lanes a row
  static constexpr int kPass = 64 / kLanes;                               // rows a load of the wavefront
  static constexpr int kMine = ROWS / NW;                                 // rows of the wavefront
  static constexpr int kN = kMine / kPass;                                // such loads
  static constexpr int kOut = kRowB<BF16> / 16 / kLanes;                  // 16-byte chunks of LDS that a lane's load makes
  static constexpr int kGroup = kMine < 16 ? kMine : 16;                  // rows with one place
  static constexpr int kGroups = kMine / kGroup;
  static constexpr uint32_t kAll = kMine == 32 ? 0xffffffffu : (1u << kMine) - 1u;

  struct Found {              // the same in all lanes
    int p0;                   // position of the wavefront's first row
    uint32_t place[kGroups];  // chunk of the pool at which a group's first row begins; 0 where there is no page
    uint32_t there;           // bit of each row
  };
  struct Held {
    Raw x[kN];
    uint32_t scale[kN];
  };
  int pg[kGroups];  // the groups' pages, one block ahead

  static __device__ __forceinline__ int row_in_wave(int i, int lane) { return i * kPass + lane / kLanes; }

  // table entries for the wavefront's rows from position p on; end: first position that is none
  __device__ __forceinline__ void look_up(const Map& m, int b, int p, int end) {
    const int32_t* table = m.table + (size_t)b * m.max_pages;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) pg[g] = table[(uint32_t)min(p + g * kGroup, end - 1) >> m.page_log2];
  }

  // what has been looked up
  __device__ __forceinline__ void find(const Args& a, int b, int kvh, int p, int end, int lane, Found& f) const {
    f.p0 = p;
    f.there = 0;
    if constexpr (SMALL) {
      uint32_t at[kN];
      f.there = find_rows(a, b, kvh, p, end, lane, at);
      return;
    }
    const uint32_t in_page = (1u << a.m.page_log2) - 1;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const uint32_t page = __builtin_amdgcn_readfirstlane(pg[g]);
      const int q = p + g * kGroup, n = page < (uint32_t)a.m.n_pages ? min(max(end - q, 0), kGroup) : 0;
      const uint32_t at = page * a.page16 + (((uint32_t)kvh << a.m.page_log2) + ((uint32_t)q & in_page)) * kRow16;
      f.place[g] = n > 0 ? at : 0;
      f.there |= ((1u << n) - 1) << (g * kGroup);
    }
  }

  // Pages of less than 16 positions: the chunk at which each of the lane's rows begins, 0 where there is none; the bits
  // of the rows that are there.
  static __device__ __forceinline__ uint32_t find_rows(const Args& a, int b, int kvh, int p, int end, int lane,
                                                       uint32_t (&at)[kN]) {
    uint32_t there = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int q = p + row_in_wave(i, lane);
      const uint32_t page = a.m.table[(size_t)b * a.m.max_pages + ((uint32_t)min(q, end - 1) >> a.m.page_log2)];
      const bool ok = (q < end) & (page < (uint32_t)a.m.n_pages);
      const uint32_t in_page = (uint32_t)q & ((1u << a.m.page_log2) - 1);
      at[i] = ok ? page * a.page16 + (((uint32_t)kvh << a.m.page_log2) + in_page) * kRow16 : 0;
      const uint64_t v = __ballot(ok);
#pragma unroll
      for (int j = 0; j < kPass; ++j) there |= (uint32_t)((v >> (j * kLanes)) & 1) << (i * kPass + j);
    }
    return there;
  }

  // the rows found, of K or of V, into registers; what is not there reads rows that do not matter
  static __device__ __forceinline__ void load(const Args& a, int b, int kvh, int end, const void* base,
                                              const uint8_t* scale, const Found& f, int lane, Held& r) {
    const int c = lane % kLanes;
    if constexpr (SMALL) {
      uint32_t at[kN];
      find_rows(a, b, kvh, f.p0, end, lane, at);
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if constexpr (PAGE != LRQK_PAGE_E2M1) {  // (sums in 64 bits cost registers and 1 to 3 % of the time; for 4 bits sums in 32 cost 4 %)
          r.x[i] = static_cast<const Raw*>(base)[(size_t)(at[i] + c)];
          if constexpr (coded(PAGE)) r.scale[i] = scale[(size_t)((at[i] + c) / (kLanes / kScales))];
        } else {
          r.x[i] = static_cast<const Raw*>(base)[(size_t)at[i] * (kLanes / kRow16) + c];
          r.scale[i] = scale[(size_t)(at[i] / (kRow16 / kScales)) + c * kScales / kLanes];
        }
      }
    } else {
      // first what all lanes share, then what a lane adds in every block, then a number that the instruction holds
      const uint32_t mine = (uint32_t)lane;  // lane / kLanes * kLanes + c
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const int g = i * kPass / kGroup, rows = i * kPass - g * kGroup;
        r.x[i] = (static_cast<const Raw*>(base) + (size_t)f.place[g] * (kLanes / kRow16))[mine + rows * kLanes];
        // (kRow16 chunks of a row and kScales scales: a lane's codes are one scale block or half of one)
        if constexpr (coded(PAGE))
          r.scale[i] = (scale + (size_t)(f.place[g] / (kRow16 / kScales)))[mine * kScales / kLanes + rows * kScales];
      }
    }
  }

  // The rows found, of the type that LDS holds, straight into LDS: a wavefront's load fills 1 KB, 16 bytes a lane, so the
  // lanes read the chunks in the order in which LDS holds them.
  template <bool V>
  static __device__ __forceinline__ void load_direct(const void* base, const Found& f, int w, int lane, char* to) {
    static_assert(kRow16 == kLanes && !SMALL, "one chunk a lane, places for whole groups");
    const int c = lane % kLanes;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int g = i * kPass / kGroup, row = w * kMine + row_in_wave(i, lane);
      const int turned = !BF16 ? (V ? c : c ^ (row & 15)) : half_turn(c ^ (V ? v_turn(row) : row & 15));
      // first what all lanes share, then what a lane adds in every block
      const char* from = static_cast<const char*>(base) + ((size_t)f.place[g] << 4) +
                         (uint32_t)(((row_in_wave(i, lane) - g * kGroup) * kRow16 + turned) << 4);
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)from,
          (__attribute__((address_space(3))) void*)(to + (w * kMine + i * kPass) * kRowB<BF16>), 16, 0, 0);
    }
  }

  // Codes as they go into LDS, in chunks; `swap`: chunks j and j ^ 2 change places.  A lane that decodes 32 codes of e2m1 stores
  // four chunks, and two rows' lanes would meet in the same banks: in every other row it begins with the third.
  static constexpr bool kSwaps = BF16 && PAGE == LRQK_PAGE_E2M1;
  static __device__ __forceinline__ int chunk_at(int c, int j, bool swap) { return c + (kSwaps && swap ? j ^ 2 : j); }
  static __device__ __forceinline__ void widen(const Raw x, uint32_t byte, bool swap, uint4 (&o)[kOut]) {
    if constexpr (!coded(PAGE)) {
      o[0] = x;
    } else if constexpr (PAGE == LRQK_PAGE_E2M1) {
      if constexpr (BF16) {
        const float s = scale_bits(byte);
        const uint32_t w[4] = {swap ? x.z : x.x, swap ? x.w : x.y, swap ? x.x : x.z, swap ? x.y : x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = decode8_bf16<PAGE>(w[j], s);
      } else {
        const float s = scale_of(byte);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float f[8];
          decode8<PAGE>(j ? x.y : x.x, s, f);
          o[2 * j] = __builtin_bit_cast(uint4, f32x4{f[0], f[1], f[2], f[3]});
          o[2 * j + 1] = __builtin_bit_cast(uint4, f32x4{f[4], f[5], f[6], f[7]});
        }
      }
    } else {
      const float s = scale_of(byte);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint2 codes = make_uint2(w[2 * j], w[2 * j + 1]);
        if constexpr (BF16) {
          o[j] = decode8_bf16<PAGE>(codes, s);
        } else {
          float f[8];
          decode8<PAGE>(codes, s, f);
          o[2 * j] = __builtin_bit_cast(uint4, f32x4{f[0], f[1], f[2], f[3]});
          o[2 * j + 1] = __builtin_bit_cast(uint4, f32x4{f[4], f[5], f[6], f[7]});
        }
      }
    }
  }

  static __device__ __forceinline__ void store_k(const Held& r, int w, int lane, char* kt) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = w * kMine + row_in_wave(i, lane), c = (lane % kLanes) * kOut;
      const bool swap = row & 1;
      uint4 o[kOut];
      widen(r.x[i], coded(PAGE) ? r.scale[i] : 0u, swap, o);
#pragma unroll
      for (int j = 0; j < kOut; ++j) *reinterpret_cast<uint4*>(kt + k_chunk<BF16>(row, chunk_at(c, j, swap))) = o[j];
    }
  }

  // V rows that are not there become zeros.  part: some rows of the problem see the block and others do not.  Returns
  // whether elements were left out for that.
  static __device__ __forceinline__ bool store_v(const Held& r, uint32_t there, bool part, int w, int lane, char* vt) {
    bool left_out = false;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int in_wave = row_in_wave(i, lane), row = w * kMine + in_wave, c = (lane % kLanes) * kOut;
      const bool swap = row & 1;
      uint4 o[kOut];
      widen(r.x[i], coded(PAGE) ? r.scale[i] : 0u, swap, o);
      if (there != kAll && !((there >> in_wave) & 1)) {
#pragma unroll
        for (int j = 0; j < kOut; ++j) o[j] = make_uint4(0, 0, 0, 0);
      }
      if (part) {
#pragma unroll
        for (int j = 0; j < kOut; ++j) {
          left_out |= odd<BF16>(o[j].x) || odd<BF16>(o[j].y) || odd<BF16>(o[j].z) || odd<BF16>(o[j].w);
          o[j] = make_uint4(clear<BF16>(o[j].x), clear<BF16>(o[j].y), clear<BF16>(o[j].z), clear<BF16>(o[j].w));
        }
      }
#pragma unroll
      for (int j = 0; j < kOut; ++j)
        *reinterpret_cast<uint4*>(vt + (BF16 ? v_chunk(row, chunk_at(c, j, swap)) : row * kRowB<false> + ((c + j) << 4))) = o[j];
    }
    return left_out;
  }
};

// ---- 32 rows of the problem in a wavefront ---------------------------------------------------------------
// Lane l: row l % 32; element e of S^T or O^T: dev::mfma_row(e, l).
template <bool BF16>
struct Rows {
  uint4 q[BF16 ? 8 : 16];  // bf16: elements 16 s + 8 h .. + 7; fp32: 8 s + 4 h .. + 3
  f32x16 o[4];             // elements 32 t .. of O^T
  float mx, sum;           // of what has been seen, in units of log2
  float near;              // mx; -infinity where that is no number below kFar
  int see;                 // positions that the lane's row sees

  __device__ __forceinline__ void start(const void* base, int64_t row, bool negate, int lane) {
    const int h = lane >> 5;
    const uint32_t flip = negate ? (BF16 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
    for (int s = 0; s < (BF16 ? 8 : 16); ++s) {
      uint4 x = static_cast<const uint4*>(base)[row * (kRowB<BF16> / 16) + 2 * s + h];
      x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
      q[s] = x;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] = 0.0f;
    mx = -INFINITY;
    near = -INFINITY;
    sum = 0.0f;
  }

  __device__ __forceinline__ f32x16 scores_step(const char* kt, int k, f32x16 s, int lane) const {
    const int i = lane & 31, h = lane >> 5;
    if constexpr (BF16) {
      return dev::mfma_bf16(__builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(kt + k_chunk<true>(i, 2 * k + h))),
                            __builtin_bit_cast(bf16x8, q[k]), s);
    } else {
      const f32x4 x = *reinterpret_cast<const f32x4*>(kt + k_chunk<false>(i, 2 * k + h));
      const f32x4 y = __builtin_bit_cast(f32x4, q[k]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], s, 0, 0, 0);
      return s;
    }
  }
  // scores of 32 positions in LDS
  __device__ __forceinline__ f32x16 scores(const char* kt, int lane) const {
    f32x16 s = zeros();
#pragma unroll
    for (int k = 0; k < (BF16 ? 8 : 16); ++k) s = scores_step(kt, k, s, lane);
    return s;
  }
  static __device__ __forceinline__ f32x16 zeros() {
    f32x16 z;
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] = 0.0f;
    return z;
  }

  // scores of the 32 positions from p0 that the row does not see, or that are not there, become -infinity
  __device__ __forceinline__ void mask(f32x16& s, int p0, uint32_t there, int lane) const {
    const int up_to = see - p0;
    const uint32_t mine = (up_to >= 32 ? there : up_to <= 0 ? 0u : there & ((1u << up_to) - 1)) >> (4 * (lane >> 5));
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = mine & (1u << (8 * (e >> 2) + (e & 3))) ? s[e] : -INFINITY;
  }

  // Weights of 32 positions at the running maximum.  That is rounded, and s c inside the instruction is not: what lies between them
  // is a factor that all weights of the row share, of 2^+-32 at most as long as the maximum is below kFar = 2^30.  Where it is not,
  // or where there is none yet, `near` makes them infinite or NaN, for who takes them to look at their sum.
  __device__ __forceinline__ f32x16 weigh(const f32x16& s, float c, float base) const {
    f32x16 w;
#pragma unroll
    for (int e = 0; e < 16; ++e) w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], c, -base));
    return w;
  }
  // The row's maximum is beyond that, or there is none.
  __device__ __forceinline__ bool far() const { return fabsf(mx) >= kFar; }
  // The same for every row: those beyond kFar with products that are rounded like the maximum, so that the largest score has the
  // weight 1.
  __device__ __forceinline__ f32x16 weigh_any(const f32x16& s, float c) const {
#pragma clang fp contract(off)
    const float base = mx == -INFINITY ? 0.0f : mx;
    const bool rounded = far();
    f32x16 w;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float y = s[e] * c;
      w[e] = __builtin_amdgcn_exp2f(rounded ? y - base : __builtin_fmaf(s[e], c, -base));
    }
    return w;
  }
  // the largest score of the row, in units of log2
  static __device__ __forceinline__ float largest(const f32x16& s, float c) {
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
    return max_halves(top) * c;
  }
  // the running maximum up to `top`
  __device__ __forceinline__ void raise(float top) {
    const float to = fmaxf(mx, top);
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mx - to);
    sum *= f;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[t][e] *= f;
    mx = to;
    near = fabsf(to) < kFar ? to : -INFINITY;
  }

  struct Weights {  // of 32 positions as the second product's operand
    uint4 half[2];
  };
  static __device__ __forceinline__ Weights pack(const f32x16& w) {
    Weights x;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      x.half[k] = make_uint4(dev::pack_bf16(w[8 * k], w[8 * k + 1]), dev::pack_bf16(w[8 * k + 2], w[8 * k + 3]),
                             dev::pack_bf16(w[8 * k + 4], w[8 * k + 5]), dev::pack_bf16(w[8 * k + 6], w[8 * k + 7]));
    return x;
  }
  // Their sum, of the weights as they are multiplied, two at a time.
  static __device__ __forceinline__ float add_up(const Weights& x) {
    const dev::bf16x2 one = __builtin_bit_cast(dev::bf16x2, 0x3f803f80u);
    float add = 0.0f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t w[4] = {x.half[k].x, x.half[k].y, x.half[k].z, x.half[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        add = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(dev::bf16x2, w[e]), one, add, false);
    }
    return add;
  }
  static __device__ __forceinline__ float add_up(const f32x16& w) {
    float add = 0.0f;
#pragma unroll
    for (int e = 0; e < 16; ++e) add += w[e];
    return add;
  }
  // the weights of s, at a maximum that is raised where it has to be
  __device__ __forceinline__ std::conditional_t<BF16, Weights, f32x16> settle(const f32x16& s, float c) {
    const auto form = [](const f32x16& w) {
      if constexpr (BF16) return pack(w);
      else return w;
    };
    const float top = largest(s, c);
    if (__any(top > mx + kLag)) raise(top);  // (-inf > -inf is false: nothing seen so far, nothing to do)
    auto x = form(weigh(s, c, mx == -INFINITY ? 0.0f : mx));
    if (__builtin_expect(__any(far()), 0)) {
      asm volatile("");  // a branch, which next to no call takes
      x = form(weigh_any(s, c));
    }
    sum += add_up(x);
    return x;
  }
  // O += weights of 16 positions (half k of 32) times 32 elements (t) of their V rows
  __device__ __forceinline__ void output_step(const char* vt, const Weights& x, int k, int t, int lane) {
    // a transposing read: the 16 lanes of a group point at 4 rows of 16 elements, lane g gets column g
    const int g = lane & 15, h = lane >> 5;
    s16x4 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int row = 16 * k + 8 * j + 4 * h + (g >> 2);
      const int chunk = 4 * t + 2 * ((lane >> 4) & 1) + ((g & 3) >> 1);
      v[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(vt + v_chunk(row, chunk) + 8 * (g & 1)));
    }
    o[t] = dev::mfma_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7)),
                          __builtin_bit_cast(bf16x8, x.half[k]), o[t]);
  }
  __device__ __forceinline__ void output(const char* vt, const Weights& x, int lane) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int t = 0; t < 4; ++t) output_step(vt, x, k, t, lane);
  }

  // 32 positions from p0 in LDS, rows `there`; c: scale in log2
  __device__ __forceinline__ void attend(const char* kt, const char* vt, int p0, uint32_t there, bool all_see, float c,
                                         int lane) {
    f32x16 s = scores(kt, lane);
    if (!(all_see && there == 0xffffffffu)) {
      asm volatile("");  // a branch: taken by few blocks
      mask(s, p0, there, lane);
    }
    const auto w = settle(s, c);
    if constexpr (BF16) {
      output(vt, w, lane);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float* row = reinterpret_cast<const float*>(vt + dev::mfma_row(e, lane) * kRowB<false>);
#pragma unroll
        for (int t = 0; t < 4; ++t)
          o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(row[32 * t + (lane & 31)], w[e], o[t], 0, 0, 0);
      }
    }
  }

  // One step of the pipeline: the weights of the scores s, between the products of the 32 positions after them (scores
  // into `next`, from kt) and of those before them (weights x, V rows from vt).  The weights are made at the maximum so
  // far, and again in the rare case that it has to be raised; x then becomes those of s.
  template <bool BEFORE>
  __device__ __forceinline__ void step(const f32x16& s, f32x16& next, Weights& x, const char* kt, const char* vt, float c,
                                       int lane) {
    next = zeros();
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      next = scores_step(kt, k, next, lane);
      if (BEFORE) output_step(vt, x, k >> 2, k & 3, lane);
    }
    x = pack(weigh(s, c, near));
    float add = add_up(x);
    // made here, between the products, and not only once the maximum is known to stand
    asm volatile("" : "+v"(x.half[0].x), "+v"(x.half[0].y), "+v"(x.half[0].z), "+v"(x.half[0].w), "+v"(x.half[1].x),
                      "+v"(x.half[1].y), "+v"(x.half[1].z), "+v"(x.half[1].w), "+v"(add));
    // reads ahead of the products, then a product, the vector instructions that go under it, a read
    __builtin_amdgcn_sched_group_barrier(0x100, BEFORE ? 6 : 4, 0);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
      __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, BEFORE ? 2 : 1, 0);
      if (BEFORE) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
        __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    // The sum says whether the maximum has to be raised, without the scores being looked through for theirs (eight of some 55
    // vector instructions).  Where there is no maximum yet, or a far one, it is no number that is less.
    if (__any(!(add <= kHeavy))) {
      raise(largest(s, c));
      x = pack(weigh_any(s, c));
      add = add_up(x);
    }
    sum += add;
  }
};

// What a state (its maximum and sum) counts for at the maximum `top` of several.  One without weights counts for nothing; a
// NaN's sum stays.
__device__ __forceinline__ float weight_of(float mx, float sum, float top) {
  return mx == -INFINITY ? (sum == 0.0f ? 0.0f : 1.0f) : __builtin_amdgcn_exp2f(mx - top);
}

// Four consecutive elements of a row of the output, or of a partial state (the row's max and sum with element 0).
template <bool BF16>
__device__ __forceinline__ void put(const Args& a, const Problem& p, int kvh, int row, int piece, int e0, f32x4 x,
                                    float mx, float sum) {
  const int t = p.s.first + row / a.G, h = kvh * a.G + row % a.G;
  const int64_t at = (int64_t)t * (a.m.Hkv * a.G) + h;
  if (a.partials) {
    float* P = a.partials + (at * a.pieces + piece) * kPartial;
    *reinterpret_cast<f32x4*>(P + 4 + e0) = x;
    if (e0 == 0) {
      P[0] = mx;
      P[1] = sum;
    }
    return;
  }
  const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = sum == 0.0f ? 0.0f : x[e] * f;
  if constexpr (BF16)
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + at * kD + e0) =
        make_uint2(dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3]));
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at * kD + e0) = x;
}

// Elements of V that are not finite at positions [from, to) that some rows of the workgroup see and others do not were left
// out: each row gets those that it sees, a thread per element.  Rare, and slow.  sums: of row r's weights, those of state v at
// v * rows_held + r; a row of the output without any (its scores are -infinity) stays 0.
template <bool BF16, int PAGE>
__device__ void add_left_out(const Args& a, const Problem& p, int kvh, int rows, int piece, int from, int to,
                             const float* sums, int states, int rows_held) {
#pragma clang fp contract(off)  // (a code times its scale is the infinity that is added: fused with the sum it would be a number of any size)
  __syncthreads();  // what this workgroup has written is read below
  const int d = threadIdx.x % kD;
  for (int r = threadIdx.x / kD; r < rows; r += kThreads / kD) {
    bool any = a.partials != nullptr;  // (the join's to say)
    for (int v = 0; v < states; ++v) any |= sums[v * rows_held + r] != 0.0f;
    if (!any) continue;
    const int row = p.r0 + r, end = min(to, sees(a, p, row));
    float x = 0.0f;
    for (int pos = from; pos < end; ++pos) {
      const int64_t at = row_of(a.m, p.b, kvh, pos);
      if (at < 0) continue;
      float v;
      if constexpr (coded(PAGE)) {  // as Block::widen makes it: a pool from elsewhere may hold what exceeds the type
        Codes8<PAGE> code;
        if constexpr (PAGE == LRQK_PAGE_E2M1) code = static_cast<const uint8_t*>(a.V)[(at * kD + d) >> 1] >> (d & 1) * 4;
        else code = make_uint2(static_cast<const uint8_t*>(a.V)[at * kD + d], 0u);
        const float scale = scale_of(a.V_scale[at * kScales + d / kScaleBlock]);
        if constexpr (BF16) {
          v = __uint_as_float(decode8_bf16<PAGE>(code, scale).x << 16);
        } else {
          float f[8];
          decode8<PAGE>(code, scale, f);
          v = f[0];
        }
      } else if constexpr (PAGE == LRQK_PAGE_BF16) {
        v = __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.V)[at * kD + d] << 16);
      } else {
        v = static_cast<const float*>(a.V)[at * kD + d];
      }
      if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) x += v;
    }
    if (x == 0.0f) continue;
    const int64_t at = (int64_t)(p.s.first + row / a.G) * (a.m.Hkv * a.G) + kvh * a.G + row % a.G;
    if (a.partials) a.partials[(at * a.pieces + piece) * kPartial + 4 + d] += x;
    else if (BF16) {
      __bf16* o = static_cast<__bf16*>(a.out) + at * kD + d;
      *o = (__bf16)((float)*o + x);
    } else {
      static_cast<float*>(a.out)[at * kD + d] += x;
    }
  }
}

// The four wavefronts' bits of a block's rows, as scalars.
template <int BITS>
__device__ __forceinline__ uint64_t gather_there(const uint16_t* there) {
  uint64_t x;
  if constexpr (BITS == 16) __builtin_memcpy(&x, there, 8);
  else x = there[0] | there[1] << 8 | there[2] << 16 | (uint64_t)there[3] << 24;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (uint64_t)hi << 32 | lo;
}

// The rounds of a tile in bf16: blocks of 64 positions, two steps (Rows::step) a round.  Round t multiplies with V of
// block t and with K of block t + 1 while K of block t + 2 and V of block t + 1 are on their way.  Even rounds read K from
// buffer 1 and V from buffer 0, odd ones the others: arrays and code of their own, so that the compiler sees that the
// rows on their way are not those that are read, and does not wait for them.
template <int PAGE>
struct TileLoop {
  static constexpr int BN = 64;
  using B = Block<true, PAGE, BN, kWaves>;
  const Args& a;
  const Problem& p;
  int kvh, w, lane, from, end, least, my_least;
  bool busy, cleared;
  float c;
  Rows<true>& r;
  uint16_t (*there)[4];  // of four blocks
  B blk;
  typename B::Found fk, fv;  // block t + 2's rows, block t + 1's
  typename B::Held hk, hv;
  f32x16 s;
  typename Rows<true>::Weights x;

  // block i's rows on their way: of K
  __device__ __forceinline__ void fetch_k(int i, char* kt) {
    const int p0 = from + i * BN + w * B::kMine;
    blk.find(a, p.b, kvh, p0, end, lane, fk);
    if constexpr (coded(PAGE)) B::load(a, p.b, kvh, end, a.K, a.K_scale, fk, lane, hk);
    else B::template load_direct<false>(a.K, fk, w, lane, kt);
    if (lane == 0) there[i & 3][w] = (uint16_t)fk.there;
    blk.look_up(a.m, p.b, p0 + BN, end);
  }
  // of V, found before
  __device__ __forceinline__ void fetch_v(int i, char* vt) {
    if constexpr (coded(PAGE)) {
      B::load(a, p.b, kvh, end, a.V, a.V_scale, fv, lane, hv);
    } else {
      const bool part = from + (i + 1) * BN > least;
      if (__builtin_expect(fv.there == B::kAll && !part, 1)) {
        B::template load_direct<true>(a.V, fv, w, lane, vt);
      } else {  // few blocks: the pieces' last, and those on missing pages
        B::load(a, p.b, kvh, end, a.V, nullptr, fv, lane, hv);
        cleared |= B::store_v(hv, fv.there, part, w, lane, vt);
      }
    }
  }
  // what came through registers goes into LDS; all that this wavefront has fetched is there
  __device__ __forceinline__ void arrive(bool k, char* kt, int i_v, char* vt) {
    if constexpr (coded(PAGE)) {
      if (k) B::store_k(hk, w, lane, kt);
      cleared |= B::store_v(hv, fv.there, from + (i_v + 1) * BN > least, w, lane, vt);
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
  }
  __device__ __forceinline__ void mask_scores(f32x16& y, int p0, uint32_t bits) {
    if (__builtin_expect(!(p0 + 32 <= my_least && bits == 0xffffffffu), 0)) {
      asm volatile("");  // a branch: taken by few blocks
      r.mask(y, p0, bits, lane);
    }
  }

  // round t of n - 1; kt, vt: what it reads; kt_to, vt_to: where the rows of blocks t + 2 and t + 1 go
  __device__ __forceinline__ void round(int t, int n, char* kt, char* vt, char* kt_to, char* vt_to) {
    arrive(true, kt, t, vt);
    __syncthreads();
    fv = fk;  // (block t + 1's rows)
    if (t + 2 < n) fetch_k(t + 2, kt_to);
    fetch_v(t + 1, vt_to);
    if (!busy) return;
    const int p0 = from + t * BN;
    f32x16 next;
    mask_scores(s, p0 + 32, (uint32_t)(gather_there<16>(there[t & 3]) >> 32));
    r.template step<true>(s, next, x, kt, vt, c, lane);
    mask_scores(next, p0 + BN, (uint32_t)gather_there<16>(there[(t + 1) & 3]));
    r.template step<true>(next, s, x, kt + 32 * kRowB<true>, vt + 32 * kRowB<true>, c, lane);
  }

  __device__ __forceinline__ void run(char* kt0, char* vt0, char* kt1, char* vt1) {
    const int n = (end - from + BN - 1) / BN;
    blk.look_up(a.m, p.b, from + w * B::kMine, end);
    fetch_k(0, kt0);
    if constexpr (coded(PAGE)) B::store_k(hk, w, lane, kt0);
    fv = fk;
    if (n > 1) fetch_k(1, kt1);
    fetch_v(0, vt0);
    if constexpr (!coded(PAGE)) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (busy) {
      f32x16 first = r.scores(kt0, lane);
      mask_scores(first, from, (uint32_t)gather_there<16>(there[0]));
      r.template step<false>(first, s, x, kt0 + 32 * kRowB<true>, nullptr, c, lane);
    }
    int t = 0;
    for (; t + 2 < n; t += 2) {
      round(t, n, kt1, vt0, kt0, vt1);
      round(t + 1, n, kt0, vt1, kt1, vt0);
    }
    if (t + 1 < n) {
      round(t, n, kt1, vt0, kt0, vt1);
      ++t;
    }
    char* const vt = t & 1 ? vt1 : vt0;
    arrive(false, nullptr, t, vt);
    __syncthreads();
    if (busy) {
      mask_scores(s, from + t * BN + 32, (uint32_t)(gather_there<16>(there[t & 3]) >> 32));
      r.output(vt, x, lane);
      x = r.settle(s, c);
      r.output(vt + 32 * kRowB<true>, x, lane);
    }
  }
};

// Rounds without a pipeline of steps, the next block on its way: tiles in fp32, which take blocks of 32 positions, and pairs,
// where a wavefront attends to one half of a block of 64.
template <bool BF16, int PAGE, int BLOCK>
struct PlainLoop {
  static constexpr int BN = BLOCK;
  using B = Block<BF16, PAGE, BN, kWaves>;
  const Args& a;
  const Problem& p;
  int kvh, w, lane, from, end, least, my_least;
  bool busy, cleared;
  float c;
  Rows<BF16>& r;
  uint16_t (*there)[4];
  int half;  // of the block that the wavefront attends to
  B blk;
  struct Way {  // a block on its way: to its buffer in LDS, or, 8-bit, through registers
    char *k, *v;
    typename B::Found f;
    typename B::Held hk, hv;
  };

  // (the table entries are asked for before the rows: who waits for them does not wait for these)
  __device__ __forceinline__ void fetch(int p0, Way& x) {
    const int mine = p0 + w * B::kMine;
    blk.find(a, p.b, kvh, mine, end, lane, x.f);
    blk.look_up(a.m, p.b, mine + BN, end);
    if constexpr (coded(PAGE)) {
      B::load(a, p.b, kvh, end, a.K, a.K_scale, x.f, lane, x.hk);
      B::load(a, p.b, kvh, end, a.V, a.V_scale, x.f, lane, x.hv);
    } else {
      B::template load_direct<false>(a.K, x.f, w, lane, x.k);
      const bool part = p0 + BN > least;
      if (__builtin_expect(x.f.there == B::kAll && !part, 1)) {
        B::template load_direct<true>(a.V, x.f, w, lane, x.v);
      } else {
        B::load(a, p.b, kvh, end, a.V, nullptr, x.f, lane, x.hv);
        cleared |= B::store_v(x.hv, x.f.there, part, w, lane, x.v);
      }
    }
    if (lane == 0) there[(p0 - from) / BN & 3][w] = (uint16_t)x.f.there;
  }
  // The block at p0; the next one is on its way, or, with 8-bit rows, the one after the next.
  __device__ __forceinline__ void round(int p0, Way& now, Way& other) {
    if constexpr (coded(PAGE)) {
      B::store_k(now.hk, w, lane, now.k);
      cleared |= B::store_v(now.hv, now.f.there, p0 + BN > least, w, lane, now.v);
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __syncthreads();
    if constexpr (coded(PAGE)) {
      if (p0 + 2 * BN < end) fetch(p0 + 2 * BN, now);
    } else {
      if (p0 + BN < end) fetch(p0 + BN, other);
    }
    const int off = 32 * half;
    if (busy)
      r.attend(now.k + off * kRowB<BF16>, now.v + off * kRowB<BF16>, p0 + off,
               (uint32_t)(gather_there<BN / kWaves>(there[(p0 - from) / BN & 3]) >> off), p0 + off + 32 <= my_least, c, lane);
  }
  __device__ __forceinline__ void run(char* kt0, char* vt0, char* kt1, char* vt1) {
    Way x{kt0, vt0, {}, {}, {}}, y{kt1, vt1, {}, {}, {}};
    blk.look_up(a.m, p.b, from + w * B::kMine, end);
    fetch(from, x);
    if (coded(PAGE) && from + BN < end) fetch(from + BN, y);
    for (int p0 = from; p0 < end; p0 += 2 * BN) {
      round(p0, x, y);
      if (p0 + BN < end) round(p0 + BN, y, x);
    }
  }
};

// 128 rows of the problem, 32 a wavefront.  Bound by the matrix cores and the vector instructions between their products: a
// step of 32 positions has 16 products (32 cycles each) and some 65 vector instructions, and two wavefronts a SIMD are what
// the registers allow.  2048 tokens at 32K, bf16, 32 + 8 heads: 1040 to 1075 us from card to card, 1.0 PFLOP/s, matrix cores busy 45% of the cycles, no
// LDS bank conflict; 8-bit rows are decoded once a workgroup, between the rounds (1024 tokens at 128K of e4m3: 2440 us,
// 0.90 PFLOP/s).  64 rows a wavefront, one a SIMD, halve the decoding and the reads of LDS and took longer (1160 and 3007 us
// where this took 1030 and 2560): what a wavefront waits for is then not covered by another one's products.  Decoding between a
// step's products does not fit the registers (90 spilled).  fp32: 1001 tokens at 5003 and 744 at 1315, 665 us with the join, 112 TFLOP/s; 2048 tokens at 16K
// 131 TFLOP/s of the 153 that a matrix product reaches.
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kThreads, 2) void attend_tile_kernel(const Args a) {
  using Loop = std::conditional_t<BF16, TileLoop<PAGE>, PlainLoop<false, PAGE, 32>>;
  constexpr int M = 128, BN = Loop::BN, kTile = BN * kRowB<BF16>;
  __shared__ __align__(16) char kt0[kTile], vt0[kTile], kt1[kTile], vt1[kTile];
  __shared__ __align__(8) uint16_t there[4][4];
  __shared__ float sums[M];
  // KV head fastest: the dies take workgroups in turn, so a head's rows stay in one die's L2
  const int kvh = blockIdx.x % a.m.Hkv;
  Problem p;
  if (!find_unit<M, true>(a, blockIdx.x / a.m.Hkv, p)) return;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = min(M, p.rows - p.r0);
  const int least = sees(a, p, p.r0), most = sees(a, p, p.r0 + rows - 1);
  const int from = p.piece * p.step, end = min(most, from + p.step);
  if (from >= end && p.piece > 0) return;  // (piece 0 writes the rows that see nothing)
  const int mine = p.r0 + w * 32 + (lane & 31), last = p.rows - 1;  // rows behind the last repeat it
  Rows<BF16> r;
  const int real = min(mine, last);
  r.see = sees(a, p, real);
  r.start(a.q, (int64_t)(p.s.first + real / a.G) * (a.m.Hkv * a.G) + kvh * a.G + real % a.G, a.scale < 0.0f, lane);
  bool cleared = false;
  if (from < end) {
    Loop loop{a, p, kvh, w, lane, from, end, least, sees(a, p, min(p.r0 + w * 32, last)), p.r0 + w * 32 <= last, false,
              log2_scale(a), r, there};
    loop.run(kt0, vt0, kt1, vt1);
    cleared = loop.cleared;
  }
  r.sum = sum_halves(r.sum);
  if (lane < 32) sums[w * 32 + lane] = r.sum;
  if (mine < p.rows) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        put<BF16>(a, p, kvh, mine, p.piece, 32 * t + 8 * e + 4 * (lane >> 5),
                  f32x4{r.o[t][4 * e], r.o[t][4 * e + 1], r.o[t][4 * e + 2], r.o[t][4 * e + 3]}, r.mx, r.sum);
  }
  if (__syncthreads_or(cleared))
    add_left_out<BF16, PAGE>(a, p, kvh, rows, p.piece, max(from, least - least % BN), end, sums, 1, M);
}

// The states of several wavefronts at the same rows joined and put: `n` of them, that of state v and row i at
// acc[(v * rows_held + i) * 128], its 16-byte chunks turned by i % 32, its maximum and sum at mx[v * rows_held + i] and sum[..].
template <bool BF16>
__device__ __forceinline__ void join_states(const Args& a, const Problem& p, int kvh, int rows, int n, int rows_held,
                                            const float* acc, const float* wm, const float* ws) {
  for (int k = threadIdx.x; k < rows * (kD / 4); k += kThreads) {
    const int row = k / (kD / 4), chunk = k % (kD / 4);
    f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
    float mx = -INFINITY, sum = 0.0f;
    for (int v = 0; v < n; ++v) mx = fmaxf(mx, wm[v * rows_held + row]);
    for (int v = 0; v < n; ++v) {
      const int i = v * rows_held + row;
      const float f = weight_of(wm[i], ws[i], mx);
      sum += ws[i] * f;
      const f32x4 y = *reinterpret_cast<const f32x4*>(acc + (size_t)i * kD + 4 * (chunk ^ (row & 31)));
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = __builtin_fmaf(f, y[e], x[e]);
    }
    put<BF16>(a, p, kvh, p.r0 + row, p.piece, 4 * chunk, x, mx, sum);
  }
}
// A wavefront's state as state v, rows i0 .. i0 + 31, of those.
template <bool BF16>
__device__ __forceinline__ void leave_state(const Rows<BF16>& r, int at, int lane, float* acc, float* wm, float* ws) {
  const int i = lane & 31, h = lane >> 5;
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4*>(acc + (size_t)(at + i) * kD + 4 * ((8 * t + 2 * e + h) ^ i)) =
          f32x4{r.o[t][4 * e], r.o[t][4 * e + 1], r.o[t][4 * e + 2], r.o[t][4 * e + 3]};
  const float sum = sum_halves(r.sum);
  if (h == 0) {
    wm[at + i] = r.mx;
    ws[at + i] = sum;
  }
}

// At most 32 rows a workgroup: K and V are read once and the matrix cores wait, so this is bound by memory where there is
// enough of it to read, and by the latency of loads that depend on each other where there is little.  No barrier between a
// wavefront's blocks, the next one in registers on its way.  One token of 16 sequences of 8K to 128K, e4m3, 2.1 GB: 383 us with
// the join, 5.6 TB/s; one token at 4K, bf16: 13 us, 8 of them here and 4 in the join.
template <bool BF16, int PAGE, bool SMALL>
__global__ __launch_bounds__(kThreads, BF16 ? 2 : 1) void attend_thin_kernel(const Args a) {
  constexpr int M = 32, BN = 32;
  constexpr int kTile = BN * kRowB<BF16>;
  extern __shared__ __align__(16) char lds[];  // per wavefront: K, V
  __shared__ float wm[kWaves * M], ws[kWaves * M];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % a.m.Hkv;
  // the grid is as large as the chip: how many units there are is known here alone
  for (int unit = blockIdx.x / a.m.Hkv;; unit += gridDim.x / a.m.Hkv) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // what follows from it is made anew for a unit, and not kept in registers over all
    Problem p;
    if (!find_unit<M, !BF16>(a, unit, p)) return;
    const int rows = min(M, p.rows - p.r0);
    const int least = sees(a, p, p.r0), most = sees(a, p, p.r0 + rows - 1);
    const int from = p.piece * p.step, end = min(most, from + p.step);
    if (from >= end && p.piece > 0) continue;  // (piece 0 writes the rows that see nothing)
    Rows<BF16> r;
    const int real = min(p.r0 + (lane & 31), p.rows - 1);
    r.see = sees(a, p, real);
    r.start(a.q, (int64_t)(p.s.first + real / a.G) * (a.m.Hkv * a.G) + kvh * a.G + real % a.G, a.scale < 0.0f, lane);
    const float c = log2_scale(a);
    char* const kt = lds + w * 2 * kTile;
    char* const vt = kt + kTile;
    bool cleared = false;
    const int mine = from + w * BN;
    if (mine < end) {
      using B = Block<BF16, PAGE, BN, 1, SMALL>;
      B blk;
      typename B::Found f;
      typename B::Held hk, hv;
      auto fetch = [&](int p0) __attribute__((always_inline)) {
        blk.find(a, p.b, kvh, p0, end, lane, f);
        B::load(a, p.b, kvh, end, a.K, a.K_scale, f, lane, hk);
        B::load(a, p.b, kvh, end, a.V, a.V_scale, f, lane, hv);
        blk.look_up(a.m, p.b, p0 + kWaves * BN, end);
      };
      blk.look_up(a.m, p.b, mine, end);
      fetch(mine);
      for (int p0 = mine; p0 < end; p0 += kWaves * BN) {
        __builtin_amdgcn_wave_barrier();  // the wavefront's LDS operations execute in order
        B::store_k(hk, 0, lane, kt);
        cleared |= B::store_v(hv, f.there, p0 + BN > least, 0, lane, vt);
        __builtin_amdgcn_wave_barrier();
        const uint32_t there = f.there;
        if (p0 + kWaves * BN < end) fetch(p0 + kWaves * BN);
        r.attend(kt, vt, p0, there, p0 + BN <= least, c, lane);
      }
    }
    __syncthreads();  // (in fp32 a state lies where another wavefront's rows were)
    leave_state(r, w * M, lane, reinterpret_cast<float*>(lds), wm, ws);
    __syncthreads();
    join_states<BF16>(a, p, kvh, rows, kWaves, M, reinterpret_cast<const float*>(lds), wm, ws);
    if (__syncthreads_or(cleared))
      add_left_out<BF16, PAGE>(a, p, kvh, rows, p.piece, max(from, least - least % BN), end, ws, kWaves, M);
  }
}

// ---- 16 rows of the problem, or 32, in a wavefront: pages of 4 bits -------------------------------------------
// Lane l: row l % 16 of a set; the 16 positions of a tile of S^T are 4 (l / 16) + v, v the register; elements of O^T likewise.
// A row of K goes straight from its load into the product: the sum over elements may run in any order, so that the lane
// that holds 32 codes of a row, one block with one scale, multiplies them eight at a time with those eight of its q.
// In fp32, K and V are exact in bf16 all the same, and q and the weights are sums of three bf16 numbers each, exactly: three bf16
// products in place of one fp32 product, which takes sixteen times as long as one.  (A term below 2^-126 may count for 0.)
template <bool BF16>
struct Set16 {
  static constexpr int kTerms = BF16 ? 1 : 3;  // of q, and of a weight
  uint4 q[kTerms][4];  // elements 32 (l / 16) + 8 s .. + 7
  f32x4 o[8];          // elements 16 t ..
  float mx, sum;
  int see;             // positions that the lane's row sees

  __device__ __forceinline__ void start(const void* base, int64_t row, bool negate, int lane) {
    const uint32_t flip = negate ? 0x80008000u : 0u;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int64_t chunk = row * 16 + 4 * (lane >> 4) + s;  // eight elements
      if constexpr (BF16) {
        uint4 x = static_cast<const uint4*>(base)[chunk];
        x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
        q[0][s] = x;
      } else {
        const float4 x = static_cast<const float4*>(base)[2 * chunk], y = static_cast<const float4*>(base)[2 * chunk + 1];
        uint32_t t[4][3];
        terms(x.x, x.y, t[0]);
        terms(x.z, x.w, t[1]);
        terms(y.x, y.y, t[2]);
        terms(y.z, y.w, t[3]);
#pragma unroll
        for (int i = 0; i < 3; ++i) q[i][s] = make_uint4(t[0][i] ^ flip, t[1][i] ^ flip, t[2][i] ^ flip, t[3][i] ^ flip);
      }
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) o[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    mx = -INFINITY;
    sum = 0.0f;
  }
  // Two fp32 numbers as three pairs of bf16 numbers that add up to them, exactly: the upper eight bits of their significands, the next
  // eight, the rest.  One that is not finite is its own first term, without others.
  static __device__ __forceinline__ void terms(float x, float y, uint32_t (&t)[3]) {
    const uint32_t u = __float_as_uint(x), v = __float_as_uint(y);
    t[0] = __builtin_amdgcn_perm(v, u, 0x07060302u);  // the upper halves
    float dx = x - __uint_as_float(u & 0xffff0000u), dy = y - __uint_as_float(v & 0xffff0000u);
    if ((u & 0x7f800000u) == 0x7f800000u) dx = 0.0f;
    if ((v & 0x7f800000u) == 0x7f800000u) dy = 0.0f;
    more_terms(dx, dy, t);
    if (((u & 0x7f800000u) == 0x7f800000u) && (u & 0x7fffffu)) t[0] |= 0x00007fffu;  // (a NaN stays one without its lower half)
    if (((v & 0x7f800000u) == 0x7f800000u) && (v & 0x7fffffu)) t[0] |= 0x7fff0000u;
  }
  static __device__ __forceinline__ void more_terms(float dx, float dy, uint32_t (&t)[3]) {
    const uint32_t u = __float_as_uint(dx), v = __float_as_uint(dy);
    t[1] = __builtin_amdgcn_perm(v, u, 0x07060302u);
    dx -= __uint_as_float(u & 0xffff0000u);
    dy -= __uint_as_float(v & 0xffff0000u);
    t[2] = __builtin_amdgcn_perm(__float_as_uint(dy), __float_as_uint(dx), 0x07060302u);
  }
  // scores of 16 positions: a tile of K, row l % 16, block l / 16, eight elements each; `low`: what q's terms after the first
  // meet, the same without elements that are not finite (an infinity times a term of 0 would be NaN)
  __device__ __forceinline__ f32x4 scores(const uint4 (&tile)[4], const uint4 (&low)[4]) const {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = kTerms - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, i > 0 ? low[k] : tile[k]), __builtin_bit_cast(bf16x8, q[i][k]), s,
                                                    0, 0, 0);
    return s;
  }
  // scores of the 16 positions from p0 that the row does not see, or that are not there, become -infinity
  __device__ __forceinline__ void mask(f32x4& s, int p0, uint32_t there, int lane) const {
    const int up_to = see - p0;
    const uint32_t mine = (up_to >= 16 ? there : up_to <= 0 ? 0u : there & ((1u << up_to) - 1)) >> (4 * (lane >> 4));
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = mine & (1u << e) ? s[e] : -INFINITY;
  }
  static __device__ __forceinline__ float over_lanes(float x) {  // the largest of the four lanes of a row
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_halves(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
  }
  static __device__ __forceinline__ float sum_lanes(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sum_halves(__uint_as_float(r[0]) + __uint_as_float(r[1]));
  }
  __device__ __forceinline__ void raise(float top) {
    const float to = fmaxf(mx, top);
    const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(mx - to);
    sum *= f;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][e] *= f;
    mx = to;
  }
  // the largest score of 64 positions, in units of log2
  static __device__ __forceinline__ float largest(const f32x4 (&s)[4], float c) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, s[i][e]);
    return over_lanes(top) * c;
  }
  // Weights of 64 positions (see Rows::weigh and weigh_any) as the second product's operands, 32 each.  FAR: some row's maximum is
  // beyond kFar.
  struct Weights {
    uint4 of[2][kTerms];
  };
  template <bool FAR>
  __device__ __forceinline__ void weigh(const f32x4 (&s)[4], float c, Weights& x) {
    const float base = mx == -INFINITY ? 0.0f : mx;
    const bool rounded = FAR && fabsf(mx) >= kFar;
    const auto weight = [&](float y) {
#pragma clang fp contract(off)
      if constexpr (FAR) {
        const float z = y * c;
        return __builtin_amdgcn_exp2f(rounded ? z - base : __builtin_fmaf(y, c, -base));
      } else {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(y, c, -base));
      }
    };
    const dev::bf16x2 one = __builtin_bit_cast(dev::bf16x2, 0x3f803f80u);
    float add[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[4][3];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float u = weight(s[2 * i + e / 2][2 * e % 4]), v = weight(s[2 * i + e / 2][2 * e % 4 + 1]);
        if constexpr (BF16) {
          w[e][0] = dev::pack_bf16(u, v);
          add[i] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(dev::bf16x2, w[e][0]), one, add[i], false);
        } else {  // (a weight that is not finite makes its row NaN through any of them)
          w[e][0] = __builtin_amdgcn_perm(__float_as_uint(v), __float_as_uint(u), 0x07060302u);
          more_terms(u - __uint_as_float(__float_as_uint(u) & 0xffff0000u), v - __uint_as_float(__float_as_uint(v) & 0xffff0000u), w[e]);
          add[i] += u + v;
        }
      }
#pragma unroll
      for (int n = 0; n < kTerms; ++n) x.of[i][n] = make_uint4(w[0][n], w[1][n], w[2][n], w[3][n]);
    }
    sum += add[0] + add[1];
  }
};
__device__ __forceinline__ uint4 cleared_chunk(uint4 x) {
  return make_uint4(clear<true>(x.x), clear<true>(x.y), clear<true>(x.z), clear<true>(x.w));
}
constexpr uint32_t kOddScale = 253;  // scale byte of e2m1 from which an element can be an infinity, or NaN
enum { kPlus = 1, kMinus = 2, kNan = 4 };
// What is not finite in the lane's 32 elements of each of the four tiles' rows, those that are there: `which`, by element.  A branch
// that few blocks take.  256 tokens of 4 heads at 8K: 32 us without such elements, 44 with one block of them in every unit's way, 228 where V
// holds nothing else (1962 with one block while a unit looked for it again at its end, position by position).
__device__ __forceinline__ void note_odd(const uint4 (&v)[4], const uint32_t (&vs)[4], const uint32_t (&there)[4], int lane,
                                         uint32_t* which, int& any) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (vs[i] < kOddScale || !((there[i] >> (lane & 15)) & 1)) continue;
    const float f = scale_bits(vs[i]);
#pragma unroll 1
    for (int j = 0; j < 4; ++j) {
      const uint32_t code = j == 0 ? v[i].x : j == 1 ? v[i].y : j == 2 ? v[i].z : v[i].w;
      const uint4 y = decode8_bf16<LRQK_PAGE_E2M1>(code, f);
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const uint32_t pair = e < 2 ? y.x : e < 4 ? y.y : e < 6 ? y.z : y.w, x = (e & 1 ? pair >> 16 : pair) & 0xffffu;
        if ((x & 0x7f80u) != 0x7f80u) continue;
        const uint32_t bit = x & 0x7fu ? kNan : x & 0x8000u ? kMinus : kPlus;
        uint32_t* const to = which + 32 * (lane >> 4) + 8 * j + e;
        if (!(*to & bit)) atomicOr(to, bit);  // (so that a context full of them does not wait for its atomics)
        any = 1;
      }
    }
  }
}
// Those given to all rows of the unit that have a weight.
__device__ __forceinline__ void add_everywhere(const Args& a, const Problem& p, int kvh, int rows, uint32_t* which, const float* sums,
                                               int rows_held) {
  const int d = threadIdx.x % kD;
  const uint32_t bits = which[d];
  const float x = bits == kPlus ? INFINITY : bits == kMinus ? -INFINITY : __uint_as_float(0x7fc00000u);
  for (int r = threadIdx.x / kD; bits && r < rows; r += kThreads / kD) {
    bool any = a.partials != nullptr;  // (the join's to say)
    for (int v = 0; v < kWaves; ++v) any |= sums[v * rows_held + r] != 0.0f;
    if (!any) continue;
    const int row = p.r0 + r;
    const int64_t at = (int64_t)(p.s.first + row / a.G) * (a.m.Hkv * a.G) + kvh * a.G + row % a.G;
    float* const to = a.partials ? a.partials + (at * a.pieces + p.piece) * kPartial + 4 + d : static_cast<float*>(a.out) + at * kD + d;
    *to += x;  // (after add_left_out, whose thread has the same elements)
  }
  __syncthreads();
  if (threadIdx.x < kD) which[threadIdx.x] = 0;
  __syncthreads();
}
// Where LDS holds chunk c of a row of V: eight rows' same chunk (as they are stored) lies in eight places mod 8, eight rows' two
// chunks (as they are read) in sixteen.
__device__ __forceinline__ int few_chunk(int row, int c) {
  return row * kRowB<true> + ((c ^ (((row & 7) << 1) | ((row >> 2) & 1))) << 4);
}

// At most 16 NS rows a workgroup, pages of 4 bits: a wavefront takes every fourth block of 64 positions, four tiles of 16, each of
// which lies in one page.  K does not touch LDS; V passes through 16 KB of it.  Two sets of rows share the
// decoded tiles; both are always worked on (with code of its own for units that have one set of rows only, 180 bytes of registers spilled
// and the whole took 1.6 to 2 times as long), and the maximum is looked at for both together.
// One set: bound by memory where there is enough of it: one token of 16 sequences of 8K to 128K, 1.10 GB, 202 us and 5 for the
// join, 5.4 TB/s (as thin workgroups 265); vector instructions are busy 37 % of the cycles, matrix cores 13 %, no LDS bank
// conflict.  Blocks two ahead changed nothing; three wavefronts a SIMD do not get the registers without spilling (340 us).  One token at
// 4K: 7.4 us and 3.4, a chain of loads that wait for each other.  Two sets: bound by the latency of what a block does one after
// the other, two wavefronts a SIMD covering it; 28 rows of 8 sequences of 32K, 285 MB, 76 to 82 us (thin 128); 1 to 5
// tokens of 8 sequences of 7K to 64K, 7 heads a group, 99 MB, 40 us and 4 (pairs 48 and 6).  Three sets spill 200 bytes.  Both
// sets are worked on for a call with n_max for more than 16 rows, also if a sequence brings one token: 265 us for 16 sequences of up to 128K
// (208 with n_max for 16 rows), 51 for 64 of up to 4K (44), 12.2 for one of 4K (11.3).
// fp32, one set, bound by the products and the vector instructions about them: with the joins, one token of 16 sequences of up to 128K
// 293 us (on the fp32 matrix cores, 32 rows a tile, 2486), the drafts 58 (399), 1001 tokens at 5003 and 744 at 1315 283 (676), 2048 tokens
// at 32K 3.3 ms, 322 TFLOP/s (8.3).
template <int NS, bool BF16>
__global__ __launch_bounds__(kThreads, 2) void attend_few_kernel(const Args a) {
  using Set = Set16<BF16>;
  constexpr int M = 16 * NS, BN = 64, kTile = BN * kRowB<true>, kStep = kWaves * BN;
  __shared__ __align__(16) char lds[kWaves * kTile];  // a wavefront's rows of V; then the states
  __shared__ float wm[kWaves * M], ws[kWaves * M];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kvh = blockIdx.x % a.m.Hkv;
  const uint4* const K = static_cast<const uint4*>(a.K);
  const uint4* const V = static_cast<const uint4*>(a.V);
  // fp32: what was left out of blocks that every row of the unit sees, by element; whether that is anything, in this unit and the next
  __shared__ uint32_t everywhere[BF16 ? 1 : kD];
  __shared__ int any_everywhere[2];
  int turn = 0;
  if constexpr (!BF16) {
    if (threadIdx.x < kD) everywhere[threadIdx.x] = 0;
    if (threadIdx.x < 2) any_everywhere[threadIdx.x] = 0;
    __syncthreads();
  }
  Problem p;
  Cursor cursor{0, 0};
  Seq first = lane_sequence(a, 0);
  p.step = piece_of<true>(a, first);
  for (int unit = blockIdx.x / a.m.Hkv;; unit += gridDim.x / a.m.Hkv) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // what follows from it is made anew for a unit, and not kept in registers over all
    if (!find_from<M>(a, unit, p, unit < gridDim.x / a.m.Hkv ? first : lane_sequence(a, cursor.i0), cursor)) return;
    const int rows = min(M, p.rows - p.r0);
    const int least = sees(a, p, p.r0), most = sees(a, p, p.r0 + rows - 1);
    const int from = p.piece * p.step, end = min(most, from + p.step);
    if (from >= end && p.piece > 0) continue;  // (piece 0 writes the rows that see nothing)
    Set r[NS];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int real = min(p.r0 + 16 * n + (lane & 15), p.rows - 1);
      r[n].see = sees(a, p, real);
      r[n].start(a.q, (int64_t)(p.s.first + real / a.G) * (a.m.Hkv * a.G) + kvh * a.G + real % a.G, a.scale < 0.0f, lane);
    }
    const float c = log2_scale(a);
    char* const vt = lds + w * kTile;
    bool cleared = false;
    const int mine = from + w * BN;
    if (mine < end) {
      const int32_t* const table = a.m.table + (size_t)p.b * a.m.max_pages;
      const uint32_t in_page = (1u << a.m.page_log2) - 1;
      const uint32_t at = 4 * (lane & 15) + (lane >> 4);  // chunk, and scale, of the lane within a tile
      int pg[4];
      uint32_t place[4], there[4];
      uint4 k[4], v[4];
      uint32_t ks[4], vs[4];
      auto look_up = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) pg[i] = table[(uint32_t)min(p0 + 16 * i, end - 1) >> a.m.page_log2];
      };
      auto find = [&](int p0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t page = __builtin_amdgcn_readfirstlane(pg[i]);
          const int q = p0 + 16 * i, n = page < (uint32_t)a.m.n_pages ? min(max(end - q, 0), 16) : 0;
          place[i] = n > 0 ? page * a.page16 + (((uint32_t)kvh << a.m.page_log2) + ((uint32_t)q & in_page)) * 4 : 0;
          there[i] = (1u << n) - 1;
        }
      };
      auto fetch = [&](const uint4* base, const uint8_t* scale, uint4 (&x)[4], uint32_t (&y)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = (base + (size_t)place[i])[at];
          y[i] = (scale + (size_t)place[i])[at];  // (a row is four chunks and has four scales)
        }
      };
      look_up(mine);
      find(mine);
      fetch(K, a.K_scale, k, ks);
      fetch(V, a.V_scale, v, vs);
      look_up(mine + kStep);
      bool far = false;
      for (int p0 = mine; p0 < end; p0 += kStep) {
        const bool part = p0 + BN > least, more = p0 + kStep < end;
        // fp32: what is not finite is left out wherever it is, since it would meet weights' terms that are 0.  In blocks that every row of
        // the unit sees it is noted here, element by element, and not looked for again
        const bool leave_out = part || (!BF16 && __any(max(max(vs[0], vs[1]), max(vs[2], vs[3])) >= kOddScale));
        const bool whole = !part && (there[0] & there[1] & there[2] & there[3]) == 0xffffu;
        bool left = false;
        uint32_t now[4];
        // V into LDS, all 64 positions, long before it is read
        __builtin_amdgcn_wave_barrier();  // the wavefront's LDS operations execute in order
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          now[i] = there[i];
          const float f = scale_bits(vs[i]);
          const uint32_t word[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            uint4 y = decode8_bf16<LRQK_PAGE_E2M1>(word[j], f);
            if (!whole || leave_out) {
              if (!((now[i] >> (lane & 15)) & 1)) y = make_uint4(0, 0, 0, 0);
              if (leave_out) {
                left |= odd<true>(y.x) || odd<true>(y.y) || odd<true>(y.z) || odd<true>(y.w);
                y = cleared_chunk(y);
              }
            }
            *reinterpret_cast<uint4*>(vt + few_chunk(16 * i + (lane & 15), 4 * (lane >> 4) + j)) = y;
          }
        }
        if (BF16 || part) {
          cleared |= left;
        } else if (__builtin_expect(leave_out, 0)) {
          if constexpr (!BF16) note_odd(v, vs, now, lane, everywhere, any_everywhere[turn]);
        }
        if (more) {
          find(p0 + kStep);
          fetch(V, a.V_scale, v, vs);
        }
        f32x4 s[NS][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float f = scale_bits(ks[i]);
          const uint32_t word[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
          uint4 tile[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) tile[j] = decode8_bf16<LRQK_PAGE_E2M1>(word[j], f);
          if (!BF16 && __builtin_expect(__any(ks[i] >= kOddScale), 0)) {
            uint4 low[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) low[j] = cleared_chunk(tile[j]);
            s[0][i] = r[0].scores(tile, low);
          } else {
#pragma unroll
            for (int n = 0; n < NS; ++n) s[n][i] = r[n].scores(tile, tile);
          }
        }
        if (more) {
          fetch(K, a.K_scale, k, ks);
          look_up(p0 + 2 * kStep);
        }
        __builtin_amdgcn_wave_barrier();
        float top[NS];
        bool raise = false;
        if (!whole) {
          asm volatile("");  // a branch: taken by few blocks
#pragma unroll
          for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) r[n].mask(s[n][i], p0 + 16 * i, now[i], lane);
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          top[n] = Set::largest(s[n], c);
          raise |= top[n] > r[n].mx + kLag;
        }
        if (__any(raise)) {
          bool beyond = false;
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            r[n].raise(top[n]);
            beyond |= fabsf(r[n].mx) >= kFar && r[n].mx != -INFINITY;
          }
          far = __any(beyond);
        }
        typename Set::Weights x[NS];
        if (__builtin_expect(far, 0)) {
#pragma unroll
          for (int n = 0; n < NS; ++n) r[n].template weigh<true>(s[n], c, x[n]);
        } else {
#pragma unroll
          for (int n = 0; n < NS; ++n) r[n].template weigh<false>(s[n], c, x[n]);
        }
        // the weights' order: 4 (l / 16) + j, then 16 + 4 (l / 16) + j
        const int g = lane & 15, row = 4 * (lane >> 4) + (g >> 2);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            s16x4 y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
              y[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(
                  vt + few_chunk(row + 16 * j + 32 * half, 2 * t + ((g & 3) >> 1)) + 8 * (g & 1)));
            const bf16x8 z = __builtin_bit_cast(bf16x8, __builtin_shufflevector(y[0], y[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
              for (int i = Set::kTerms - 1; i >= 0; --i)
                r[n].o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(z, __builtin_bit_cast(bf16x8, x[n].of[half][i]), r[n].o[t], 0, 0, 0);
          }
        }
      }
    }
    __syncthreads();  // (a state lies where other wavefronts' rows were)
    float* const acc = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int i = 16 * n + (lane & 15), to = w * M + i;
#pragma unroll
      for (int t = 0; t < 8; ++t)
        *reinterpret_cast<f32x4*>(acc + (size_t)to * kD + 4 * ((4 * t + (lane >> 4)) ^ i)) = r[n].o[t];
      const float sum = Set::sum_lanes(r[n].sum);
      if (lane < 16) {
        wm[to] = r[n].mx;
        ws[to] = sum;
      }
    }
    __syncthreads();
    join_states<BF16>(a, p, kvh, rows, kWaves, M, acc, wm, ws);
    if (a.partials && p.piece == 0 && (int)threadIdx.x < rows) {  // what attend_join_few_kernel goes by
      const int row = p.r0 + threadIdx.x;
      const int64_t at = (int64_t)(p.s.first + row / a.G) * (a.m.Hkv * a.G) + kvh * a.G + row % a.G;
      a.partials[at * a.pieces * kPartial + 2] = __int_as_float(max(1, (most + p.step - 1) / p.step));
    }
    if (!BF16 && threadIdx.x == 0) any_everywhere[turn ^ 1] = 0;  // (nobody looks at that one before the next unit)
    if (__syncthreads_or(cleared))
      add_left_out<BF16, LRQK_PAGE_E2M1>(a, p, kvh, rows, p.piece, max(from, least - least % BN), end, ws, kWaves, M);
    if constexpr (!BF16) {
      if (any_everywhere[turn]) add_everywhere(a, p, kvh, rows, everywhere, ws, M);
    }
    turn ^= 1;
  }
}

// 33 to 64 rows: rows of the pool are read and decoded once for all of them, which a thin workgroup per 32 rows would do
// twice.  Bound by the decoding and the barriers between blocks more than by memory.  1 to 5 tokens of 8 sequences of 7K to 64K,
// 7 heads a group, i8, 192 MB: 64 us with the join, 3.0 TB/s (75 with pieces from the longest sequence alone: no more than 372 of the 512
// workgroups had any; as thin workgroups with two sets of rows a wavefront 101).
template <int PAGE>
__global__ __launch_bounds__(kThreads, 2) void attend_pair_kernel(const Args a) {
  using Loop = PlainLoop<true, PAGE, 64>;
  constexpr int M = 64, BN = Loop::BN, kTile = BN * kRowB<true>;
  __shared__ __align__(16) char lds[4 * kTile];  // two buffers of K and V; then the states
  __shared__ __align__(8) uint16_t there[4][4];
  __shared__ float wm[2 * M], ws[2 * M];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), set = w & 1, half = w >> 1;
  const int kvh = blockIdx.x % a.m.Hkv;
  for (int unit = blockIdx.x / a.m.Hkv;; unit += gridDim.x / a.m.Hkv) {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));  // (as above)
    Problem p;
    if (!find_unit<M, true>(a, unit, p)) return;
    const int rows = min(M, p.rows - p.r0);
    const int least = sees(a, p, p.r0), most = sees(a, p, p.r0 + rows - 1);
    const int from = p.piece * p.step, end = min(most, from + p.step);
    if (from >= end && p.piece > 0) continue;
    Rows<true> r;
    const int real = min(p.r0 + 32 * set + (lane & 31), p.rows - 1);
    r.see = sees(a, p, real);
    r.start(a.q, (int64_t)(p.s.first + real / a.G) * (a.m.Hkv * a.G) + kvh * a.G + real % a.G, a.scale < 0.0f, lane);
    bool cleared = false;
    if (from < end) {
      Loop loop{a,     p,    kvh, w, lane, from, end, least, sees(a, p, min(p.r0 + 32 * set, p.rows - 1)), 32 * set < rows,
                false, log2_scale(a), r, there, half};
      loop.run(lds, lds + kTile, lds + 2 * kTile, lds + 3 * kTile);
      cleared = loop.cleared;
    }
    __syncthreads();
    leave_state(r, half * M + 32 * set, lane, reinterpret_cast<float*>(lds), wm, ws);
    __syncthreads();
    join_states<true>(a, p, kvh, rows, 2, M, reinterpret_cast<const float*>(lds), wm, ws);
    if (__syncthreads_or(cleared))
      add_left_out<true, PAGE>(a, p, kvh, rows, p.piece, max(from, least - least % BN), end, ws, 2, M);
  }
}

// The pieces of a row's context joined: W wavefronts a row, each takes its share of the pieces, a piece's maximum and sum
// in a lane, two elements a lane.  All loads of a share are independent of each other: bound by latency, 4 us of the 13 of one
// token at 4K (32 pieces), 8 of 383 at 16 sequences of up to 128K.
template <bool BF16, int W>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(const Args a, int64_t n_rows) {
  __shared__ float part[kWaves][2 + kD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
  const int64_t at = (int64_t)blockIdx.x * (kWaves / W) + wave / W;
  const int Hq = a.m.Hkv * a.G;
  const int t = (int)min(at / Hq, (int64_t)a.m.T);
  const int step = piece_of<true>(a, lane_sequence(a, 0));
  const int b = sequence_of(a.m, t);
  bool mine = at < n_rows && b >= 0;
  int pieces = 0;
  if (mine) {
    const Seq s = sequence(a.m, b);
    mine = t >= s.first && t < s.first + s.n;
    const int see = min(max(s.len - s.n + (t - s.first) + 1, 0), a.m.l_max);
    pieces = max(1, (see + step - 1) / step);
  }
  if (W == 1 && !mine) return;
  float mx = -INFINITY, sum = 0.0f, x0 = 0.0f, x1 = 0.0f;
  if (mine) {
    const float* P = a.partials + at * a.pieces * kPartial;
    const int share = (pieces + W - 1) / W, lo = min(pieces, w * share), hi = min(pieces, lo + share);
    for (int i0 = lo; i0 < hi; i0 += 64) {
      const int n = min(64, hi - i0);
      const float* p = P + (int64_t)(i0 + min(lane, n - 1)) * kPartial;
      const float m = lane < n ? p[0] : -INFINITY, l = lane < n ? p[1] : 0.0f;
      float top = fmaxf(mx, m);
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
      const float f = weight_of(m, l, top), g = weight_of(mx, sum, top);
      float add = l * f;
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) add += __shfl_xor(add, i);
      sum = sum * g + add;
      x0 *= g;
      x1 *= g;
      mx = top;
      p = P + (int64_t)i0 * kPartial + 4 + 2 * lane;
      for (int i = 0; i < n; i += 4) {
        float2 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const float2*>(p + (int64_t)min(i + j, n - 1) * kPartial);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i + j < n) {
            const float k = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i + j));
            x0 = __builtin_fmaf(k, x[j].x, x0);
            x1 = __builtin_fmaf(k, x[j].y, x1);
          }
      }
    }
  }
  if constexpr (W > 1) {
    if (lane == 0) {
      part[wave][0] = mx;
      part[wave][1] = sum;
    }
    part[wave][2 + 2 * lane] = x0;
    part[wave][3 + 2 * lane] = x1;
    __syncthreads();
    if (!mine || w != 0) return;
    float top = mx;
#pragma unroll
    for (int i = 1; i < W; ++i) top = fmaxf(top, part[wave + i][0]);
    sum = x0 = x1 = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const float f = weight_of(part[wave + i][0], part[wave + i][1], top);
      sum += part[wave + i][1] * f;
      x0 = __builtin_fmaf(f, part[wave + i][2 + 2 * lane], x0);
      x1 = __builtin_fmaf(f, part[wave + i][3 + 2 * lane], x1);
    }
  }
  x0 = sum == 0.0f ? 0.0f : x0 / sum;
  x1 = sum == 0.0f ? 0.0f : x1 / sum;
  if constexpr (BF16) static_cast<uint32_t*>(a.out)[at * (kD / 2) + lane] = dev::pack_bf16(x0, x1);
  else static_cast<float2*>(a.out)[at * (kD / 2) + lane] = make_float2(x0, x1);
}

// The same for attend_few_kernel's states: the number of a row's pieces stands with its first one, so that a row asks for
// everything at once, its first states before it knows how many there are, and nothing depends on the number of sequences (a
// token of 256 sequences, 8192 rows: 101 us in attend_join_kernel, where every row looks through their lengths; the whole call 281 us with
// that and 198 with this).  2.4 to 3.4 us for a token at 4K, 16 pieces.  W wavefronts a row:
// all of them weigh all pieces, each adds up every W-th.
template <bool BF16, int W>
__global__ __launch_bounds__(kThreads) void attend_join_few_kernel(const Args a, int64_t n_rows) {
  constexpr int kAhead = 8;
  __shared__ float2 part[kWaves][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % W;
  const int64_t at = (int64_t)blockIdx.x * (kWaves / W) + wave / W, row = min(at, n_rows - 1);
  const float* const P = a.partials + row * a.pieces * kPartial;
  auto state = [&](int i) { return P + (int64_t)min(i, a.pieces - 1) * kPartial; };
  float m = state(lane)[0], l = state(lane)[1];
  const int count = __float_as_int(P[2]);
  float2 x[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) x[j] = *reinterpret_cast<const float2*>(state(w + j * W) + 4 + 2 * lane);
  const int t = (int)(row / (a.m.Hkv * a.G));
  const bool mine = at < n_rows && t >= max(a.m.start[0], 0) && t < min(a.m.start[a.m.B], a.m.T);
  if (W == 1 && !mine) return;
  const int pieces = __builtin_amdgcn_readfirstlane(min(max(count, 1), a.pieces));
  float mx = -INFINITY, sum = 0.0f, x0 = 0.0f, x1 = 0.0f;
  for (int i0 = 0; i0 < pieces; i0 += 64) {
    if (i0 > 0) {
      m = state(i0 + lane)[0];
      l = state(i0 + lane)[1];
    }
    if (i0 + lane >= pieces) {
      m = -INFINITY;
      l = 0.0f;
    }
    float top = fmaxf(mx, m);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    const float f = weight_of(m, l, top), g = weight_of(mx, sum, top);
    float add = l * f;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) add += __shfl_xor(add, i);
    sum = sum * g + add;
    x0 *= g;
    x1 *= g;
    mx = top;
    const int n = min(64, pieces - i0);
    for (int i = w; i < n; i += kAhead * W) {
      if (i0 > 0 || i > w) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) x[j] = *reinterpret_cast<const float2*>(state(i0 + i + j * W) + 4 + 2 * lane);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j * W < n) {
          const float k = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), i + j * W));
          x0 = __builtin_fmaf(k, x[j].x, x0);
          x1 = __builtin_fmaf(k, x[j].y, x1);
        }
    }
  }
  if constexpr (W > 1) {
    part[wave][lane] = make_float2(x0, x1);
    __syncthreads();
    if (!mine || w != 0) return;
#pragma unroll
    for (int i = 1; i < W; ++i) {
      x0 += part[wave + i][lane].x;
      x1 += part[wave + i][lane].y;
    }
  }
  x0 = sum == 0.0f ? 0.0f : x0 / sum;
  x1 = sum == 0.0f ? 0.0f : x1 / sum;
  if constexpr (BF16) static_cast<uint32_t*>(a.out)[at * (kD / 2) + lane] = dev::pack_bf16(x0, x1);
  else static_cast<float2*>(a.out)[at * (kD / 2) + lane] = make_float2(x0, x1);
}

constexpr int kFewJoin = 1024; // rows up to which a workgroup joins one of them (1536 rows of 64 sequences: 58 us so, 54 with a wavefront each)
constexpr int kFewRows = 64;   // rows of the problem up to which pages of 4 bits are attended to by attend_few_kernel
constexpr int kFewGrid = 512;  // workgroups of a thin or pair launch, at most

// How a call is cut up.  Pages of 4 bits in bf16 go the few way up to 64 rows: 4 rows 265 us as thin workgroups and 209 so, 28 rows
// 128 and 82, 32 rows 76 and 52, 35 rows in pairs 73 and 75, 1 to 35 rows 56 and 48, 63 rows 34.6 and 34.1; in fp32 all calls (see
// attend_few_kernel).  Else at most 32 rows a
// sequence and KV head go the thin way, and all calls with pages of less than 16 positions, whose rows have a place each (2048 tokens at 32K, bf16: 2360 us, and 1050 with pages of 16 and more; 12 tokens 38 and
// 35; one token at 128K 114 and 106; pages of 4 bits with 8 and with 16 positions: one token of 16 sequences of 32K 206 and 121, five of 8
// of 16K, 7 heads a group, 97 and 50, 1024 at 8K 258 and 185, in fp32 818 and 152, 215 and 67, 1397 and 431); up to 64 in pairs (bf16; in fp32 a pair's registers do not go twice on a compute unit);
// more in tiles.
struct Cut {
  int rows;  // 16: few, 32: few or thin, 64: pair, 128: tile
  bool few;
  int units, pieces, prefer, want, least;  // units: of a KV head, at most; the others: piece_of
};
Cut cut(const lrqk_pages_shape& s) {
  const int G = s.Hq / s.Hkv;
  const int64_t most = (int64_t)s.n_max * G;
  const bool f32 = s.kv_dtype == LRQK_KV_F32;
  Cut c;
  c.few = s.page_dtype == LRQK_PAGE_E2M1 && s.page >= 16 && (f32 || most <= kFewRows);
  c.rows = c.few ? (most <= 16 || f32 ? 16 : 32) : most <= 32 || s.page < 16 ? 32 : most <= 64 && !f32 ? 64 : 128;
  const int full = (int)(((int64_t)s.T * G + c.rows - 1) / c.rows), tiles = full + s.B;  // sum_b ceil(n_b G / rows) is no more
  const int64_t units = (int64_t)std::max(s.B, full) * s.Hkv;
  // workgroups that the chip holds at a time: two on each of 256 compute units where registers allow it
  const int held = c.rows == 32 && f32 ? 256 : 512;
  const int64_t state = (int64_t)s.T * s.Hq * kPartial * (int64_t)sizeof(float);
  // In a batch there may be sequences of few new tokens and a long context among the others, which a workgroup a head would
  // be left with (a chunk of 4096 and seven single tokens at 120K: 1073 us, and 818 with pieces of 16384).  Not at the
  // price of partial states of more than a gigabyte.
  const int64_t few = s.B > 1 ? std::min<int64_t>((s.l_max + 16383) / 16384, (1ll << 30) / state) : 1;
  c.least = most > 128 ? 512 : s.B > 1 || c.few ? 256 : 128;
  const int64_t least = (s.l_max + c.least - 1) / c.least;  // pieces, with those
  c.prefer = 1;
  c.want = 0;
  if (most <= 128 && s.B <= (c.rows == 16 ? 2048 : 4096) && (c.rows > 32 || f32 || c.few)) {
    // Workgroups that are bound by more than memory: as many units as the chip holds, one each.  In us with as many / twice /
    // three times as many: 1 to 5 tokens of 8 sequences of 7K to 64K, i8, 64 / 72 / 79; 12 tokens of 2 sequences of 32K
    // 63 / 76 / 86; fp32, one token of 4 sequences of 32K 206 / 218 / 234; few, one token of 4 sequences of 16K 24 / 29 / -, 16 rows of
    // 8 of 32K 64 / 75 / - (eight times as many, as thin workgroups have: 113).  States of 64 MiB at most.
    c.want = std::max((held + s.Hkv - 1) / s.Hkv, 2 * tiles);
    c.pieces = (int)std::max(few, std::min<int64_t>({c.want, least, std::max<int64_t>((1ll << 26) / state, 1)}));
    c.units = c.want;
  } else {
    if (most <= 128) {
      // Bound by memory where a batch has enough of it: more units than the chip holds, so that all of it reads to the end.
      // With as many / twice / eight times as many: one token of 16 sequences of 8K to 128K, 8-bit rows, 512 / 427 / 384; of
      // one sequence of 128K 103 / 110 / 136.
      c.prefer = (int)std::min<int64_t>(((int64_t)held * (s.B == 1 ? 1 : 8) + units - 1) / units, least);
    } else {
      // many tiles: the fewest rounds of `held` workgroups per piece; a piece more costs some hundredths (700 tokens at 20K,
      // 176 tiles of 8 heads: 347 us with 3 pieces, which make 528 workgroups, and 274 with 5); the few way deals its units out as
      // workgroups end, and has one piece from four rounds on (2100 tokens at 20K, fp32: 2062 us with two, 2041 with one)
      double best = 0.0;
      for (int n = 1; n <= (c.few && units >= 4 * held ? 1 : 16); ++n) {
        const double cost = (double)((units * n + held - 1) / held) / n * (1.0 + 0.04 * (n - 1));
        if (n == 1 || cost < best) {
          c.prefer = n;
          best = cost;
        }
      }
      c.prefer = (int)std::min<int64_t>(c.prefer, least);
    }
    c.pieces = (int)std::max<int64_t>(c.prefer, few);
    c.units = tiles * c.pieces;
  }
  if (c.pieces == 1) c.least = s.l_max;
  return c;
}
size_t partial_bytes(const lrqk_pages_shape& s) {
  const Cut c = cut(s);
  return c.pieces > 1 ? (size_t)s.T * s.Hq * c.pieces * kPartial * sizeof(float) : 0;
}

template <bool BF16, int PAGE, bool SMALL>
hipError_t launch_thin(const dim3 grid, const Args& a, hipStream_t st) {
  constexpr size_t kLds = (size_t)kWaves * 2 * 32 * kRowB<BF16>;
  static std::atomic<uint64_t> done{0};
  const auto kernel = attend_thin_kernel<BF16, PAGE, SMALL>;
  const hipError_t e = raise_dynamic_lds_once(kernel, kLds, done);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), kLds, st, a);
  return hipSuccess;
}

template <bool BF16, int PAGE>
hipError_t launch(const lrqk_pages_shape& s, const Cut& c, const Args& a, hipStream_t st) {
  // as large as the chip, but for the few way with many units: there the next workgroup takes the next one (2048 tokens at 32K in fp32
  // 3.29 ms with 512 workgroups, 3.18 so, prompts of up to 2000 510 and 481 us)
  // (not more than a launch may have)
  const int most = std::max(1, (c.few && c.want == 0 ? 1 << 20 : kFewGrid) / s.Hkv);
  const dim3 grid((unsigned)(s.Hkv * (c.rows == 128 ? c.units : std::min(c.units, most))));
  hipError_t e = hipSuccess;
  constexpr bool k4 = PAGE == LRQK_PAGE_E2M1;  // (those go the few way wherever others go thin or in pairs, and in fp32 always: cut)
  if (s.page < 16) e = launch_thin<BF16, PAGE, true>(grid, a, st);
  else if (c.few) {
    if constexpr (k4) {
      if (c.rows == 16) hipLaunchKernelGGL((attend_few_kernel<1, BF16>), grid, dim3(kThreads), 0, st, a);
      else if constexpr (BF16) hipLaunchKernelGGL((attend_few_kernel<2, BF16>), grid, dim3(kThreads), 0, st, a);
    }
  } else if (c.rows == 128) {
    if constexpr (BF16 || !k4) hipLaunchKernelGGL((attend_tile_kernel<BF16, PAGE>), grid, dim3(kThreads), 0, st, a);
  } else if constexpr (!k4) {
    if (c.rows == 32) e = launch_thin<BF16, PAGE, false>(grid, a, st);
    else if constexpr (BF16) hipLaunchKernelGGL((attend_pair_kernel<PAGE>), grid, dim3(kThreads), 0, st, a);
  }
  if (e != hipSuccess) return e;
  if (a.partials) {
    const int64_t rows = (int64_t)s.T * s.Hq;
    if (c.few) {
      if constexpr (PAGE == LRQK_PAGE_E2M1) {
        if (c.pieces > 8 && rows <= kFewJoin)
          hipLaunchKernelGGL((attend_join_few_kernel<BF16, kWaves>), dim3((unsigned)rows), dim3(kThreads), 0, st, a, rows);
        else
          hipLaunchKernelGGL((attend_join_few_kernel<BF16, 1>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0, st, a, rows);
      }
    } else if (c.pieces > 8)  // a workgroup per row
      hipLaunchKernelGGL((attend_join_kernel<BF16, kWaves>), dim3((unsigned)rows), dim3(kThreads), 0, st, a, rows);
    else
      hipLaunchKernelGGL((attend_join_kernel<BF16, 1>), dim3((unsigned)((rows + kWaves - 1) / kWaves)), dim3(kThreads), 0,
                         st, a, rows);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API size_t lrqk_pages_workspace_bytes(const lrqk_pages_shape* shape) {
  using namespace lrqk;
  if (check_pages(shape) != LRQK_OK) return 0;
  return std::max<size_t>(256, partial_bytes(*shape));
}

LRQK_API int lrqk_chunk_attend(const lrqk_pages_shape* shape, const lrqk_pages* pg, const void* q, void* out,
                               void* workspace, size_t ws_bytes, void* stream) {
  using namespace lrqk;
  const int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  const lrqk_pages_shape& s = *shape;
  if (!pages_given(s, pg) || !q || !out || !aligned16(q) || !aligned16(out)) return LRQK_EINVAL;
  if (!workspace || !aligned256(workspace)) return LRQK_EINVAL;
  if (ws_bytes < lrqk_pages_workspace_bytes(shape)) return LRQK_ENOMEM;
  const Cut c = cut(s);
  const Args a{make_map(s, *pg), pg->K, pg->V, pg->K_scale, pg->V_scale, q, out,
               c.pieces > 1 ? static_cast<float*>(workspace) : nullptr, s.Hq / s.Hkv,
               __builtin_ctz((unsigned)c.rows), c.pieces, c.prefer, c.want, c.least,
               (uint32_t)s.Hkv * (uint32_t)s.page * (uint32_t)(row_bytes(s.page_dtype) / 16), s.scale};
  hipError_t e = hipSuccess;
  by_type(s, [&](auto bf16, auto page) {
    e = launch<bf16.value, page.value>(s, c, a, static_cast<hipStream_t>(stream));
  });
  LRQK_HIP(e);
  return LRQK_OK;
}
