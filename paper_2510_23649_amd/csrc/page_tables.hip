// g5 -- block tables and slot maps of the paged cache, made on the device (include/lrqk.h).
//
// A few kilobytes that depend on each other: bound by latency.  One workgroup does all of it for one call, with barriers in
// place of launches; the maps of many rows are a launch more, the counts of a large pool two.  Which page a sequence gets depends on
// nothing but the set of free pages, so the order in which atomics give pages back does not show.
#include "pages.h"

#include <algorithm>

namespace lrqk {
namespace {

using namespace pages;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSeqs = 2048;           // sequences whose numbers LDS holds
constexpr int kTile = kThreads * 16;  // pages looked at together: a wavefront takes 1024 of them, four loads of four a lane
// Rows whose maps the one workgroup makes (256 sequences, 4096 rows: 10.0 us, and 12.0 with a launch of their own; 6144: 12.1 and 12.7; 8448: 14.4 and 13.8).
constexpr int kRowsHere = 6144;
constexpr int kSmall = 2;  // pages of a sequence that its own thread gives back or takes
// Pages that the one workgroup looks through itself, as far as it has to: 3.6 us for 64K of them.  Two launches before it that give pages
// back and count take 5, however many there are.  256 sequences that ask for a page each, in us a call without / with counts: a tenth
// of the pool free, all over (requests come and go) 10.6 / 15.7 at 20K to 144K pages; the last tenth free (a pool that is filled from the front)
// 14.8 / 15.3 at 20K, 15.2 / 15.6 at 64K and 90K, 18.9 / 15.5 at 144K; 1M pages at their end 113 / 15.4.
constexpr int kPagesHere = 9 * kTile;

struct Args {
  int32_t *refs, *table, *kv_len, *start, *status, *seq, *pos, *slot;
  const int32_t *keep, *n_new;
  int32_t* work;    // B > kSeqs: what LDS does not hold
  int32_t* counts;  // n_pages > kPagesHere: free pages of each tile, after what is given back; else null
  int B, T, n_max, l_max, n_pages, max_pages, page_log2;
  bool maps;      // of the rows, here
};

__device__ __forceinline__ int pages_of(const Args& a, int len) { return (len + (1 << a.page_log2) - 1) >> a.page_log2; }

// Sums over the workgroup's threads before this one, and of all, of two numbers at a time: a wavefront's sum of numbers up to 2^24
// fits 32 bits; the workgroup's need not and stays at the largest, above all that it is compared with.  Each wavefront reads a total a
// lane and adds them up along a row of 16.  One barrier, at which nothing waits for memory: the totals of one scan are read while
// the next one writes the others.  MEM: what threads exchange lies in memory.
struct Totals {
  uint2 of[2][kWaves];
};
struct Sums {
  uint64_t x, y;
  uint32_t all_x, all_y;
};
__device__ __forceinline__ uint32_t sum_row(uint32_t v) {
  v = __builtin_elementwise_add_sat(v, dev::dpp_zero_fill<0x111, 0xf>(v));  // row_shr:1
  v = __builtin_elementwise_add_sat(v, dev::dpp_zero_fill<0x112, 0xf>(v));
  v = __builtin_elementwise_add_sat(v, dev::dpp_zero_fill<0x114, 0xf>(v));
  return __builtin_elementwise_add_sat(v, dev::dpp_zero_fill<0x118, 0xf>(v));
}
template <bool MEM = false>
__device__ __forceinline__ Sums scan(uint32_t x, uint32_t y, Totals& tot, int& turn) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ux = dev::wave_inclusive_scan(x), uy = dev::wave_inclusive_scan(y);
  uint2* const of = tot.of[turn];
  turn ^= 1;
  if (lane == 63) of[w] = make_uint2(ux, uy);
  if constexpr (MEM) {
    __syncthreads();
  } else {
    dev::lds_barrier();
  }
  const uint2 t = of[lane & 15];
  const uint32_t tx = sum_row(t.x), ty = sum_row(t.y);
  const uint32_t bx = w ? __builtin_amdgcn_readlane(tx, w - 1) : 0, by = w ? __builtin_amdgcn_readlane(ty, w - 1) : 0;
  return Sums{(uint64_t)bx + (ux - x), (uint64_t)by + (uy - y), (uint32_t)__builtin_amdgcn_readlane(tx, 15),
              (uint32_t)__builtin_amdgcn_readlane(ty, 15)};
}

// The last of x[0 .. n) (ascending, x[0] <= v) that is not above v.
__device__ __forceinline__ int last_upto(const int32_t* x, int n, int v) {
  int lo = 0, len = n;
  while (len > 1) {
    const int half = len >> 1;
    if (x[lo + half] <= v) lo += half;
    len -= half;
  }
  return lo;
}

// Free pages among the 16 of a lane in the tile from `base`: bit 4 i + j is page base + 1024 w + 256 i + 4 lane + j.
__device__ __forceinline__ uint32_t free_mask(const Args& a, int64_t base, int w, int lane) {
  uint32_t mask = 0;
  const int64_t first = base + w * 1024 + 4 * lane;
  int4 r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t p = first + 256 * i;
    if (p + 4 <= a.n_pages) {
      r[i] = *reinterpret_cast<const int4*>(a.refs + p);
    } else {
      r[i].x = p < a.n_pages ? a.refs[p] : 1;
      r[i].y = p + 1 < a.n_pages ? a.refs[p + 1] : 1;
      r[i].z = p + 2 < a.n_pages ? a.refs[p + 2] : 1;
      r[i].w = 1;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    mask |= ((r[i].x <= 0 ? 1u : 0u) | (r[i].y <= 0 ? 2u : 0u) | (r[i].z <= 0 ? 4u : 0u) | (r[i].w <= 0 ? 8u : 0u)) << (4 * i);
  return mask;
}
// Free pages of the wavefront in front of each of the lane's four groups of four; returns those of the wavefront.
__device__ __forceinline__ uint32_t in_wave(uint32_t mask, uint32_t (&before)[4]) {
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t k = (uint32_t)__builtin_popcount(mask >> (4 * i) & 15u), upto = dev::wave_inclusive_scan(k);
    before[i] = n + upto - k;
    n += __builtin_amdgcn_readlane(upto, 63);
  }
  return n;
}

// The maps of rows t0 .. t0 + 3.  `at(b)`: what a row's number has to be added to for its position.  Found with one search: the
// rows after the first are its sequence's or those of one of the next.
template <typename F>
__device__ __forceinline__ void put_maps(const Args& a, int t0, const int32_t* start, int n_rows, F at) {
  int b[4], pos[4], pg[4];
  int s = t0 < n_rows ? last_upto(start, a.B, t0) : 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int t = t0 + j;
    b[j] = pos[j] = pg[j] = -1;
    if (t < n_rows) {
      for (int i = 0; t >= start[s + 1]; ++i) s = i < 2 ? s + 1 : last_upto(start, a.B, t);
      b[j] = s;
      pos[j] = at(s) + t;
    }
  }
  if (a.slot) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (b[j] >= 0) pg[j] = a.table[(size_t)b[j] * a.max_pages + (pos[j] >> a.page_log2)];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      pg[j] = (unsigned)pg[j] >= (unsigned)a.n_pages ? -1 : (pg[j] << a.page_log2) + (pos[j] & ((1 << a.page_log2) - 1));
  }
  auto put = [&](int32_t* map, const int (&x)[4]) {
    if (!map) return;
    if (t0 + 4 <= a.T) {
      *reinterpret_cast<int4*>(map + t0) = make_int4(x[0], x[1], x[2], x[3]);
    } else {
      for (int j = 0; j < 4 && t0 + j < a.T; ++j) map[t0 + j] = x[j];
    }
  };
  put(a.seq, b);
  put(a.pos, pos);
  put(a.slot, pg);
}

// Positions kept of b's `old`.
__device__ __forceinline__ int kept_of(const Args& a, int b, int& old) {
  old = min(max(a.kv_len[b], 0), a.l_max);
  return a.keep ? min(max(a.keep[b], 0), old) : old;
}

// Step 1 by a wavefront a sequence, and the tiles' counts, of a large pool.
__global__ __launch_bounds__(256) void cut_kernel(const Args a) {
  const int lane = threadIdx.x & 63, b = (int)(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (b >= a.B) return;
  int old;
  const int k = kept_of(a, b, old), to = pages_of(a, old);
  int32_t* const row = a.table + (size_t)b * a.max_pages;
  for (int i = pages_of(a, k) + lane; i < to; i += 64) {
    const int pg = row[i];
    row[i] = -1;
    if ((unsigned)pg < (unsigned)a.n_pages) atomicSub(a.refs + pg, 1);
  }
}
__global__ __launch_bounds__(kThreads) void count_kernel(const Args a) {
  __shared__ Totals tot;
  int turn = 0;
  const uint32_t mask = free_mask(a, (int64_t)blockIdx.x * kTile, threadIdx.x >> 6, threadIdx.x & 63);
  const Sums s = scan((uint32_t)__builtin_popcount(mask), 0u, tot, turn);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = (int32_t)s.all_x;
}

// 6.5 us for one sequence of one token and a page, 9.6 for 256 (3.6 for a launch that finds nothing to do): a round trip to memory each for the
// lengths, the entries given back, their references, the pool's, the table and its entries for the slots, and ten barriers.  What
// most of them share lies in LDS, so that they wait for no store or load; with barriers that do, and all sixteen totals of a scan read by
// every thread (128 registers and 19 spilled; now 86), 8.5 and 11.6.
template <bool LDS>
__global__ __launch_bounds__(kThreads) void advance_kernel(const Args a) {
  __shared__ int32_t lds[LDS ? 4 * (kSeqs + 1) : 1];
  __shared__ uint16_t pick[kTile];  // free pages of a tile, ascending
  __shared__ Totals tot;
  __shared__ int32_t most, first_tile, big;
  const int size = LDS ? kSeqs + 1 : a.B + 1;
  int32_t* const kept = LDS ? lds : a.work;  // [B] positions kept
  int32_t* const want = kept + size;         // [B] new tokens, or -status
  int32_t* const rank = want + size;         // [B] table entries given back, then new pages, of the sequences before
  int32_t* const start = rank + size;        // [B+1]
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, page = 1 << a.page_log2;
  int turn = 0;

  // 1: cut back.  A sequence's thread gives back a page or two; the entries of those that give back more are dealt out to
  // all threads, since a loop over a sequence's would wait for one load after the other (256 sequences, of which a third give something
  // back: 28 us with such loops).
  uint64_t gone = 0;
  int last = -1;  // the page of position `kept`, if that is no page's first (one sequence a thread: looked up on the way)
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int n_gone = 0;
    if (b < a.B) {
      const int n = max(a.n_new[b], 0);
      int old;
      const int k = kept_of(a, b, old);
      n_gone = a.counts ? 0 : pages_of(a, old) - pages_of(a, k);
      kept[b] = k;
      want[b] = n > 0 && (n > a.n_max || n > a.l_max - k) ? -LRQK_ADVANCE_LONG : n;
      int32_t* const row = a.table + (size_t)b * a.max_pages;
      if ((k & (page - 1)) != 0) last = row[k >> a.page_log2];
      if (n_gone <= kSmall) {
        int pg[kSmall];
#pragma unroll
        for (int i = 0; i < kSmall; ++i) pg[i] = i < n_gone ? row[pages_of(a, k) + i] : -1;
#pragma unroll
        for (int i = 0; i < kSmall; ++i) {
          if (i < n_gone) row[pages_of(a, k) + i] = -1;
          if ((unsigned)pg[i] < (unsigned)a.n_pages) atomicSub(a.refs + pg[i], 1);
        }
        n_gone = 0;
      }
    }
    const Sums s = scan<!LDS>((uint32_t)n_gone, 0u, tot, turn);
    if (b < a.B) rank[b] = (int32_t)min(gone + s.x, (uint64_t)INT32_MAX);
    gone += s.all_x;
  }
  if (threadIdx.x == 0) {
    most = 0;
    big = 0;
    first_tile = INT32_MAX;
  }
  __syncthreads();
  for (uint64_t i = threadIdx.x; i < gone; i += kThreads) {
    if (i >= INT32_MAX) break;  // (2^31 entries: no table has them)
    const int b = last_upto(rank, a.B, (int)i);
    int32_t* const entry = a.table + (size_t)b * a.max_pages + pages_of(a, kept[b]) + ((int)i - rank[b]);
    const int pg = *entry;
    *entry = -1;
    if ((unsigned)pg < (unsigned)a.n_pages) atomicSub(a.refs + pg, 1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the atomics have arrived in the L2, past which nothing has read refs
  __syncthreads();

  // 2: what is asked for
  uint64_t asked = 0, rows = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int n = 0, need = 0;
    if (b < a.B) {
      n = want[b];
      const int k = kept[b];
      if (n > 0 && (k & (page - 1)) != 0) {
        const int pg = a.B <= kThreads ? last : a.table[(size_t)b * a.max_pages + (k >> a.page_log2)];
        if ((unsigned)pg < (unsigned)a.n_pages && a.refs[pg] > 1) want[b] = n = -LRQK_ADVANCE_SHARED;
      }
      need = n > 0 ? pages_of(a, k + n) - pages_of(a, k) : 0;
      n = max(n, 0);
      if (need > kSmall) big = 1;
    }
    const Sums s = scan<!LDS>((uint32_t)need, (uint32_t)n, tot, turn);
    if (b < a.B) {
      rank[b] = (int32_t)min(asked + s.x, (uint64_t)INT32_MAX);
      start[b] = n > 0 && rows + s.y + n > (uint64_t)a.T ? LRQK_ADVANCE_ROWS : 0;
    }
    asked += s.all_x;
    rows += s.all_y;
  }

  // free pages: as many as are asked for, or all
  uint64_t there = 0;
  int64_t from = 0, at = -1;  // the first tile that has any; the one that `mask` is of
  uint32_t mask = 0, before[4];
  uint64_t ahead = 0, in_tile = 0;
  auto count = [&]() __attribute__((always_inline)) {  // what `mask` says
    const uint32_t n = in_wave(mask, before);
    const Sums s = scan<!LDS>(lane == 0 ? n : 0u, 0u, tot, turn);
    ahead = __builtin_amdgcn_readfirstlane((uint32_t)s.x);  // of lane 0: the wavefronts before
    in_tile = s.all_x;
  };
  if (a.counts && asked > 0) {
    const int tiles = (int)((a.n_pages + (int64_t)kTile - 1) / kTile);
    for (int i0 = 0; i0 < tiles && there < asked; i0 += kThreads) {
      const int n = i0 + (int)threadIdx.x < tiles ? a.counts[i0 + threadIdx.x] : 0;
      if (n > 0) atomicMin(&first_tile, i0 + (int)threadIdx.x);
      there += scan<!LDS>((uint32_t)n, 0u, tot, turn).all_x;
    }
    from = first_tile == INT32_MAX ? 0 : (int64_t)first_tile * kTile;
  } else if (asked > 0) {
    mask = free_mask(a, 0, w, lane);
    count();
    there = in_tile;
    at = 0;
    // four tiles a round (144K pages: 18.8 us, and 21.5 where they come one by one); a tile's 16384 fit 16 bits
    for (int64_t base = kTile; base < a.n_pages && there < asked; base += 4 * kTile) {
      uint32_t n[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) n[i] = (uint32_t)__builtin_popcount(free_mask(a, base + i * kTile, w, lane));
      const Sums s = scan<!LDS>(n[0] | n[1] << 16, n[2] | n[3] << 16, tot, turn);
      const uint32_t in[4] = {s.all_x & 0xffffu, s.all_x >> 16, s.all_y & 0xffffu, s.all_y >> 16};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (there == 0) from = base + i * kTile;
        there += in[i];
      }
    }
  }

  // 2, 4: who gets what
  rows = 0;
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int n = 0;
    if (b < a.B) {
      n = want[b];
      const int k = kept[b], need = n > 0 ? pages_of(a, k + n) - pages_of(a, k) : 0;
      int status = n < 0 ? -n : 0;
      if (status == 0 && need > 0 && (uint64_t)rank[b] + need > there) status = LRQK_ADVANCE_PAGES;
      if (status == 0 && n > 0) status = start[b];
      n = status == 0 ? n : 0;
      want[b] = n;
      a.status[b] = status;
      a.kv_len[b] = k + n;
      // those that are refused pages or rows are the last ones that ask for any: the others' pages are the first ones
      if (n > 0 && need > 0) atomicMax(&most, rank[b] + need);
    }
    const Sums s = scan<!LDS>((uint32_t)n, 0u, tot, turn);
    if (b < a.B) {
      start[b] = (int32_t)(rows + s.x);
      a.start[b] = (int32_t)(rows + s.x);
    }
    rows += s.all_x;
  }
  if (threadIdx.x == 0) {
    start[a.B] = (int32_t)rows;
    a.start[a.B] = (int32_t)rows;
  }
  __syncthreads();

  // 3: the pages: a tile's free ones in order; a sequence's thread takes a page or two, a thread for each those of the others
  const int give = most;
  int64_t found = 0;
  for (int64_t base = from; base < a.n_pages && found < give; base += kTile) {
    if (a.counts && a.counts[base / kTile] == 0) continue;
    if (base != at) {
      mask = free_mask(a, base, w, lane);
      count();
    }
    at = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t r = (uint32_t)ahead + before[i];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (mask >> (4 * i + j) & 1) pick[r++] = (uint16_t)(w * 1024 + 256 * i + 4 * lane + j);
    }
    __syncthreads();
    const int n = (int)min((int64_t)in_tile, give - found);  // of this tile
    for (int b = threadIdx.x; b < a.B; b += kThreads) {
      const int need = want[b] > 0 ? pages_of(a, kept[b] + want[b]) - pages_of(a, kept[b]) : 0;
#pragma unroll
      for (int i = 0; i < kSmall; ++i) {
        const int64_t r = rank[b] + i - found;
        if (need > kSmall || i >= need || r < 0 || r >= n) continue;
        const int pg = (int)base + pick[r];
        a.refs[pg] = 1;
        a.table[(size_t)b * a.max_pages + pages_of(a, kept[b]) + i] = pg;
      }
    }
    if (big) {
      for (int i = threadIdx.x; i < n; i += kThreads) {
        const int r = (int)found + i, pg = (int)base + pick[i];
        const int b = last_upto(rank, a.B, r), first = pages_of(a, kept[b]);
        if (pages_of(a, kept[b] + want[b]) - first <= kSmall) continue;
        a.refs[pg] = 1;
        a.table[(size_t)b * a.max_pages + first + (r - rank[b])] = pg;
      }
    }
    found += (int64_t)in_tile;
    __syncthreads();
  }
  if (!a.maps) return;
  for (int t = 4 * threadIdx.x; t < a.T; t += 4 * kThreads)
    put_maps(a, t, start, start[a.B], [&](int i) { return kept[i] - start[i]; });
}

// The maps of many rows, from the tables.
constexpr int kMapThreads = 256;
__global__ __launch_bounds__(kMapThreads) void maps_kernel(const Args a) {
  __shared__ int32_t lds[kSeqs + 1];
  const int32_t* start = a.start;
  if (a.B <= kSeqs) {
    for (int i = threadIdx.x; i <= a.B; i += kMapThreads) lds[i] = a.start[i];
    __syncthreads();
    start = lds;
  }
  for (int t = 4 * (blockIdx.x * kMapThreads + threadIdx.x); t < a.T; t += 4 * gridDim.x * kMapThreads)
    put_maps(a, t, start, start[a.B], [&](int i) { return a.kv_len[i] - start[i + 1]; });
}

__global__ __launch_bounds__(kMapThreads) void tables_init_kernel(const Args a) {
  const int64_t step = (int64_t)gridDim.x * kMapThreads, i0 = (int64_t)blockIdx.x * kMapThreads + threadIdx.x;
  for (int64_t i = i0; i < a.n_pages; i += step) a.refs[i] = 0;
  for (int64_t i = i0; i < (int64_t)a.B * a.max_pages; i += step) a.table[i] = -1;
  for (int64_t i = i0; i < a.B; i += step) a.kv_len[i] = 0;
}

size_t work_bytes(const lrqk_pages_shape& s) {
  return s.B <= kSeqs ? 0 : round_up((size_t)4 * (s.B + 1) * sizeof(int32_t), 256);
}
size_t count_bytes(const lrqk_pages_shape& s) {
  return s.n_pages <= kPagesHere ? 0 : ((size_t)s.n_pages + kTile - 1) / kTile * sizeof(int32_t);
}

bool given(std::initializer_list<const void*> p) {
  for (const void* x : p)
    if (!x || !aligned16(x)) return false;
  return true;
}
Args make_args(const lrqk_pages_shape& s, const lrqk_pages_tables& t) {
  return Args{t.refs, t.table, t.kv_len, t.start, t.status, t.seq, t.pos, t.slot, nullptr, nullptr, nullptr, nullptr,
              s.B, s.T, s.n_max, s.l_max, s.n_pages, s.max_pages, __builtin_ctz((unsigned)s.page), true};
}

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API size_t lrqk_pages_advance_workspace_bytes(const lrqk_pages_shape* shape) {
  using namespace lrqk;
  if (check_pages(shape) != LRQK_OK) return 0;
  return round_up(256 + work_bytes(*shape) + count_bytes(*shape), 256);
}

LRQK_API int lrqk_pages_tables_init(const lrqk_pages_shape* shape, const lrqk_pages_tables* tables, void* stream) {
  using namespace lrqk;
  const int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  if (!tables || !given({tables->refs, tables->table, tables->kv_len})) return LRQK_EINVAL;
  const Args a = make_args(*shape, *tables);
  const int64_t most = std::max<int64_t>(a.n_pages, (int64_t)a.B * a.max_pages);
  hipLaunchKernelGGL(tables_init_kernel, dim3((unsigned)std::min<int64_t>((most + kMapThreads - 1) / kMapThreads, 4096)),
                     dim3(kMapThreads), 0, static_cast<hipStream_t>(stream), a);
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}

LRQK_API int lrqk_pages_advance(const lrqk_pages_shape* shape, const lrqk_pages_tables* tables, const int32_t* keep,
                                const int32_t* n_new, void* workspace, size_t ws_bytes, void* stream) {
  using namespace lrqk;
  const int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  if (!tables || !given({tables->refs, tables->table, tables->kv_len, tables->start, tables->status, n_new})) return LRQK_EINVAL;
  if (!aligned16(tables->seq) || !aligned16(tables->pos) || !aligned16(tables->slot) || !aligned16(keep)) return LRQK_EINVAL;
  if (!workspace || !aligned256(workspace)) return LRQK_EINVAL;
  if (ws_bytes < lrqk_pages_advance_workspace_bytes(shape)) return LRQK_ENOMEM;
  Args a = make_args(*shape, *tables);
  a.keep = keep;
  a.n_new = n_new;
  a.work = static_cast<int32_t*>(workspace);
  const bool any = a.seq || a.pos || a.slot;
  a.maps = any && a.T <= kRowsHere;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (count_bytes(*shape) > 0) {
    a.counts = a.work + work_bytes(*shape) / sizeof(int32_t);
    hipLaunchKernelGGL(cut_kernel, dim3((unsigned)ceil_div(a.B, 4)), dim3(256), 0, st, a);
    hipLaunchKernelGGL(count_kernel, dim3((unsigned)((a.n_pages + (int64_t)kTile - 1) / kTile)), dim3(kThreads), 0, st, a);
  }
  if (a.B <= kSeqs) hipLaunchKernelGGL(advance_kernel<true>, dim3(1), dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(advance_kernel<false>, dim3(1), dim3(kThreads), 0, st, a);
  if (any && !a.maps)
    hipLaunchKernelGGL(maps_kernel, dim3((unsigned)std::min(ceil_div(a.T, 4 * kMapThreads), 2048)), dim3(kMapThreads), 0, st, a);
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}
