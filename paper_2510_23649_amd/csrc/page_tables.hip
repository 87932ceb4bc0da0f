// g5 -- block tables and slot maps of the paged cache, made on the device (include/lrqk.h).
//
// A few kilobytes that depend on each other: bound by latency.  One workgroup does all of it for one call, with barriers in
// place of launches; the maps of many rows are a second launch.  Which page a sequence gets depends on nothing but the set of
// free pages, so the order in which atomics give pages back does not show.
#include "pages.h"

#include <algorithm>

namespace lrqk {
namespace {

using namespace pages;

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSeqs = 2048;        // sequences whose numbers LDS holds
constexpr int kTile = kThreads * 16;  // pages looked at a time: a wavefront takes 1024 of them, four loads of four a lane
constexpr int kRowsHere = 8192;    // rows whose maps the one workgroup makes

struct Args {
  int32_t *refs, *table, *kv_len, *start, *status, *seq, *pos, *slot;
  const int32_t *keep, *n_new;
  int32_t* work;  // B > kSeqs: what LDS does not hold
  int B, T, n_max, l_max, n_pages, max_pages, page_log2;
  bool maps;      // of the rows, here
};

__device__ __forceinline__ int pages_of(const Args& a, int len) { return (len + (1 << a.page_log2) - 1) >> a.page_log2; }

// Sum over the workgroup's threads before this one, and of all: a wavefront's sum of numbers below 2^24 fits 32 bits, the
// workgroup's need not.
__device__ __forceinline__ uint64_t scan(uint32_t v, uint32_t* tot, uint64_t& all) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const uint32_t upto = dev::wave_inclusive_scan(v);
  __syncthreads();  // (tot may still be read)
  if (lane == 63) tot[w] = upto;
  __syncthreads();
  uint64_t before = 0;
  all = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    before += i < w ? tot[i] : 0u;
    all += tot[i];
  }
  return before + upto - v;
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
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t p = first + 256 * i;
    if (p + 4 <= a.n_pages) {
      const int4 r = *reinterpret_cast<const int4*>(a.refs + p);
      mask |= ((r.x <= 0 ? 1u : 0u) | (r.y <= 0 ? 2u : 0u) | (r.z <= 0 ? 4u : 0u) | (r.w <= 0 ? 8u : 0u)) << (4 * i);
    } else {
      for (int j = 0; j < 4; ++j)
        if (p + j < a.n_pages && a.refs[p + j] <= 0) mask |= 1u << (4 * i + j);
    }
  }
  return mask;
}

__device__ __forceinline__ void put_maps(const Args& a, int t, int b, int pos, int page) {
  if (a.seq) a.seq[t] = b;
  if (a.pos) a.pos[t] = pos;
  if (a.slot) a.slot[t] = (unsigned)page >= (unsigned)a.n_pages ? -1 : (page << a.page_log2) + (pos & ((1 << a.page_log2) - 1));
}

__global__ __launch_bounds__(kThreads) void advance_kernel(const Args a) {
  __shared__ int32_t lds[4 * (kSeqs + 1)];
  __shared__ uint32_t tot[kWaves];
  __shared__ int32_t most;
  int32_t* const own = a.B <= kSeqs ? lds : a.work;
  int32_t* const kept = own;                // [B] positions kept
  int32_t* const want = kept + (a.B + 1);   // [B] new tokens, or -status
  int32_t* const rank = want + (a.B + 1);   // [B] new pages of the sequences before
  int32_t* const start = rank + (a.B + 1);  // [B+1]
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;

  // 1: cut back
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int held = 0, keep_pages = 0;
    if (b < a.B) {
      const int old = min(max(a.kv_len[b], 0), a.l_max), n = max(a.n_new[b], 0);
      const int k = a.keep ? min(max(a.keep[b], 0), old) : old;
      held = pages_of(a, old);
      keep_pages = pages_of(a, k);
      kept[b] = k;
      want[b] = n > 0 && (n > a.n_max || n > a.l_max - k) ? -LRQK_ADVANCE_LONG : n;
    }
    uint64_t todo = __ballot(held > keep_pages);
    while (todo) {
      const int j = __builtin_ctzll(todo);
      todo &= todo - 1;
      const int to = __builtin_amdgcn_readlane(held, j);
      int32_t* row = a.table + (size_t)(b0 + w * 64 + j) * a.max_pages;
      for (int i = __builtin_amdgcn_readlane(keep_pages, j) + lane; i < to; i += 64) {
        const int pg = row[i];
        row[i] = -1;
        if ((unsigned)pg < (unsigned)a.n_pages) atomicSub(a.refs + pg, 1);
      }
    }
  }
  if (threadIdx.x == 0) most = 0;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the atomics have arrived in the L2, past which nothing has read refs
  __syncthreads();

  // 2: what is asked for
  uint64_t pages = 0, rows = 0;  // of the sequences so far
  for (int b0 = 0; b0 < a.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    int n = 0, need = 0;
    if (b < a.B) {
      n = want[b];
      const int k = kept[b], kp = pages_of(a, k);
      if (n > 0 && (k & ((1 << a.page_log2) - 1)) != 0) {
        const int pg = a.table[(size_t)b * a.max_pages + kp - 1];
        if ((unsigned)pg < (unsigned)a.n_pages && a.refs[pg] > 1) want[b] = n = -LRQK_ADVANCE_SHARED;
      }
      need = n > 0 ? pages_of(a, k + n) - kp : 0;
      n = max(n, 0);
    }
    uint64_t all;
    const uint64_t p = pages + scan((uint32_t)need, tot, all);
    pages += all;
    const uint64_t r = rows + scan((uint32_t)n, tot, all);
    rows += all;
    if (b < a.B) {
      rank[b] = (int32_t)min(p, (uint64_t)INT32_MAX);
      if (n > 0 && r + n > (uint64_t)a.T) start[b] = LRQK_ADVANCE_ROWS;
      else start[b] = 0;
    }
  }
  const uint64_t asked = pages;

  // free pages: as many as are asked for, or all
  uint64_t there = 0;
  int64_t from = 0;  // the first tile that has any
  for (int64_t base = 0; base < a.n_pages && there < asked; base += kTile) {
    uint64_t all;
    scan((uint32_t)__builtin_popcount(free_mask(a, base, w, lane)), tot, all);
    if (there == 0) from = base;
    there += all;
  }
  __syncthreads();

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
    uint64_t all;
    const uint64_t r = rows + scan((uint32_t)n, tot, all);
    rows += all;
    if (b < a.B) {
      start[b] = (int32_t)r;
      a.start[b] = (int32_t)r;
    }
  }
  if (threadIdx.x == 0) {
    start[a.B] = (int32_t)rows;
    a.start[a.B] = (int32_t)rows;
  }
  __syncthreads();

  // 3: the pages
  const int give = most;
  int64_t found = 0;
  for (int64_t base = from; base < a.n_pages && found < give; base += kTile) {
    const uint32_t mask = free_mask(a, base, w, lane);
    uint32_t before[4], in_wave = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t n = (uint32_t)__builtin_popcount(mask >> (4 * i) & 15u), upto = dev::wave_inclusive_scan(n);
      before[i] = in_wave + upto - n;
      in_wave += __builtin_amdgcn_readlane(upto, 63);
    }
    uint64_t all;
    uint64_t ahead = scan(lane == 0 ? in_wave : 0u, tot, all);  // of lane 0: the wavefronts before
    ahead = __builtin_amdgcn_readfirstlane((uint32_t)ahead);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int64_t r = found + (int64_t)ahead + before[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (!(mask >> (4 * i + j) & 1)) continue;
        if (r < give) {
          const int page = (int)(base + w * 1024 + 256 * i + 4 * lane + j);
          const int b = last_upto(rank, a.B, (int)r);
          a.refs[page] = 1;
          a.table[(size_t)b * a.max_pages + pages_of(a, kept[b]) + ((int)r - rank[b])] = page;
        }
        ++r;
      }
    }
    found += (int64_t)all;
  }
  if (!a.maps) return;
  __syncthreads();
  const int n_rows = start[a.B];
  for (int t = threadIdx.x; t < a.T; t += kThreads) {
    if (t >= n_rows) {
      put_maps(a, t, -1, -1, -1);
      continue;
    }
    const int b = last_upto(start, a.B, t);
    const int pos = kept[b] + (t - start[b]);
    put_maps(a, t, b, pos, a.slot ? a.table[(size_t)b * a.max_pages + (pos >> a.page_log2)] : 0);
  }
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
  const int n_rows = start[a.B];
  for (int t = blockIdx.x * kMapThreads + threadIdx.x; t < a.T; t += gridDim.x * kMapThreads) {
    if (t >= n_rows) {
      put_maps(a, t, -1, -1, -1);
      continue;
    }
    const int b = last_upto(start, a.B, t);
    const int pos = a.kv_len[b] - start[b + 1] + t;
    put_maps(a, t, b, pos, a.slot ? a.table[(size_t)b * a.max_pages + (pos >> a.page_log2)] : 0);
  }
}

__global__ __launch_bounds__(kMapThreads) void tables_init_kernel(const Args a) {
  const int64_t step = (int64_t)gridDim.x * kMapThreads, i0 = (int64_t)blockIdx.x * kMapThreads + threadIdx.x;
  for (int64_t i = i0; i < a.n_pages; i += step) a.refs[i] = 0;
  for (int64_t i = i0; i < (int64_t)a.B * a.max_pages; i += step) a.table[i] = -1;
  for (int64_t i = i0; i < a.B; i += step) a.kv_len[i] = 0;
}

bool given(std::initializer_list<const void*> p) {
  for (const void* x : p)
    if (!x || !aligned16(x)) return false;
  return true;
}
Args make_args(const lrqk_pages_shape& s, const lrqk_pages_tables& t) {
  return Args{t.refs, t.table, t.kv_len, t.start, t.status, t.seq, t.pos, t.slot, nullptr, nullptr, nullptr,
              s.B, s.T, s.n_max, s.l_max, s.n_pages, s.max_pages, __builtin_ctz((unsigned)s.page), true};
}

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API size_t lrqk_pages_advance_workspace_bytes(const lrqk_pages_shape* shape) {
  using namespace lrqk;
  if (check_pages(shape) != LRQK_OK) return 0;
  return shape->B <= kSeqs ? 256 : round_up((size_t)4 * (shape->B + 1) * sizeof(int32_t), 256);
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
  hipLaunchKernelGGL(advance_kernel, dim3(1), dim3(kThreads), 0, st, a);
  if (any && !a.maps)
    hipLaunchKernelGGL(maps_kernel, dim3((unsigned)std::min(ceil_div(a.T, kMapThreads), 2048)), dim3(kMapThreads), 0, st, a);
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}
