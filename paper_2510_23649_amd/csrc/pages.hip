// g1, g2 -- the paged K/V cache is written and read back (include/lrqk.h).
//
// Both move rows of 128 elements and are bound by memory: by its latency where a lane has one row in flight, by its
// bandwidth with several.
#include "pages.h"

#include <cmath>

namespace lrqk {

int check_pages(const lrqk_pages_shape* s) {
  if (!s) return LRQK_EINVAL;
  if (s->kv_dtype != LRQK_KV_BF16 && s->kv_dtype != LRQK_KV_F32) return LRQK_EINVAL;
  if (s->page_dtype < LRQK_PAGE_BF16 || s->page_dtype > LRQK_PAGE_I8) return LRQK_EINVAL;
  if (s->page_dtype == LRQK_PAGE_BF16 && s->kv_dtype != LRQK_KV_BF16) return LRQK_EINVAL;
  if (s->page_dtype == LRQK_PAGE_F32 && s->kv_dtype != LRQK_KV_F32) return LRQK_EINVAL;
  if (s->B < 1 || s->Hq < 1 || s->Hkv < 1 || s->n_max < 1 || s->n_pages < 1) return LRQK_ESHAPE;
  if (s->Hq % s->Hkv != 0 || s->Hq / s->Hkv > kMaxG) return LRQK_ESHAPE;
  if (s->d != kD) return LRQK_ESHAPE;
  if ((int64_t)s->B * s->Hq > 65535) return LRQK_ESHAPE;
  if (s->T < 1 || s->T >= (1 << 24) || (int64_t)s->T * s->Hq > INT32_MAX) return LRQK_ESHAPE;
  if (s->l_max < 1 || s->l_max >= (1 << 24)) return LRQK_ESHAPE;
  if (s->l_cap != 0 && (s->l_cap < s->l_max || s->l_cap >= (1 << 24))) return LRQK_ESHAPE;
  if (s->page < 1 || s->page > 1024 || (s->page & (s->page - 1)) != 0) return LRQK_ESHAPE;
  if (s->max_pages < 1 || (int64_t)s->max_pages * s->page < s->l_max) return LRQK_ESHAPE;
  if (!std::isfinite(s->scale)) return LRQK_ESHAPE;
  // 16-byte chunks of a pool are counted in 32 bits
  const int64_t page16 = (int64_t)s->Hkv * s->page * (kD * pages::page_elem_bytes(s->page_dtype) / 16);
  if (page16 * s->n_pages > (int64_t)1 << 32) return LRQK_ESHAPE;
  return LRQK_OK;
}

bool pages_given(const lrqk_pages_shape& s, const lrqk_pages* p) {
  if (!p) return false;
  auto ok = [](const void* x) { return x && aligned16(x); };
  if (pages::is8(s.page_dtype) && (!ok(p->K_scale) || !ok(p->V_scale))) return false;
  return ok(p->K) && ok(p->V) && ok(p->table) && ok(p->start) && ok(p->kv_len);
}

namespace {

using namespace pages;

constexpr int kMoveThreads = 256;

// ---- g1 ----------------------------------------------------------------------------------------------------
constexpr int kAppendEach = 4;                                   // rows of K and of V a 16-lane group has in flight
constexpr int kAppendRows = kMoveThreads / 16 * kAppendEach;     // rows of K (and of V) a workgroup

// Eight elements of a row, chunk c of 16, as they are, and as fp32.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t row, int c, uint4& a, uint4& b) {
  const uint4* p = static_cast<const uint4*>(base) + (row * 16 + c) * (BF16 ? 1 : 2);
  a = p[0];
  if (!BF16) b = p[1];
}
template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t row, int c, uint4 a, uint4 b) {
  uint4* p = static_cast<uint4*>(base) + (row * 16 + c) * (BF16 ? 1 : 2);
  p[0] = a;
  if (!BF16) p[1] = b;
}
template <bool BF16>
__device__ __forceinline__ void get8(uint4 a, uint4 b, float (&x)[8]) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = __uint_as_float(!BF16 ? w[i] : i % 2 == 0 ? w[i / 2] << 16 : w[i / 2] & 0xffff0000u);
}

// A 16-lane group takes rows of k_new and v_new, 8 elements a lane; the rows are on their way while their places are found.
// An 8-bit row has its four blocks of 32 elements in four lanes each: a block's largest magnitude takes two DPP steps.
// Bound by memory: 4 prompts of up to 8192 tokens, bf16 to e4m3 (K and V, 99 MB), 22 us.  One
// token of 16 sequences is 5 us of loads that wait for each other (start, then length and table, then the row's place).
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kMoveThreads) void pages_append_kernel(const Map m, const void* k_new,
                                                                    const void* v_new, void* K, void* V,
                                                                    uint8_t* K_scale, uint8_t* V_scale) {
  const int grp = threadIdx.x >> 4, c = threadIdx.x & 15;
  const int64_t rows = (int64_t)m.T * m.Hkv;
  for (int64_t r0 = (int64_t)blockIdx.x * kAppendRows; r0 < rows; r0 += (int64_t)gridDim.x * kAppendRows) {
    uint4 k[kAppendEach], v[kAppendEach], k2[kAppendEach], v2[kAppendEach];  // (2: fp32 rows only)
    int t[kAppendEach], b[kAppendEach];
#pragma unroll
    for (int j = 0; j < kAppendEach; ++j) {
      const int64_t r = min(r0 + j * (kMoveThreads / 16) + grp, rows - 1);
      k2[j] = v2[j] = make_uint4(0, 0, 0, 0);
      load8<BF16>(k_new, r, c, k[j], k2[j]);
      load8<BF16>(v_new, r, c, v[j], v2[j]);
      t[j] = (int)((uint32_t)r / (uint32_t)m.Hkv);
    }
    sequences_of(m, t, b);  // the whole wavefront takes part
#pragma unroll
    for (int j = 0; j < kAppendEach; ++j) {
      const int64_t r = r0 + j * (kMoveThreads / 16) + grp;
      if (r >= rows || b[j] < 0) continue;
      const Seq q = sequence(m, b[j]);
      const int p = q.len - q.n + (t[j] - q.first);
      if (t[j] < q.first || t[j] >= q.first + q.n || p < 0 || p >= m.l_max) continue;
      const int64_t row = row_of(m, b[j], (int)((uint32_t)r % (uint32_t)m.Hkv), p);
      if (row < 0) continue;
      if constexpr (!is8(PAGE)) {
        store8<BF16>(K, row, c, k[j], k2[j]);
        store8<BF16>(V, row, c, v[j], v2[j]);
      } else {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
          float x[8];
          get8<BF16>(which ? v[j] : k[j], which ? v2[j] : k2[j], x);
          uint32_t top = 0;
#pragma unroll
          for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
          top = max(top, dev::dpp_u32<0xB1>(top));  // over the four lanes of a block
          top = max(top, dev::dpp_u32<0x4E>(top));
          const uint32_t byte = scale_byte<PAGE>(top);
          static_cast<uint2*>(which ? V : K)[row * 16 + c] = encode8<PAGE>(x, byte);
          if ((c & 3) == 0) (which ? V_scale : K_scale)[row * kScales + (c >> 2)] = (uint8_t)byte;
        }
      }
    }
  }
}

// ---- g2 ----------------------------------------------------------------------------------------------------
constexpr int kReadSpan = 32;  // positions of a workgroup

// Workgroups: (KV head, stretch of positions, sequence).  All rows of K and V of a workgroup are on their way before the first
// is stored.  A lane makes 16 bytes of a dense row, so that the wavefront's stores are whole, and they are streamed past
// the caches.  A prompt of 32K, e4m3 to bf16 (204 MB): 31 us, 6.6 TB/s, the codes from the Infinity Cache (a context of 256K from
// memory: 287 us, 5.7 TB/s); with ordinary stores 43, with lanes that make
// 32 bytes in two stores 50 (66 streamed: halves of lines).
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kMoveThreads) void pages_read_kernel(const Map m, const void* K, const void* V,
                                                                  const uint8_t* K_scale,
                                                                  const uint8_t* V_scale, int first,
                                                                  int stretches, int64_t units, int lrows,
                                                                  void* K_out, void* V_out) {
  constexpr int kLanes = kD * (BF16 ? 2 : 4) / 16, kPass = kMoveThreads / kLanes, kN = kReadSpan / kPass;
  using Raw = std::conditional_t<!is8(PAGE), uint4, std::conditional_t<BF16, uint2, uint32_t>>;
  const int grp = threadIdx.x / kLanes, c = threadIdx.x % kLanes;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int kvh = (int)(u % m.Hkv);
    const int64_t v = u / m.Hkv;
    const int b = (int)(v / stretches), p0 = first + (int)(v % stretches) * kReadSpan;
    const int len = min(m.kv_len[b], m.l_max);
    if (p0 >= len) continue;
    int64_t row[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int p = p0 + i * kPass + grp;
      row[i] = row_of(m, b, kvh, min(p, len - 1));
      if (p >= len) row[i] = -1;
    }
    Raw x[2][kN];
    uint32_t sc[2][kN];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      if (!(which ? V_out : K_out)) continue;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (row[i] < 0) continue;
        x[which][i] = static_cast<const Raw*>(which ? V : K)[row[i] * kLanes + c];
        if constexpr (is8(PAGE)) sc[which][i] = (which ? V_scale : K_scale)[row[i] * kScales + c / (kLanes / kScales)];
      }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      void* const out = which ? V_out : K_out;
      if (!out) continue;
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        if (row[i] < 0) continue;
        uint4 y;
        if constexpr (!is8(PAGE)) {
          y = x[which][i];
        } else if constexpr (BF16) {
          y = decode8_bf16<PAGE>(x[which][i], scale_of(sc[which][i]));
        } else {
          float f[8];
          decode8<PAGE>(make_uint2(x[which][i], 0u), scale_of(sc[which][i]), f);
          y = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        }
        const dev::u32x4 z = {y.x, y.y, y.z, y.w};
        __builtin_nontemporal_store(
            z, reinterpret_cast<dev::u32x4*>(out) +
                   (((int64_t)b * m.Hkv + kvh) * lrows + p0 + i * kPass + grp) * kLanes + c);
      }
    }
  }
}

constexpr int64_t kMostBlocks = 1 << 20;

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API int lrqk_validate_pages(const lrqk_pages_shape* shape) { return lrqk::check_pages(shape); }

LRQK_API int lrqk_pages_append(const lrqk_pages_shape* shape, const lrqk_pages* pg, const void* k_new,
                               const void* v_new, void* stream) {
  using namespace lrqk;
  const int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  const lrqk_pages_shape& s = *shape;
  if (!pages_given(s, pg) || !k_new || !v_new || !aligned16(k_new) || !aligned16(v_new)) return LRQK_EINVAL;
  const Map m = make_map(s, *pg);
  const int64_t blocks = ((int64_t)s.T * s.Hkv + kAppendRows - 1) / kAppendRows;
  const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks));
  by_type(s, [&](auto bf16, auto page) {
    hipLaunchKernelGGL((pages_append_kernel<bf16.value, page.value>), grid, dim3(kMoveThreads), 0,
                       static_cast<hipStream_t>(stream), m, k_new, v_new, pg->K, pg->V, pg->K_scale,
                       pg->V_scale);
  });
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}

LRQK_API int lrqk_pages_read(const lrqk_pages_shape* shape, const lrqk_pages* pg, int32_t first, void* K_out,
                             void* V_out, void* stream) {
  using namespace lrqk;
  const int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  const lrqk_pages_shape& s = *shape;
  if (!pages_given(s, pg) || first < 0 || (!K_out && !V_out)) return LRQK_EINVAL;
  if ((K_out && !aligned16(K_out)) || (V_out && !aligned16(V_out))) return LRQK_EINVAL;
  if (first >= s.l_max) return LRQK_OK;  // no such position
  const Map m = make_map(s, *pg);
  const int stretches = ceil_div(s.l_max - first, kReadSpan);
  const int64_t units = (int64_t)s.B * s.Hkv * stretches;
  const dim3 grid((unsigned)(units < kMostBlocks ? units : kMostBlocks));
  by_type(s, [&](auto bf16, auto page) {
    hipLaunchKernelGGL((pages_read_kernel<bf16.value, page.value>), grid, dim3(kMoveThreads), 0,
                       static_cast<hipStream_t>(stream), m, pg->K, pg->V, pg->K_scale, pg->V_scale, first,
                       stretches, units, s.l_cap > 0 ? s.l_cap : s.l_max, K_out, V_out);
  });
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}
