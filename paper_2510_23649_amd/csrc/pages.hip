// g1, g2 -- the paged K/V cache is written and read back (include/lrqk.h).
//
// Both move rows of 128 elements and are bound by memory.  16 lanes share a row, 8 elements each: 16-byte
// loads and stores of bf16 rows, full rows of 256 bytes per 16 lanes.  An 8-bit row has its four
// blocks of 32 elements in four lanes each: the block's largest magnitude takes two DPP steps, its
// scale is a power of two read off the bits (see pages.h), so that nothing but the rounding to the
// code is rounded.
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
constexpr int kRowsPerBlock = kMoveThreads / 16;

// Eight elements of a row, chunk c of 16.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t row, int c, float (&x)[8]) {
  if constexpr (BF16) {
    const uint4 u = static_cast<const uint4*>(base)[row * 16 + c];
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const float4 a = static_cast<const float4*>(base)[(row * 16 + c) * 2];
    const float4 b = static_cast<const float4*>(base)[(row * 16 + c) * 2 + 1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t row, int c, const float (&x)[8]) {
  if constexpr (BF16) {
    static_cast<uint4*>(base)[row * 16 + c] =
        make_uint4(dev::pack_bf16(x[0], x[1]), dev::pack_bf16(x[2], x[3]), dev::pack_bf16(x[4], x[5]),
                   dev::pack_bf16(x[6], x[7]));
  } else {
    static_cast<float4*>(base)[(row * 16 + c) * 2] = make_float4(x[0], x[1], x[2], x[3]);
    static_cast<float4*>(base)[(row * 16 + c) * 2 + 1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// One 16-lane group per row of k_new (blockIdx.y == 0) or v_new (1).
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kMoveThreads) void pages_append_kernel(const Map m, const void* k_new,
                                                                    const void* v_new, void* K, void* V,
                                                                    uint8_t* K_scale, uint8_t* V_scale) {
  const int grp = threadIdx.x >> 4, c = threadIdx.x & 15;
  const void* src = blockIdx.y ? v_new : k_new;
  void* dst = blockIdx.y ? V : K;
  uint8_t* sc = blockIdx.y ? V_scale : K_scale;
  const int64_t rows = (int64_t)m.T * m.Hkv;
  for (int64_t r0 = (int64_t)blockIdx.x * kRowsPerBlock; r0 < rows; r0 += (int64_t)gridDim.x * kRowsPerBlock) {
    const int64_t r = r0 + grp;
    const int t = (int)min(r / m.Hkv, (int64_t)m.T), kvh = (int)(r % m.Hkv);
    const int b = sequence_of(m, t);  // the whole wavefront takes part
    if (b < 0) continue;
    const Seq q = sequence(m, b);
    if (t < q.first || t >= q.first + q.n) continue;
    const int p = q.len - q.n + (t - q.first);
    if (p < 0 || p >= m.l_max) continue;
    const int64_t row = row_of(m, b, kvh, p);
    if (row < 0) continue;
    if constexpr (!is8(PAGE)) {
      constexpr int kChunks = BF16 ? 1 : 2;
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        static_cast<uint4*>(dst)[(row * 16 + c) * kChunks + i] =
            static_cast<const uint4*>(src)[(r * 16 + c) * kChunks + i];
    } else {
      float x[8];
      load8<BF16>(src, r, c, x);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
      top = max(top, dev::dpp_u32<0xB1>(top));  // over the four lanes of a block
      top = max(top, dev::dpp_u32<0x4E>(top));
      const uint32_t byte = scale_byte<PAGE>(top);
      static_cast<uint2*>(dst)[row * 16 + c] = encode8<PAGE>(x, byte);
      if ((c & 3) == 0) sc[row * kScales + (c >> 2)] = (uint8_t)byte;
    }
  }
}

// One 16-lane group per position; K and V of it.  Workgroups: (sequence, stretch of positions, KV head).
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kMoveThreads) void pages_read_kernel(const Map m, const void* K, const void* V,
                                                                  const uint8_t* K_scale,
                                                                  const uint8_t* V_scale, int first,
                                                                  int stretches, int64_t units, int lrows,
                                                                  void* K_out, void* V_out) {
  const int grp = threadIdx.x >> 4, c = threadIdx.x & 15;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int kvh = (int)(u % m.Hkv);
    const int64_t v = u / m.Hkv;
    const int b = (int)(v / stretches), st = (int)(v % stretches);
    const int p = first + st * kRowsPerBlock + grp;
    const int len = min(m.kv_len[b], m.l_max);
    if (p >= len) continue;
    const int64_t row = row_of(m, b, kvh, p);
    if (row < 0) continue;
    const int64_t to = ((int64_t)b * m.Hkv + kvh) * lrows + p;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const void* src = which ? V : K;
      void* dst = which ? V_out : K_out;
      if (!dst) continue;
      if constexpr (!is8(PAGE)) {
        constexpr int kChunks = BF16 ? 1 : 2;
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
          static_cast<uint4*>(dst)[(to * 16 + c) * kChunks + i] =
              static_cast<const uint4*>(src)[(row * 16 + c) * kChunks + i];
      } else {
        const uint8_t* sc = which ? V_scale : K_scale;
        float x[8];
        decode8<PAGE>(static_cast<const uint2*>(src)[row * 16 + c], scale_of(sc[row * kScales + (c >> 2)]), x);
        store8<BF16>(dst, to, c, x);
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
  const int64_t blocks = ((int64_t)s.T * s.Hkv + kRowsPerBlock - 1) / kRowsPerBlock;
  const dim3 grid((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), 2);
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
  const int stretches = ceil_div(s.l_max - first, kRowsPerBlock);
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
