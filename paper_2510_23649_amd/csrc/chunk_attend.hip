// g3 -- exact causal attention of new tokens over the paged cache (include/lrqk.h).
//
// One workgroup per (new token, query head).  16 lanes share a row of K and of V, 8 elements each; the
// 16 groups of a workgroup take positions in turn, keep a running (max, sum, acc) each and merge at
// the end.  Everything in fp32.
#include "pages.h"

namespace lrqk {
namespace {

using namespace pages;

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

struct Args {
  Map m;
  const void *K, *V;
  const uint8_t *K_scale, *V_scale;
  const void* q;
  void* out;
  int Hq;
  float scale;
};

template <bool BF16, int PAGE>
__device__ __forceinline__ void load_row8(const void* base, const uint8_t* sc, int64_t row, int c, float (&x)[8]) {
  if constexpr (is8(PAGE)) {
    decode8<PAGE>(static_cast<const uint2*>(base)[row * 16 + c], scale_of(sc[row * kScales + (c >> 2)]), x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = BF16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(base)[row * kD + 8 * c + i] << 16)
                  : static_cast<const float*>(base)[row * kD + 8 * c + i];
  }
}

template <bool BF16, int PAGE>
__global__ __launch_bounds__(kThreads) void chunk_attend_kernel(const Args a) {
  __shared__ float gm[16], gs[16], gacc[16][kD];
  const Map& m = a.m;
  const int t = blockIdx.x, h = blockIdx.y, grp = threadIdx.x >> 4, c = threadIdx.x & 15;
  const int kvh = h / (a.Hq / m.Hkv);
  const int b = sequence_of(m, t);
  if (b < 0) return;
  const Seq s = sequence(m, b);
  if (t < s.first || t >= s.first + s.n) return;
  const int see = min(max(s.len - s.n + (t - s.first) + 1, 0), m.l_max);
  float q[8];
  load_row8<BF16, BF16 ? LRQK_PAGE_BF16 : LRQK_PAGE_F32>(a.q, nullptr, (int64_t)t * a.Hq + h, c, q);
  float mx = -INFINITY, sum = 0.0f, acc[8] = {};
  for (int p = grp; p < see; p += 16) {
    const int64_t row = row_of(m, b, kvh, p);
    if (row < 0) continue;
    float x[8], d = 0.0f;
    load_row8<BF16, PAGE>(a.K, a.K_scale, row, c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) d = __builtin_fmaf(q[i], x[i], d);
#pragma unroll
    for (int i = 1; i < 16; i <<= 1) d += __shfl_xor(d, i);
    d *= a.scale * kLog2e;
    const float mn = fmaxf(mx, d);
    if (mn == -INFINITY) continue;
    const float f = exp2f(mx - mn), w = exp2f(d - mn);
    load_row8<BF16, PAGE>(a.V, a.V_scale, row, c, x);
    sum = sum * f + w;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(w, x[i], acc[i] * f);
    mx = d != d ? d : mn;
  }
  if (c == 0) {
    gm[grp] = mx;
    gs[grp] = sum;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) gacc[grp][8 * c + i] = acc[i];
  __syncthreads();
  if (threadIdx.x >= kD) return;
  float M = -INFINITY, S = 0.0f, A = 0.0f;
  for (int i = 0; i < 16; ++i) M = gm[i] != gm[i] ? gm[i] : fmaxf(M, gm[i]);
  for (int i = 0; i < 16; ++i)
    if (gm[i] != -INFINITY) {
      const float f = exp2f(gm[i] - M);
      S += gs[i] * f;
      A += gacc[i][threadIdx.x] * f;
    }
  const float y = S == 0.0f ? 0.0f : A / S;
  const size_t at = ((size_t)t * a.Hq + h) * kD + threadIdx.x;
  if (BF16) static_cast<__bf16*>(a.out)[at] = (__bf16)y;
  else static_cast<float*>(a.out)[at] = y;
}

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API size_t lrqk_pages_workspace_bytes(const lrqk_pages_shape* shape) {
  return lrqk::check_pages(shape) == LRQK_OK ? 256 : 0;
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
  const Args a{make_map(s, *pg), pg->K, pg->V, pg->K_scale, pg->V_scale, q, out, s.Hq, s.scale};
  by_type(s, [&](auto bf16, auto page) {
    hipLaunchKernelGGL((chunk_attend_kernel<bf16.value, page.value>), dim3(s.T, s.Hq), dim3(kThreads), 0,
                       static_cast<hipStream_t>(stream), a);
  });
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}
