// r0, r1, g4 -- rotary positions: their table, queries and keys turned, and a layer's new rows turned and written into their
// pages in one call (include/lrqk.h).
//
// A position's angle for pair j is p turns[j] mod 2^64, a fraction of a turn: the product of two integers, so nothing is
// lost at far positions and no argument reduction is needed beyond taking its nearest quarter off.  A wavefront takes one token
// (or some of its heads): lane j makes the cosine and sine of pair j once, LDS deals them out, and sixteen lanes turn a row of 128
// elements, eight each, four rows at a time.
// Bound by memory: 32768 tokens of 32 + 8 heads, bf16, 671 MB, 122 us (5.5 TB/s), 16384 in fp32 131 us; for few tokens by the latency of
// a launch, the positions and the angles: 1 token 2.7 us, 16 and 64 tokens 3.6 by a kernel trace, 3.0 to 3.3 a call in a captured run of twenty.
#include "pages.h"

#include <cmath>

namespace lrqk {
namespace {

using namespace pages;

constexpr int kThreads = 256;
constexpr int kWaves = 4;
constexpr int kEach = 4;   // quads of rows that a wavefront has in flight
constexpr int kMaxHeads = 1024;

struct Rope {
  const uint64_t* turns;
  int rot, layout, back;
  float amplitude;
};

// Cosine and sine of a fraction of a turn (in units of 2^-64), off by at most 3.2 2^-24.  The nearest quarter is taken off; what
// is left is within an eighth of a turn, |x| <= pi / 4, where the Taylor series to x^9 and x^10 leave less than 2^-29.
__device__ __forceinline__ float2 cos_sin(uint64_t turn) {
  const uint32_t quarter = (uint32_t)((turn + (1ull << 61)) >> 62);
  const int32_t rest = (int32_t)((int64_t)(turn - ((uint64_t)quarter << 62)) >> 32);
  const float x = (float)rest * 1.46291807926715968e-9f;  // 2 pi / 2^32
  const float z = x * x;
  const float s = __builtin_fmaf(
      x * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
  const float c = __builtin_fmaf(
      z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f),
                                          1.0f / 24.0f),
                        -0.5f),
      1.0f);
  const float a = quarter & 1 ? -s : c, b = quarter & 1 ? c : s;
  return quarter & 2 ? make_float2(-a, -b) : make_float2(a, b);
}

// What a lane multiplies its eight elements, chunk c of 16, and their partners with; `turned`: how many of the eight are.
struct Angles {
  float cs[8], sn[8];
  int turned;
};

// The wavefront's token is at position pos; lds: 64 pairs of the wavefront's own.
__device__ __forceinline__ void make_angles(const Rope& r, uint64_t turn, int pos, int lane, float2* lds, Angles& a) {
  const int half = r.rot >> 1, c = lane & 15;
  if (lane < half) {
    const float2 x = cos_sin(turn * (uint64_t)(int64_t)pos);
    lds[lane] = make_float2(x.x * r.amplitude, (r.back ? -x.y : x.y) * r.amplitude);
  }
  __builtin_amdgcn_wave_barrier();  // (a wavefront's LDS operations execute in order)
  a.turned = min(max(r.rot - 8 * c, 0), 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = 8 * c + i;
    const bool first = r.layout == LRQK_ROPE_PAIRS ? e % 2 == 0 : e < half;
    const int j = r.layout == LRQK_ROPE_PAIRS ? e >> 1 : first ? e : e - half;
    const float2 x = lds[e < r.rot ? j : 0];
    a.cs[i] = x.x;
    a.sn[i] = first ? -x.y : x.y;
  }
  __builtin_amdgcn_wave_barrier();
}

template <bool BF16>
struct Chunk {
  uint4 a, b;  // b: fp32 only
};
template <bool BF16>
__device__ __forceinline__ Chunk<BF16> load_chunk(const void* row, int c) {
  Chunk<BF16> x;
  x.b = make_uint4(0, 0, 0, 0);
  load8<BF16>(row, 0, c, x.a, x.b);
  return x;
}
template <bool BF16>
__device__ __forceinline__ Chunk<BF16> make_chunk(const float (&y)[8]) {
  Chunk<BF16> x;
  if constexpr (BF16) {
    x.a = make_uint4(dev::pack_bf16(y[0], y[1]), dev::pack_bf16(y[2], y[3]), dev::pack_bf16(y[4], y[5]), dev::pack_bf16(y[6], y[7]));
  } else {
    x.a = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
    x.b = make_uint4(__float_as_uint(y[4]), __float_as_uint(y[5]), __float_as_uint(y[6]), __float_as_uint(y[7]));
  }
  return x;
}
__device__ __forceinline__ uint4 from_lane(uint4 x, int lane) {
  auto get = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_ds_bpermute(lane << 2, (int)v); };
  return make_uint4(get(x.x), get(x.y), get(x.z), get(x.w));
}

// Chunk c of a row, turned.  In halves the partners of a chunk are another lane's chunk if rot / 2 is a multiple of 8; else
// they are loaded one by one, before anything of the row is stored (32768 tokens: rot = 112 127 us, rot = 126 183).
template <bool IN, bool OUT>
__device__ __forceinline__ Chunk<OUT> turned(const Rope& r, const Angles& a, const Chunk<IN>& in, const void* row, int lane) {
  float x[8], p[8], y[8];
  get8<IN>(in.a, in.b, x);
  const int half = r.rot >> 1, c = lane & 15;
  if (r.layout == LRQK_ROPE_PAIRS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = x[i ^ 1];
  } else if (half % 8 == 0) {
    const int other = 8 * c < half ? c + (half >> 3) : c - (half >> 3);
    const int from = (lane & 48) | (other & 15);
    Chunk<IN> q;
    q.a = from_lane(in.a, from);
    q.b = IN ? q.a : from_lane(in.b, from);
    get8<IN>(q.a, q.b, p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int e = 8 * c + i, o = e < half ? e + half : e < r.rot ? e - half : e;
      p[i] = IN ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(row)[o] << 16) : static_cast<const float*>(row)[o];
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = __builtin_fmaf(x[i], a.cs[i], p[i] * a.sn[i]);
    y[i] = i < a.turned ? t : x[i];
  }
  Chunk<OUT> out = make_chunk<OUT>(y);
  if constexpr (IN == OUT) {
    if (a.turned == 0) {  // as they are, bit for bit
      out.a = in.a;
      out.b = in.b;
    }
  }
  return out;
}

// ---- r1 ----------------------------------------------------------------------------------------------------
struct Rows {
  const char* in;
  char* out;
  int64_t in_stride, out_stride;  // bytes from one token to the next
  int heads;
};
struct RotateArgs {
  Rope rope;
  const int32_t* pos;
  Rows q, k;
  int T, parts, q_quads, quads;  // quads: four heads of q or k; a wavefront has every parts-th run of them
};

template <bool IN, bool OUT>
__device__ __forceinline__ void turn_heads(const Rope& r, const Rows& x, int t, int from, int to, uint64_t turn, int pos, int lane,
                                           float2* lds, Angles& a, bool& made) {
  const int g = lane >> 4, c = lane & 15;
  const char* in = x.in + t * x.in_stride;
  char* out = x.out + t * x.out_stride;
  for (int i0 = from; i0 < to; i0 += kEach) {
    Chunk<IN> v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int h = min(4 * min(i0 + i, to - 1) + g, x.heads - 1);
      v[i] = load_chunk<IN>(in + (int64_t)h * (kD * (IN ? 2 : 4)), c);
    }
    if (!made) make_angles(r, turn, pos, lane, lds, a);  // while the rows are on their way
    made = true;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int h = 4 * (i0 + i) + g;
      if (i0 + i >= to || h >= x.heads) continue;
      const Chunk<OUT> y = turned<IN, OUT>(r, a, v[i], in + (int64_t)h * (kD * (IN ? 2 : 4)), lane);
      store8<OUT>(out + (int64_t)h * (kD * (OUT ? 2 : 4)), 0, c, y.a, y.b);
    }
  }
}

template <bool QIN, bool QOUT, bool KT>
__global__ __launch_bounds__(kThreads) void rotate_kernel(const RotateArgs s) {
  __shared__ float2 angles[kWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + w;
  const int t = (int)(unit / s.parts), part = (int)(unit % s.parts);
  if (t >= s.T) return;
  const int pos = s.pos[t];
  const uint64_t turn = s.rope.turns[min(lane, (s.rope.rot >> 1) - 1)];
  const int each = (s.quads + s.parts - 1) / s.parts, from = part * each, to = min(s.quads, from + each);
  Angles a;
  bool made = false;
  if (from < s.q_quads) turn_heads<QIN, QOUT>(s.rope, s.q, t, from, min(to, s.q_quads), turn, pos, lane, angles[w], a, made);
  if (to > s.q_quads)
    turn_heads<KT, KT>(s.rope, s.k, t, max(from - s.q_quads, 0), to - s.q_quads, turn, pos, lane, angles[w], a, made);
}

// ---- g4 ----------------------------------------------------------------------------------------------------
struct NewArgs {
  Map m;
  Rope rope;
  Rows q;
  const char *k, *v;
  int64_t k_stride, v_stride;
  void *K, *V;
  uint8_t *K_scale, *V_scale;
  const int32_t *pos, *slot;
  int parts, q_quads, kv_quads;
};

// As r1; k and v go on into their pages.  Bound by memory: 15939 tokens of 4 prompts into pages of 4 bits, 343 MB, 66 us (5.2 TB/s); one
// token of 16 sequences 3.7 us with positions and slots at hand, 4.6 from the tables (start, then length, then table).
template <bool BF16, int PAGE>
__global__ __launch_bounds__(kThreads) void rotate_append_kernel(const NewArgs s) {
  constexpr int kRow = kD * (BF16 ? 2 : 4);
  __shared__ float2 angles[kWaves][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = (int64_t)blockIdx.x * kWaves + w;
  const int t = (int)(unit / s.parts), part = (int)(unit % s.parts);
  if (t >= s.m.T) return;
  const uint64_t turn = s.rope.turns[min(lane, (s.rope.rot >> 1) - 1)];
  const int page = 1 << s.m.page_log2;
  int pos, pg = -1, off = 0;  // pg: no page
  if (s.pos) {
    pos = s.pos[t];
    const int slot = s.slot[t];
    if (slot >= 0) {
      pg = slot >> s.m.page_log2;
      off = slot & (page - 1);
    }
    if (pos >= s.m.l_max) pg = -1;
  } else {
    const int b = sequence_of(s.m, t);
    if (b < 0) return;
    const Seq q = sequence(s.m, b);
    if (t < q.first || t >= q.first + q.n) return;
    pos = q.len - q.n + (t - q.first);
    if (pos >= 0 && pos < s.m.l_max) pg = s.m.table[(size_t)b * s.m.max_pages + (pos >> s.m.page_log2)];
    off = pos & (page - 1);
  }
  if (pos < 0) return;
  if ((unsigned)pg >= (unsigned)s.m.n_pages) pg = -1;
  const int quads = s.q_quads + 2 * s.kv_quads;
  const int each = (quads + s.parts - 1) / s.parts, from = part * each, to = min(quads, from + each);
  Angles a;
  bool made = false;
  if (from < s.q_quads)
    turn_heads<BF16, BF16>(s.rope, s.q, t, from, min(to, s.q_quads), turn, pos, lane, angles[w], a, made);
  if (pg < 0) return;
  const int g = lane >> 4, c = lane & 15;
  auto rows = [&](bool key, const char* base, void* pool, uint8_t* scale, int lo, int hi) __attribute__((always_inline)) {
    for (int i0 = lo; i0 < hi; i0 += kEach) {
      Chunk<BF16> v[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int h = min(4 * min(i0 + i, hi - 1) + g, s.m.Hkv - 1);
        v[i] = load_chunk<BF16>(base + (int64_t)h * kRow, c);
      }
      if (key && !made) make_angles(s.rope, turn, pos, lane, angles[w], a);
      made = made || key;
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int h = 4 * (i0 + i) + g;
        if (i0 + i >= hi || h >= s.m.Hkv) continue;
        if (key) v[i] = turned<BF16, BF16>(s.rope, a, v[i], base + (int64_t)h * kRow, lane);
        const int64_t row = (((int64_t)pg * s.m.Hkv + h) << s.m.page_log2) + off;
        put_row<BF16, PAGE>(pool, scale, row, c, v[i].a, v[i].b);
      }
    }
  };
  const int k0 = s.q_quads, v0 = k0 + s.kv_quads;
  rows(true, s.k + t * s.k_stride, s.K, s.K_scale, max(from, k0) - k0, min(to, v0) - k0);
  rows(false, s.v + t * s.v_stride, s.V, s.V_scale, max(from, v0) - v0, min(to, quads) - v0);
}

// Wavefronts a token: two for each of the chip's 1024 SIMDs, a quad of rows each at least.  In us a call of a captured run of twenty
// with 1 / 512 / 2048 / 8192 of them, bf16: 64 tokens 5.6 / 3.2 / 3.0 / 3.0, 256 5.9 / 4.5 / 3.8 / 3.8, 1024 6.9 / 6.9 / 5.9 / 7.4, 4096 15.0 / 14.9 / 15.0 / 14.5.
int parts_of(int T, int quads) {
  const int want = (2048 + T - 1) / T;
  return want < 1 ? 1 : want > quads ? quads : want;
}

int check_rope(const lrqk_rope* r) {
  if (!r || !r->turns || !aligned16(r->turns)) return LRQK_EINVAL;
  if (r->layout != LRQK_ROPE_HALVES && r->layout != LRQK_ROPE_PAIRS) return LRQK_EINVAL;
  if (r->back != 0 && r->back != 1) return LRQK_EINVAL;
  if (r->rot < 2 || r->rot > kD || r->rot % 2 != 0 || !std::isfinite(r->amplitude)) return LRQK_ESHAPE;
  return LRQK_OK;
}
Rope make_rope(const lrqk_rope& r) { return Rope{r.turns, r.rot, r.layout, r.back, r.amplitude}; }

bool kv_type(int t) { return t == LRQK_KV_BF16 || t == LRQK_KV_F32; }
// A stride in elements: 0 means dense; whether it will do.
bool stride_ok(int32_t stride, int heads, int type) {
  return stride == 0 || (stride >= heads * kD && (stride * (int64_t)kv_elem_bytes(type)) % 16 == 0);
}
int64_t stride_bytes(int32_t stride, int heads, int type) {
  return (int64_t)(stride ? stride : heads * kD) * (int64_t)kv_elem_bytes(type);
}

}  // namespace
}  // namespace lrqk

#define LRQK_API extern "C" __attribute__((visibility("default")))

LRQK_API int lrqk_rope_turns(int32_t rot, int32_t scaling, double base, double factor, double low, double high, int32_t l_orig,
                             uint64_t* turns, float* amplitude) {
  using namespace lrqk;
  if (!turns || scaling < LRQK_ROPE_PLAIN || scaling > LRQK_ROPE_RAMP) return LRQK_EINVAL;
  if (rot < 2 || rot > kD || rot % 2 != 0) return LRQK_ESHAPE;
  if (!(base > 1.0) || !std::isfinite(base)) return LRQK_EINVAL;
  if (scaling != LRQK_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return LRQK_EINVAL;
  const bool blend = scaling == LRQK_ROPE_BANDS || scaling == LRQK_ROPE_RAMP;
  if (blend && (!(low > 0.0) || !(high > low) || !std::isfinite(high) || l_orig < 1)) return LRQK_EINVAL;
  typedef long double real;
  const real two_pi = 2 * acosl(-1.0L);
  real b = base;
  if (scaling == LRQK_ROPE_BASE && rot > 2) b = (real)base * powl((real)factor, (real)rot / (rot - 2));
  if (!std::isfinite(b)) return LRQK_EINVAL;
  real j0 = 0, j1 = 0;
  if (scaling == LRQK_ROPE_RAMP) {
    auto index = [&](real n) { return rot * logl(l_orig / (two_pi * n)) / (2 * logl((real)base)); };
    j0 = std::fmax(floorl(index(high)), (real)0);
    j1 = std::fmin(ceill(index(low)), (real)(rot - 1));  // (may lie behind the last pair, rot / 2 - 1: the pairs have a part of the ramp then)
  }
  for (int j = 0; j < rot / 2; ++j) {
    real f = powl(b, (real)(-2 * j) / rot);
    real s = 1;
    if (scaling == LRQK_ROPE_LINEAR) s = 0;
    if (scaling == LRQK_ROPE_BANDS) s = (l_orig * f / two_pi - low) / ((real)high - low);
    if (scaling == LRQK_ROPE_RAMP) s = 1 - (j - j0) / std::fmax(j1 - j0, (real)0.001L);
    s = std::fmin(std::fmax(s, (real)0), (real)1);
    if (scaling != LRQK_ROPE_BASE && scaling != LRQK_ROPE_PLAIN) f = f * (s + (1 - s) / factor);
    real turn = f / two_pi;
    turn -= floorl(turn);
    const real whole = roundl(ldexpl(turn, 64));  // (of 64 bits: nothing is lost)
    turns[j] = whole >= ldexpl((real)1, 64) ? 0 : (uint64_t)whole;
  }
  if (amplitude) *amplitude = scaling == LRQK_ROPE_RAMP && factor > 1.0 ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return LRQK_OK;
}

LRQK_API int lrqk_rotate(const lrqk_rotate_shape* shape, const lrqk_rope* rope, const int32_t* pos, const void* q, void* q_out,
                         const void* k, void* k_out, void* stream) {
  using namespace lrqk;
  if (!shape) return LRQK_EINVAL;
  const lrqk_rotate_shape& s = *shape;
  int rc = check_rope(rope);
  if (rc != LRQK_OK) return rc;
  if (s.T < 1 || s.T >= (1 << 24) || s.d != kD) return LRQK_ESHAPE;
  if (!q != !q_out || !k != !k_out || (!q && !k) || !pos || !aligned16(pos)) return LRQK_EINVAL;
  if (!aligned16(q) || !aligned16(q_out) || !aligned16(k) || !aligned16(k_out)) return LRQK_EINVAL;
  if (q && (!kv_type(s.q_type) || !kv_type(s.q_out_type))) return LRQK_EINVAL;
  if (k && !kv_type(s.k_type)) return LRQK_EINVAL;
  if (q && (s.Hq < 1 || s.Hq > kMaxHeads || !stride_ok(s.q_stride, s.Hq, s.q_type) || !stride_ok(s.q_out_stride, s.Hq, s.q_out_type)))
    return LRQK_ESHAPE;
  if (k && (s.Hkv < 1 || s.Hkv > kMaxHeads || !stride_ok(s.k_stride, s.Hkv, s.k_type) || !stride_ok(s.k_out_stride, s.Hkv, s.k_type)))
    return LRQK_ESHAPE;
  RotateArgs a{make_rope(*rope), pos, {}, {}, s.T, 1, 0, 0};
  if (q)
    a.q = Rows{static_cast<const char*>(q), static_cast<char*>(q_out), stride_bytes(s.q_stride, s.Hq, s.q_type),
               stride_bytes(s.q_out_stride, s.Hq, s.q_out_type), s.Hq};
  if (k)
    a.k = Rows{static_cast<const char*>(k), static_cast<char*>(k_out), stride_bytes(s.k_stride, s.Hkv, s.k_type),
               stride_bytes(s.k_out_stride, s.Hkv, s.k_type), s.Hkv};
  if (q == q_out && q && (s.q_type != s.q_out_type || a.q.in_stride != a.q.out_stride)) return LRQK_EINVAL;
  if (k == k_out && k && a.k.in_stride != a.k.out_stride) return LRQK_EINVAL;
  a.q_quads = ceil_div(a.q.heads, 4);
  a.quads = a.q_quads + ceil_div(a.k.heads, 4);
  a.parts = parts_of(s.T, a.quads);
  const dim3 grid((unsigned)(((int64_t)s.T * a.parts + kWaves - 1) / kWaves));
  auto go = [&](auto in, auto out, auto kt) {
    hipLaunchKernelGGL((rotate_kernel<in.value, out.value, kt.value>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  };
  auto type = [](int t, auto f) { t == LRQK_KV_BF16 ? f(std::true_type{}) : f(std::false_type{}); };
  const int qi = q ? s.q_type : s.k_type, qo = q ? s.q_out_type : s.k_type, kt = k ? s.k_type : s.q_type;
  type(qi, [&](auto i) { type(qo, [&](auto o) { type(kt, [&](auto x) { go(i, o, x); }); }); });
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}

LRQK_API int lrqk_pages_rotate_append(const lrqk_pages_shape* shape, const lrqk_pages* pg, const lrqk_rope* rope,
                                      const lrqk_new_rows* rows, void* stream) {
  using namespace lrqk;
  int rc = check_pages(shape);
  if (rc != LRQK_OK) return rc;
  const lrqk_pages_shape& s = *shape;
  if (!rows) return LRQK_EINVAL;
  const lrqk_new_rows& n = *rows;
  if (!n.pos != !n.slot || !aligned16(n.pos) || !aligned16(n.slot)) return LRQK_EINVAL;
  if (!pg) return LRQK_EINVAL;
  lrqk_pages given = *pg;
  if (n.pos) given.table = given.start = given.kv_len = n.pos;  // not looked at
  if (!pages_given(s, &given)) return LRQK_EINVAL;
  rc = check_rope(rope);
  if (rc != LRQK_OK) return rc;
  if (!n.k || !n.v || !n.q != !n.q_out || !aligned16(n.q) || !aligned16(n.k) || !aligned16(n.v) || !aligned16(n.q_out)) return LRQK_EINVAL;
  if (!stride_ok(n.k_stride, s.Hkv, s.kv_dtype) || !stride_ok(n.v_stride, s.Hkv, s.kv_dtype)) return LRQK_ESHAPE;
  if (n.q && !stride_ok(n.q_stride, s.Hq, s.kv_dtype)) return LRQK_ESHAPE;
  NewArgs a{make_map(s, *pg), make_rope(*rope), {}, static_cast<const char*>(n.k), static_cast<const char*>(n.v),
            stride_bytes(n.k_stride, s.Hkv, s.kv_dtype), stride_bytes(n.v_stride, s.Hkv, s.kv_dtype), pg->K, pg->V, pg->K_scale,
            pg->V_scale, n.pos, n.slot, 1, 0, ceil_div(s.Hkv, 4)};
  if (n.q) {
    a.q = Rows{static_cast<const char*>(n.q), static_cast<char*>(n.q_out), stride_bytes(n.q_stride, s.Hq, s.kv_dtype),
               stride_bytes(0, s.Hq, s.kv_dtype), s.Hq};
    if (n.q == n.q_out && a.q.in_stride != a.q.out_stride) return LRQK_EINVAL;
    a.q_quads = ceil_div(s.Hq, 4);
  }
  a.parts = parts_of(s.T, a.q_quads + 2 * a.kv_quads);
  const dim3 grid((unsigned)(((int64_t)s.T * a.parts + kWaves - 1) / kWaves));
  by_type(s, [&](auto bf16, auto page) {
    hipLaunchKernelGGL((rotate_append_kernel<bf16.value, page.value>), grid, dim3(kThreads), 0, static_cast<hipStream_t>(stream), a);
  });
  LRQK_HIP(hipGetLastError());
  return LRQK_OK;
}
