// Attention of a chunk of new tokens over a paged cache.
#include "paged.h"

namespace reflex {

namespace {

// Running maxima start here instead of at -infinity, so that a row that sees
// nothing has exp2(-infinity - m) = 0 and not NaN.
constexpr float kFloor = -3.0e38f;

// Keys that a query at token `pos` of a sequence of `len` sees: [lo, hi).
struct Span { int lo, hi; };
RFX_DEV Span span_of(const PagedAttnArgs& a, int pos, int len) {
  Span s;
  const int64_t cap = (int64_t)a.q.max_pages << a.c.shift;
  s.hi = (int)min((int64_t)(a.causal ? min(pos, len - 1) + 1 : len), cap);
  s.lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  return s;
}

template <typename T, int ST> struct Elem { typedef T type; };
template <typename T> struct Elem<T, REFLEX_STORE_FP8> { typedef uint8_t type; };
template <typename T> struct Elem<T, REFLEX_STORE_INT8> { typedef int8_t type; };

template <int ST, typename E> RFX_DEV float elem_f(E v) {
  if (ST == REFLEX_STORE_FP8) return __builtin_amdgcn_cvt_f32_fp8((int)(uint32_t)v, 0);
  if (ST == REFLEX_STORE_INT8) return (float)v;
  return to_f(v);
}
template <> RFX_DEV float elem_f<REFLEX_STORE_INT8, int8_t>(int8_t v) { return (float)v; }
template <> RFX_DEV float elem_f<REFLEX_STORE_FP8, uint8_t>(uint8_t v) {
  return __builtin_amdgcn_cvt_f32_fp8((int)(uint32_t)v, 0);
}

// One (row, query head) by one wave, key by key; each lane holds DH / 64 dims.
template <typename T, int ST, int DH>
RFX_DEV void scalar_row(const PagedAttnArgs& a, int64_t row, int head, int b, Span sp, float& m, float& l, float* o) {
  typedef typename Elem<T, ST>::type E;
  constexpr int N = DH / 64;
  constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  const int lane = threadIdx.x & 63;
  const T* qp = reinterpret_cast<const T*>(a.x.p) + row * a.x.rs + head * a.x.hs + lane * N;
  float q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = to_f(qp[i]);
    o[i] = 0.f;
  }
  m = kFloor;
  l = 0.f;
  const int64_t hoff = (int64_t)(head / a.group) << a.c.shift;
  for (int j = sp.lo; j < sp.hi; ++j) {
    const int r = page_row(a.c, a.q, b, j);
    if (r < 0) continue;
    const int64_t prow = r + hoff;
    const E* kp = reinterpret_cast<const E*>(a.c.k) + prow * DH + lane * N;
    const E* vp = reinterpret_cast<const E*>(a.c.v) + prow * DH + lane * N;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) s += q[i] * elem_f<ST>(kp[i]);
    s = warp_sum(s) * a.scale2;
    if (Q8) s *= a.c.k_scale[prow];
    const float m2 = fmaxf(m, s);
    const float c = exp2f(m - m2);
    float p = exp2f(s - m2);
    m = m2;
    l = l * c + p;
    if (Q8) p *= a.c.v_scale[prow];
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * c + p * elem_f<ST>(vp[i]);
  }
}

template <typename T, int ST, int DH>
__global__ __launch_bounds__(256) void paged_attn_row_kernel(const PagedAttnArgs a) {
  constexpr int N = DH / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row = id / a.n_q;
  const int head = (int)(id - row * a.n_q);
  if (row >= a.n_rows) return;
  const int b = seq_of_row(a.q, row, lane);
  if (b < 0 || b >= a.q.n) return;
  const int len = a.q.len[b];
  const int pos = (int)((int64_t)len - a.q.cu[b + 1] + row);
  float m, l, o[N];
  scalar_row<T, ST, DH>(a, row, head, b, span_of(a, pos, len), m, l, o);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = reinterpret_cast<T*>(const_cast<char*>(a.o.p)) + row * a.o.rs + head * a.o.hs + lane * N;
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = from_f<T>(o[i] * inv);
}

template <typename T, int ST>
hipError_t launch_store(const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_rows * a.n_q + 3) / 4));
  if (a.c.dh == 64)
    RFX_LAUNCH((paged_attn_row_kernel<T, ST, 64>), grid, dim3(256), 0, s, a);
  else if (a.c.dh == 128)
    RFX_LAUNCH((paged_attn_row_kernel<T, ST, 128>), grid, dim3(256), 0, s, a);
  else
    RFX_LAUNCH((paged_attn_row_kernel<T, ST, 256>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

PagedAttnPlan paged_attention_plan(const reflex_paged_cache&, const reflex_paged_batch&, int64_t, int, int) {
  PagedAttnPlan p;
  p.nsplit = 1;
  p.split_keys = 0;
  p.bytes = 0;
  return p;
}

template <typename T>
hipError_t launch_paged_attention(const PagedAttnArgs& a, int store, hipStream_t s) {
  if (store == REFLEX_STORE_FP8) return launch_store<T, REFLEX_STORE_FP8>(a, s);
  if (store == REFLEX_STORE_INT8) return launch_store<T, REFLEX_STORE_INT8>(a, s);
  return launch_store<T, REFLEX_STORE_BF16>(a, s);
}
template hipError_t launch_paged_attention<float>(const PagedAttnArgs&, int, hipStream_t);
template hipError_t launch_paged_attention<bf16_t>(const PagedAttnArgs&, int, hipStream_t);

}  // namespace reflex
