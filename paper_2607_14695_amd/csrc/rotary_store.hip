// Rotary positions over several axes, and the paged cache's writer and reader.
//
// All three move rows of head_dim values once and are bound by that traffic.
// A thread holds 8 values of each half of a head (two 16-byte accesses in
// bf16), so it has both members of 8 rotary pairs, and head_dim / 16 threads
// make a row: its maximum is a few shuffles.  A thread goes over several heads
// of its token where there are enough tokens, because the angles' sines are
// the arithmetic of these kernels and belong to the token alone.
#include "paged.h"

namespace reflex {

namespace {

// 8 consecutive elements as fp32
RFX_DEV void ld8(const float* p, float* o) {
  frag_to_f(ld16(p), o, 0.f);
  frag_to_f(ld16(p + 4), o + 4, 0.f);
}
RFX_DEV void ld8(const bf16_t* p, float* o) { frag_to_f(ld16(p), o, bf16_t(0)); }
RFX_DEV void st8(float* p, const float* v) {
  st16(p, f_to_frag(v, 0.f));
  st16(p + 4, f_to_frag(v + 4, 0.f));
}
RFX_DEV void st8(bf16_t* p, const float* v) { st16(p, f_to_frag(v, bf16_t(0))); }

// Angle of a pair at a position, as a fraction of a turn in [-1/2, 1/2]: the
// product and its reduction in 64 bits, so far positions keep 2^-53 of the
// product (a position of 10^6 keeps the angle to 2e-10).
RFX_DEV double turn_of(int64_t pos, double turns) {
  const double t = (double)pos * turns;
  return t - rint(t);
}

// ---------------------------------------------------------------------------
// rotary
// ---------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a) {
  const int G = a.plan.head_dim >> 4;
  const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = t / G;
  const int g = (int)(t - row * G);
  if (row >= a.n_rows) return;
  const int half = a.plan.head_dim >> 1;
  const int h0 = blockIdx.y * a.heads_per, h1 = min(a.n_heads, h0 + a.heads_per);
  const T* x = reinterpret_cast<const T*>(a.x.p) + row * a.x.rs + 8 * g;
  T* y = reinterpret_cast<T*>(const_cast<char*>(a.y.p)) + row * a.y.rs + 8 * g;
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pair = 8 * g + i;
    const double f = turn_of(a.pos[a.plan.axis[pair] * a.ps + row], a.plan.turns[pair]);
    sincospif(2.f * (float)f, &sn[i], &cs[i]);
    if (a.inverse) sn[i] = -sn[i];
  }
  for (int h = h0; h < h1; ++h) {
    float u[8], w[8], p[8], q[8];
    ld8(x + h * a.x.hs, u);
    ld8(x + h * a.x.hs + half, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = u[i] * cs[i] - w[i] * sn[i];
      q[i] = w[i] * cs[i] + u[i] * sn[i];
    }
    st8(y + h * a.y.hs, p);
    st8(y + h * a.y.hs + half, q);
  }
}

// ---------------------------------------------------------------------------
// paged write
// ---------------------------------------------------------------------------
// Nearest fp32 to x whose rounding to fewer bits is that of x itself: where
// the conversion is inexact the last bit is set (rounding to odd).
RFX_DEV float odd_float(double x) {
  float f = (float)x;
  const double d = (double)f;
  if (d != x) {
    uint32_t u = __float_as_uint(f);
    if (fabs(d) > fabs(x)) u -= 1;
    f = __uint_as_float(u | 1u);
  }
  return f;
}

// x / scale to the nearest integer, ties to even: the product with the
// reciprocal is within 2^-50 of the quotient, so only a quotient that close
// to a border needs the division
RFX_DEV int code_int8(double x, double scale, double inv) {
  const double t = x * inv;
  double r = rint(t);
  if (fabs(fabs(t - r) - 0.5) < 1e-9) r = rint(x / scale);
  return max(-127, min(127, (int)r));
}

// Scale of a row from the bits of its largest magnitude; NaN for a row with a
// value that is not finite.
template <int ST>
RFX_DEV float row_scale(uint32_t amax) {
  if (amax >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  if (ST == REFLEX_STORE_INT8) return fmaxf(__uint_as_float(amax) * (1.f / 127.f), 0x1p-126f);
  // amax = m * 2^e with m in [1, 2), 448 = 1.75 * 2^8: the scale is 2^(e - 8), or
  // twice that above 1.75
  int k = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
  k = max(k, -126);
  return __uint_as_float((uint32_t)(k + 127) << 23);
}

// The codes of 8 values as 8 bytes.
template <int ST>
RFX_DEV uint2 codes8(const double* x, float scale) {
  uint32_t w[2] = {0, 0};
  if (!(scale < INFINITY)) return make_uint2(0u, 0u);
  const double s = (double)scale, inv = 1.0 / s;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (ST == REFLEX_STORE_INT8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[i] |= (uint32_t)(code_int8(x[4 * i + j], s, inv) & 255) << (8 * j);
    } else {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = fminf(fmaxf(odd_float(x[4 * i + j] * inv), -448.f), 448.f);  // inv: a power of two
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], v, true);
    }
  }
  return make_uint2(w[0], w[1]);
}

// blockIdx.z: 0 = K (rotated), 1 = V.  A wave holds 64 / G whole rows.
template <typename T, int ST>
__global__ __launch_bounds__(256) void paged_write_kernel(const PagedWriteArgs a) {
  const int G = a.c.dh >> 4;  // 4, 8 or 16
  const int lane = threadIdx.x & 63;
  const int g = lane & (G - 1);
  const int R = 64 / G;  // rows of a wave
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * R;
  if (row0 >= a.n_rows) return;
  const int64_t row = row0 + lane / G;
  // sequences of the wave's rows: that of the first one, and how many of the
  // next 64 begin at or before each other row
  const int s0 = seq_of_row(a.q, row0, lane);
  const int nx = s0 + 1 + lane <= a.q.n ? a.q.cu[s0 + 1 + lane] : INT32_MAX;
  int b = s0;
  for (int j = 0; j < R; ++j) {
    const int c = __popcll(__ballot((int64_t)nx <= row0 + j));
    if (lane / G == j) b = s0 + c;
  }
  if (b == s0 + 64)
    while (b < a.q.n && a.q.cu[b + 1] <= row) ++b;  // many empty sequences
  const bool is_k = blockIdx.z == 0;
  const int half = a.c.dh >> 1;
  bool live = row < a.n_rows && b >= 0 && b < a.q.n;
  int64_t tok = 0;
  int at = -1;
  if (live) {
    tok = (int64_t)a.q.len[b] - a.q.cu[b + 1] + row;
    at = page_row(a.c, a.q, b, tok);
    live = at >= 0;
  }
  const Rows& in = is_k ? a.k : a.v;
  const T* x = reinterpret_cast<const T*>(in.p) + row * in.rs + 8 * g;
  char* const out = is_k ? a.c.k : a.c.v;
  float* const scales = is_k ? a.c.k_scale : a.c.v_scale;
  const bool rot = is_k && a.rotate;
  constexpr bool Q = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  double cs[8], sn[8];
  if (rot && live) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pair = 8 * g + i;
      const double f = turn_of(a.pos ? a.pos[a.plan.axis[pair] * a.ps + row] : tok, a.plan.turns[pair]);
      if (Q) {
        sincospi(2.0 * f, &sn[i], &cs[i]);
      } else {
        float s1, c1;
        sincospif(2.f * (float)f, &s1, &c1);
        sn[i] = s1;
        cs[i] = c1;
      }
    }
  }
  const int h0 = blockIdx.y * a.heads_per, h1 = min(a.c.n_kv, h0 + a.heads_per);
  for (int h = h0; h < h1; ++h) {
    float u[8], w[8];
    const int64_t prow = (int64_t)at + ((int64_t)h << a.c.shift);
    if (live) {
      ld8(x + h * in.hs, u);
      ld8(x + h * in.hs + half, w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = w[i] = 0.f;
    }
    if (!Q) {
      if (rot && live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float c = (float)cs[i], s = (float)sn[i], p = u[i] * c - w[i] * s;
          w[i] = w[i] * c + u[i] * s;
          u[i] = p;
        }
      }
      if (live) {
        T* y = reinterpret_cast<T*>(out) + prow * a.c.dh + 8 * g;
        st8(y, u);
        st8(y + half, w);
      }
      continue;
    }
    double p[8], q[8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = u[i];
      q[i] = w[i];
      if (rot && live) {
        p[i] = (double)u[i] * cs[i] - (double)w[i] * sn[i];
        q[i] = (double)w[i] * cs[i] + (double)u[i] * sn[i];
      }
      amax = max(amax, max(__float_as_uint((float)p[i]) & 0x7fffffffu, __float_as_uint((float)q[i]) & 0x7fffffffu));
    }
    for (int o = 1; o < G; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
    if (live) {
      const float scale = row_scale<ST>(amax);
      char* y = out + prow * a.c.dh + 8 * g;
      *reinterpret_cast<uint2*>(y) = codes8<ST>(p, scale);
      *reinterpret_cast<uint2*>(y + half) = codes8<ST>(q, scale);
      if (g == 0) scales[prow] = scale;
    }
  }
}

// ---------------------------------------------------------------------------
// paged read
// ---------------------------------------------------------------------------
template <int ST>
RFX_DEV void decode8(const uint2& c, float scale, float* o) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (ST == REFLEX_STORE_INT8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[4 * i + j] = (float)(int)(int8_t)(w[i] >> (8 * j)) * scale;
    } else {
      o[4 * i] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 0) * scale;
      o[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1) * scale;
      o[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2) * scale;
      o[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3) * scale;
    }
  }
}

// blockIdx.z: 0 = K, 1 = V; blockIdx.y: the head.  Rows as in the writer.
template <typename T, int ST>
__global__ __launch_bounds__(256) void paged_read_kernel(const PagedReadArgs a) {
  const int G = a.c.dh >> 4;
  const int lane = threadIdx.x & 63;
  const int g = lane & (G - 1);
  const int R = 64 / G;
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * R;
  if (row0 >= a.n_rows) return;
  const int64_t row = row0 + lane / G;
  const int s0 = seq_of_row(a.q, row0, lane);
  const int nx = s0 + 1 + lane <= a.q.n ? a.q.cu[s0 + 1 + lane] : INT32_MAX;
  int b = s0;
  for (int j = 0; j < R; ++j) {
    const int c = __popcll(__ballot((int64_t)nx <= row0 + j));
    if (lane / G == j) b = s0 + c;
  }
  if (b == s0 + 64)
    while (b < a.q.n && a.q.cu[b + 1] <= row) ++b;
  if (row >= a.n_rows || b < 0 || b >= a.q.n) return;
  const int64_t tok = (int64_t)a.q.len[b] - a.q.cu[b + 1] + row;
  const int at = page_row(a.c, a.q, b, tok);
  const bool is_k = blockIdx.z == 0;
  const int half = a.c.dh >> 1, h = blockIdx.y;
  const Rows& dst = is_k ? a.k : a.v;
  T* y = reinterpret_cast<T*>(const_cast<char*>(dst.p)) + row * dst.rs + h * dst.hs + 8 * g;
  float u[8], w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = w[i] = 0.f;
  if (at >= 0) {
    const int64_t prow = (int64_t)at + ((int64_t)h << a.c.shift);
    const char* src = is_k ? a.c.k : a.c.v;
    if (ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8) {
      const float scale = (is_k ? a.c.k_scale : a.c.v_scale)[prow];
      const char* p = src + prow * a.c.dh + 8 * g;
      decode8<ST>(*reinterpret_cast<const uint2*>(p), scale, u);
      decode8<ST>(*reinterpret_cast<const uint2*>(p + half), scale, w);
    } else {
      const T* p = reinterpret_cast<const T*>(src) + prow * a.c.dh + 8 * g;
      ld8(p, u);
      ld8(p + half, w);
    }
  }
  st8(y, u);
  st8(y + half, w);
}

// Heads a thread goes over: all of them where the tokens alone fill the chip
// (256 CUs, 1024 threads each), fewer otherwise.
int pick_heads_per(int64_t threads_per_head, int heads) {
  const int64_t want = 256 * 1024;
  int64_t groups = (want + threads_per_head - 1) / threads_per_head;
  if (groups > heads) groups = heads;
  return (int)((heads + groups - 1) / groups);
}

}  // namespace

template <typename T>
hipError_t launch_rotary(const RotaryArgs& args, hipStream_t s) {
  RotaryArgs a = args;
  const int64_t threads = a.n_rows * (a.plan.head_dim >> 4);
  a.heads_per = pick_heads_per(threads, a.n_heads);
  const dim3 grid((unsigned)((threads + 255) / 256), (a.n_heads + a.heads_per - 1) / a.heads_per);
  RFX_LAUNCH(rotary_kernel<T>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template hipError_t launch_rotary<float>(const RotaryArgs&, hipStream_t);
template hipError_t launch_rotary<bf16_t>(const RotaryArgs&, hipStream_t);

template <typename T>
hipError_t launch_paged_write(const PagedWriteArgs& args, int store, hipStream_t s) {
  PagedWriteArgs a = args;
  const int G = a.c.dh >> 4;
  const int rows_per_block = 4 * (64 / G);
  a.heads_per = pick_heads_per(2 * a.n_rows * G, a.c.n_kv);
  const dim3 grid((unsigned)((a.n_rows + rows_per_block - 1) / rows_per_block),
                  (a.c.n_kv + a.heads_per - 1) / a.heads_per, 2);
  if (store == REFLEX_STORE_FP8)
    RFX_LAUNCH((paged_write_kernel<T, REFLEX_STORE_FP8>), grid, dim3(256), 0, s, a);
  else if (store == REFLEX_STORE_INT8)
    RFX_LAUNCH((paged_write_kernel<T, REFLEX_STORE_INT8>), grid, dim3(256), 0, s, a);
  else
    RFX_LAUNCH((paged_write_kernel<T, REFLEX_STORE_F32>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template hipError_t launch_paged_write<float>(const PagedWriteArgs&, int, hipStream_t);
template hipError_t launch_paged_write<bf16_t>(const PagedWriteArgs&, int, hipStream_t);

template <typename T>
hipError_t launch_paged_read(const PagedReadArgs& a, int store, hipStream_t s) {
  const int rows_per_block = 4 * (64 / (a.c.dh >> 4));
  const dim3 grid((unsigned)((a.n_rows + rows_per_block - 1) / rows_per_block), a.c.n_kv, 2);
  if (store == REFLEX_STORE_FP8)
    RFX_LAUNCH((paged_read_kernel<T, REFLEX_STORE_FP8>), grid, dim3(256), 0, s, a);
  else if (store == REFLEX_STORE_INT8)
    RFX_LAUNCH((paged_read_kernel<T, REFLEX_STORE_INT8>), grid, dim3(256), 0, s, a);
  else
    RFX_LAUNCH((paged_read_kernel<T, REFLEX_STORE_F32>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template hipError_t launch_paged_read<float>(const PagedReadArgs&, int, hipStream_t);
template hipError_t launch_paged_read<bf16_t>(const PagedReadArgs&, int, hipStream_t);

}  // namespace reflex
