// Rotary positions over several axes, and the paged cache's writer and reader.
//
// All three move rows of head_dim values once and are bound by that traffic.
// A thread holds 8 values of each half of a head (two 16-byte accesses in
// bf16), so it has both members of 8 rotary pairs, and head_dim / 16 threads
// make a row: its maximum is a few shuffles.  A thread goes over several heads
// of its token where there are enough tokens, because the angles' sines are
// the arithmetic of these kernels and belong to the token alone.
#include <type_traits>

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
RFX_DEV uint32_t pack2(float a, float b) {  // to nearest even, NaN kept
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;
  const bf16x2_v v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
RFX_DEV void st8(bf16_t* p, const float* v) {
  st16(p, make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])));
}

// Angle of a pair at a position, as a fraction of a turn in [-1/2, 1/2]: the
// product and its reduction in 64 bits, so far positions keep 2^-53 of the
// product (a position of 10^6 keeps the angle to 2e-10).
RFX_DEV double turn_of(double pos, double turns) {
  const double t = pos * turns;
  return t - rint(t);
}

// The turns of a thread's 8 pairs (8 g ..) at a row's positions; with no
// positions every axis counts the token.  All axes' positions are loaded at
// once, and the pair's one is selected.
RFX_DEV void turns_of(const reflex_rotary& plan, const int64_t* pos, int64_t ps, int64_t row, int64_t tok, int g,
                      double* f) {
  const double* const turns = plan.turns + 8 * g;
  const double first = (double)(pos ? pos[row] : tok);
  if (plan.n_axes == 1 || !pos) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = turn_of(first, turns[i]);
    return;
  }
  double p[REFLEX_MAX_AXES];
  p[0] = first;
#pragma unroll
  for (int a = 1; a < REFLEX_MAX_AXES; ++a) p[a] = (double)pos[(a < plan.n_axes ? a : 0) * ps + row];
  const uint64_t axes = *reinterpret_cast<const uint64_t*>(plan.axis + 8 * g);
  auto of = [&](int a) __attribute__((always_inline)) {
    const double lo = a & 1 ? p[1] : p[0], hi = a & 1 ? p[3] : p[2];
    return a & 2 ? hi : lo;
  };
  if (axes == (axes & 255) * 0x0101010101010101ull) {  // sections of whole eights
    const double q = of((int)axes & 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = turn_of(q, turns[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = turn_of(of((int)(axes >> (8 * i)) & 3), turns[i]);
  }
}

// Sine and cosine of a fraction of a turn in [-1/2, 1/2]: the
// nearest quarter turn is taken off, and the Taylor series of both functions
// (sine to x^15, cosine to x^14) hold the rest, |x| <= pi / 4, to 2^-49 of 1.
RFX_DEV void sincos_turn(double f, double* sn, double* cs) {
  const double q = rint(4.0 * f);
  const double x = fma(q, -0.25, f) * 6.283185307179586477;
  const double z = x * x;
  double s = -1.0 / 1307674368000.0;
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, x, x);
  double c = -1.0 / 87178291200.0;
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int n = (int)q;  // -2 .. 2
  const double a = n & 1 ? c : s, b = n & 1 ? s : c;
  auto flip = [](double v, int by) __attribute__((always_inline)) {  // bit 1 of `by` on the sign
    return __hiloint2double(__double2hiint(v) ^ ((by & 2) << 30), __double2loint(v));
  };
  *sn = flip(a, n);
  *cs = flip(b, n + 1);
}

// The same for values of type T, in fp32: rounded from 64 bits for fp32 values (a
// fraction rounded to fp32 first is off by 2^-26 of a turn, all of a small sine
// next to half a turn), from an fp32 fraction for bf16 ones.
template <typename T> RFX_DEV void sincos_for(double f, float* sn, float* cs) {
  if constexpr (sizeof(T) == 4) {
    double s, c;
    sincos_turn(f, &s, &c);
    *sn = (float)s;
    *cs = (float)c;
  } else {
    sincospif(2.f * (float)f, sn, cs);
  }
}

// ---------------------------------------------------------------------------
// rotary
// ---------------------------------------------------------------------------
// 24,576 rows of 8 heads of 256 in fp32 (403 MB read and written) take 87 us,
// 4.6 TB/s, where a large copy reaches 4.9-5.0; 768 rows in bf16 5 us and eight
// rows 4 us, the latency of positions, frequencies and rows.  (Products in 64
// bits too would leave only the result's rounding, 2.5e-8 of it instead of
// 3.3e-8, and take 5 % longer.)
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
  double f[8];
  turns_of(a.plan, a.pos, a.ps, row, 0, g, f);
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    sincos_for<T>(f[i], &sn[i], &cs[i]);
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

// The codes of 8 values as 8 bytes, from their fp32 form f and the values x
// themselves (a rotated key comes in 64 bits).  No border between codes can lie
// between x and f unless f is next to it: in int8 within 2^-14 of a half (the
// product's error is under 2^-15), in fp8 on it (borders have five significant
// bits).  Those few are decided from x.
template <int ST, typename F>
RFX_DEV uint2 codes8(const float* f, const F* x, float scale) {
  uint32_t w[2] = {0, 0};
  if (!(scale < INFINITY)) return make_uint2(0u, 0u);
  const float inv = 1.f / scale;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (ST == REFLEX_STORE_INT8) {
      int c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float t = f[4 * i + j] * inv;
        float r = rintf(t);
        if (fabsf(fabsf(t - r) - 0.5f) < 0x1p-14f) r = (float)rint((double)x[4 * i + j] / (double)scale);
        c[j] = (int)r;  // -127 .. 127: f is at most the row's maximum
      }
      w[i] = (uint32_t)(c[0] & 255) | (uint32_t)(c[1] & 255) << 8 | (uint32_t)(c[2] & 255) << 16 | (uint32_t)c[3] << 24;
    } else {
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] = f[4 * i + j];
        if (sizeof(F) == 8 && !(__float_as_uint(y[j]) & 0xffffu)) y[j] = odd_float((double)x[4 * i + j]);
        y[j] *= inv;  // a power of two
      }
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
    }
  }
  return make_uint2(w[0], w[1]);
}

// Token and page row (head 0) of row row0 + lane: -2 where the row belongs to
// no sequence, -1 where the token is absent.  Lanes past `rows` look at no
// table.  Up to 63 sequences lie in the lanes themselves, with one load; of
// more, the 64 after that of the wave's first row do.  A lane finds its own by
// halving over them.
RFX_DEV int rows_of_wave(const Pages& c, const Seqs& q, int64_t row0, int rows, int64_t n_rows, int lane, int64_t& tok) {
  const int64_t row = row0 + lane;
  const bool few = q.n < 64;
  const int first = few ? 0 : seq_of_row(q, row0, lane) + 1;
  const int v = first + lane <= q.n ? q.cu[first + lane] : INT32_MAX;
  const int ln = few && lane < q.n ? q.len[lane] : 0;
  int lo = 0;
#pragma unroll
  for (int step = 32; step > 0; step >>= 1)
    if ((int64_t)__shfl(v, lo + step - 1, 64) <= row) lo += step;
  lo += (int64_t)__shfl(v, lo, 64) <= row;
  int b = first + lo - 1;
  int len = __shfl(ln, max(b, 0), 64), end = __shfl(v, min(lo, 63), 64);
  tok = 0;
  if (!few && lo == 64)
    while (b < q.n && q.cu[b + 1] <= row) ++b;  // many empty sequences
  if (lane >= rows || row >= n_rows || b < 0 || b >= q.n) return -2;
  if (!few) {
    len = q.len[b];
    end = q.cu[b + 1];
  }
  tok = (int64_t)len - end + row;
  return page_row(c, q, b, tok);
}

// 8 elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<float> {
  uint4 a, b;
  RFX_DEV void load(const float* p) { a = ld16(p); b = ld16(p + 4); }
  RFX_DEV void to_f(float* o) const { frag_to_f(a, o, 0.f); frag_to_f(b, o + 4, 0.f); }
};
template <> struct Raw8<bf16_t> {
  uint4 a;
  RFX_DEV void load(const bf16_t* p) { a = ld16(p); }
  RFX_DEV void to_f(float* o) const { frag_to_f(a, o, bf16_t(0)); }
};

// blockIdx.z: 0 = K (rotated), 1 = V.  A wave takes 64 / G rows.  Bound by the
// vector unit where keys are rotated for an 8-bit store: 32 frames of 768 keys
// of 256 take 20 us with V, 8 us of them memory's.  Eight prompts with eight
// heads of 128 (44,000 rows) take 70 us into int8 pages (273 MB), 3.9 TB/s, and 76
// into bf16 ones (360 MB), 4.8 TB/s: the angles' sines are taken once for all
// heads.  (Measured slower: four times the rows a wave, 22 us and, with eight
// 128-wide heads, 89 against 78 us; K and V side by side in turn, 25 us.)
template <typename T, int ST>
__global__ __launch_bounds__(256) void paged_write_kernel(const PagedWriteArgs a) {
  const int G = a.c.dh >> 4;  // 4, 8 or 16
  const int lane = threadIdx.x & 63;
  const int g = lane & (G - 1), sub = lane / G;
  const int R = 64 / G;
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * R;
  if (row0 >= a.n_rows) return;
  const bool is_k = blockIdx.z == 0;
  const int half = a.c.dh >> 1;
  const Rows& in = is_k ? a.k : a.v;
  char* const out = is_k ? a.c.k : a.c.v;
  float* const scales = is_k ? a.c.k_scale : a.c.v_scale;
  const bool rot = is_k && a.rotate;
  constexpr bool Q = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  typedef typename std::conditional<Q, double, float>::type F;  // what a rotation is computed in
  const int h0 = blockIdx.y * a.heads_per, h1 = min(a.c.n_kv, h0 + a.heads_per);
  // the next head's values are always under way, the first ones while the rows'
  // places are looked up
  Raw8<T> nu, nw;
  const int64_t row = row0 + sub;
  const T* const x = reinterpret_cast<const T*>(in.p) + min(row, a.n_rows - 1) * in.rs + 8 * g;
  auto fetch = [&](int h) __attribute__((always_inline)) {
    nu.load(x + h * in.hs);
    nw.load(x + h * in.hs + half);
  };
  fetch(h0);
  int64_t wave_tok;
  const int wave_at = rows_of_wave(a.c, a.q, row0, R, a.n_rows, lane, wave_tok);
  const int at = __shfl(wave_at, sub, 64);
  const int64_t tok = (int64_t)__shfl((long long)wave_tok, sub, 64);
  const bool live = at >= 0;
  F cs[8], sn[8];
  if (rot && live) {
    double f[8];
    turns_of(a.plan, a.pos, a.ps, row, tok, g, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (Q) sincos_turn(f[i], &sn[i], &cs[i]);
      else sincos_for<T>(f[i], &sn[i], &cs[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = sn[i] = F(0);
  }
  for (int h = h0; h < h1; ++h) {
    float u[8], w[8];
    const int64_t prow = (int64_t)at + ((int64_t)h << a.c.shift);
    nu.to_f(u);
    nw.to_f(w);
    if (h + 1 < h1) fetch(h + 1);
    auto put = [&](const auto* p, const auto* q) __attribute__((always_inline)) {
      uint32_t amax = 0;
      float fp[8], fq[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        fp[i] = (float)p[i];
        fq[i] = (float)q[i];
        amax = max(amax, max(__float_as_uint(fp[i]) & 0x7fffffffu, __float_as_uint(fq[i]) & 0x7fffffffu));
      }
      for (int o = 1; o < G; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
      if (live) {
        const float scale = row_scale<ST>(amax);
        char* y = out + prow * a.c.dh + 8 * g;
        *reinterpret_cast<uint2*>(y) = codes8<ST>(fp, p, scale);
        *reinterpret_cast<uint2*>(y + half) = codes8<ST>(fq, q, scale);
        if (g == 0) scales[prow] = scale;
      }
    };
    if (rot) {
      F p[8], q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = (F)u[i] * cs[i] - (F)w[i] * sn[i];
        q[i] = (F)w[i] * cs[i] + (F)u[i] * sn[i];
      }
      if constexpr (Q) {
        put(p, q);
        continue;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] = p[i];
          w[i] = q[i];
        }
      }
    }
    if constexpr (Q) {
      put(u, w);
    } else if (live) {
      T* y = reinterpret_cast<T*>(out) + prow * a.c.dh + 8 * g;
      st8(y, u);
      st8(y + half, w);
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
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      o[4 * i] = a[0] * scale;
      o[4 * i + 1] = a[1] * scale;
      o[4 * i + 2] = b[0] * scale;
      o[4 * i + 3] = b[1] * scale;
    }
  }
}

// blockIdx.z: 0 = K, 1 = V; blockIdx.y: the head.  A wave takes U times 64 / G
// rows, whose loads are all under way before the first is used.  The same prompts
// 50 us from int8 pages, 5.4 TB/s; 69 from bf16 and 171 from fp32 ones, 5.2 and 4.2.
template <typename T, int ST, int U>
__global__ __launch_bounds__(256) void paged_read_kernel(const PagedReadArgs a) {
  constexpr bool Q = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  const int G = a.c.dh >> 4;
  const int lane = threadIdx.x & 63;
  const int g = lane & (G - 1), sub = lane / G;
  const int R = 64 / G;
  const int64_t row0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (R * U);
  if (row0 >= a.n_rows) return;
  int64_t tok;
  const int wave_at = rows_of_wave(a.c, a.q, row0, R * U, a.n_rows, lane, tok);
  const bool is_k = blockIdx.z == 0;
  const int half = a.c.dh >> 1, h = blockIdx.y;
  const Rows& dst = is_k ? a.k : a.v;
  const char* src = is_k ? a.c.k : a.c.v;
  const float* scales = is_k ? a.c.k_scale : a.c.v_scale;
  int at[U];
  float u[U][8], w[U][8], scale[U];
  uint2 c[U][2];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    at[i] = __shfl(wave_at, i * R + sub, 64);
    // (an absent row loads what its first head's page begins with)
    const int64_t prow = (int64_t)max(at[i], 0) + ((int64_t)h << a.c.shift);
    if (Q) {
      scale[i] = scales[prow];
      const char* p = src + prow * a.c.dh + 8 * g;
      c[i][0] = *reinterpret_cast<const uint2*>(p);
      c[i][1] = *reinterpret_cast<const uint2*>(p + half);
    } else {
      const T* p = reinterpret_cast<const T*>(src) + prow * a.c.dh + 8 * g;
      ld8(p, u[i]);
      ld8(p + half, w[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (at[i] == -2) continue;  // of no sequence
    if (Q) {
      decode8<ST>(c[i][0], scale[i], u[i]);
      decode8<ST>(c[i][1], scale[i], w[i]);
    }
    if (at[i] < 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) u[i][e] = w[i][e] = 0.f;
    }
    const int64_t row = row0 + i * R + sub;
    T* y = reinterpret_cast<T*>(const_cast<char*>(dst.p)) + row * dst.rs + h * dst.hs + 8 * g;
    st8(y, u[i]);
    st8(y + half, w[i]);
  }
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

// Rows of a wave, in units of 64 / G: four where that leaves two waves to a
// SIMD (looking up the rows' places is a third of a single unit's work).
int pick_unroll(int64_t threads) { return threads >= 4 * 2 * 1024 * 64 ? 4 : 1; }

template <typename T>
hipError_t launch_paged_write(const PagedWriteArgs& args, int store, hipStream_t s) {
  PagedWriteArgs a = args;
  const int G = a.c.dh >> 4;
  a.heads_per = pick_heads_per(2 * a.n_rows * G, a.c.n_kv);
  const unsigned heads = (a.c.n_kv + a.heads_per - 1) / a.heads_per;
  const int rows_per_block = 4 * (64 / G);
  const unsigned blocks = (unsigned)((a.n_rows + rows_per_block - 1) / rows_per_block);
  const dim3 grid(blocks, heads, 2);
  auto go = [&](auto S) {
    RFX_LAUNCH((paged_write_kernel<T, decltype(S)::value>), grid, dim3(256), 0, s, a);
  };
  if (store == REFLEX_STORE_FP8) go(std::integral_constant<int, REFLEX_STORE_FP8>{});
  else if (store == REFLEX_STORE_INT8) go(std::integral_constant<int, REFLEX_STORE_INT8>{});
  else go(std::integral_constant<int, REFLEX_STORE_F32>{});  // (the inputs' own type)
  return hipGetLastError();
}
template hipError_t launch_paged_write<float>(const PagedWriteArgs&, int, hipStream_t);
template hipError_t launch_paged_write<bf16_t>(const PagedWriteArgs&, int, hipStream_t);

template <typename T>
hipError_t launch_paged_read(const PagedReadArgs& a, int store, hipStream_t s) {
  const int G = a.c.dh >> 4;
  const int U = pick_unroll(2 * a.n_rows * G * a.c.n_kv);
  const int rows_per_block = 4 * (64 / G) * U;
  const dim3 grid((unsigned)((a.n_rows + rows_per_block - 1) / rows_per_block), a.c.n_kv, 2);
  auto go = [&](auto S) {
    constexpr int ST = decltype(S)::value;
    if (U == 4)
      RFX_LAUNCH((paged_read_kernel<T, ST, 4>), grid, dim3(256), 0, s, a);
    else
      RFX_LAUNCH((paged_read_kernel<T, ST, 1>), grid, dim3(256), 0, s, a);
  };
  if (store == REFLEX_STORE_FP8) go(std::integral_constant<int, REFLEX_STORE_FP8>{});
  else if (store == REFLEX_STORE_INT8) go(std::integral_constant<int, REFLEX_STORE_INT8>{});
  else go(std::integral_constant<int, REFLEX_STORE_F32>{});
  return hipGetLastError();
}
template hipError_t launch_paged_read<float>(const PagedReadArgs&, int, hipStream_t);
template hipError_t launch_paged_read<bf16_t>(const PagedReadArgs&, int, hipStream_t);

}  // namespace reflex
