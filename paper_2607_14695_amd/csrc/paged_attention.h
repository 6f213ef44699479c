// Attention of a chunk of new tokens over a paged cache: softmax(scale q k^T) v
// over the present keys that a row sees, in one pass over the keys with a
// running maximum m and sum l (an earlier tile's results are scaled by
// 2^(m_old - m_new) when the maximum is raised).
//
// Two kernels.  The few-row one (one workgroup per 16 or 32 rows) is bound by
// reading the cache; the many-row one (128 rows, bf16) by the matrix products
// and the softmax.  Keys are split over workgroups where rows are few; a merge
// kernel joins the splits in fp32, always in the same order.
//
// MODE says what a row sees and what is kept beside its result: kPlain a run of
// keys, kTree the cached tokens and those of the call's rows whose bits are set,
// kWeigh a run of keys, with every row's maximum and sum written for the sums of
// its probabilities, kKept (few rows) its scores too.  Each mode is compiled in a file of its own.
#pragma once

#include <algorithm>
#include <type_traits>

#include "paged.h"

namespace reflex {

namespace {

constexpr int kPlain = 0, kTree = 1, kWeigh = 2, kKept = 3;

// Running maxima start here instead of at -infinity, so that a row that sees
// nothing has exp2(-infinity - m) = 0 and not NaN.
constexpr float kFloor = -3.0e38f;

// The running maximum of a row is raised only when a score exceeds it by 2^8:
// probabilities then stay below 2^8, and the output is rescaled in few tiles.
constexpr float kSlack = 8.f;

// what a copy into LDS reads in place of a row that is not there
__device__ const uint4 kZeros[1] = {};

// Keys that a query at token `pos` of a sequence of `len` sees: [lo, hi).
struct Span { int lo, hi; };
RFX_DEV Span span_of(const PagedAttnArgs& a, int pos, int len) {
  Span s;
  const int64_t cap = (int64_t)a.q.max_pages << a.c.shift;
  s.hi = (int)min((int64_t)(a.causal ? min(pos, len - 1) + 1 : len), cap);
  s.lo = a.window > 0 ? (int)max((int64_t)0, (int64_t)pos - a.window + 1) : 0;
  return s;
}

// The keys of split `split` of a tile that sees [lo, hi): equal runs of whole
// 128s, so that a window, a causal mask or a short sequence leaves no split
// without work before the others are down to 128.  (64 single tokens with a
// window of 1,024 over 15,409 keys took 29 us, where equal runs of the longest
// sequence took 42; now 26.)
RFX_DEV Span split_of(const PagedAttnArgs& a, int lo, int hi, int split) {
  const int from = lo & ~127;
  const int per = (max(hi - from, 1) + 128 * a.nsplit - 1) / (128 * a.nsplit) * 128;
  Span s;
  s.lo = max(lo, from + split * per);
  s.hi = min(hi, from + (split + 1) * per);
  return s;
}

// kTree: the keys that packed row `row` sees among the 64 from key0 on, as bits;
// its sequence's first row is token `first`.
RFX_DEV uint64_t tree_bits(const PagedAttnArgs& a, int64_t row, int key0, int first) {
  const uint64_t* const m = a.tree + row * a.tree_words;
  const int d = key0 - first;
  if (d <= -64) return ~0ull;
  if (d < 0) return (~0ull >> (64 + d)) | (m[0] << -d);
  const int w = d >> 6, s = d & 63;
  uint64_t x = w < a.tree_words ? m[w] >> s : 0;
  if (s && w + 1 < a.tree_words) x |= m[w + 1] << (64 - s);
  return x;
}

template <int ST> RFX_DEV float code_to_f32(uint32_t c) {
  return ST == REFLEX_STORE_FP8 ? __builtin_amdgcn_cvt_f32_fp8((int)c, 0) : (float)(int8_t)c;
}

// Element `at` of the pages as fp32, without its row's scale.
template <typename T, int ST> RFX_DEV float page_elem(const char* p, int64_t at) {
  if constexpr (ST == REFLEX_STORE_FP8) return code_to_f32<ST>(reinterpret_cast<const uint8_t*>(p)[at]);
  else return to_f(reinterpret_cast<const T*>(p)[at]);
}

// One (row, query head) by one wave, key by key, which reads nothing but what
// the row sees; each lane holds DH / 64 dims.  Four keys' loads are under way at
// a time.
template <int MODE, typename T, int ST, int DH>
RFX_DEV void scalar_row(const PagedAttnArgs& a, int64_t row, int head, int b, int first, Span sp, float& m, float& l,
                        float* o) {
  constexpr int N = DH / 64, U = 4;
  const int lane = threadIdx.x & 63;
  const T* qp = reinterpret_cast<const T*>(a.x.p) + row * a.x.rs + head * a.x.hs + lane * N;
  float q[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = to_f(qp[i]) * a.factor;
    o[i] = 0.f;
  }
  m = kFloor;
  l = 0.f;
  const int64_t hoff = (int64_t)(head / a.group) << a.c.shift;
  for (int j = sp.lo; j < sp.hi; j += U) {
    int r[U];
    float k[U][N], v[U][N], ks[U], vs[U];
#pragma unroll
    for (int u = 0; u < U; ++u) r[u] = j + u < sp.hi ? page_row(a.c, a.q, b, j + u) : -1;
    if constexpr (MODE == kTree) {
      const uint64_t bits = tree_bits(a, row, j, first);
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = (bits >> u) & 1 ? r[u] : -1;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t pr = max(r[u], 0) + hoff;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        k[u][i] = page_elem<T, ST>(a.c.k, pr * DH + lane * N + i);
        v[u][i] = page_elem<T, ST>(a.c.v, pr * DH + lane * N + i);
      }
      ks[u] = ST == REFLEX_STORE_FP8 ? a.c.k_scale[pr] : 1.f;
      vs[u] = ST == REFLEX_STORE_FP8 ? a.c.v_scale[pr] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (r[u] < 0) continue;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) s += q[i] * k[u][i];
      s = warp_sum(s) * a.scale2 * ks[u];
      const float m2 = fmaxf(m, s);
      const float c = exp2f(m - m2), p = exp2f(s - m2);
      m = m2;
      l = l * c + p;
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = o[i] * c + p * vs[u] * v[u][i];
    }
  }
}

// Whether one of the present keys [lo, hi) has an infinity or a NaN among its
// values (in fp8 a NaN among its codes).
template <typename T, int ST, int DH>
RFX_DEV bool values_not_finite(const PagedAttnArgs& a, int head, int b, int lo, int hi) {
  constexpr int N = DH / 64;
  const int lane = threadIdx.x & 63;
  const int64_t hoff = (int64_t)(head / a.group) << a.c.shift;
  for (int j = lo; j < hi; ++j) {
    const int r = page_row(a.c, a.q, b, j);
    if (r < 0) continue;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N; ++i)
      odd |= !(fabsf(page_elem<T, ST>(a.c.v, (r + hoff) * DH + lane * N + i)) < INFINITY);
    if (__ballot(odd)) return true;
  }
  return false;
}

// out[row][head] = o / l; each lane holds DH / 64 dims.
template <typename T, int DH>
RFX_DEV void store_row(const PagedAttnArgs& a, int64_t row, int head, float l, const float* o) {
  constexpr int N = DH / 64;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = reinterpret_cast<T*>(const_cast<char*>(a.o.p)) + row * a.o.rs + head * a.o.hs + (threadIdx.x & 63) * N;
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = from_f<T>(o[i] * inv);
}

// ---------------------------------------------------------------------------
// shared pieces of the tiled kernels
// ---------------------------------------------------------------------------
// N copies as lds_dma16's from a wave-uniform base, each 1 KB further than the
// one before on both sides: one run of bytes
template <int N> RFX_DEV void lds_dma16_run(const void* base, const uint32_t (&off)[N], void* lds) {
  static_assert(N == 1 || N == 2 || N == 4, "up to four copies");
  const unsigned m0 = (unsigned)(size_t)lds;
  if constexpr (N == 1) {
    lds_dma16(base, off[0], lds);
  } else if constexpr (N == 2) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %2\n\t"
                 "global_load_lds_dwordx4 %1, %2 offset:1024"
                 :: "v"(off[0]), "v"(off[1]), "s"(base), "s"(m0) : "memory");
  } else {
    asm volatile("s_mov_b32 m0, %5\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %0, %4\n\t"
                 "global_load_lds_dwordx4 %1, %4 offset:1024\n\tglobal_load_lds_dwordx4 %2, %4 offset:2048\n\t"
                 "global_load_lds_dwordx4 %3, %4 offset:%6"
                 :: "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base), "s"(m0), "n"(3 * 1024) : "memory");
  }
}

template <int N, typename F> RFX_DEV void static_for(F&& f) {
  if constexpr (N > 0) {
    static_for<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// all but this wave's newest N copies have landed
template <int N> RFX_DEV void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// A store of 16 bytes per lane that the counts of wait_copies may include: all
// lanes' and one instruction, at its place.  (Stores are counted with the loads,
// in order.  The last of the four wait states before its data may be written
// again is taken here.)
RFX_DEV void store_counted(float* p, const f32x4_v& v) {
  asm volatile("global_store_dwordx4 %0, %1, off\n\ts_nop 3" :: "v"(p), "v"(v) : "memory");
}
// LDS reads issued so far have their values: what they read may be overwritten
RFX_DEV void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// 4 bytes per lane from global memory into LDS (as lds_dma16)
RFX_DEV void lds_dma4(const void* g, void* lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off"
               :: "v"(g), "s"((unsigned)(size_t)lds) : "memory");
}

// A lane's value combined with those of the lanes 16 and 32 further (mod 64),
// by the two row swaps of the vector unit.
template <typename F> RFX_DEV float across_rows(float x, F f) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
RFX_DEV float max2(float a, float b) { return fmaxf(a, b); }
RFX_DEV float add2(float a, float b) { return a + b; }

typedef __attribute__((ext_vector_type(4))) short s16x4_v;
typedef __attribute__((ext_vector_type(2))) int i32x2_v;
#define RFX_LDS __attribute__((address_space(3)))
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_v;

// 8 bytes per lane read so that each lane gets one column: of every 16 lanes,
// four rows of 16 two-byte elements (lane i gives the address of elements
// 4 (i % 4) .. of row i / 4), or eight rows of 16 one-byte elements (lane i:
// elements 8 (i % 2) .. of row i / 2); lane i gets column i.
RFX_DEV uint2 ld_tr16(const unsigned char* lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((RFX_LDS s16x4_v*)lds));
}
RFX_DEV uint2 ld_tr8(const unsigned char* lds) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((RFX_LDS i32x2_v*)lds));
}

// n fragments times a power of two or its negative, mostly 1
template <int N, typename T> RFX_DEV void scale_frags(uint4 (&v)[N], float factor, T) {
  if (factor == 1.f) return;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    float x[ElemT<T>::kPerFrag];
    frag_to_f(v[k], x, T(0));
#pragma unroll
    for (int i = 0; i < ElemT<T>::kPerFrag; ++i) x[i] *= factor;
    v[k] = f_to_frag(x, T(0));
  }
}

RFX_DEV uint32_t pack_bf16(float a, float b) {
  bf16x2_v v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// what the packed roundings of a and b left of them, rounded itself
RFX_DEV uint32_t rest_bf16(float a, float b, uint32_t w) {
  return pack_bf16(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
}

// 8 codes -> 8 bf16 (exact: codes have at most 7 significant bits and a sign)
template <int ST> RFX_DEV uint4 codes_to_bf16(uint2 c) {
  uint32_t w[4];
  if (ST == REFLEX_STORE_FP8) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, 1.f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, 1.f, true));
  } else {
    const uint32_t u[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int v = (int)u[i];
      w[2 * i] = pack_bf16((float)(int8_t)v, (float)(int8_t)(v >> 8));
      w[2 * i + 1] = pack_bf16((float)(int8_t)(v >> 16), (float)(v >> 24));
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// codes -> fp32
template <int ST> RFX_DEV uint4 codes_to_f32(uint32_t c) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = code_to_f32<ST>(c >> (8 * i) & 255);
  return f_to_frag(f, 0.f);
}

// The tile of a workgroup: rows r0 .. of sequence b, where a sequence's rows
// are its tokens in turn with the query heads of one K/V head within (row =
// token * group + head), BM rows a tile; tiles are numbered over the sequences
// in order.  Every wave finds it by itself: 64 sequences per step, a sum over
// the lanes.
struct Tile { int b, r0, rows, len, first_pos; int64_t first_row; };
RFX_DEV bool find_tile(const PagedAttnArgs& a, int tile, int bm, int lane, Tile& t) {
  int before = 0;
  for (int b0 = 0; b0 < a.q.n; b0 += 64) {
    const int b = b0 + lane;
    int c0 = 0, c1 = 0, end = 0, len = 0;
    if (b < a.q.n) {
      c0 = (int)min((int64_t)max(a.q.cu[b], 0), a.n_rows);
      end = a.q.cu[b + 1];
      c1 = (int)min((int64_t)max(end, 0), a.n_rows);
      len = a.q.len[b];
    }
    const int mine = c1 > c0 ? ((c1 - c0) * a.group + bm - 1) / bm : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    const uint64_t past = __ballot(before + sum > tile);
    if (past) {
      const int src = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
      t.b = b0 + src;
      t.r0 = (tile - before - (__shfl(sum, src, 64) - __shfl(mine, src, 64))) * bm;
      const int f0 = __shfl(c0, src, 64), f1 = __shfl(c1, src, 64);
      t.b = __builtin_amdgcn_readfirstlane(t.b);
      t.r0 = __builtin_amdgcn_readfirstlane(t.r0);
      t.first_row = __builtin_amdgcn_readfirstlane(f0);
      t.rows = __builtin_amdgcn_readfirstlane((f1 - f0) * a.group);
      t.len = __builtin_amdgcn_readfirstlane(__shfl(len, src, 64));
      t.first_pos = __builtin_amdgcn_readfirstlane((int)((int64_t)t.len - __shfl(end, src, 64) + f0));
      return true;
    }
    before += __shfl(sum, 63, 64);
  }
  return false;
}


// How many such tiles the batch has: at most tile_bound.
RFX_DEV int count_tiles(const PagedAttnArgs& a, int bm, int lane) {
  int sum = 0;
  for (int b = lane; b < a.q.n; b += 64) {
    const int c0 = (int)min((int64_t)max(a.q.cu[b], 0), a.n_rows), c1 = (int)min((int64_t)max(a.q.cu[b + 1], 0), a.n_rows);
    sum += c1 > c0 ? ((c1 - c0) * a.group + bm - 1) / bm : 0;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  return __builtin_amdgcn_readfirstlane(sum);
}

// kTree: trees are small, and the sequences below them differ in length, so tiles
// are not split alike: the batch's work (tiles x keys) is divided by the number of
// workgroups that the chip holds, and every tile has as many splits, alike ones, as
// that many keys to a split ask for.  32 ragged trees of 26 to 64 rows of 8 heads
// of 256 over 3,344 to 15,409 fp8 keys take 228 us in a row of calls, with their
// merge (530 TFLOP/s; by the profiler, which leaves pauses between the calls, 241
// and 9); with two splits each they took 327 against 234, the longest ones' time.
//
// A unit is a tile's split; units are numbered over the sequences, in each over
// the splits and in these over the tiles, which share the split's keys.
struct Units { int per, total; };  // keys of a split, units of a K/V head
struct UnitSeq { int c0, c1, end, len, tiles, keys; };
RFX_DEV UnitSeq unit_seq(const PagedAttnArgs& a, int b, int bm) {
  UnitSeq s{0, 0, 0, 0, 0, 0};
  if (b < a.q.n) {
    s.c0 = (int)min((int64_t)max(a.q.cu[b], 0), a.n_rows);
    s.end = a.q.cu[b + 1];
    s.c1 = (int)min((int64_t)max(s.end, 0), a.n_rows);
    s.len = a.q.len[b];
    s.tiles = s.c1 > s.c0 ? ((s.c1 - s.c0) * a.group + bm - 1) / bm : 0;
    s.keys = max(min(s.len, a.q.max_pages << a.c.shift), 1);  // (a table holds 2^30 tokens at most)
  }
  return s;
}
RFX_DEV int lanes_sum(int x) { return __builtin_amdgcn_readlane(lanes_up_to(x), 63); }
RFX_DEV Units count_units(const PagedAttnArgs& a, int bm, int lane, const UnitSeq& first) {
  if (a.nsplit == 1) {
    Units u{1 << 30, 0};
    for (int b0 = 0; b0 < a.q.n; b0 += 64) u.total += lanes_sum((b0 ? unit_seq(a, b0 + lane, bm) : first).tiles);
    return u;
  }
  // in units of 128 keys, of which 2^23 rows in tiles of 16 over 2^30 keys make less than 2^43
  int64_t work = 0;
  int longest = 0;
  for (int b0 = 0; b0 < a.q.n; b0 += 64) {
    const UnitSeq s = b0 ? unit_seq(a, b0 + lane, bm) : first;
    const int k = (s.keys + 127) >> 7;
    const int64_t x = (int64_t)s.tiles * k;
    work += (int64_t)lanes_sum((int)(x & 0xfffff)) + ((int64_t)lanes_sum((int)(x >> 20)) << 20);
    int m = s.tiles ? k : 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = max(m, __shfl_xor(m, o, 64));
    longest = max(longest, __builtin_amdgcn_readfirstlane(m));
  }
  // keys of a split in 128s, at first
  auto rounded_up = [](int64_t x, int d) __attribute__((always_inline)) {
    if (x < 1 << 22) return (int64_t)divided((int)x + d - 1, d, __builtin_amdgcn_rcpf((float)d));
    return (x + d - 1) / d;
  };
  int64_t per = max(max(rounded_up(work, a.units), rounded_up(longest, a.nsplit)), (int64_t)1);
  Units u;
  // (each tile's last split may be short: once more with what there then are too many)
  for (int turn = 0;; ++turn) {
    u.per = __builtin_amdgcn_readfirstlane((int)min(per * 128, (int64_t)1 << 30));
    u.total = 0;
    const float inv = __builtin_amdgcn_rcpf((float)u.per);
    for (int b0 = 0; b0 < a.q.n; b0 += 64) {
      const UnitSeq s = b0 ? unit_seq(a, b0 + lane, bm) : first;
      u.total += lanes_sum(s.tiles * (s.tiles ? divided(s.keys - 1, u.per, inv) + 1 : 0));
    }
    if (turn == 2 || u.total <= a.units || per >= longest) return u;
    per = max(per + 1, rounded_up(per * u.total, a.units));
  }
}
// `splits`: how many the tile has; `part`: the unit's keys, of those that any row may see.
RFX_DEV bool find_unit(const PagedAttnArgs& a, int unit, int bm, int lane, const UnitSeq& first, int per, Tile& t,
                       int& split, int& splits, Span& part) {
  int before = 0;
  const float inv = __builtin_amdgcn_rcpf((float)per);
  for (int b0 = 0; b0 < a.q.n; b0 += 64) {
    const UnitSeq s = b0 ? unit_seq(a, b0 + lane, bm) : first;
    const int ns = s.tiles ? divided(s.keys - 1, per, inv) + 1 : 0, mine = s.tiles * ns, sum = lanes_up_to(mine);
    const uint64_t past = __ballot(before + sum > unit);
    if (past) {
      const int src = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)past) - 1);
      auto of = [&](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, src); };
      const int local = unit - before - (of(sum) - of(mine)), tiles = of(s.tiles);
      split = __builtin_amdgcn_readfirstlane(divided(local, tiles, __builtin_amdgcn_rcpf((float)tiles)));
      splits = of(ns);
      const int keys = of(s.keys);
      const int alike = __builtin_amdgcn_readfirstlane(
          (divided(keys - 1, 128 * splits, __builtin_amdgcn_rcpf((float)(128 * splits))) + 1) * 128);
      part.lo = min(split * alike, keys);
      part.hi = min(part.lo + alike, keys);
      t.b = b0 + src;
      t.r0 = __builtin_amdgcn_readfirstlane((local - split * tiles) * bm);
      t.first_row = of(s.c0);
      t.rows = (of(s.c1) - of(s.c0)) * a.group;
      t.len = of(s.len);
      t.first_pos = (int)((int64_t)t.len - of(s.end) + of(s.c0));
      return true;
    }
    before += __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

// Row `q` of a tile done again where its result is not finite: key by key, which
// reads only what the row sees.  Needed where a key that this row does not see,
// but another row of the tile does, has a value that is not finite, which has met
// a probability of 0 in the matrix product; and with `halves`, probabilities
// taken as two bf16, of which the second, being 0 or of either sign, makes a NaN
// of an infinite value.  (Codes in fp8 are finite or NaN, in int8 finite; the
// scale of a value that the row does not see never meets its probability of 0.)
//
// All of it starts from the arguments (the kernel's first parameter lies at the
// start of the argument segment) and the tile's number, so that this rare path
// keeps nothing alive through the loops before it: what it needs held from there
// cost 29 spilled scalar registers and 5 to 8 % with many rows over fp8 pages.
// It is slow, a key at a time by one wave: 64 single tokens over 8,000 bf16 keys
// of which one has a NaN 1.1 ms instead of 0.11, two prompts of 8,192 rows whose
// last token has one 132 ms instead of 1.1.
template <int MODE, typename T, int ST, int DH>
RFX_DEV void redo_row(int tile, int bm, int q, int64_t row, int head, int split, bool halves, float& M, float& L,
                      float* y) {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  const PagedAttnArgs& a = *reinterpret_cast<const PagedAttnArgs*>(at);
  const int lane = threadIdx.x & 63;
  Tile t;
  Span part;
  if constexpr (MODE == kTree) {
    const UnitSeq first = unit_seq(a, lane, bm);
    const int per = count_units(a, bm, lane, first).per;
    int splits;
    if (!find_unit(a, tile, bm, lane, first, per, t, split, splits, part)) return;
  } else {
    if (!find_tile(a, tile, bm, lane, t)) return;
  }
  const int last = min(bm, t.rows - t.r0) - 1;
  const Span first_sees = span_of(a, t.first_pos + t.r0 / a.group, t.len);
  const Span last_sees = span_of(a, t.first_pos + (t.r0 + last) / a.group, t.len);
  if constexpr (MODE != kTree) part = split_of(a, first_sees.lo, last_sees.hi, split);
  Span sp = span_of(a, t.first_pos + (t.r0 + q) / a.group, t.len);
  sp.lo = max(sp.lo, part.lo);
  sp.hi = min(sp.hi, part.hi);
  // (in a tree the keys that the row does not see lie between those it does)
  if (MODE == kTree || (halves && ST != REFLEX_STORE_FP8) ||
      values_not_finite<T, ST, DH>(a, head, t.b, part.lo, min(sp.lo, part.hi)) ||
      values_not_finite<T, ST, DH>(a, head, t.b, max(sp.hi, part.lo), part.hi))
    scalar_row<MODE, T, ST, DH>(a, row, head, t.b, t.first_pos, sp, M, L, y);
}

// A row's result of one split: stored, or kept for the merge.  Where the sum is
// not finite a score that the row does see was not, and all of the row is NaN.
template <int MODE, typename T, int ST, int DH>
RFX_DEV void finish_row(const PagedAttnArgs& a, int tile, int bm, int q, int64_t row, int head, int split, bool halves,
                        float M, float L, float* y, int splits = 0) {
  constexpr int N = DH / 64;
  if constexpr (ST != REFLEX_STORE_INT8) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N; ++i) odd |= !(fabsf(y[i]) < INFINITY);
    if (__ballot(odd) && L < INFINITY) redo_row<MODE, T, ST, DH>(tile, bm, q, row, head, split, halves, M, L, y);
  }
  const int lane = threadIdx.x & 63;
  if (a.nsplit == 1) {
    store_row<T, DH>(a, row, head, L, y);
    if constexpr (MODE == kWeigh || MODE == kKept)
      if (lane == 0) a.stats[row * a.n_q + head] = make_float2(M, L == 0.f ? 0.f : 1.f / L);
    return;
  }
  const int64_t at = (row * a.n_q + head) * a.nsplit + split;
  if (lane == 0) a.part_ml[at] = make_float2(M, L);
  // (splits that the tile does not have)
  if (MODE == kTree && split == 0 && lane >= splits && lane < a.nsplit) a.part_ml[at + lane] = make_float2(kFloor, 0.f);
  if (L == 0.f) return;
  float* p = a.part_o + at * DH + lane * N;
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = y[i];
}

// ---------------------------------------------------------------------------
// few rows: one workgroup per 16 or 32 rows and key split
// ---------------------------------------------------------------------------
// Bound by reading the cache once.  Four waves hold the same query rows and
// take every fourth tile of KT keys, each on its own: the tile's K and V go
// straight from the pages into the wave's part of LDS (no barrier in the loop,
// only a wait on the wave's own copies), the next K tile is under way while
// the softmax and P.V run, the next V tile during the next scores.  Scores are
// formed transposed, S^T = K Q^T, so that a lane holds four keys of one query
// row: what the softmax leaves is in the right lanes to be the B operand of
// O^T = V^T P^T, with V^T taken from row-major V by transposing LDS reads.
// 8-bit codes become bf16 exactly on the way from LDS; the keys' scales enter
// the scores and the values' scales the probabilities, in fp32, so a code is
// never rounded.  The waves' results meet in LDS at the end.
//
// 64 single tokens, 8 query heads of 256 on one K/V head: over 15,409 fp8 keys
// at most (310 MB) 66 us, 4.7 TB/s; over 8,000 bf16 keys (525 MB) 102 us with the
// merge, 5.1 TB/s, and fp32 keys (1.05 GB) 194 us, 5.4 TB/s, as a large copy.  One
// token over 817 keys 9 us, a chain of latencies (lengths, table, K, V, the
// exchange).  fp32 with many rows is bound by its matrix products at one wave to
// a SIMD: four chunks of 1,000 rows over 2,000 keys, 8 heads of 128 on two K/V
// heads, 342 us, 72 TFLOP/s of the 154 that a large fp32 product reaches.
template <typename T, int ST, int DH>
struct FewCfg {
  static constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  static constexpr int ES = Q8 ? 1 : (int)sizeof(T);
  static constexpr int RB = DH * ES;                                          // bytes of a K or V row
  static constexpr int KT = RB >= 1024 ? 16 : RB >= 256 ? 32 : 64;            // keys of a tile
  static constexpr int NCH = RB / 16;                                         // 16-byte chunks of a row
  static constexpr int RPC = 64 / NCH;                                        // rows of a copy
  static constexpr int NI = KT * RB / 1024;                                   // copies of a tile
  static constexpr int TB = KT * RB;                                          // bytes of a tile
  static constexpr int SC = Q8 ? 2 * 64 * 4 : 0;                              // scales of a tile
  static constexpr int WAVE = 2 * TB + SC;                                    // LDS of a wave
  static constexpr int kTable = 1024;                                         // page table entries held in LDS
};

// workgroups that a CU holds where their LDS allows it
template <typename T, int ST, int DH, int MR>
constexpr int few_occupancy = MR == 1 && FewCfg<T, ST, DH>::WAVE <= 18 * 1024 ? 2 : 1;

template <int MODE, typename T, int ST, int DH, int MR>
__global__ __launch_bounds__(256, (few_occupancy<T, ST, DH, MR>)) void paged_attn_few_kernel(const PagedAttnArgs a) {
  typedef FewCfg<T, ST, DH> C;
  constexpr bool Q8 = C::Q8, BF = sizeof(T) == 2;
  constexpr int KT = C::KT, RB = C::RB, NCH = C::NCH, NI = C::NI;
  constexpr int NKB = KT / 16, NDB = DH / 16;
  constexpr int QS = BF ? 32 : 16;     // head dims of an MFMA step
  constexpr int NKS = DH / QS;
  constexpr int BM = 16 * MR;
  constexpr int OP = DH + 4;           // row pitch of the exchange, in floats
  constexpr int XB = 4 * BM * OP * 4;
  constexpr int MAIN = 4 * C::WAVE > XB ? 4 * C::WAVE : XB;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[MAIN];
  __shared__ int table[C::kTable];
  __shared__ float2 ml[4][BM];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int kvh = MODE == kTree ? blockIdx.y : blockIdx.y / a.nsplit;
  int split = MODE == kTree ? 0 : blockIdx.y - kvh * a.nsplit, splits = 0;
  Span part;
  Tile t;
  if constexpr (MODE == kTree) {
    const UnitSeq first = unit_seq(a, lane, BM);
    const int per = count_units(a, BM, lane, first).per;
    if (!find_unit(a, blockIdx.x, BM, lane, first, per, t, split, splits, part)) return;
  } else {
    if (!find_tile(a, blockIdx.x, BM, lane, t)) return;
  }

  // keys that any row of the tile sees, cut to this split
  const int rows_here = min(BM, t.rows - t.r0);
  const int p0 = t.first_pos + t.r0 / a.group, p1 = t.first_pos + (t.r0 + rows_here - 1) / a.group;
  const int lo_min = span_of(a, p0, t.len).lo, hi_max = span_of(a, p1, t.len).hi;
  const int lo_max = span_of(a, p1, t.len).lo;
  // (in a tree every row sees the cached tokens)
  const int hi_min = MODE == kTree ? min(t.first_pos, hi_max) : span_of(a, p0, t.len).hi;
  if constexpr (MODE == kTree) part.hi = min(part.hi, hi_max);
  else part = split_of(a, lo_min, hi_max, split);
  const int k_beg = part.lo, k_end = part.hi;

  // query rows: column c16 of block m
  int lo[MR], hi[MR];
  uint4 qf[MR][NKS];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    const int r = t.r0 + 16 * m + c16;
    const int tok = r / a.group;
    const Span sp = span_of(a, t.first_pos + tok, t.len);
    lo[m] = sp.lo;
    hi[m] = r < t.rows ? sp.hi : 0;
    const T* qp = reinterpret_cast<const T*>(a.x.p) + (t.first_row + tok) * a.x.rs +
                  (int64_t)(kvh * a.group + (r - tok * a.group)) * a.x.hs;
#pragma unroll
    for (int k = 0; k < NKS; ++k) {
      // a lane's contraction elements follow the K fragments: 16 bytes of a
      // row hold two bf16 steps of codes, or four fp32 steps
      int d;
      if (!Q8) d = QS * k + (QS / 4) * g;
      else if (BF) d = 64 * (k >> 1) + 16 * g + 8 * (k & 1);
      else d = 64 * (k >> 2) + 16 * g + 4 * (k & 3);
      qf[m][k] = r < t.rows ? ld16(qp + d) : zero16();
    }
    scale_frags(qf[m], a.factor, T(0));
    // (the compiler's own wait for the queries has to lie here: in the loop it would
    // be one for the copies and the counted stores too)
    if constexpr (MODE != kPlain) {
#pragma unroll
      for (int k = 0; k < NKS; ++k)
        asm volatile("" : "+v"(qf[m][k].x), "+v"(qf[m][k].y), "+v"(qf[m][k].z), "+v"(qf[m][k].w));
    }
  }
  float* score_row[MR];  // kKept: where a row's scores go; those of no row go behind the others, where none reads them
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    if constexpr (MODE == kKept) {
      const int r = t.r0 + 16 * m + c16, tok = r / a.group;
      const int64_t id = r < t.rows ? (t.first_row + tok) * a.n_q + kvh * a.group + (r - tok * a.group) : a.n_rows * a.n_q;
      score_row[m] = a.scores + id * a.score_pitch;
    }
  }
  f32x4_v o[MR][NDB];
  float mx[MR], sum[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    mx[m] = kFloor;
    sum[m] = 0.f;
#pragma unroll
    for (int d = 0; d < NDB; ++d) o[m][d] = f32x4_v{0.f, 0.f, 0.f, 0.f};
  }

  unsigned char* const kb = smem + wave * C::WAVE;
  unsigned char* const vb = kb + C::TB;
  float* const ksc = reinterpret_cast<float*>(vb + C::TB);
  float* const vsc = ksc + 64;
  const int64_t hoff = (int64_t)kvh << a.c.shift;
  auto swz = [](int row) __attribute__((always_inline)) { return (Q8 ? row : 2 * row) & (NCH - 1); };
  // copies after which the swizzle of a copy's rows repeats
  constexpr int NSW = (Q8 ? NCH : NCH / 2) / C::RPC < 1 ? 1 : (Q8 ? NCH : NCH / 2) / C::RPC;
  const int shift = a.c.shift, n_pages = a.c.n_pages, n_kv = a.c.n_kv;
  const char *const pk = a.c.k, *const pv = a.c.v;
  const float *const psk = a.c.k_scale, *const psv = a.c.v_scale;
  const float scale2 = a.scale2;
  const bool in_page = (1 << shift) >= C::RPC;  // the rows of a copy lie in one page
  // this lane's offset within copy j; the swizzle repeats after NO copies
  constexpr int NO = NI < 1 ? 1 : NI < NSW ? NI : NSW;
  uint32_t off[NO];
#pragma unroll
  for (int j = 0; j < NO; ++j) {
    const int sub = lane / NCH;  // (rows of 1 KB: a copy is a row)
    off[j] = sub * RB + (((lane % NCH) ^ swz(j * C::RPC + sub)) << 4);
  }

  for (int seg = k_beg & ~(KT - 1); seg < k_end;) {
    // the segment's table entries, checked once: -1 where the page is absent
    const int e0 = seg >> shift;
    const int seg_end = (int)min((int64_t)k_end, (int64_t)(e0 + C::kTable) << shift);
    const int ne = ((seg_end - 1) >> shift) - e0 + 1;
    __syncthreads();
    for (int i = threadIdx.x; i < ne; i += 256) {
      const int pg = a.q.table[(int64_t)t.b * a.q.max_pages + e0 + i];
      table[i] = (unsigned)pg < (unsigned)n_pages ? pg : -1;
    }
    __syncthreads();
    const int n_t = (seg_end - seg + KT - 1) / KT;

    // this lane's key of tile `x`: its page row, or -1 where no row of the tile
    // sees it: such values must not meet a probability of 0
    const int v_lo = max(k_beg, lo_min), v_hi = min(hi_max, seg_end);
    auto row_of = [&](int x) __attribute__((always_inline)) {
      const int key = seg + x * KT + lane;
      if (lane >= KT || key < v_lo || key >= v_hi) return -1;
      const int pg = table[(key >> shift) - e0];
      return pg < 0 ? -1 : ((pg * n_kv) << shift) + (key & ((1 << shift) - 1));
    };
    // Copy a tile's K or V; r: this lane's page row; zeros where it has none.
    // Mostly all rows are there and those of a copy lie in one page: then the
    // copy needs only a uniform base and the lane's offset.
    auto copy = [&](const char* base, const float* sc, int r, bool easy, unsigned char* dst, float* sdst)
        __attribute__((always_inline)) {
      if (easy) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
          lds_dma16(base + ((int64_t)__builtin_amdgcn_readlane(r, j * 64 / NCH) + hoff) * RB, off[j % NO], dst + j * 1024);
      } else {
#pragma unroll 4
        for (int j = 0; j < NI; ++j) {
          const int row = (j * 64 + lane) / NCH, ch = lane % NCH;
          const int pr = __shfl(r, row, 64);
          const char* src = base + ((int64_t)pr + hoff) * RB + ((ch ^ swz(row)) << 4);
          lds_dma16(pr < 0 ? reinterpret_cast<const char*>(kZeros) : src, dst + j * 1024);
        }
      }
      if (Q8) lds_dma4(sc + (int64_t)max(r, 0) + hoff, sdst);
    };
    constexpr uint64_t kAll = KT == 64 ? ~0ull : (1ull << KT) - 1;
    constexpr int NC = NI + (Q8 ? 1 : 0);
    // stores of a tile's scores, between the next K copies and the next V copies
    constexpr int NST = MODE == kKept ? MR * NKB : 0;
    static_assert(NC + NST < 64, "the counter's range");

    int r_cur = row_of(wave);
    if (wave < n_t) {
      const bool easy = in_page && __ballot(r_cur >= 0) == kAll;
      copy(pk, psk, r_cur, easy, kb, ksc);
      copy(pv, psv, r_cur, easy, vb, vsc);
    }
    for (int x = wave; x < n_t; x += 4) {
      const int r_next = row_of(x + 4);
      const bool more = x + 4 < n_t;
      const bool easy = in_page && __ballot(r_next >= 0) == kAll;
      const int key0 = seg + x * KT;
      const uint64_t present = __ballot(r_cur >= 0);
      if (NST > 0 && x != wave) wait_copies<NC + NST>();
      else wait_copies<NC>();
      // S^T: block kb holds keys 16 kb + 4 g + i of query row c16
      f32x4_v s[MR][NKB];
#pragma unroll
      for (int b = 0; b < NKB; ++b)
#pragma unroll
        for (int m = 0; m < MR; ++m) s[m][b] = f32x4_v{0.f, 0.f, 0.f, 0.f};
      auto k_read = [&](int b, int k) __attribute__((always_inline)) {
        const int row = 16 * b + c16;
        return ld16(kb + row * RB + (((4 * k + g) ^ swz(row)) << 4));
      };
      constexpr int NR = Q8 ? DH / 64 : NKS;  // reads of a row
      if constexpr (BF) {
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int k = 0; k < NR; ++k) {
            const uint4 c = k_read(b, k);
            if (!Q8) {
#pragma unroll
              for (int m = 0; m < MR; ++m) mfma_step(s[m][b], c, qf[m][k], T(0));
            } else {
              const uint4 f0 = codes_to_bf16<ST>(make_uint2(c.x, c.y)), f1 = codes_to_bf16<ST>(make_uint2(c.z, c.w));
#pragma unroll
              for (int m = 0; m < MR; ++m) {
                mfma_step(s[m][b], f0, qf[m][2 * k], T(0));
                mfma_step(s[m][b], f1, qf[m][2 * k + 1], T(0));
              }
            }
          }
      } else {
        // fp32 is bound by its products: the next group of reads is under way
        // while one is multiplied
        constexpr int RG = Q8 ? 1 : 4, NG = NKB * NR / RG;
        uint4 kf[2][RG];
        auto request = [&](int n) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < RG; ++i) kf[n & 1][i] = k_read((n * RG + i) / NR, (n * RG + i) % NR);
        };
        request(0);
#pragma unroll
        for (int n = 0; n < NG; ++n) {
          if (n + 1 < NG) request(n + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < RG; ++i) {
            const int b = (n * RG + i) / NR, k = (n * RG + i) % NR;
            const uint4 c = kf[n & 1][i];
            if (!Q8) {
#pragma unroll
              for (int m = 0; m < MR; ++m) mfma_step(s[m][b], c, qf[m][k], T(0));
            } else {
              const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint4 f = codes_to_f32<ST>(w[e]);
#pragma unroll
                for (int m = 0; m < MR; ++m) mfma_step(s[m][b], f, qf[m][4 * k + e], T(0));
              }
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      float4 ks[NKB];
#pragma unroll
      for (int b = 0; b < NKB; ++b) ks[b] = Q8 ? *reinterpret_cast<const float4*>(ksc + 16 * b + 4 * g) : make_float4(1.f, 1.f, 1.f, 1.f);
      wait_lds();
      if (more) copy(pk, psk, r_next, easy, kb, ksc);

      // softmax: scores in units of log2 e
      const bool whole = key0 >= max(lo_max, k_beg) && key0 + KT <= min(hi_min, k_end) && present == kAll;
      uint64_t bits[MR];
      if constexpr (MODE == kTree) {
        if (!whole) {
#pragma unroll
          for (int m = 0; m < MR; ++m) {
            const int r = min(t.r0 + 16 * m + c16, t.rows - 1);
            bits[m] = tree_bits(a, t.first_row + r / a.group, key0, t.first_pos);
          }
        }
      }
      // whether row m sees key `at` of the tile
      auto sees = [&](int m, int at) __attribute__((always_inline)) {
        const int key = key0 + at;
        return key >= max(lo[m], k_beg) && key < min(hi[m], seg_end) && ((present >> at) & 1) &&
               (MODE != kTree || ((bits[m] >> at) & 1));
      };
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        float top = kFloor;
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
          const float kk[4] = {ks[b].x, ks[b].y, ks[b].z, ks[b].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = s[m][b][i] * scale2;
            if (Q8) v *= kk[i];
            if (!whole) v = sees(m, 16 * b + 4 * g + i) ? v : -INFINITY;
            s[m][b][i] = v;
            top = fmaxf(top, v);
          }
          if constexpr (MODE == kKept) store_counted(score_row[m] + key0 + 16 * b + 4 * g, s[m][b]);
        }
        top = across_rows(top, max2);
        if (__ballot(top > mx[m] + kSlack)) {
          const float nm = top > mx[m] + kSlack ? top : mx[m];
          const float f = __builtin_amdgcn_exp2f(mx[m] - nm);
          mx[m] = nm;
          sum[m] *= f;
#pragma unroll
          for (int d = 0; d < NDB; ++d) o[m][d] *= f;
        }
        float add = 0.f;
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(s[m][b][i] - mx[m]);
            add += p;
            s[m][b][i] = p;
          }
        sum[m] += add;
      }

      if (more) wait_copies<NC + NST>();  // (the last tile has no newer copies under way)
      else wait_copies<NST>();
      if (Q8) {
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
          const float4 v4 = *reinterpret_cast<const float4*>(vsc + 16 * b + 4 * g);
          const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[m][b][i] *= vv[i];
        }
      }
      if (Q8 && !whole) {  // a key that the row does not see may have any scale
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
          for (int b = 0; b < NKB; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[m][b][i] = sees(m, 16 * b + 4 * g + i) ? s[m][b][i] : 0.f;
      }
      // O^T += V^T P^T
      if (BF) {
#pragma unroll
        for (int j = 0; j < KT / 32; ++j) {
          // The probabilities as two bf16 each, the second what the first's
          // rounding left: 16 bits of them.  The products this adds are hidden
          // by the cache's reads, and the result is then as exact as its own
          // rounding.
          uint4 pf[MR], pl[MR];
#pragma unroll
          for (int m = 0; m < MR; ++m) {
            const f32x4_v &u = s[m][2 * j], &w = s[m][2 * j + 1];
            pf[m] = make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]));
            pl[m] = make_uint4(rest_bf16(u[0], u[1], pf[m].x), rest_bf16(u[2], u[3], pf[m].y),
                               rest_bf16(w[0], w[1], pf[m].z), rest_bf16(w[2], w[3], pf[m].w));
          }
#pragma unroll
          for (int d = 0; d < NDB; ++d) {
            uint4 f;
            if (Q8) {
              const int rr = c16 >> 1, row = 32 * j + (rr < 4 ? 4 * g + rr : 12 + 4 * g + rr);
              f = codes_to_bf16<ST>(ld_tr8(vb + row * RB + ((d ^ swz(row)) << 4) + (c16 & 1) * 8));
            } else {
              const int row = 32 * j + 4 * g + (c16 >> 2), ch = 2 * d + ((c16 >> 1) & 1), sub = (c16 & 1) * 8;
              const uint2 f0 = ld_tr16(vb + row * RB + ((ch ^ swz(row)) << 4) + sub);
              const uint2 f1 = ld_tr16(vb + (row + 16) * RB + ((ch ^ swz(row + 16)) << 4) + sub);
              f = make_uint4(f0.x, f0.y, f1.x, f1.y);
            }
#pragma unroll
            for (int m = 0; m < MR; ++m) {
              mfma_step(o[m][d], f, pf[m], bf16_t(0));
              mfma_step(o[m][d], f, pl[m], bf16_t(0));
            }
          }
        }
      } else {
        // element (row 16 b + 4 g + e, column 16 d + c16): the swizzle of a row
        // does not depend on b, and is an XOR
        constexpr int SH = Q8 ? 4 : 6;  // 16 columns are one chunk of codes, four of fp32
        uint32_t base[4], vf[2][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int row = 4 * g + e;
          base[e] = row * RB + (Q8 ? (swz(row) << 4) + c16 : (((c16 >> 2) ^ swz(row)) << 4) + (c16 & 3) * 4);
        }
        auto request = [&](int n) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const unsigned char* at = vb + (base[e] ^ (n % NDB << SH)) + 16 * (n / NDB) * RB;
            vf[n & 1][e] = Q8 ? (uint32_t)*at : *reinterpret_cast<const uint32_t*>(at);
          }
        };
        request(0);
#pragma unroll
        for (int n = 0; n < NKB * NDB; ++n) {
          if (n + 1 < NKB * NDB) request(n + 1);
          __builtin_amdgcn_sched_barrier(0);
          const int b = n / NDB, d = n % NDB;
          float f[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) f[e] = Q8 ? code_to_f32<ST>(vf[n & 1][e]) : __uint_as_float(vf[n & 1][e]);
          const uint4 v = f_to_frag(f, 0.f);
#pragma unroll
          for (int m = 0; m < MR; ++m) {
            const float p[4] = {s[m][b][0], s[m][b][1], s[m][b][2], s[m][b][3]};
            mfma_step(o[m][d], v, f_to_frag(p, 0.f), 0.f);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      wait_lds();
      if (more) copy(pv, psv, r_next, easy, vb, vsc);
      r_cur = r_next;
    }
    seg = seg_end;
  }

  // join the four waves: rows of the tile over the waves, DH / 64 dims a lane
  __syncthreads();
  float* const ex = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    const float l = across_rows(sum[m], add2);
    const int q = 16 * m + c16;
    if (g == 0) ml[wave][q] = make_float2(mx[m], l);
#pragma unroll
    for (int d = 0; d < NDB; ++d)
      *reinterpret_cast<float4*>(ex + (wave * BM + q) * OP + 16 * d + 4 * g) =
          make_float4(o[m][d][0], o[m][d][1], o[m][d][2], o[m][d][3]);
  }
  __syncthreads();
  constexpr int N = DH / 64;
  if constexpr (MODE == kTree) {
    // (Four rows' reads at once: a tree of 16 rows of 8 heads of 256 over 833 keys 11.5
    // instead of 12.6 us; single weighed tokens, which have one or two rows a wave, no less.)
    for (int q0 = wave; q0 < rows_here; q0 += 16) {
      float M[4], L[4], y[4][N];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + 4 * u;
        M[u] = kFloor;
#pragma unroll
        for (int w = 0; w < 4; ++w) M[u] = fmaxf(M[u], ml[w][q].x);
        L[u] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) y[u][i] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = __builtin_amdgcn_exp2f(ml[w][q].x - M[u]);
          L[u] += ml[w][q].y * f;
#pragma unroll
          for (int i = 0; i < N; ++i) y[u][i] += f * ex[(w * BM + q) * OP + lane * N + i];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + 4 * u;
        if (q >= rows_here) break;
        const int r = t.r0 + q, tok = r / a.group, head = kvh * a.group + (r - tok * a.group);
        const int64_t row = t.first_row + tok;
        finish_row<MODE, T, ST, DH>(a, blockIdx.x, BM, q, row, head, split, BF, M[u], L[u], y[u], splits);
      }
    }
  } else {
    for (int q = wave; q < rows_here; q += 4) {
      float M = kFloor;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w][q].x);
      float L = 0.f, y[N];
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[w][q].x - M);
        L += ml[w][q].y * f;
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] += f * ex[(w * BM + q) * OP + lane * N + i];
      }
      const int r = t.r0 + q, tok = r / a.group, head = kvh * a.group + (r - tok * a.group);
      const int64_t row = t.first_row + tok;
      finish_row<MODE, T, ST, DH>(a, blockIdx.x, BM, q, row, head, split, BF, M, L, y, splits);
    }
  }
}

// ---------------------------------------------------------------------------
// many rows (bf16): one workgroup per 128 rows, K/V head and key split
// ---------------------------------------------------------------------------
// Bound by the matrix products.  Four waves hold 32 query rows each and share
// tiles of 64 keys, copied straight from the pages into two buffers of LDS.
// As in the few-row kernel scores are formed transposed and V is read through
// transposing LDS reads, so that probabilities stay in registers; here with
// the 32x32x16 product.  A wave forms the scores of tile t + 1 while it takes
// the softmax of tile t, so that its vector work runs under its matrix work;
// K of tile t + 2 and V of tile t + 1 are on their way meanwhile, with one
// barrier a tile.  The probabilities are rounded to bf16 once: two halves, as
// with few rows, double the second product and bring the error against 64 bits
// from 0.0023 to the 0.0017 of the result's own rounding (32 ragged trees over fp8
// keys 228 and 269 us, 8 trees of 95 to 128 rows of 32 heads of 128 over 8,192 bf16
// keys 160 and 203).
//
// Two prompts of 8,192 rows with 32 heads of 128, causal: 1.09-1.13 ms, 975-1,010
// TFLOP/s, matrix units busy for 54 % and vector issue for 56 % of the cycles:
// the two overlap little, although two waves share a SIMD.  One chunk of 768 rows
// with 8 heads of 256 over 15,408 keys: 121 us, 800 TFLOP/s, matrix units busy
// for 42 % and vector issue for 31 %; without softmax, copies and LDS reads the
// one wave of a SIMD took 96.  8-bit pages cost a conversion of every fragment
// in every wave: prompts 1.31 (fp8) and 1.63 ms (int8).
template <int ST, int DH>
struct ManyCfg {
  static constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  static constexpr int ES = Q8 ? 1 : 2;
  static constexpr int RB = DH * ES;
  static constexpr int KT = 64;
  static constexpr int NCH = RB / 16;
  static constexpr int RPC = 64 / NCH;           // rows of a copy
  static constexpr int TB = KT * RB;
  static constexpr int NI = TB / 1024 / 4;       // copies of a wave and tile (K or V)
  static constexpr int XB = 128 * (DH + 4) * 4;  // the exchange at the end
  static constexpr int SMEM = 4 * TB > XB ? 4 * TB : XB;
  static constexpr int kTable = 1024;
};

template <int MODE, int ST, int DH>
__global__ __launch_bounds__(256, DH <= 128 ? 2 : 1) void paged_attn_many_kernel(const PagedAttnArgs a, int grid_tiles) {
  typedef ManyCfg<ST, DH> C;
  typedef bf16_t T;
  constexpr bool Q8 = C::Q8;
  constexpr int KT = C::KT, RB = C::RB, NCH = C::NCH, NI = C::NI, RPC = C::RPC, TB = C::TB;
  constexpr int NKS = DH / 16, NDB = DH / 32, BM = 128, OP = DH + 4;
  constexpr int NKH = NCH / 2;  // K reads of a row: 32 bytes each, two lanes' chunks
  constexpr int T2 = DH / 8;                  // products of a tile's scores, and of its values
  constexpr int KA = DH > 128 ? 4 : 2;        // K reads under way, of each block of 32 keys
  constexpr int VA = 4;                       // V fragments under way
  // 256-wide heads run one wave per SIMD, with accumulators in the upper half
  // of the registers
  constexpr bool WIDE = DH > 128;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[C::SMEM];
  __shared__ float scales[2][4][KT];  // a ring of four tiles' K scales, and of V's
  __shared__ int table[C::kTable];
  __shared__ float2 ml[BM];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  // consecutive workgroups go to the eight XCDs in turn: each XCD takes a run
  // of (head, split) groups, so that a group's tiles share its L2, and a
  // group's last tiles (with a causal mask the longest) first.  One workgroup to
  // a CU may fill the chip exactly, and then the runs have to be of the tiles
  // that the batch has, not of the grid's: with those a chunk of 1,024 rows of 8
  // heads over 8,192 keys gave some XCDs one too many and took 159 us instead of
  // 93 (now 88).  (Narrower heads, two workgroups to a CU, lose 2 % to the counting.)
  int split, splits = 0;
  UnitSeq first;
  Units units;
  if constexpr (MODE == kTree) {
    first = unit_seq(a, lane, BM);
    units = count_units(a, BM, lane, first);
  }
  const int tiles = MODE == kTree ? units.total : WIDE ? count_tiles(a, BM, lane) : grid_tiles;
  const int all = tiles * a.c.n_kv * (MODE == kTree ? 1 : a.nsplit), per = (all + 7) >> 3;
  const int id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= per || id >= all) return;
  const int grp = id / tiles;
  const int kvh = MODE == kTree ? __builtin_amdgcn_readfirstlane(grp) : grp / a.nsplit;
  if constexpr (MODE != kTree) split = grp - kvh * a.nsplit;
  Tile t;
  Span part;
  const int tile = MODE == kTree ? id - grp * tiles : tiles - 1 - (id - grp * tiles);
  if constexpr (MODE == kTree) {
    if (!find_unit(a, tile, BM, lane, first, units.per, t, split, splits, part)) return;
  } else {
    if (!find_tile(a, tile, BM, lane, t)) return;
  }

  const int rows_here = min(BM, t.rows - t.r0);
  const int p0 = t.first_pos + t.r0 / a.group, p1 = t.first_pos + (t.r0 + rows_here - 1) / a.group;
  const Span sp0 = span_of(a, p0, t.len), sp1 = span_of(a, p1, t.len);
  if constexpr (MODE == kTree) part.hi = min(part.hi, sp1.hi);
  else part = split_of(a, sp0.lo, sp1.hi, split);
  const int k_beg = part.lo, k_end = part.hi;

  const int r = t.r0 + 32 * wave + r32;
  const int tok = r / a.group;
  const Span sp = span_of(a, t.first_pos + tok, t.len);
  const int lo = max(sp.lo, k_beg), hi = r < t.rows ? min(sp.hi, k_end) : 0;
  // the keys that all of the wave's rows see
  const int w0 = min(t.r0 + 32 * wave, t.rows - 1), w1 = min(w0 + 31, t.rows - 1);
  const int all_lo = max(span_of(a, t.first_pos + w1 / a.group, t.len).lo, k_beg);
  const int all_hi = min(MODE == kTree ? t.first_pos : span_of(a, t.first_pos + w0 / a.group, t.len).hi, k_end);
  uint4 qf[NKS];
  {
    const T* qp = reinterpret_cast<const T*>(a.x.p) + (t.first_row + tok) * a.x.rs +
                  (int64_t)(kvh * a.group + (r - tok * a.group)) * a.x.hs;
#pragma unroll
    for (int k = 0; k < NKS; ++k) {
      const int d = Q8 ? 32 * (k >> 1) + 16 * h + 8 * (k & 1) : 16 * k + 8 * h;
      qf[k] = r < t.rows ? ld16(qp + d) : zero16();
    }
    scale_frags(qf, a.factor, T(0));
  }
  f32x16_v o[NDB];
#pragma unroll
  for (int d = 0; d < NDB; ++d) o[d] = f32x16_v{};
  float mx = kFloor, sum = 0.f;

  const int64_t hoff = (int64_t)kvh << a.c.shift;
  const int shift = a.c.shift, n_pages = a.c.n_pages, n_kv = a.c.n_kv;
  const char *const pk = a.c.k, *const pv = a.c.v;
  const float *const psk = a.c.k_scale, *const psv = a.c.v_scale;
  const float scale2 = a.scale2;
  const bool in_page = (1 << shift) >= KT / 4;  // the rows a wave copies lie in one page
  // Swizzles of the 16-byte chunks of a row in LDS: K reads take one chunk of
  // 32 rows at a time, V reads 64 bytes of 8 rows.  They are XORs, and rows
  // are powers of two apart, so the address of every read is one of few
  // registers plus a constant.
  auto swk = [](int row) __attribute__((always_inline)) { return row & (NCH - 1) & 15; };
  auto swv = [](int row) __attribute__((always_inline)) { return (Q8 ? row : 2 * row) & (NCH - 1); };
  constexpr int NKR = NCH / 2 < 8 ? NCH / 2 : 8;   // K reads: chunk pairs 2 k, by their low four bits
  constexpr int NVR = Q8 ? NDB : NDB < 4 ? NDB : 4;  // V reads: blocks d, in bf16 by their low two bits
  uint32_t kreg[NKR], vreg[NVR];
#pragma unroll
  for (int k = 0; k < NKR; ++k) kreg[k] = r32 * RB + (((2 * k + h) ^ swk(r32)) << 4);
  {
    const int i16 = lane & 15, dh16 = (lane >> 4) & 1, r8 = i16 >> 1;
    const int row = 4 * h + (Q8 ? (r8 < 4 ? r8 : r8 + 4) : i16 >> 2);
#pragma unroll
    for (int d = 0; d < NVR; ++d) {
      const int ch = Q8 ? 2 * d + dh16 : 4 * d + 2 * dh16 + ((i16 >> 1) & 1);
      vreg[d] = 2 * TB + row * RB + ((ch ^ swv(row)) << 4) + (i16 & 1) * 8;
    }
  }
  // this lane's offset within its wave's copies of a tile, four at a time
  const int sub = lane / NCH;
  constexpr int NO = NI < 4 ? NI : 4;
  uint32_t koff[NO], voff[NO];
#pragma unroll
  for (int j = 0; j < NO; ++j) {
    koff[j] = sub * RB + (((lane % NCH) ^ swk(j * RPC + sub)) << 4);
    voff[j] = sub * RB + (((lane % NCH) ^ swv(j * RPC + sub)) << 4);
  }

  for (int seg = k_beg & ~(KT - 1); seg < k_end;) {
    const int e0 = seg >> shift;
    const int seg_end = (int)min((int64_t)k_end, (int64_t)(e0 + C::kTable) << shift);
    const int ne = ((seg_end - 1) >> shift) - e0 + 1;
    __syncthreads();
    int good = 1;
    for (int i = threadIdx.x; i < ne; i += 256) {
      const int pg = a.q.table[(int64_t)t.b * a.q.max_pages + e0 + i];
      const bool ok = (unsigned)pg < (unsigned)n_pages;
      table[i] = ok ? pg : -1;
      good &= ok;
    }
    const bool seg_ok = __syncthreads_and(good);
    const int n_t = (seg_end - seg + KT - 1) / KT;

    auto row_of = [&](int x) __attribute__((always_inline)) {
      const int key = seg + x * KT + lane;
      const int pg = table[(min(key, seg_end - 1) >> shift) - e0];
      return key < k_beg || key >= seg_end || pg < 0 ? -1 : ((pg * n_kv) << shift) + (key & ((1 << shift) - 1));
    };
    // A tile's copies; rr: the lane's page row of it.  Mostly all 64 are there
    // and the 16 rows that a wave copies lie in one page (`plain`): then they
    // are one run of bytes, and copy j needs the run's base and the lane's
    // offset.
    auto plain = [&](int rr) __attribute__((always_inline)) { return in_page && !__ballot(rr < 0); };
    auto run_of = [&](const char* base, int rr) __attribute__((always_inline)) {
      return base + ((int64_t)__builtin_amdgcn_readlane(rr, wave * (KT / 4)) + hoff) * RB;
    };
    // NB copies from the B-th group on
    constexpr int NB = NI < 4 ? NI : 4;
    auto copy_some = [&](const char* run, auto sw, const uint32_t (&off)[NO], unsigned char* dst, auto B)
        __attribute__((always_inline)) {
      constexpr int b = decltype(B)::value;
      // (beyond the first four copies the swizzle differs by the bits above theirs)
      const uint32_t x = b ? (sw(4 * b * RPC) ^ sw(0)) << 4 : 0;
      uint32_t o[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) o[j] = off[j] ^ x;
      lds_dma16_run<NB>(run + b * 4096, o, dst + wave * NI * 1024 + b * 4096);
    };
    auto copy_any = [&](const char* base, auto sw, int rr, unsigned char* dst) __attribute__((always_inline)) {
#pragma unroll 4
      for (int j = 0; j < NI; ++j) {
        const int row = j * RPC + sub;
        const int pr = __shfl(rr, wave * (KT / 4) + row, 64);
        const char* src = base + ((int64_t)pr + hoff) * RB + (((lane % NCH) ^ sw(row)) << 4);
        lds_dma16(pr < 0 ? reinterpret_cast<const char*>(kZeros) : src, dst + (wave * NI + j) * 1024);
      }
    };
    // scales of tile x, two steps before its values are taken
    auto copy_scales = [&](int rr, int x) __attribute__((always_inline)) {
      if (Q8 && wave < 2) lds_dma4((wave == 0 ? psk : psv) + max(rr, 0) + hoff, scales[wave][x & 3]);
    };
    // S^T of a tile: block b, register i holds key 32 b + 8 (i / 4) + 4 h + i % 4.
    // K fragments are requested KA steps ahead.
    auto k_load = [&](uint32_t buf, int k, uint4 (&kf)[KA][2]) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
        kf[k % KA][b] = ld16(smem + (kreg[k % NKR] ^ buf) + (k / NKR) * 256 + b * 32 * RB);
    };
    // product g of the scores: block g % 2, head dims 16 (g / 2) ..
    auto k_mfma = [&](int g, const uint4 (&kf)[KA][2], f32x16_v (&s)[2]) __attribute__((always_inline)) {
      const int b = g & 1, k = g >> 1;
      if (!Q8) {
        mfma32_step(s[b], kf[k % KA][b], qf[k]);
      } else {
        const uint4 c = kf[(k >> 1) % KA][b];
        mfma32_step(s[b], codes_to_bf16<ST>(k & 1 ? make_uint2(c.z, c.w) : make_uint2(c.x, c.y)), qf[k]);
      }
    };
    // O^T += V^T P^T: fragment n = u * NDB + d, step u covers keys 16 u + {4 h ..,
    // 8 + 4 h ..}; requested VA ahead
    auto v_load = [&](uint32_t buf, int n, uint4 (&vf)[VA]) __attribute__((always_inline)) {
      const int u = n / NDB, d = n % NDB;
      if (Q8) {
        const uint2 c = ld_tr8(smem + (vreg[d % NVR] ^ buf) + 16 * u * RB);
        vf[n % VA] = make_uint4(c.x, c.y, 0u, 0u);
      } else {
        // rows 8 further: the swizzle differs by 16 of the chunk's bits, if it has that many
        const unsigned char* at = smem + (vreg[d % NVR] ^ buf) + 16 * u * RB;
        constexpr int flip = NCH > 16 ? 1 : 0;
        const uint2 f0 = ld_tr16(at + (d / NVR) * 256), f1 = ld_tr16(at + 8 * RB + ((d / NVR) ^ flip) * 256);
        vf[n % VA] = make_uint4(f0.x, f0.y, f1.x, f1.y);
      }
    };
    auto v_mfma = [&](int n, const uint4 (&vf)[VA], const uint4& pf) __attribute__((always_inline)) {
      const uint4 f = vf[n % VA];
      mfma32_step(o[n % NDB], Q8 ? codes_to_bf16<ST>(make_uint2(f.x, f.y)) : f, pf);
    };

    // the softmax in pieces.  Scores stay as the product left them (times the
    // keys' scales); `scale2` enters with the maximum's subtraction.
    auto is_whole = [&](int x) __attribute__((always_inline)) {
      const int key0 = seg + x * KT;
      return seg_ok && key0 >= all_lo && key0 + KT <= all_hi && key0 + KT <= seg_end;
    };
    auto key_scales = [&](int x, f32x16_v (&s)[2]) __attribute__((always_inline)) {
      if (Q8) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 k4 = *reinterpret_cast<const float4*>(&scales[0][x & 3][32 * b + 8 * i + 4 * h]);
            s[b][4 * i] *= k4.x; s[b][4 * i + 1] *= k4.y; s[b][4 * i + 2] *= k4.z; s[b][4 * i + 3] *= k4.w;
          }
      }
    };
    auto mask = [&](int x, f32x16_v (&s)[2]) __attribute__((always_inline)) {
      const int key0 = seg + x * KT;
      const int l0 = lo - key0 - 4 * h, h0 = min(hi, seg_end) - key0 - 4 * h;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 32 * b + 8 * (i >> 2) + (i & 3);
          s[b][i] = at >= l0 && at < h0 ? s[b][i] : -INFINITY;
        }
      if (!seg_ok) {
        const uint64_t present = __ballot(row_of(x) >= 0) >> (4 * h);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!((present >> (32 * b + 8 * (i >> 2) + (i & 3))) & 1)) s[b][i] = -INFINITY;
      }
      if constexpr (MODE == kTree) {
        const int tk = min(r, t.rows - 1) / a.group;
        const uint64_t bits = tree_bits(a, t.first_row + tk, key0, t.first_pos) >> (4 * h);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!((bits >> (32 * b + 8 * (i >> 2) + (i & 3))) & 1)) s[b][i] = -INFINITY;
      }
    };
    auto block_max = [&](const f32x16_v& s) __attribute__((always_inline)) {
      float m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = fmaxf(fmaxf(fmaxf(s[4 * i], s[4 * i + 1]), s[4 * i + 2]), s[4 * i + 3]);
      return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
    };
    // the row's maximum, in the unit of the exponent
    auto row_top = [&](float top) __attribute__((always_inline)) {
      auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
      return fmaxf(fmaxf(__uint_as_float(z[0]), __uint_as_float(z[1])) * scale2, kFloor);
    };
    auto raise = [&](float top) __attribute__((always_inline)) {
      const float nm = top > mx + kSlack ? top : mx;
      const float f = __builtin_amdgcn_exp2f(mx - nm);
      mx = nm;
      sum *= f;
#pragma unroll
      for (int d = 0; d < NDB; ++d) o[d] *= f;
    };
    // probabilities of registers 2 (q % 8) and the next of block q / 8; the
    // empty statement keeps them at their place among the products
    auto pair = [&](int x, int q, const f32x16_v (&s)[2], uint32_t (&pw)[16]) __attribute__((always_inline)) {
      const int i = 2 * (q & 7);
      float p0 = __builtin_amdgcn_exp2f(fmaf(s[q >> 3][i], scale2, -mx));
      float p1 = __builtin_amdgcn_exp2f(fmaf(s[q >> 3][i + 1], scale2, -mx));
      sum += p0 + p1;
      if (Q8) {
        const float2 v = *reinterpret_cast<const float2*>(&scales[1][x & 3][32 * (q >> 3) + 8 * (i >> 2) + 4 * h + (i & 3)]);
        // (a key that the row does not see may have any scale)
        p0 = s[q >> 3][i] == -INFINITY ? 0.f : p0 * v.x;
        p1 = s[q >> 3][i + 1] == -INFINITY ? 0.f : p1 * v.y;
      }
      pw[q] = pack_bf16(p0, p1);
      asm volatile("" : "+v"(pw[q]), "+v"(sum));
    };
    auto pfrag = [](const uint32_t (&pw)[16], int u) __attribute__((always_inline)) {
      return make_uint4(pw[4 * u], pw[4 * u + 1], pw[4 * u + 2], pw[4 * u + 3]);
    };
    auto fence = [&]() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    // all of the wave's copies have landed and its reads are done, in every wave
    auto turn = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };

    int rr1 = row_of(0);
    copy_any(pk, swk, rr1, smem);
    copy_any(pv, swv, rr1, smem + 2 * TB);
    copy_scales(rr1, 0);
    rr1 = row_of(1);  // page rows of tile x + 1 in the loop
    copy_scales(rr1, 1);
    if (n_t > 1) copy_any(pk, swk, rr1, smem + TB);
    turn();
    f32x16_v sa[2], sb[2];
    sa[0] = f32x16_v{};
    sa[1] = f32x16_v{};
    {
      uint4 kf[KA][2];
#pragma unroll
      for (int k = 0; k < KA; ++k) k_load(0, k, kf);
#pragma unroll
      for (int g = 0; g < T2; ++g) {
        k_mfma(g, kf, sa);
        if ((Q8 ? g & 1 && g >> 1 & 1 : g & 1) && g / (T2 / NKH) + KA < NKH) k_load(0, g / (T2 / NKH) + KA, kf);
      }
    }
    // scores of tile x as the softmax takes them; returns the rows' maxima
    auto ready = [&](int x, f32x16_v (&s)[2]) __attribute__((always_inline)) {
      key_scales(x, s);
      if (!is_whole(x)) mask(x, s);
      return row_top(fmaxf(block_max(s[0]), block_max(s[1])));
    };
    {
      const float top = ready(0, sa);
      if (__ballot(top > mx + kSlack)) raise(top);
    }
    turn();
    uint32_t pw[16];
    // Step x: probabilities and values of tile x, scores of tile x + 1, copies
    // of K of tile x + 2 and of V of tile x + 1.  The vector work lies between
    // the products by hand; the fences keep it there.  Returns the maxima of
    // the new scores.
    auto step = [&](int x, f32x16_v (&cur)[2], f32x16_v (&nxt)[2]) __attribute__((always_inline)) {
      const uint32_t bx = x & 1 ? TB : 0, by = TB - bx;
      const int rr2 = row_of(x + 2);
      uint4 kf[KA][2], vf[VA];
#pragma unroll
      for (int k = 0; k < KA; ++k) k_load(by, k, kf);
      const bool easy = x + 2 < n_t && plain(rr1) && plain(rr2);
      const char *run_k = run_of(pk, rr2), *run_v = run_of(pv, rr1);
      unsigned char *const dk = smem + bx, *const dv = smem + 2 * TB + by;
      if (!easy) {
        if (x + 2 < n_t) copy_any(pk, swk, rr2, dk);
        copy_any(pv, swv, rr1, dv);
      }
      copy_scales(rr2, x + 2);
      nxt[0] = f32x16_v{};
      nxt[1] = f32x16_v{};
      fence();
      // what goes with product g of the tile's 2 T2
      auto beside = [&](auto G) __attribute__((always_inline)) {
        constexpr int g = decltype(G)::value;
#pragma unroll
        for (int q = 0; q < 16; ++q)
          if (g == T2 / 16 + q * 11 * T2 / 128) pair(x, q, cur, pw);
        // copies over the first three quarters
        constexpr int NG = 2 * NI / NB, STEP = 3 * T2 / 2 / NG;
        if constexpr (g % STEP == STEP / 2 && g / STEP < NG) {
          constexpr int c = g / STEP;
          if (easy) {
            if constexpr (c < NG / 2) copy_some(run_k, swk, koff, dk, std::integral_constant<int, c>{});
            else copy_some(run_v, swv, voff, dv, std::integral_constant<int, c - NG / 2>{});
          }
        }
      };
      static_for<T2>([&](auto G) __attribute__((always_inline)) {
        constexpr int g = decltype(G)::value;
        constexpr int per = T2 / NKH;  // products to a K read of both blocks
        k_mfma(g, kf, nxt);
        if constexpr (g % per == per - 1 && g / per + KA < NKH) k_load(by, g / per + KA, kf);
        if constexpr (g == T2 - 1) {
#pragma unroll
          for (int n = 0; n < VA; ++n) v_load(bx, n, vf);
        }
        beside(G);
        fence();
      });
      static_for<T2>([&](auto N) __attribute__((always_inline)) {
        constexpr int n = decltype(N)::value;
        v_mfma(n, vf, pfrag(pw, n / NDB));
        if constexpr (n + VA < T2) v_load(bx, n + VA, vf);
        beside(std::integral_constant<int, T2 + n>{});
        fence();
      });
      rr1 = rr2;
      return ready(x + 1, nxt);
    };
    int x = 0;
    if constexpr (WIDE) {
      // the loop without a rescaling: one within it would move the
      // accumulators about at every turn
      while (x + 1 < n_t) {
        float top;
        bool high;
        do {
          top = step(x, sa, sb);
          turn();
          sa[0] = sb[0];
          sa[1] = sb[1];
          high = __ballot(top > mx + kSlack) != 0;
          ++x;
        } while (x + 1 < n_t && !high);
        if (high) raise(top);
      }
    } else {
      for (; x + 2 < n_t; x += 2) {
        float top = step(x, sa, sb);
        if (__ballot(top > mx + kSlack)) raise(top);
        turn();
        top = step(x + 1, sb, sa);
        if (__ballot(top > mx + kSlack)) raise(top);
        turn();
      }
      if (x + 1 < n_t) {
        const float top = step(x, sa, sb);
        if (__ballot(top > mx + kSlack)) raise(top);
        turn();
        ++x;
        sa[0] = sb[0];
        sa[1] = sb[1];
      }
    }
    {
      const uint32_t bx = x & 1 ? TB : 0;
#pragma unroll
      for (int q = 0; q < 16; ++q) pair(x, q, sa, pw);
      uint4 vf[VA];
#pragma unroll
      for (int n = 0; n < VA; ++n) v_load(bx, n, vf);
#pragma unroll
      for (int n = 0; n < T2; ++n) {
        v_mfma(n, vf, pfrag(pw, n / NDB));
        if (n + VA < T2) v_load(bx, n + VA, vf);
      }
    }
    seg = seg_end;
  }

  if constexpr (MODE != kPlain) {
    // Mostly every lane stores its row's dims as it holds them, 16 bytes at a time: a
    // row at a time by the whole wave, as below, 32 rows take 8 us (8 trees of 64
    // rows of 32 heads over 8,192 keys 96 us that way, 87 this way).
    auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    const float l = __uint_as_float(z[0]) + __uint_as_float(z[1]);
    bool odd = false;
    if constexpr (ST != REFLEX_STORE_INT8) {
#pragma unroll
      for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) odd |= !(fabsf(o[d][i]) < INFINITY);
    }
    if (!__syncthreads_or(odd && l < INFINITY && r < t.rows)) {
      if (r >= t.rows) return;
      const int64_t row = t.first_row + tok;
      const int head = kvh * a.group + (r - tok * a.group);
      if (a.nsplit == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* const y = reinterpret_cast<T*>(const_cast<char*>(a.o.p)) + row * a.o.rs + head * a.o.hs + 4 * h;
#pragma unroll
        for (int d = 0; d < NDB; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            *reinterpret_cast<uint2*>(y + 32 * d + 8 * i) =
                make_uint2(pack_bf16(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                           pack_bf16(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
        if (MODE == kWeigh && h == 0) a.stats[row * a.n_q + head] = make_float2(mx, inv);
        return;
      }
      const int64_t at = (row * a.n_q + head) * a.nsplit + split;
      if (h == 0) a.part_ml[at] = make_float2(mx, l);
      if (MODE == kTree && split == 0)  // (splits that the tile does not have)
        for (int s = splits + h; s < a.nsplit; s += 2) a.part_ml[at + s] = make_float2(kFloor, 0.f);
      if (l == 0.f) return;
      float* const y = a.part_o + at * DH + 4 * h;
#pragma unroll
      for (int d = 0; d < NDB; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(y + 32 * d + 8 * i) =
              make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
      return;
    }
  }
  __syncthreads();
  float* const ex = reinterpret_cast<float*>(smem) + wave * 32 * OP;
  {
    auto z = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    if (h == 0) ml[32 * wave + r32] = make_float2(mx, __uint_as_float(z[0]) + __uint_as_float(z[1]));
  }
#pragma unroll
  for (int d = 0; d < NDB; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<float4*>(ex + r32 * OP + 32 * d + 8 * i + 4 * h) =
          make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
  __syncthreads();
  constexpr int N = DH / 64;
  for (int q = 0; q < 32 && 32 * wave + q < rows_here; ++q) {
    const int rq = t.r0 + 32 * wave + q, tq = rq / a.group;
    const float2 w = ml[32 * wave + q];
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = ex[q * OP + lane * N + i];
    finish_row<MODE, T, ST, DH>(a, tile, BM, 32 * wave + q, t.first_row + tq, kvh * a.group + (rq - tq * a.group), split, false,
                          w.x, w.y, y, splits);
  }
}

// One wave per (row, head): the splits' partial results joined in order.  Those
// of the first eight splits are requested with the maxima and sums, so that
// most rows take one memory round trip: 6,144 rows of 256 in five splits 8 us,
// 32 MB of partial results.
template <int MODE, typename T, int DH>
RFX_DEV void merge_row(const PagedAttnArgs& a, int64_t id) {
  constexpr int N = DH / 64, G = 8;
  const int lane = threadIdx.x & 63;
  // (there are 2^23 at most: a quotient in 64 bits was most of the instructions)
  const int64_t row = MODE == kPlain ? id / a.n_q
                                     : divided((int)id, a.n_q, 1.f / (float)a.n_q);
  if (row >= a.n_rows) return;
  const float* p = a.part_o + id * a.nsplit * DH + lane * N;
  float v[G][N];
  int splits = a.nsplit;
  auto request = [&](int s0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < G; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (MODE != kTree || s0 + u < splits) v[u][i] = p[(int64_t)min(s0 + u, splits - 1) * DH + i];
  };
  if constexpr (MODE != kTree) request(0);
  const float2 w = lane < a.nsplit ? a.part_ml[id * a.nsplit + lane] : make_float2(kFloor, 0.f);
  if (row < a.q.cu[0] || row >= a.q.cu[a.q.n]) return;
  if constexpr (MODE == kTree) {  // a tile may have few of the splits that there is room for
    splits = max(64 - (int)__clzll(__ballot(w.y != 0.f)), 1);
    if (splits <= G) request(0);
  }
  float y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = 0.f;
  auto finish = [&](float M, float L) __attribute__((always_inline)) {
    store_row<T, DH>(a, row, (int)(id - row * a.n_q), L, y);
    if constexpr (MODE == kWeigh || MODE == kKept)
      if (lane == 0) a.stats[id] = make_float2(M, L == 0.f ? 0.f : 1.f / L);
  };
  if constexpr (MODE == kTree) {  // (weighed results stay the attention's, bit by bit)
    if (splits <= G) {
      // few splits: from lane to lane by scalar reads, which takes a third of the
      // instructions (28,700 rows of 128 in two splits took 12 us, 94 % vector issue)
      auto of = [&](float x, int u) __attribute__((always_inline)) {
        return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), u));
      };
      float M = kFloor, L = 0.f;
#pragma unroll
      for (int u = 0; u < G; ++u)
        if (u < splits) M = fmaxf(M, of(w.x, u));
#pragma unroll
      for (int u = 0; u < G; ++u)
        if (u < splits && of(w.y, u) != 0.f) {  // (others have stored no partial sums)
          const float f = __builtin_amdgcn_exp2f(of(w.x, u) - M);
          L += of(w.y, u) * f;
#pragma unroll
          for (int i = 0; i < N; ++i) y[i] += f * v[u][i];
        }
      finish(M, L);
      return;
    }
  }
  float M = w.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float f = __builtin_amdgcn_exp2f(w.x - M);
  const float L = warp_sum(w.y * f);
  const uint64_t live = __ballot(w.y != 0.f);  // others have stored no partial sums
  if constexpr (MODE == kTree) {
    // Many splits: four are added and asked for anew while four are under way.  For one
    // that is not live the last one, which is, is read, without a branch, and not added
    // (64 rows of 8 heads of 256 in 64 splits 7.6 instead of 14.0 us, eight at a time).
    auto fetch = [&](int u0, int s0) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < G / 2; ++u) {
        const int s = s0 + u < splits && ((live >> ((s0 + u) & 63)) & 1) ? s0 + u : splits - 1;
#pragma unroll
        for (int i = 0; i < N; ++i) v[u0 + u][i] = p[s * DH + i];
      }
    };
    auto add = [&](int u0, int s0) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < G / 2; ++u) {
        const int s = s0 + u;
        if (s >= splits || !((live >> s) & 1)) continue;
        const float fs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), s));
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] += fs * v[u0 + u][i];
      }
    };
    fetch(0, 0);
    fetch(G / 2, G / 2);
    for (int s0 = 0; s0 < splits; s0 += G) {
      add(0, s0);
      fetch(0, s0 + G);
      add(G / 2, s0 + G / 2);
      fetch(G / 2, s0 + G + G / 2);
    }
    finish(M, L);
    return;
  }
  for (int s0 = 0; s0 < a.nsplit; s0 += G) {
    if (s0) {
      if (!(live >> s0)) break;
      request(s0);
    }
#pragma unroll
    for (int u = 0; u < G; ++u) {
      const float fs = __shfl(f, (s0 + u) & 63, 64);
      if (s0 + u < a.nsplit && ((live >> (s0 + u)) & 1))
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] += fs * v[u][i];
    }
  }
  finish(M, L);
}

template <int MODE, typename T, int DH>
__global__ __launch_bounds__(256) void paged_attn_merge_kernel(const PagedAttnArgs a) {
  merge_row<MODE, T, DH>(a, (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6));
}

// Tiles that a batch can have at most: every sequence's last one may be partial.
inline int64_t tile_bound(int64_t n_rows, int n_seqs, int group, int bm) {
  return n_rows * group / bm + std::min<int64_t>(n_seqs, n_rows);
}

// Rows of a tile, by the rows of an average sequence (with one K/V head): 16 or
// 32 with the few-row kernel, 128 with the many-row one.  fp32, which only the
// first has, takes 32 where that makes two workgroups for every CU: seven
// ragged chunks of up to 450 rows 23 us with 16 against 31, four of 4,000 rows
// 419 against 342.  256-wide heads stay at 16, as queries and sums of 32 such
// rows do not fit a wave's registers: four of 8,000 rows 730 us against 736,
// over int8 pages 594 against 705.
inline int rows_of_tile(int64_t n_rows, int n_seqs, int group, int n_kv, int dh, int dtype) {
  const int64_t rows = n_rows * group / std::max<int64_t>(1, std::min<int64_t>(n_seqs, n_rows));
  if (rows <= 16) return 16;
  if (dtype != REFLEX_DTYPE_BF16) return dh <= 128 && tile_bound(n_rows, n_seqs, group, 32) * n_kv >= 512 ? 32 : 16;
  return rows <= 32 ? 32 : 128;
}

template <int MODE, typename T, int ST, int DH>
hipError_t launch_shape(const PagedAttnArgs& a, hipStream_t s) {
  const int bm = MODE == kTree ? a.tile_rows
                               : rows_of_tile(a.n_rows, a.q.n, a.group, a.c.n_kv, DH,
                                              sizeof(T) == 2 ? REFLEX_DTYPE_BF16 : REFLEX_DTYPE_F32);
  // (units: what the division gives, and a short last split of every tile)
  const int64_t tiles = tile_bound(a.n_rows, a.q.n, a.group, bm) + (MODE == kTree ? a.units : 0);
  const int splits = MODE == kTree ? 1 : a.nsplit;
  const dim3 grid((unsigned)tiles, (unsigned)(a.c.n_kv * splits));
  if constexpr (sizeof(T) == 2 && MODE != kKept) {
    if (bm == 128) {
      const unsigned n = (unsigned)((tiles * a.c.n_kv * splits + 7) / 8 * 8);
      RFX_LAUNCH((paged_attn_many_kernel<MODE, ST, DH>), dim3(n), dim3(256), 0, s, a, (int)tiles);
    }
  }
  if (bm == 16)
    RFX_LAUNCH((paged_attn_few_kernel<MODE, T, ST, DH, 1>), grid, dim3(256), 0, s, a);
  if constexpr (sizeof(T) == 2 || DH <= 128) {
    if (bm == 32) RFX_LAUNCH((paged_attn_few_kernel<MODE, T, ST, DH, 2>), grid, dim3(256), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.nsplit > 1 && !(MODE == kKept && a.merge_with_sums)) {
    RFX_LAUNCH((paged_attn_merge_kernel<MODE, T, DH>), dim3((unsigned)((a.n_rows * a.n_q + 3) / 4)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <int MODE, typename T, int ST>
hipError_t launch_store(const PagedAttnArgs& a, hipStream_t s) {
  if (a.c.dh == 64) return launch_shape<MODE, T, ST, 64>(a, s);
  if (a.c.dh == 128) return launch_shape<MODE, T, ST, 128>(a, s);
  return launch_shape<MODE, T, ST, 256>(a, s);
}

template <int MODE, typename T>
hipError_t launch_mode(const PagedAttnArgs& a, int store, hipStream_t s) {
  if (store == REFLEX_STORE_FP8) return launch_store<MODE, T, REFLEX_STORE_FP8>(a, s);
  if (store == REFLEX_STORE_INT8) return launch_store<MODE, T, REFLEX_STORE_INT8>(a, s);
  return launch_store<MODE, T, REFLEX_STORE_BF16>(a, s);
}

}  // namespace

}  // namespace reflex
