// Attention of a chunk of new tokens over a paged cache.
#include <algorithm>

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

// out[row][head] = o / l; each lane holds DH / 64 dims.
template <typename T, int DH>
RFX_DEV void store_row(const PagedAttnArgs& a, int64_t row, int head, float l, const float* o) {
  constexpr int N = DH / 64;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* y = reinterpret_cast<T*>(const_cast<char*>(a.o.p)) + row * a.o.rs + head * a.o.hs + (threadIdx.x & 63) * N;
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = from_f<T>(o[i] * inv);
}

template <int N> RFX_DEV void wait_copies_if(bool newer) {
  // the last tile has nothing newer under way
  if (newer) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// ---------------------------------------------------------------------------
// shared pieces of the tiled kernels
// ---------------------------------------------------------------------------
template <int N> RFX_DEV void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
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

RFX_DEV uint32_t pack_bf16(float a, float b) {
  bf16x2_v v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
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

// 4 codes (or 4 fp32) -> 4 fp32
template <int ST> RFX_DEV uint4 codes_to_f32(uint32_t c) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    f[i] = ST == REFLEX_STORE_FP8 ? elem_f<REFLEX_STORE_FP8, uint8_t>((uint8_t)(c >> (8 * i)))
                                  : (float)(int8_t)(c >> (8 * i));
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
    int c0 = 0, c1 = 0;
    if (b < a.q.n) {
      c0 = (int)min((int64_t)max(a.q.cu[b], 0), a.n_rows);
      c1 = (int)min((int64_t)max(a.q.cu[b + 1], 0), a.n_rows);
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
      t.len = __builtin_amdgcn_readfirstlane(a.q.len[t.b]);
      t.first_pos = __builtin_amdgcn_readfirstlane((int)((int64_t)t.len - a.q.cu[t.b + 1] + f0));
      return true;
    }
    before += __shfl(sum, 63, 64);
  }
  return false;
}


// A row's result of one split: stored, or kept for the merge.  `mixed`: the
// tile's rows do not all see the same keys, so a NaN or an infinity among the
// values of a key that this row does not see has met a probability of 0 in the
// matrix product.  Such a row is done again key by key, which reads only what
// the row sees.  (Values in 8 bits are finite codes; their scales never meet a
// probability of 0.)
template <typename T, int ST, int DH>
RFX_DEV void finish_row(const PagedAttnArgs& a, const Tile& t, int64_t row, int head, int pos, int k_beg, int k_end,
                        int split, bool mixed, float M, float L, float* y) {
  constexpr int N = DH / 64;
  constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  if (!Q8 && mixed) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < N; ++i) odd |= !(fabsf(y[i]) < INFINITY);
    if (__ballot(odd)) {
      Span sp = span_of(a, pos, t.len);
      sp.lo = max(sp.lo, k_beg);
      sp.hi = min(sp.hi, k_end);
      scalar_row<T, ST, DH>(a, row, head, t.b, sp, M, L, y);
    }
  }
  if (a.nsplit == 1) {
    store_row<T, DH>(a, row, head, L, y);
    return;
  }
  const int lane = threadIdx.x & 63;
  const int64_t at = (row * a.n_q + head) * a.nsplit + split;
  if (lane == 0) a.part_ml[at] = make_float2(M, L);
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
template <typename T, int ST, int DH>
struct FewCfg {
  static constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8;
  static constexpr int ES = Q8 ? 1 : (int)sizeof(T);
  static constexpr int RB = DH * ES;                                          // bytes of a K or V row
  static constexpr int KT = RB >= 1024 ? 16 : RB >= 512 ? 32 : 64;            // keys of a tile
  static constexpr int NCH = RB / 16;                                         // 16-byte chunks of a row
  static constexpr int RPC = 64 / NCH;                                        // rows of a copy (0: half a row)
  static constexpr int NI = KT * RB / 1024;                                   // copies of a tile
  static constexpr int TB = KT * RB;                                          // bytes of a tile
  static constexpr int SC = Q8 ? 2 * 64 * 4 : 0;                              // scales of a tile
  static constexpr int WAVE = 2 * TB + SC;                                    // LDS of a wave
  static constexpr int kTable = 1024;                                         // page table entries held in LDS
};

template <typename T, int ST, int DH, int MR>
__global__ __launch_bounds__(256) void paged_attn_few_kernel(const PagedAttnArgs a) {
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
  const int kvh = blockIdx.y / a.nsplit, split = blockIdx.y - kvh * a.nsplit;
  Tile t;
  if (!find_tile(a, blockIdx.x, BM, lane, t)) return;

  // keys that any row of the tile sees, cut to this split
  const int rows_here = min(BM, t.rows - t.r0);
  const int p0 = t.first_pos + t.r0 / a.group, p1 = t.first_pos + (t.r0 + rows_here - 1) / a.group;
  const int lo_min = span_of(a, p0, t.len).lo, hi_max = span_of(a, p1, t.len).hi;
  const int lo_max = span_of(a, p1, t.len).lo, hi_min = span_of(a, p0, t.len).hi;
  const int s_beg = split * a.split_keys;
  const int s_end = split == a.nsplit - 1 ? INT32_MAX : s_beg + a.split_keys;
  const int k_beg = max(lo_min, s_beg), k_end = min(hi_max, s_end);

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
  const int shift = a.c.shift, n_pages = a.c.n_pages, n_kv = a.c.n_kv;

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

    // this lane's key of tile `x`: its page row, or -1
    auto row_of = [&](int x) __attribute__((always_inline)) {
      const int key = seg + x * KT + lane;
      if (lane >= KT || key >= seg_end) return -1;
      const int pg = table[(key >> shift) - e0];
      return pg < 0 ? -1 : ((pg * n_kv) << shift) + (key & ((1 << shift) - 1));
    };
    // copy a tile's K or V; r: this lane's page row (or -1: any row will do)
    auto copy = [&](const char* base, const float* sc, int r, unsigned char* dst, float* sdst)
        __attribute__((always_inline)) {
      const int64_t rr = (int64_t)max(r, 0) + hoff;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        const int row = (j * 64 + lane) / NCH, ch = (lane + j * 64) % NCH;
        const int pr = __shfl(max(r, 0), row, 64);
        lds_dma16(base + ((int64_t)pr + hoff) * RB + ((ch ^ swz(row)) << 4), dst + j * 1024);
      }
      if (Q8) lds_dma4(sc + rr, sdst);
    };
    constexpr int NC = NI + (Q8 ? 1 : 0);

    int r_cur = row_of(wave);
    if (wave < n_t) {
      copy(a.c.k, a.c.k_scale, r_cur, kb, ksc);
      copy(a.c.v, a.c.v_scale, r_cur, vb, vsc);
    }
    for (int x = wave; x < n_t; x += 4) {
      const int r_next = row_of(x + 4);
      const bool more = x + 4 < n_t;
      const int key0 = seg + x * KT;
      const uint64_t present = __ballot(r_cur >= 0);
      wait_copies<NC>();
      // S^T: block kb holds keys 16 kb + 4 g + i of query row c16
      f32x4_v s[MR][NKB];
#pragma unroll
      for (int b = 0; b < NKB; ++b) {
#pragma unroll
        for (int m = 0; m < MR; ++m) s[m][b] = f32x4_v{0.f, 0.f, 0.f, 0.f};
        const int row = 16 * b + c16;
        const unsigned char* kr = kb + row * RB;
        if (!Q8) {
#pragma unroll
          for (int k = 0; k < NKS; ++k) {
            const uint4 f = ld16(kr + (((4 * k + g) ^ swz(row)) << 4));
#pragma unroll
            for (int m = 0; m < MR; ++m) mfma_step(s[m][b], f, qf[m][k], T(0));
          }
        } else {
#pragma unroll
          for (int k = 0; k < DH / 64; ++k) {
            const uint4 c = ld16(kr + (((4 * k + g) ^ swz(row)) << 4));
            if (BF) {
              const uint4 f0 = codes_to_bf16<ST>(make_uint2(c.x, c.y)), f1 = codes_to_bf16<ST>(make_uint2(c.z, c.w));
#pragma unroll
              for (int m = 0; m < MR; ++m) {
                mfma_step(s[m][b], f0, qf[m][2 * k], T(0));
                mfma_step(s[m][b], f1, qf[m][2 * k + 1], T(0));
              }
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
        }
      }
      float4 ks[NKB];
#pragma unroll
      for (int b = 0; b < NKB; ++b) ks[b] = Q8 ? *reinterpret_cast<const float4*>(ksc + 16 * b + 4 * g) : make_float4(1.f, 1.f, 1.f, 1.f);
      wait_lds();
      if (more) copy(a.c.k, a.c.k_scale, r_next, kb, ksc);

      // softmax: scores in units of log2 e
      const bool whole = key0 >= lo_max && key0 + KT <= hi_min && key0 + KT <= s_end && key0 >= s_beg &&
                         present == (KT == 64 ? ~0ull : (1ull << KT) - 1);
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        float top = kFloor;
        const int l0 = max(lo[m], k_beg), h0 = min(hi[m], seg_end);
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
          const float kk[4] = {ks[b].x, ks[b].y, ks[b].z, ks[b].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = s[m][b][i] * a.scale2;
            if (Q8) v *= kk[i];
            if (!whole) {
              const int at = 16 * b + 4 * g + i, key = key0 + at;
              const bool see = key >= l0 && key < h0 && ((present >> at) & 1);
              v = see ? v : -INFINITY;
            }
            s[m][b][i] = v;
            top = fmaxf(top, v);
          }
        }
        top = fmaxf(mx[m], across_rows(top, max2));
        const float scale = __builtin_amdgcn_exp2f(mx[m] - top);
        mx[m] = top;
        float add = 0.f;
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(s[m][b][i] - top);
            add += p;
            s[m][b][i] = p;
          }
        sum[m] = sum[m] * scale + add;
#pragma unroll
        for (int d = 0; d < NDB; ++d) o[m][d] *= scale;
      }

      wait_copies_if<NC>(more);
      if (!whole) {
        // values that no row of the tile sees must not meet a probability of 0
        const int v_lo = max(k_beg, lo_min), v_hi = min(hi_max, seg_end);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
          const int at = (j * 64 + lane) / NCH, key = key0 + at;
          if (key < v_lo || key >= v_hi || !((present >> at) & 1)) st16(vb + j * 1024 + lane * 16, zero16());
        }
      }
      if (Q8) {
#pragma unroll
        for (int b = 0; b < NKB; ++b) {
          const float4 v4 = *reinterpret_cast<const float4*>(vsc + 16 * b + 4 * g);
          const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
#pragma unroll
          for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float p = s[m][b][i];
              // (a key that the row does not see may have any scale)
              s[m][b][i] = whole || p > 0.f || p != p ? p * vv[i] : 0.f;
            }
        }
      }
      // O^T += V^T P^T
      if (BF) {
#pragma unroll
        for (int j = 0; j < KT / 32; ++j) {
          uint4 pf[MR];
#pragma unroll
          for (int m = 0; m < MR; ++m) {
            const f32x4_v &u = s[m][2 * j], &w = s[m][2 * j + 1];
            pf[m] = make_uint4(pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]));
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
            for (int m = 0; m < MR; ++m) mfma_step(o[m][d], f, pf[m], bf16_t(0));
          }
        }
      } else {
#pragma unroll
        for (int b = 0; b < NKB; ++b)
#pragma unroll
          for (int d = 0; d < NDB; ++d) {
            float f[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int row = 16 * b + 4 * g + e, col = 16 * d + c16;
              if (Q8) {
                const unsigned char c = vb[row * RB + (((col >> 4) ^ swz(row)) << 4) + (col & 15)];
                f[e] = ST == REFLEX_STORE_FP8 ? elem_f<REFLEX_STORE_FP8, uint8_t>(c) : (float)(int8_t)c;
              } else {
                f[e] = *reinterpret_cast<const float*>(vb + row * RB + (((col >> 2) ^ swz(row)) << 4) + (col & 3) * 4);
              }
            }
            const uint4 vf = f_to_frag(f, 0.f);
#pragma unroll
            for (int m = 0; m < MR; ++m) {
              const float p[4] = {s[m][b][0], s[m][b][1], s[m][b][2], s[m][b][3]};
              mfma_step(o[m][d], vf, f_to_frag(p, 0.f), 0.f);
            }
          }
      }
      wait_lds();
      if (more) copy(a.c.v, a.c.v_scale, r_next, vb, vsc);
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
    finish_row<T, ST, DH>(a, t, row, head, t.first_pos + tok, k_beg, k_end, split, lo_min != lo_max || hi_min != hi_max, M, L,
                          y);
  }
}

// One wave per (row, head): the splits' partial results joined.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_attn_merge_kernel(const PagedAttnArgs a) {
  constexpr int N = DH / 64;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t row = id / a.n_q;
  if (row >= a.n_rows || row < a.q.cu[0] || row >= a.q.cu[a.q.n]) return;
  const float2 w = lane < a.nsplit ? a.part_ml[id * a.nsplit + lane] : make_float2(kFloor, 0.f);
  float M = w.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float f = __builtin_amdgcn_exp2f(w.x - M);
  const float L = warp_sum(w.y * f);
  float y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = 0.f;
  const float* p = a.part_o + id * a.nsplit * DH + lane * N;
  // splits without keys for this row hold no partial sums
  uint64_t live = __ballot(w.y != 0.f);
  while (live) {
    float v[4][N], fs[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = live ? __ffsll((unsigned long long)live) - 1 : -1;
      live &= live - 1;
      fs[u] = s < 0 ? 0.f : __shfl(f, max(s, 0), 64);
#pragma unroll
      for (int i = 0; i < N; ++i) v[u][i] = s < 0 ? 0.f : p[(int64_t)s * DH + i];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) y[i] += fs[u] * v[u][i];
  }
  store_row<T, DH>(a, row, (int)(id - row * a.n_q), L, y);
}

// Key splits at most: a merging wave holds one in each lane.
constexpr int kMaxSplits = 64;

// Tiles that a batch can have at most: every sequence's last one may be partial.
int64_t tile_bound(int64_t n_rows, int n_seqs, int group, int bm) {
  return n_rows * group / bm + std::min<int64_t>(n_seqs, n_rows);
}

// 16-row blocks of a workgroup of the few-row kernel.
int few_blocks(int64_t n_rows, int n_seqs, int group) {
  return n_rows * group > 16 * (int64_t)std::max(1, n_seqs) ? 2 : 1;
}

template <typename T, int ST, int DH>
hipError_t launch_shape(const PagedAttnArgs& a, hipStream_t s) {
  const int mr = few_blocks(a.n_rows, a.q.n, a.group);
  const int64_t tiles = tile_bound(a.n_rows, a.q.n, a.group, 16 * mr);
  const dim3 grid((unsigned)tiles, (unsigned)(a.c.n_kv * a.nsplit));
  if (mr == 1)
    RFX_LAUNCH((paged_attn_few_kernel<T, ST, DH, 1>), grid, dim3(256), 0, s, a);
  else
    RFX_LAUNCH((paged_attn_few_kernel<T, ST, DH, 2>), grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.nsplit > 1) {
    RFX_LAUNCH((paged_attn_merge_kernel<T, DH>), dim3((unsigned)((a.n_rows * a.n_q + 3) / 4)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int ST>
hipError_t launch_store(const PagedAttnArgs& a, hipStream_t s) {
  if (a.c.dh == 64) return launch_shape<T, ST, 64>(a, s);
  if (a.c.dh == 128) return launch_shape<T, ST, 128>(a, s);
  return launch_shape<T, ST, 256>(a, s);
}

}  // namespace

PagedAttnPlan paged_attention_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q,
                                   int dtype) {
  PagedAttnPlan p;
  const int group = n_q / c.n_kv_heads;
  const int64_t cap = (int64_t)b.max_pages * c.page_size;
  const int64_t len = b.max_length > 0 && b.max_length < cap ? b.max_length : cap;
  const int mr = few_blocks(n_rows, b.n_seqs, group);
  const int64_t blocks = tile_bound(n_rows, b.n_seqs, group, 16 * mr) * c.n_kv_heads;
  // enough workgroups for every CU four times over, each with 128 keys at least
  int64_t want = (1024 + blocks - 1) / blocks;
  want = std::min<int64_t>(want, (len + 127) / 128);
  want = std::min<int64_t>(want, std::min<int64_t>(kMaxSplits, 65535 / c.n_kv_heads));
  want = std::max<int64_t>(want, 1);
  int64_t keys = ((len + want - 1) / want + 127) / 128 * 128;
  keys = std::max<int64_t>(keys, 128);
  p.nsplit = (int)std::max<int64_t>(1, (len + keys - 1) / keys);
  p.split_keys = (int)keys;
  p.bytes = p.nsplit == 1 ? 0 : (size_t)n_rows * n_q * p.nsplit * (c.head_dim + 2) * sizeof(float);
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
