// Attention that also adds up the weight that every key got: the kernels of
// paged_attention.h, which leave every row's maximum and sum, and the sums of
// the rows' probabilities for each key.
#include "paged_attention.h"

namespace reflex {

namespace {

// Sums over the rows (tokens and query heads of a K/V head) of p(row, key) =
// 2^(score - maximum) / sum, added to the keys' weights.  The scores are formed
// again: a wave holds the fragments of its keys in registers and goes over the
// query rows that see any of them, 16 at a time, S^T = K Q^T as in the
// attention, so that a lane holds four keys of one query row and sums its own
// column of rows; the columns are joined at the end, over the lanes and then over
// the waves, always in the same order, and one thread adds a key's sum.
template <typename T, int ST, int DH>
struct WeighCfg {
  static constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8, BF = sizeof(T) == 2;
  static constexpr int ES = Q8 ? 1 : (int)sizeof(T);
  static constexpr int RB = DH * ES;
  static constexpr int QS = BF ? 32 : 16;              // head dims of a product
  static constexpr int NKS = DH / QS;
  static constexpr int NKB = !BF && DH > 128 ? 2 : 4;  // blocks of 16 keys of a wave
  static constexpr int KPW = 16 * NKB;
};

template <typename T, int ST, int DH>
__global__ __launch_bounds__(256) void paged_weigh_kernel(const PagedAttnArgs a, float* weights, int key_waves,
                                                          int tiles) {
  typedef WeighCfg<T, ST, DH> C;
  constexpr bool Q8 = C::Q8, BF = C::BF;
  constexpr int RB = C::RB, QS = C::QS, NKS = C::NKS, NKB = C::NKB, KPW = C::KPW;
  __shared__ float red[4][KPW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  const int list = blockIdx.x / tiles, b = list / a.c.n_kv, kvh = list - b * a.c.n_kv;
  const int64_t c0 = min((int64_t)max(a.q.cu[b], 0), a.n_rows), c1 = min((int64_t)max(a.q.cu[b + 1], 0), a.n_rows);
  if (c1 <= c0) return;
  const int n = (int)(c1 - c0), rows = n * a.group, len = a.q.len[b];
  const int first = (int)((int64_t)len - a.q.cu[b + 1] + c0);
  const int lo_all = span_of(a, first, len).lo, hi_all = span_of(a, first + n - 1, len).hi;
  const int kt = KPW * key_waves, phases = 4 / key_waves;
  const int64_t hoff = (int64_t)kvh << a.c.shift;
  for (int64_t t0 = (lo_all & ~(kt - 1)) + (int64_t)(blockIdx.x - list * tiles) * kt; t0 < hi_all;
       t0 += (int64_t)tiles * kt) {
    const int k0 = (int)t0 + (wave % key_waves) * KPW, phase = wave / key_waves;
    const int key = k0 + lane;
    const int pr = lane < KPW && key >= lo_all && key < hi_all ? page_row(a.c, a.q, b, key) : -1;
    constexpr uint64_t kAll = KPW == 64 ? ~0ull : (1ull << KPW) - 1;
    const uint64_t present = __ballot(pr >= 0);
    uint4 kf[NKB][NKS];
    float ks[NKB][4];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      const int r = __shfl(pr, 16 * kb + c16, 64);
      const char* const at = a.c.k + ((int64_t)max(r, 0) + hoff) * RB;
#pragma unroll
      for (int k = 0; k < NKS; ++k) {
        const int d = QS * k + (QS / 4) * g;
        if (!Q8) kf[kb][k] = r >= 0 ? ld16(at + d * C::ES) : zero16();
        else if constexpr (BF) kf[kb][k] = codes_to_bf16<ST>(r >= 0 ? *reinterpret_cast<const uint2*>(at + d) : make_uint2(0, 0));
        else kf[kb][k] = codes_to_f32<ST>(r >= 0 ? *reinterpret_cast<const uint32_t*>(at + d) : 0u);
      }
      const float mine = Q8 && r >= 0 ? a.c.k_scale[(int64_t)r + hoff] : 1.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) ks[kb][i] = __shfl(mine, 4 * g + i, 64);
    }
    f32x4_v acc[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) acc[kb] = f32x4_v{0.f, 0.f, 0.f, 0.f};
    // tokens that see any of the wave's keys
    const int tok_lo = a.causal ? max(k0 - first, 0) : 0;
    const int tok_hi = (int)min((int64_t)n, a.window > 0 ? (int64_t)k0 + KPW - 1 + a.window - first : (int64_t)n);
    const int r_lo = (tok_lo * a.group) & ~15, r_hi = tok_hi * a.group;
    for (int r0 = r_lo + 16 * phase; r0 < r_hi; r0 += 16 * phases) {
      const int r = min(r0 + c16, rows - 1), tok = r / a.group;
      const int64_t row = c0 + tok;
      const int head = kvh * a.group + (r - tok * a.group);
      const T* const qp = reinterpret_cast<const T*>(a.x.p) + row * a.x.rs + (int64_t)head * a.x.hs;
      uint4 qf[NKS];
#pragma unroll
      for (int k = 0; k < NKS; ++k) qf[k] = ld16(qp + QS * k + (QS / 4) * g);
      const float2 st = a.stats[row * a.n_q + head];
      scale_frags(qf, a.factor, T(0));
      const Span sp = span_of(a, first + tok, len);
      const bool whole = present == kAll && !__ballot(r0 + c16 >= rows || sp.lo > k0 || sp.hi < k0 + KPW);
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) {
        f32x4_v s = f32x4_v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < NKS; ++k) mfma_step(s, kf[kb][k], qf[k], T(0));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (Q8) s[i] *= ks[kb][i];
          const float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale2, -st.x));
          if (whole) {
            acc[kb][i] = fmaf(e, st.y, acc[kb][i]);
          } else {
            const int at = 16 * kb + 4 * g + i;
            const bool sees = r0 + c16 < rows && k0 + at >= sp.lo && k0 + at < sp.hi && ((present >> at) & 1);
            acc[kb][i] += sees ? e * st.y : 0.f;
          }
        }
      }
    }
    __syncthreads();  // the last tile's sums have been read
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = acc[kb][i];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        if (c16 == 0) red[wave][16 * kb + 4 * g + i] = v;
      }
    __syncthreads();
    if (wave < key_waves && pr >= 0) {
      float v = 0.f;
      for (int p = 0; p < phases; ++p) v += red[wave + p * key_waves][lane];
      weights[pr + hoff] += v;
    }
  }
}

template <typename T, int ST, int DH>
hipError_t weigh_shape(const PagedAttnArgs& a, float* weights, int64_t keys, hipStream_t s) {
  typedef WeighCfg<T, ST, DH> C;
  const int64_t lists = (int64_t)a.c.n_kv * a.q.n;
  int kw = 4;
  while (kw > 1 && lists * ((keys + kw * C::KPW - 1) / (kw * C::KPW)) < 1024) kw /= 2;
  // (one more where the first key lies inside a tile)
  const int64_t tiles = std::min<int64_t>((keys + kw * C::KPW - 1) / (kw * C::KPW) + 1, std::max<int64_t>(1, (1 << 30) / lists));
  RFX_LAUNCH((paged_weigh_kernel<T, ST, DH>), dim3((unsigned)(tiles * lists)), dim3(256), 0, s, a, weights, kw, (int)tiles);
  return hipGetLastError();
}

template <typename T, int ST>
hipError_t weigh_store(const PagedAttnArgs& a, float* weights, int64_t keys, hipStream_t s) {
  if (a.c.dh == 64) return weigh_shape<T, ST, 64>(a, weights, keys, s);
  if (a.c.dh == 128) return weigh_shape<T, ST, 128>(a, weights, keys, s);
  return weigh_shape<T, ST, 256>(a, weights, keys, s);
}

}  // namespace

template <typename T>
hipError_t launch_paged_weighed_attention(const PagedAttnArgs& a, int store, float* weights, int64_t keys, hipStream_t s) {
  const hipError_t e = launch_mode<kWeigh, T>(a, store, s);
  if (e != hipSuccess) return e;
  if (store == REFLEX_STORE_FP8) return weigh_store<T, REFLEX_STORE_FP8>(a, weights, keys, s);
  if (store == REFLEX_STORE_INT8) return weigh_store<T, REFLEX_STORE_INT8>(a, weights, keys, s);
  return weigh_store<T, REFLEX_STORE_BF16>(a, weights, keys, s);
}
template hipError_t launch_paged_weighed_attention<float>(const PagedAttnArgs&, int, float*, int64_t, hipStream_t);
template hipError_t launch_paged_weighed_attention<bf16_t>(const PagedAttnArgs&, int, float*, int64_t, hipStream_t);

}  // namespace reflex
