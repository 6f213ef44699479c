// Attention that also adds up the weight that every key got: the kernels of
// paged_attention.h, which leave every row's maximum and sum, and the sums of
// the rows' probabilities for each key.
#include "paged_attention.h"

namespace reflex {

namespace {

// What the sums of a (sequence, K/V head) are about.
struct List {
  int b, kvh, n, rows, len, first;  // `n` tokens, the first of them token `first`; rows = tokens * group
  int64_t row;                      // first packed row
  int lo, hi;                       // keys that any of its rows sees
};
RFX_DEV bool list_of(const PagedAttnArgs& a, int list, List& q) {
  q.b = list / a.c.n_kv;
  q.kvh = list - q.b * a.c.n_kv;
  const int64_t c0 = min((int64_t)max(a.q.cu[q.b], 0), a.n_rows), c1 = min((int64_t)max(a.q.cu[q.b + 1], 0), a.n_rows);
  if (c1 <= c0) return false;
  q.row = c0;
  q.n = (int)(c1 - c0);
  q.rows = q.n * a.group;
  q.len = a.q.len[q.b];
  q.first = (int)((int64_t)q.len - a.q.cu[q.b + 1] + c0);
  q.lo = span_of(a, q.first, q.len).lo;
  q.hi = span_of(a, q.first + q.n - 1, q.len).hi;
  return true;
}

// From kept scores: a workgroup sums 4 LANES keys of one list, four of them a lane,
// and its 256 / LANES groups of lanes take the rows in turn.  64 lanes where rows
// are few, 16 where they are not: then there are more workgroups, with more rows
// under way in each (four chunks of 1,000 rows of 4 heads over 2,000 keys, 256 MB of
// scores, 536 us with 64 lanes, 65 with 16).  With few rows the maxima and sums
// are joined from the splits' here too, 16 rows at a time under the loads of their
// scores, so that this need not wait for the merge.
template <int LANES>
RFX_DEV void sum_kept(const PagedAttnArgs& a, float* weights, int tiles, int block) {
  constexpr int KT = 4 * LANES, G = 256 / LANES, SR = 16, PER = SR / G;
  __shared__ float red[G][KT];
  const int sub = threadIdx.x % LANES, grp = threadIdx.x / LANES, lane = threadIdx.x & 63;
  const int list = block / tiles;
  List q;
  if (!list_of(a, list, q)) return;
  const float inv_group = 1.f / (float)a.group;
  auto id_of = [&](int r, int& tok) __attribute__((always_inline)) {
    tok = divided(r, a.group, inv_group);
    return (q.row + tok) * a.n_q + q.kvh * a.group + (r - tok * a.group);
  };
  for (int64_t t0 = (q.lo & ~(KT - 1)) + (int64_t)(block - list * tiles) * KT; t0 < q.hi; t0 += (int64_t)tiles * KT) {
    const int key = (int)t0 + 4 * sub;
    const float* const at = a.scores + min((int64_t)key, a.score_pitch - 4);
    // rows of the tokens that see any of these keys
    const int r_lo = (a.causal ? max((int)t0 - q.first, 0) : 0) * a.group;
    const int r_hi = (int)min((int64_t)q.n, a.window > 0 ? t0 + KT - 1 + a.window - q.first : (int64_t)q.n) * a.group;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    auto load = [&](int r) __attribute__((always_inline)) {
      int tok;
      const int64_t id = id_of(r, tok);
      return *reinterpret_cast<const float4*>(at + id * a.score_pitch);
    };
    auto add = [&](int r, const float4& v, const float2& st) __attribute__((always_inline)) {
      Span sp = span_of(a, q.first + divided(r, a.group, inv_group), q.len);
      if (r >= r_hi) sp.hi = 0;
      const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc[i] += key + i >= sp.lo && key + i < sp.hi ? __builtin_amdgcn_exp2f(x[i] - st.x) * st.y : 0.f;
    };
    if (LANES == 64 && a.merge_with_sums) {
      for (int r0 = r_lo; r0 < r_hi; r0 += SR) {
        // (wave `grp` has rows r0 + 4 u + grp, here and in the sums)
        float4 v[PER];
        float2 w[PER];
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int r = min(r0 + G * u + grp, r_hi - 1);
          int tok;
          const int64_t id = id_of(r, tok);
          w[u] = lane < a.nsplit ? a.part_ml[id * a.nsplit + lane] : make_float2(kFloor, 0.f);
        }
#pragma unroll
        for (int u = 0; u < PER; ++u) v[u] = load(min(r0 + G * u + grp, r_hi - 1));
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const int r = r0 + G * u + grp;
          if (r >= r_hi) break;  // (alike in all of the wave)
          float M = w[u].x;
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, 64));
          const float L = warp_sum(w[u].y * __builtin_amdgcn_exp2f(w[u].x - M));
          add(r, v[u], make_float2(M, L == 0.f ? 0.f : 1.f / L));
        }
      }
    } else {
      constexpr int U = 4;  // rows of a thread under way
      for (int r0 = r_lo + grp; r0 < r_hi; r0 += U * G) {
        float4 v[U];
        float2 st[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          int tok;
          const int64_t id = id_of(min(r0 + u * G, r_hi - 1), tok);
          v[u] = *reinterpret_cast<const float4*>(at + id * a.score_pitch);
          st[u] = a.stats[id];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) add(r0 + u * G, v[u], st[u]);
      }
    }
    __syncthreads();  // the last tile's sums have been read
    *reinterpret_cast<float4*>(&red[grp][4 * sub]) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    __syncthreads();
    const int mine = (int)t0 + threadIdx.x;
    const int r = threadIdx.x < KT && mine >= q.lo && mine < q.hi ? page_row(a.c, a.q, q.b, mine) : -1;
    if (r >= 0) {
      float v = 0.f;
#pragma unroll
      for (int p = 0; p < G; ++p) v += red[p][threadIdx.x];
      weights[r + ((int64_t)q.kvh << a.c.shift)] += v;
    }
  }
}

template <int LANES>
__global__ __launch_bounds__(256) void paged_weigh_kept_kernel(const PagedAttnArgs a, float* weights, int tiles) {
  sum_kept<LANES>(a, weights, tiles, blockIdx.x);
}

// The same for few rows, and the merge of their results in the first workgroups:
// neither waits for the other (64 tokens over 15,409 fp8 keys: 13.5 us together,
// apart 5 and 10 and the gap between them).
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_weigh_merge_kernel(const PagedAttnArgs a, float* weights, int tiles, int merges) {
  if ((int)blockIdx.x < merges) merge_row<kKept, T, DH>(a, (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6));
  else sum_kept<64>(a, weights, tiles, blockIdx.x - merges);
}

// Without kept scores: they are formed again.  Each wave holds the fragments of
// its KPW keys in registers, and the four go over the query rows that see any of
// the workgroup's keys, 16 at a time, S^T = K Q^T as in the attention, so that a
// lane holds four keys of one query row and sums its own column of rows; the
// columns are joined at the end, over the lanes, always in the same order.  The
// query rows, and their maxima and sums, come through LDS, 64 a stage in two
// buffers.  The exponentials are what bounds it (16 cycles of the vector unit
// for 64 of them, with 8 for the rest, against 16 of the matrix unit): those of
// one block of rows stand between the products of the next.  Two pieces of 4,096
// rows of 32 heads of 128 over 8,192 keys (412 GFLOP, 1.6e9 exponentials) 465 us,
// vector issue 72 % and matrix units busy for 47 % of the cycles; with the
// exponentials behind the products 788, with each score's operations in a row 527.
// Three waves to a SIMD, which spill, 604.
template <typename T, int ST, int DH>
struct WeighCfg {
  static constexpr bool Q8 = ST == REFLEX_STORE_FP8 || ST == REFLEX_STORE_INT8, BF = sizeof(T) == 2;
  static constexpr int ES = Q8 ? 1 : (int)sizeof(T);
  static constexpr int RB = DH * ES;
  static constexpr int QS = BF ? 32 : 16;              // head dims of a product
  static constexpr int NKS = DH / QS;
  // blocks of 16 keys of a wave, with 64 registers of fragments at most
  static constexpr int NKB = DH * (int)sizeof(T) <= 256 ? 4 : 1024 / (DH * (int)sizeof(T));
  static constexpr int KPW = 16 * NKB, KT = 4 * KPW;   // keys of a wave, of a workgroup
  static constexpr int QR = 64;                        // query rows of a stage
  static constexpr int QB = DH * (int)sizeof(T);       // bytes of a query row
  static constexpr int NCH = QB / 16;
  static constexpr int STAGE = QR * QB;
};

struct WeighArgs {
  PagedAttnArgs a;
  float* weights;
  int lists, tiles;       // tiles of KT keys that the launch has for a list
  int row_splits;         // workgroups that divide a tile's rows; with more than one their sums go to `part`
  float* part;            // [row_splits][lists][pitch]
  int64_t pitch;          // keys that the table holds
};

template <typename T, int ST, int DH>
__global__ __launch_bounds__(256, (WeighCfg<T, ST, DH>::STAGE > 32 * 1024 ? 1 : 2)) void paged_weigh_kernel(const WeighArgs w) {
  typedef WeighCfg<T, ST, DH> C;
  constexpr bool Q8 = C::Q8, BF = C::BF;
  constexpr int RB = C::RB, QS = C::QS, NKS = C::NKS, NKB = C::NKB, KPW = C::KPW, KT = C::KT;
  constexpr int QR = C::QR, QB = C::QB, NCH = C::NCH;
  __shared__ __attribute__((aligned(1024))) unsigned char smem[2 * C::STAGE];
  __shared__ __attribute__((aligned(16))) float2 stats[2][QR];
  const PagedAttnArgs& a = w.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, c16 = lane & 15;
  // each XCD takes a run of lists, whose query rows its L2 then holds
  const int per_list = w.tiles * w.row_splits, all = per_list * w.lists;
  const int run = (all + 7) >> 3, id = (blockIdx.x & 7) * run + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= run || id >= all) return;
  const int list = id / per_list, rs = (id - list * per_list) % w.row_splits;
  List q;
  if (!list_of(a, list, q)) return;
  const int64_t hoff = (int64_t)q.kvh << a.c.shift;
  const float inv_group = 1.f / (float)a.group, scale2 = a.scale2;
  for (int64_t t0 = (q.lo & ~(KT - 1)) + (int64_t)((id - list * per_list) / w.row_splits) * KT; t0 < q.hi;
       t0 += (int64_t)w.tiles * KT) {
    const int k0 = (int)t0 + wave * KPW, key = k0 + lane;
    const int pr = lane < KPW && key >= q.lo && key < q.hi ? page_row(a.c, a.q, q.b, key) : -1;
    constexpr uint64_t kAll = ~0ull >> (64 - KPW);
    const uint64_t present = __ballot(pr >= 0);

    // rows that see any of the workgroup's keys: this workgroup's share of them, and
    // those that see all of the wave's keys
    const int tok_lo = a.causal ? max((int)t0 - q.first, 0) : 0;
    const int tok_hi = (int)min((int64_t)q.n, a.window > 0 ? t0 + KT - 1 + a.window - q.first : (int64_t)q.n);
    const int share = (max(tok_hi - tok_lo, 0) * a.group + QR * w.row_splits - 1) / (QR * w.row_splits) * QR;
    const int r_lo = min(tok_lo * a.group + rs * share, tok_hi * a.group), r_hi = min(r_lo + share, tok_hi * a.group);
    const int64_t sees_lo = a.causal ? (int64_t)(k0 + KPW - 1 - q.first) * a.group : 0;
    const int64_t sees_hi = a.window > 0 ? ((int64_t)k0 + a.window - q.first) * a.group : q.rows;
    const bool keys_whole = present == kAll && k0 + KPW <= q.hi && k0 >= q.lo;
    // (rows as 32 bits: a list has fewer than 2^23)
    const int all_lo = keys_whole ? (int)max(sees_lo, (int64_t)r_lo) : r_hi;
    const int all_hi = (int)min(sees_hi, (int64_t)r_hi);

    // A stage's copies.  Where the group divides 64 a stage's rows are whole tokens,
    // and each copy needs the stage's base and the lane's offset, which stays; else,
    // and where the last stage is not full, each lane finds the place of one row.
    auto place = [&](int r, int& stat) __attribute__((always_inline)) {
      const int tok = divided(r, a.group, inv_group), head = q.kvh * a.group + r - tok * a.group;
      stat = (int)((q.row + tok) * a.n_q) + head;
      return a.x.p + ((q.row + tok) * a.x.rs + (int64_t)head * a.x.hs) * (int64_t)sizeof(T);
    };
    constexpr int NC = C::STAGE / 4096;  // copies of a wave
    const int64_t stage_bytes = (int64_t)(QR / a.group) * a.x.rs * (int64_t)sizeof(T);
    const bool easy = QR % a.group == 0 && r_lo % a.group == 0 && a.x.rs >= 0 && a.x.hs >= 0 &&
                      stage_bytes + a.group * a.x.hs * (int64_t)sizeof(T) < (int64_t)1 << 31;
    int base_stat;
    const char* base_at = place(min(r_lo, q.rows - 1), base_stat);
    const float* base_stats = reinterpret_cast<const float*>(a.stats + base_stat);
    uint32_t off[NC], stat_off;
    {
      const int r = wave * 32 + (lane >> 1), tok = divided(r, a.group, inv_group);
      stat_off = (uint32_t)(tok * a.n_q + r - tok * a.group) * 8 + (lane & 1) * 4;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int p = wave * (C::STAGE / 64) + j * 64 + lane, rj = p / NCH, tj = divided(rj, a.group, inv_group);
        off[j] = (uint32_t)((tj * a.x.rs + (rj - tj * a.group) * a.x.hs) * (int64_t)sizeof(T)) +
                 (((p % NCH) ^ (rj & (NCH - 1) & 15)) << 4);
      }
    }
    auto copy = [&](int r0, int buf) __attribute__((always_inline)) {
      unsigned char* const dst = smem + buf * C::STAGE + wave * (C::STAGE / 4);
      float* const dst_stats = reinterpret_cast<float*>(stats[buf]) + wave * 64;
      if (easy && r0 + QR <= q.rows) {
        const int64_t n = (r0 - r_lo) / QR;
        const char* const at = base_at + n * stage_bytes;
#pragma unroll
        for (int j = 0; j < NC; ++j) lds_dma16(at, off[j], dst + j * 1024);
        if (wave < 2) lds_dma4(reinterpret_cast<const char*>(base_stats + n * (QR / a.group) * 2 * a.n_q) + stat_off, dst_stats);
      } else {
        int stat;
        const uint64_t mine = (uint64_t)place(min(r0 + lane, q.rows - 1), stat);
        const int lo32 = (int)mine, hi32 = (int)(mine >> 32);
#pragma unroll 1
        for (int j = 0; j < NC; ++j) {
          const int p = wave * (C::STAGE / 64) + j * 64 + lane, rj = p / NCH, ch = (p % NCH) ^ (rj & (NCH - 1) & 15);
          const uint64_t src = (uint32_t)__shfl(lo32, rj, 64) | (uint64_t)(uint32_t)__shfl(hi32, rj, 64) << 32;
          lds_dma16(reinterpret_cast<const char*>(src) + ch * 16, dst + j * 1024);
        }
        if (wave < 2) {
          const int at = __shfl(stat, wave * 32 + (lane >> 1), 64);
          lds_dma4(reinterpret_cast<const float*>(a.stats + at) + (lane & 1), dst_stats);
        }
      }
    };
    auto turn = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    __syncthreads();  // the last tile's stage has been read
    if (r_lo < r_hi) copy(r_lo, 0);

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
      scale_frags(kf[kb], a.factor, T(0));  // (as well as the queries)
      const float mine = Q8 && r >= 0 ? a.c.k_scale[(int64_t)r + hoff] : 1.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) ks[kb][i] = __shfl(mine, 4 * g + i, 64);
    }
    f32x4_v acc[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) acc[kb] = f32x4_v{0.f, 0.f, 0.f, 0.f};
    turn();
    // (the compiler's own wait for the fragments has to lie before the loop: it
    // would be one for the stage's copies too)
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int k = 0; k < NKS; ++k)
        asm volatile("" : "+v"(kf[kb][k].x), "+v"(kf[kb][k].y), "+v"(kf[kb][k].z), "+v"(kf[kb][k].w));
    // scores of a block whose sums are not taken yet, at first of none
    f32x4_v sa[NKB], sb[NKB];
    float2 sta = make_float2(INFINITY, 0.f), stb;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) sa[kb] = f32x4_v{0.f, 0.f, 0.f, 0.f};
    constexpr int NV = 4 * NKB;  // scores of a lane in a block
    auto exponent = [&](const f32x4_v (&s)[NKB], const float2& st, int v) __attribute__((always_inline)) {
      const int kb = v >> 2, i = v & 3;
      return fmaf(Q8 ? s[kb][i] * ks[kb][i] : s[kb][i], scale2, -st.x);
    };
    auto fragments = [&](int buf, int u, uint4 (&qf)[NKS]) __attribute__((always_inline)) {
      const unsigned char* const at = smem + buf * C::STAGE + (16 * u + c16) * QB;
#pragma unroll
      for (int k = 0; k < NKS; ++k) qf[k] = ld16(at + (((4 * k + g) ^ (c16 & (NCH - 1))) << 4));
    };
    auto block = [&](int buf, int u, const f32x4_v (&s)[NKB], const float2& st, f32x4_v (&z)[NKB], float2& zst)
        __attribute__((always_inline)) {
      uint4 qf[NKS];
      fragments(buf, u, qf);
      zst = stats[buf][16 * u + c16];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) z[kb] = f32x4_v{0.f, 0.f, 0.f, 0.f};
      // a step takes the exponent of one score, 2 to the power of the one before and
      // the sum of that before it, so that no operation waits for its neighbour
      constexpr int NM = NKB * NKS;
      float x[NV + 2], e[NV + 1];
      x[0] = exponent(s, st, 0);
#pragma unroll
      for (int m = 0; m < NM; ++m) {
        mfma_step(z[m % NKB], kf[m % NKB][m / NKB], qf[m / NKB], T(0));
#pragma unroll
        for (int v = m * (NV + 1) / NM; v < (m + 1) * (NV + 1) / NM; ++v) {
          if (v + 1 < NV) x[v + 1] = exponent(s, st, v + 1);
          if (v < NV) e[v] = __builtin_amdgcn_exp2f(x[v]);
          if (v > 0) acc[(v - 1) >> 2][(v - 1) & 3] = fmaf(e[v - 1], st.y, acc[(v - 1) >> 2][(v - 1) & 3]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    int buf = 0;
#pragma unroll 1
    for (int s0 = r_lo; s0 < r_hi; s0 += QR) {
      if (s0 + QR < r_hi) copy(s0 + QR, buf ^ 1);
      if (s0 >= all_lo && s0 + QR <= all_hi) {
        block(buf, 0, sa, sta, sb, stb);
        block(buf, 1, sb, stb, sa, sta);
        block(buf, 2, sa, sta, sb, stb);
        block(buf, 3, sb, stb, sa, sta);
      } else {
#pragma unroll 1
        for (int u = 0; u < QR / 16; ++u) {
          const int r0 = s0 + 16 * u;
          uint4 qf[NKS];
          fragments(buf, u, qf);
          const float2 st = stats[buf][16 * u + c16];
          const Span sp = span_of(a, q.first + divided(min(r0 + c16, q.rows - 1), a.group, inv_group), q.len);
          // this lane's keys that the row sees, as bits 16 kb + i
          uint64_t seen = present;
          const int lo = max(sp.lo - k0, 0), hi = min(sp.hi - k0, KPW);
          seen = hi > lo && r0 + c16 < r_hi ? seen & (~0ull << lo) & (~0ull >> (64 - hi)) : 0;
          seen >>= 4 * g;
          asm volatile("" : "+v"(seen));  // (not formed ahead of the loop)
#pragma unroll
          for (int kb = 0; kb < NKB; ++kb) {
            f32x4_v s = f32x4_v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NKS; ++k) mfma_step(s, kf[kb][k], qf[k], T(0));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float e = __builtin_amdgcn_exp2f(fmaf(Q8 ? s[i] * ks[kb][i] : s[i], scale2, -st.x)) * st.y;
              acc[kb][i] += (seen >> (16 * kb + i)) & 1 ? e : 0.f;
            }
          }
        }
      }
      turn();
      buf ^= 1;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
      acc[v >> 2][v & 3] = fmaf(__builtin_amdgcn_exp2f(exponent(sa, sta, v)), sta.y, acc[v >> 2][v & 3]);
    // over the lanes; lane 16 g' has keys 16 kb + 4 g' + i
    float mine = 0.f;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float v = acc[kb][i];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        // to lane 16 kb + 4 g + i
        v = __shfl(v, (lane >> 2 & 3) * 16, 64);
        mine = lane >> 4 == kb && (lane & 3) == i ? v : mine;
      }
    if (pr >= 0) {
      if (w.row_splits == 1) w.weights[pr + hoff] += mine;
      else w.part[((int64_t)rs * w.lists + list) * w.pitch + key] = mine;
    }
  }
}

// The row splits' sums joined, in order.
__global__ __launch_bounds__(256) void paged_weigh_join_kernel(const WeighArgs w, int tiles) {
  const PagedAttnArgs& a = w.a;
  const int list = blockIdx.x / tiles;
  List q;
  if (!list_of(a, list, q)) return;
  for (int64_t key = q.lo + (int64_t)(blockIdx.x - list * tiles) * 256 + threadIdx.x; key < q.hi; key += (int64_t)tiles * 256) {
    const int r = page_row(a.c, a.q, q.b, key);
    if (r < 0) continue;
    float v = 0.f;
    for (int s = 0; s < w.row_splits; ++s) v += w.part[((int64_t)s * w.lists + list) * w.pitch + key];
    w.weights[r + ((int64_t)q.kvh << a.c.shift)] += v;
  }
}

template <typename T, int ST, int DH>
hipError_t weigh_shape(const PagedAttnArgs& a, float* weights, int64_t keys, hipStream_t s) {
  typedef WeighCfg<T, ST, DH> C;
  WeighArgs w;
  w.a = a;
  w.weights = weights;
  w.lists = a.c.n_kv * a.q.n;
  // (one more where the first key lies inside a tile)
  w.tiles = (int)std::min<int64_t>((keys + C::KT - 1) / C::KT + 1, std::max<int64_t>(1, (1 << 22) / w.lists));
  w.part = a.scores;
  w.pitch = a.score_pitch;
  w.row_splits = a.row_splits;
  const int64_t blocks = (int64_t)w.tiles * w.lists * w.row_splits;
  RFX_LAUNCH((paged_weigh_kernel<T, ST, DH>), dim3((unsigned)((blocks + 7) / 8 * 8)), dim3(256), 0, s, w);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && w.row_splits > 1) {
    const int tiles = (int)std::min<int64_t>((keys + 255) / 256, std::max<int64_t>(1, (1 << 22) / w.lists));
    RFX_LAUNCH(paged_weigh_join_kernel, dim3((unsigned)(tiles * w.lists)), dim3(256), 0, s, w, std::max(tiles, 1));
    e = hipGetLastError();
  }
  return e;
}

template <typename T, int ST>
hipError_t weigh_store(const PagedAttnArgs& a, float* weights, int64_t keys, hipStream_t s) {
  if (a.c.dh == 64) return weigh_shape<T, ST, 64>(a, weights, keys, s);
  if (a.c.dh == 128) return weigh_shape<T, ST, 128>(a, weights, keys, s);
  return weigh_shape<T, ST, 256>(a, weights, keys, s);
}

}  // namespace

// Few rows a sequence are bound by reading the keys, and to write and read their
// scores is less than to read the keys again (64 tokens of 8 heads of 256: 32
// bytes a key against 256 to 1,024; over fp8 pages 11 us more in the attention and
// 10 for the sums against 136 with the scores formed again).  fp32 has the
// products to save.  256 MB of
// scores at most: a table for much longer sequences than there are would ask
// for a workspace that is hardly used.
//
// Else the rows of a list are divided where lists and tiles of 256 keys alone
// would not make sixteen workgroups for every CU, with 512 rows at least to each
// (and not over a table of no pages, which leaves no sums to join).
PagedWeighPlan paged_weigh_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q, int dtype) {
  const int group = n_q / c.n_kv_heads;
  const int bm = rows_of_tile(n_rows, b.n_seqs, group, c.n_kv_heads, c.head_dim, dtype);
  const int64_t cap = (int64_t)b.max_pages * c.page_size, pitch = (cap + 63) / 64 * 64;
  const int64_t keys = b.max_length > 0 && b.max_length < cap ? b.max_length : cap;
  PagedWeighPlan p{0, pitch, (size_t)(pitch * (n_rows * n_q + 1) * 4),  // (and one that rows of no tile write to)
                   n_rows * group <= 16 * (int64_t)b.n_seqs};
  if (bm <= 32 && p.bytes <= (256 << 20)) return p;
  const int64_t lists = (int64_t)c.n_kv_heads * b.n_seqs;
  const int64_t rows = n_rows * group / std::max<int64_t>(1, std::min<int64_t>(b.n_seqs, n_rows));
  p.row_splits = (int)std::max<int64_t>(1, std::min<int64_t>({4096 / (lists * ((keys + 255) / 256) + 1), rows / 512, 64}));
  p.bytes = (size_t)(lists * p.row_splits * pitch * 4);
  if (p.row_splits == 1 || p.bytes == 0 || p.bytes > (64 << 20)) p = {1, 0, 0, false};
  return p;
}

template <typename T>
hipError_t launch_paged_weighed_attention(const PagedAttnArgs& a, int store, float* weights, int64_t keys, bool few,
                                          hipStream_t s) {
  const hipError_t e = a.row_splits ? launch_mode<kWeigh, T>(a, store, s) : launch_mode<kKept, T>(a, store, s);
  if (e != hipSuccess) return e;
  if (a.row_splits == 0) {
    const int64_t lists = (int64_t)a.c.n_kv * a.q.n;
    const int64_t kt = few ? 256 : 64;
    const int64_t tiles = std::min<int64_t>((keys + kt - 1) / kt + 1, std::max<int64_t>(1, (1 << 22) / lists));
    const unsigned grid = (unsigned)(tiles * lists);
    if (a.merge_with_sums) {
      const unsigned merges = (unsigned)((a.n_rows * a.n_q + 3) / 4);
      if (a.c.dh == 64) RFX_LAUNCH((paged_weigh_merge_kernel<T, 64>), dim3(merges + grid), dim3(256), 0, s, a, weights, (int)tiles, (int)merges);
      else if (a.c.dh == 128) RFX_LAUNCH((paged_weigh_merge_kernel<T, 128>), dim3(merges + grid), dim3(256), 0, s, a, weights, (int)tiles, (int)merges);
      else RFX_LAUNCH((paged_weigh_merge_kernel<T, 256>), dim3(merges + grid), dim3(256), 0, s, a, weights, (int)tiles, (int)merges);
    } else if (few) {
      RFX_LAUNCH(paged_weigh_kept_kernel<64>, dim3(grid), dim3(256), 0, s, a, weights, (int)tiles);
    } else {
      RFX_LAUNCH(paged_weigh_kept_kernel<16>, dim3(grid), dim3(256), 0, s, a, weights, (int)tiles);
    }
    return hipGetLastError();
  }
  if (store == REFLEX_STORE_FP8) return weigh_store<T, REFLEX_STORE_FP8>(a, weights, keys, s);
  if (store == REFLEX_STORE_INT8) return weigh_store<T, REFLEX_STORE_INT8>(a, weights, keys, s);
  return weigh_store<T, REFLEX_STORE_BF16>(a, weights, keys, s);
}
template hipError_t launch_paged_weighed_attention<float>(const PagedAttnArgs&, int, float*, int64_t, bool, hipStream_t);
template hipError_t launch_paged_weighed_attention<bf16_t>(const PagedAttnArgs&, int, float*, int64_t, bool, hipStream_t);

}  // namespace reflex
