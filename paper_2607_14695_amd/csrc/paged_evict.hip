// Eviction: a long sequence keeps, for each K/V head, its first tokens, its last
// ones and those of greatest weight between them, moved together in order.
//
// Two kernels.  The first chooses (one workgroup to a sequence and K/V head);
// the second moves rows, scales and weights and writes the lengths.
#include <algorithm>

#include "paged.h"

namespace reflex {

namespace {

// Unsigned keys in the order of the weights: -0 is 0, and a NaN is -infinity.
// A token whose page is absent has the key 0, below all of them.
RFX_DEV uint32_t order_of(float w) {
  if (!(w == w)) w = -INFINITY;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

constexpr int kBins = 2048;
constexpr int kCopies = 4;        // of the histogram: a lane adds to copy lane % 4, which divides the conflicts of
constexpr int kPitch = kBins + 16;  // equal digits; the copies' equal bins lie in different banks
constexpr int kTable = 4096;      // table entries held in LDS, if that is all of them

// The least of the `need` greatest keys is found digit by digit (11, 11 and 10
// bits): a histogram of the digits of those keys that agree so far, summed from
// the top.  Counts are whole numbers, so the order of the additions does not
// matter.  Then every wave counts the greater and the equal keys of its tokens,
// and writes the chosen ones behind those of the waves before it.
//
// A wave has a run of tokens, 64 at a time, the first HELD of these in registers
// with their page rows (longer sequences than the launch expected read the others
// again).  32 lists of 6,360 to 15,408 tokens 14 us, with keys in LDS 24: vector
// issue bounds it, 60 % of the cycles of the CUs that it runs on, one to a list.
// Places behind the last token have the key 0 as absent tokens do: they come after
// all others, and there are tokens enough before them.
template <int HELD>
__global__ __launch_bounds__(1024) void paged_choose_kernel(const PagedEvictArgs a) {
  __shared__ uint32_t hist[kCopies * kPitch];
  __shared__ int32_t table[kTable];
  __shared__ __attribute__((aligned(16))) int part[16], part_eq[16];
  __shared__ int found, above;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t list = blockIdx.x;
  const int b = (int)(list / a.c.n_kv), g = (int)(list - (int64_t)b * a.c.n_kv);
  const int raw = a.q.len[b];
  const int64_t cap = (int64_t)a.q.max_pages << a.c.shift;
  const int len = (int)min((int64_t)max(raw, 0), cap);
  int32_t* const kept = a.kept ? a.kept + list * a.keep : nullptr;
  int32_t* const from = a.from + list * a.keep;
  if (tid == 0) a.cut[list] = make_int2(raw, len > a.keep ? len : 0);
  if (len <= a.keep) {
    if (kept)
      for (int i = tid; i < a.keep; i += 1024) kept[i] = i < len ? i : -1;
    return;
  }
  const int lo = a.sinks, hi = len - a.recent, n = hi - lo;
  const int need = a.keep - a.sinks - a.recent;
  const int shift = a.c.shift, n_kv = a.c.n_kv, n_pages = a.c.n_pages;
  const int hoff = g << shift;
  const int entries = ((len - 1) >> shift) + 1;
  const bool in_lds = entries <= kTable;
  const int32_t* const mine = a.q.table + (int64_t)b * a.q.max_pages;
  if (in_lds)
    for (int e = tid; e < entries; e += 1024) table[e] = mine[e];
  for (int i = tid; i < kCopies * kPitch; i += 1024) hist[i] = 0;
  __syncthreads();
  // page row of token j < len, or -1
  auto row_of = [&](int j) __attribute__((always_inline)) {
    const int page = in_lds ? table[j >> shift] : mine[j >> shift];
    return (unsigned)page < (unsigned)n_pages ? ((page * n_kv) << shift) + (j & ((1 << shift) - 1)) + hoff : -1;
  };
  const int chunks = (n + 1023) / 1024, first = wave * chunks * 64 + lane;
  uint32_t key[HELD];
  int place[HELD];
  {
    float w[HELD];
#pragma unroll
    for (int t = 0; t < HELD; ++t) place[t] = t < chunks ? row_of(lo + min(first + 64 * t, n - 1)) : -1;
#pragma unroll
    for (int t = 0; t < HELD; ++t) w[t] = a.weights[max(place[t], 0)];
#pragma unroll
    for (int t = 0; t < HELD; ++t) key[t] = place[t] < 0 || first + 64 * t >= n ? 0u : order_of(w[t]);
  }
  // f(token, page row, key) of the run's places; all of the wave's lanes come to it
  auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < HELD; ++t)
      if (t < chunks) f(first + 64 * t, place[t], key[t]);
    for (int t = HELD; t < chunks; ++t) {
      const int j = first + 64 * t, r = j < n ? row_of(lo + j) : -1;
      f(j, r, r < 0 ? 0u : order_of(a.weights[r]));
    }
  };
  // sum of the waves before this one
  auto before_wave = [&](const int* p) __attribute__((always_inline)) {
    int s = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += w < wave ? p[w] : 0;
    return s;
  };

  uint32_t top = 0;  // the digits found so far
  int left = need;   // of the keys that have them, how many are chosen
  uint32_t* const bins = hist + (lane & (kCopies - 1)) * kPitch;
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int at = pass == 0 ? 21 : pass == 1 ? 10 : 0, last = pass == 2 ? 1023 : 2047;
    if (pass == 0)
      each([&](int, int, uint32_t k) __attribute__((always_inline)) { atomicAdd(&bins[k >> 21], 1u); });
    else
      each([&](int, int, uint32_t k) __attribute__((always_inline)) {
        if (k >> (pass == 1 ? 21 : 10) == top) atomicAdd(&bins[(k >> at) & last], 1u);
      });
    __syncthreads();
    // thread t has bins 2 t', 2 t' + 1 with t' counted from the top; it leaves zeros
    const int t = 1023 - tid;
    int h0 = 0, h1 = 0;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      uint2* const p = reinterpret_cast<uint2*>(&hist[c * kPitch + 2 * t]);
      const uint2 h = *p;
      *p = make_uint2(0, 0);
      h0 += (int)h.x;
      h1 += (int)h.y;
    }
    const int sum = lanes_up_to(h0 + h1);
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    const int before = sum - h0 - h1 + before_wave(part);
    // exactly one bin holds the left-th key from the top
    if (before < left && before + h1 >= left) {
      found = 2 * t + 1;
      above = before;
    } else if (before + h1 < left && before + h1 + h0 >= left) {
      found = 2 * t;
      above = before + h1;
    }
    __syncthreads();
    top = top << (pass == 2 ? 10 : 11) | (uint32_t)found;
    left -= above;
  }
  if (need == 0) {
    top = 0xffffffffu;
    left = 0;
  }

  int more = 0, same = 0;
  each([&](int, int, uint32_t k) __attribute__((always_inline)) {
    more += k > top;
    same += k == top;
  });
  more = lanes_up_to(more);
  same = lanes_up_to(same);
  __syncthreads();  // (the last pass's sums have been read)
  if (lane == 63) {
    part[wave] = more;
    part_eq[wave] = same;
  }
  __syncthreads();
  more = before_wave(part);
  same = before_wave(part_eq);
  const uint64_t below = (1ull << lane) - 1;
  auto put = [&](int i, int j, int r) __attribute__((always_inline)) {
    from[i] = r;
    if (kept) kept[i] = j;
  };
  each([&](int j, int r, uint32_t k) __attribute__((always_inline)) {
    const uint64_t gt = __ballot(k > top), eq = __ballot(k == top);
    const int eq_before = same + __popcll(eq & below);
    if (k > top || (k == top && eq_before < left))
      put(lo + more + __popcll(gt & below) + min(eq_before, left), lo + j, r);
    more += __popcll(gt);
    same += __popcll(eq);
  });
  for (int i = tid; i < a.sinks; i += 1024) put(i, i, row_of(i));
  for (int i = tid; i < a.recent; i += 1024) put(a.keep - a.recent + i, hi + i, row_of(hi + i));
}

// Token i of a list from page row from[i], in order: from[i] is that of a token
// >= i, so a place is never read after a later step has written it, and within a
// step everything is read before anything is written.  A workgroup moves a
// column of the rows: kColumn bytes of K or of V, the scales of one of them, or
// the weights, so that the columns need not wait for each other.  The next
// step's values are under way while this one's are stored (the places of this
// step's tokens are behind it, the next step's come from further on), and the
// places of the step after that.
//
// Bound by memory: 32 lists of 7,000 rows of 512 bytes, K and V (418 MB read and
// written), 94 us, 4.4 TB/s of rows that lie apart, of the 5.1 of a large copy.
// Columns of 64 bytes take 125 us, of 256 98, of 512 141 (too few workgroups); 1,024
// threads 103; without the next step's loads ahead 165.
constexpr int kColumn = 128, kMoveThreads = 512;
constexpr int kMoveUnits = 8;  // pieces of a thread and step
template <typename U>
RFX_DEV void move_column(const PagedEvictArgs& a, int b, const int32_t* from, int64_t hoff, char* base, int64_t row_bytes,
                         int lanes, int offset) {
  const int tid = threadIdx.x, per = kMoveThreads / lanes, step = per * kMoveUnits;
  const int sub = tid / lanes, at = offset + (tid - sub * lanes) * (int)sizeof(U);
  const int64_t table = (int64_t)b * a.q.max_pages;
  const int slots = 1 << a.c.shift;
  // what is behind the last token takes the last one's place, and is not stored
  int src[2][kMoveUnits], page[2][kMoveUnits];
  auto places = [&](int i0, int (&s)[kMoveUnits], int (&p)[kMoveUnits]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {
      const int i = min(i0 + u * per + sub, a.keep - 1);
      s[u] = from[i];
      p[u] = a.q.table[table + (i >> a.c.shift)];  // (a sequence that is cut has a table for more than `keep`)
    }
  };
  U v[kMoveUnits], next[kMoveUnits];
  auto load = [&](const int (&s)[kMoveUnits], U (&x)[kMoveUnits]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u)
      x[u] = *reinterpret_cast<const U*>(base + (int64_t)max(s[u], 0) * row_bytes + at);
  };
  places(0, src[0], page[0]);
  places(step, src[1], page[1]);
  load(src[0], v);
  for (int i0 = 0; i0 < a.keep; i0 += step) {
    int src2[kMoveUnits], page2[kMoveUnits];
    load(src[1], next);
    places(i0 + 2 * step, src2, page2);
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {  // this step's values are there
      if constexpr (sizeof(U) == 16) asm volatile("" : "+v"(v[u].x), "+v"(v[u].y), "+v"(v[u].z), "+v"(v[u].w));
      else asm volatile("" : "+v"(v[u]));
    }
    asm volatile("s_barrier" ::: "memory");  // in every wave
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {
      const int i = i0 + u * per + sub;
      const int dst = ((page[0][u] * a.c.n_kv) << a.c.shift) + (i & (slots - 1)) + (int)hoff;
      if (i < a.keep && (unsigned)page[0][u] < (unsigned)a.c.n_pages && dst != src[0][u])
        *reinterpret_cast<U*>(base + (int64_t)dst * row_bytes + at) = src[0][u] < 0 ? U{} : v[u];
    }
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {
      v[u] = next[u];
      src[0][u] = src[1][u];
      page[0][u] = page[1][u];
      src[1][u] = src2[u];
      page[1][u] = page2[u];
    }
  }
}

__global__ __launch_bounds__(kMoveThreads) void paged_move_kernel(const PagedEvictArgs a, int row_bytes, int column, int scaled) {
  const int columns = row_bytes / column, all = 2 * columns + 2 * scaled + 1;
  const int64_t list = blockIdx.x / all;
  const int col = blockIdx.x - (int)list * all;
  const int b = (int)(list / a.c.n_kv), g = (int)(list - (int64_t)b * a.c.n_kv);
  const int2 cut = a.cut[list];  // (length as it was given, length that is cut or 0)
  // (a length past the table may be longer than `keep` without a token to move)
  if (g == 0 && col == all - 1 && threadIdx.x == 0) a.lengths[b] = min(cut.x, a.keep);
  if (!cut.y) return;
  const int32_t* const from = a.from + list * a.keep;
  const int64_t hoff = (int64_t)g << a.c.shift;
  if (col < 2 * columns) {
    const int side = col / columns, x = col - side * columns;
    move_column<uint4>(a, b, from, hoff, side ? a.c.v : a.c.k, row_bytes, column / 16, x * column);
  } else if (col < all - 1) {
    move_column<float>(a, b, from, hoff, reinterpret_cast<char*>(col == 2 * columns ? a.c.k_scale : a.c.v_scale), 4, 1, 0);
  } else {
    move_column<float>(a, b, from, hoff, reinterpret_cast<char*>(a.weights), 4, 1, 0);
    __syncthreads();
    for (int j = a.keep + threadIdx.x; j < cut.y; j += kMoveThreads) {
      const int r = page_row(a.c, a.q, b, j);
      if (r >= 0) a.weights[r + hoff] = 0.f;
    }
  }
}

}  // namespace

hipError_t launch_paged_evict(const PagedEvictArgs& a, int elem_bytes, int scaled, int64_t keys, hipStream_t s) {
  const dim3 lists((unsigned)(a.c.n_kv * a.q.n));
  if (keys <= 4096) RFX_LAUNCH(paged_choose_kernel<4>, lists, dim3(1024), 0, s, a);
  else if (keys <= 16384) RFX_LAUNCH(paged_choose_kernel<16>, lists, dim3(1024), 0, s, a);
  else RFX_LAUNCH(paged_choose_kernel<32>, lists, dim3(1024), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int row_bytes = a.c.dh * elem_bytes, column = std::min(row_bytes, kColumn);
  const dim3 grid((unsigned)((int64_t)a.q.n * a.c.n_kv * (2 * (row_bytes / column) + 2 * scaled + 1)));
  RFX_LAUNCH(paged_move_kernel, grid, dim3(kMoveThreads), 0, s, a, row_bytes, column, scaled);
  return hipGetLastError();
}

}  // namespace reflex
