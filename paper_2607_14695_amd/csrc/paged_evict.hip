// Eviction: a long sequence keeps, for each K/V head, its first tokens, its last
// ones and those of greatest weight between them, moved together in order.
//
// Two kernels.  The first chooses (one workgroup to a sequence and K/V head);
// the second moves rows, scales and weights and writes the lengths.
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

constexpr int kHeld = 32768;  // keys held in LDS; those of a longer sequence are read again
constexpr int kBins = 2048;

// The least of the `need` greatest keys is found digit by digit (11, 11 and 10
// bits): a histogram of the digits of those keys that agree so far, summed from
// the top.  Counts are whole numbers, so the order of the additions does not
// matter.  Then every wave counts the greater and the equal keys of a run of
// tokens, and writes the chosen ones behind those of the waves before it.
__global__ __launch_bounds__(1024) void paged_choose_kernel(const PagedEvictArgs a) {
  __shared__ uint32_t held[kHeld];
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part[16];
  __shared__ int found, above;
  __shared__ int2 waves[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  const int64_t hoff = (int64_t)g << a.c.shift;
  auto row_of = [&](int j) __attribute__((always_inline)) {
    const int r = page_row(a.c, a.q, b, j);
    return r < 0 ? -1 : r + (int)hoff;
  };
  auto read = [&](int j) __attribute__((always_inline)) {
    const int r = row_of(lo + j);
    return r < 0 ? 0u : order_of(a.weights[r]);
  };
  for (int j = tid; j < min(n, kHeld); j += 1024) held[j] = read(j);
  auto key_of = [&](int j) __attribute__((always_inline)) { return j < kHeld ? held[j] : read(j); };

  uint32_t top = 0;   // the digits found so far
  int left = need;    // of the keys that have them, how many are chosen
  for (int pass = 0; pass < 3 && need > 0; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
    for (int i = tid; i < kBins; i += 1024) hist[i] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += 1024) {
      const uint32_t k = key_of(j);
      if (pass == 0 || k >> (pass == 1 ? 21 : 10) == top) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    // thread t has bins 2 t', 2 t' + 1 with t' counted from the top
    const int t = 1023 - tid;
    const uint32_t h1 = hist[2 * t + 1], h0 = hist[2 * t];
    uint32_t sum = h0 + h1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t v = __shfl_up(sum, o, 64);
      if (lane >= o) sum += v;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    uint32_t before = sum - h0 - h1;
    for (int w = 0; w < wave; ++w) before += part[w];
    // exactly one bin holds the left-th key from the top
    if (before < (uint32_t)left && before + h1 >= (uint32_t)left) {
      found = 2 * t + 1;
      above = (int)before;
    } else if (before + h1 < (uint32_t)left && before + h1 + h0 >= (uint32_t)left) {
      found = 2 * t;
      above = (int)(before + h1);
    }
    __syncthreads();
    top = top << (pass == 2 ? 10 : 11) | (uint32_t)found;
    left -= above;
  }
  if (need == 0) {
    top = 0xffffffffu;
    left = 0;
  }
  __syncthreads();

  // runs of whole 64s
  const int run = (n + 1023) / 1024 * 64, j0 = min(wave * run, n), j1 = min(j0 + run, n);
  int more = 0, same = 0;
  for (int j = j0; j < j1; j += 64) {
    const uint32_t k = j + lane < j1 ? key_of(j + lane) : 0;
    more += __popcll(__ballot(j + lane < j1 && k > top));
    same += __popcll(__ballot(j + lane < j1 && k == top));
  }
  if (lane == 0) waves[wave] = make_int2(more, same);
  __syncthreads();
  more = same = 0;
  for (int w = 0; w < wave; ++w) {
    more += waves[w].x;
    same += waves[w].y;
  }
  const uint64_t below = (1ull << lane) - 1;
  auto put = [&](int i, int j) __attribute__((always_inline)) {
    from[i] = row_of(j);
    if (kept) kept[i] = j;
  };
  for (int j = j0; j < j1; j += 64) {
    const bool in = j + lane < j1;
    const uint32_t k = in ? key_of(j + lane) : 0;
    const uint64_t gt = __ballot(in && k > top), eq = __ballot(in && k == top);
    const int eq_before = same + __popcll(eq & below);
    const bool take = in && (k > top || (k == top && eq_before < left));
    if (take) put(lo + more + __popcll(gt & below) + min(eq_before, left), lo + j + lane);
    more += __popcll(gt);
    same += __popcll(eq);
  }
  for (int i = tid; i < a.sinks; i += 1024) put(i, i);
  for (int i = tid; i < a.recent; i += 1024) put(a.keep - a.recent + i, hi + i);
}

// Token i of a list from page row from[i], in order: from[i] is that of a token
// >= i, so a place is never read after a later step has written it, and within a
// step everything is read before anything is written.  A workgroup moves a
// column of the rows: COLUMN bytes of K or of V, the scales of one of them, or
// the weights, so that the columns need not wait for each other.
constexpr int kColumn = 128, kMoveThreads = 512, kMoveUnits = 4;
template <typename U>
RFX_DEV void move_column(const PagedEvictArgs& a, int b, const int32_t* from, int64_t hoff, char* base, int64_t row_bytes,
                         int lanes, int offset) {
  const int tid = threadIdx.x, per = kMoveThreads / lanes;
  const int sub = tid / lanes, at = offset + (tid - sub * lanes) * (int)sizeof(U);
  for (int i0 = 0; i0 < a.keep; i0 += per * kMoveUnits) {
    U v[kMoveUnits];
    char* to[kMoveUnits];
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {
      const int i = i0 + u * per + sub;
      to[u] = nullptr;
      v[u] = U{};
      if (i >= a.keep) continue;
      const int src = from[i];
      int dst = page_row(a.c, a.q, b, i);
      if (dst < 0) continue;
      dst += (int)hoff;
      if (src == dst) continue;
      to[u] = base + (int64_t)dst * row_bytes + at;
      if (src >= 0) v[u] = *reinterpret_cast<const U*>(base + (int64_t)src * row_bytes + at);
    }
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u) {
      if constexpr (sizeof(U) == 16) asm volatile("" : "+v"(v[u].x), "+v"(v[u].y), "+v"(v[u].z), "+v"(v[u].w));
      else asm volatile("" : "+v"(v[u]));
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMoveUnits; ++u)
      if (to[u]) *reinterpret_cast<U*>(to[u]) = v[u];
  }
}

__global__ __launch_bounds__(kMoveThreads) void paged_move_kernel(const PagedEvictArgs a, int row_bytes, int columns, int scaled) {
  const int all = 2 * columns + 2 * scaled + 1;
  const int64_t list = blockIdx.x / all;
  const int col = blockIdx.x - (int)list * all;
  const int b = (int)(list / a.c.n_kv), g = (int)(list - (int64_t)b * a.c.n_kv);
  const int2 cut = a.cut[list];  // (length as it was given, length that is cut or 0)
  if (g == 0 && col == all - 1 && threadIdx.x == 0) a.lengths[b] = cut.y ? a.keep : cut.x;
  if (!cut.y) return;
  const int32_t* const from = a.from + list * a.keep;
  const int64_t hoff = (int64_t)g << a.c.shift;
  if (col < 2 * columns) {
    const int side = col / columns, x = col - side * columns;
    move_column<uint4>(a, b, from, hoff, side ? a.c.v : a.c.k, row_bytes, min(row_bytes, kColumn) / 16, x * kColumn);
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

hipError_t launch_paged_evict(const PagedEvictArgs& a, int elem_bytes, int scaled, hipStream_t s) {
  RFX_LAUNCH(paged_choose_kernel, dim3((unsigned)(a.c.n_kv * a.q.n)), dim3(1024), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int row_bytes = a.c.dh * elem_bytes, columns = row_bytes < kColumn ? 1 : row_bytes / kColumn;
  const int64_t blocks = (int64_t)a.q.n * a.c.n_kv * (2 * columns + 2 * scaled + 1);
  RFX_LAUNCH(paged_move_kernel, dim3((unsigned)blocks), dim3(kMoveThreads), 0, s, a, row_bytes, columns, scaled);
  return hipGetLastError();
}

}  // namespace reflex
