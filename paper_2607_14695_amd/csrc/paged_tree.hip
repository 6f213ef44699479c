// Drafted tokens over a paged cache: which of them see which, their attention
// (the kernels of paged_attention.h in their tree mode) and the move of the
// accepted ones to the end of their sequence.
#include "paged_attention.h"

namespace reflex {

namespace {

// The visibility bits and position of every drafted token: a thread follows its
// row's parents down to the root.  Parents lie before their children, so the
// words of a row are finished from the last to the first, and the walk ends; a
// chain of 4,096 is the longest.  One workgroup to a sequence, whose parents
// are held in LDS: the walk is a chain of LDS reads, the kernel all latency (16
// rows 2.2 us, 64 trees of 78 to 256 rows 5 us, a launch among them; a chain's
// walks are as long as it is: of 256 rows 26 us, of 1,024 255, of 4,096 3.6 ms).
__global__ __launch_bounds__(256) void paged_tree_kernel(const PagedTreeArgs a) {
  __shared__ int32_t parent[kMaxTreeRows];
  const int b = blockIdx.x;
  const int64_t c0 = min((int64_t)max(a.q.cu[b], 0), a.n_rows), c1 = min((int64_t)max(a.q.cu[b + 1], 0), a.n_rows);
  const int64_t first = (int64_t)a.q.len[b] - ((int64_t)a.q.cu[b + 1] - a.q.cu[b]);
  const int64_t n = c1 - c0;
  const int most = 64 * a.words;  // rows that the bits can name
  for (int64_t i = threadIdx.x; i < min(n, (int64_t)most); i += 256) parent[i] = a.parents[c0 + i];
  __syncthreads();
  for (int64_t i = threadIdx.x; i < n; i += 256) {
    uint64_t* const m = a.mask + (c0 + i) * a.words;
    int depth = 0;
    if (i >= most) {
      for (int w = 0; w < a.words; ++w) m[w] = 0;
    } else {
      int at = (int)i >> 6;
      for (int w = a.words - 1; w > at; --w) m[w] = 0;
      uint64_t bits = 0;
      depth = -1;
      for (int j = (int)i; j >= 0;) {
        const int w = j >> 6;
        if (w != at) {
          m[at] = bits;
          while (--at > w) m[at] = 0;
          bits = 0;
        }
        bits |= 1ull << (j & 63);
        ++depth;
        const int p = parent[j];
        j = p < j ? p : -1;
      }
      m[at] = bits;
      while (--at >= 0) m[at] = 0;
    }
    if (a.pos) a.pos[c0 + i] = first + depth;
  }
}

// Accepted rows of a sequence moved to its end: token first + i from token first
// + path[i].  The path goes up, so path[i] - i never falls: tokens that come from
// a lower place (none, unless the path begins with negative entries, which read as
// zeros) are the first `up` ones, and these come from places among their own.  They
// are taken from the last to the first, the others, with path[i] >= i, from the
// first to the last: either way a place is never read after a later step has
// written it.  A step is some thousands of bytes, and is stored only when all of it
// was read.  One workgroup to a sequence, which also writes its length (32
// sequences of 6 tokens of one 256-wide head 4 us, a chain of latencies); where
// that would be many bytes, one to each `per_part` heads, and the lengths in a
// launch of their own (8 sequences of up to 90 tokens of 8 heads of 128 took 31 us
// in 8 workgroups).
struct Accepted { int64_t n, first; int c; };
RFX_DEV Accepted accepted_of(const PagedAcceptArgs& a, int b) {
  Accepted x;
  x.n = max((int64_t)a.q.cu[b + 1] - a.q.cu[b], (int64_t)0);
  x.first = (int64_t)a.q.len[b] - x.n;
  x.c = (int)min((int64_t)max(a.counts[b], 0), min(x.n, (int64_t)a.max_path));
  return x;
}

// How many of the accepted tokens come from a lower place than theirs.
RFX_DEV int from_below(const int32_t* path, int p0, int c) {
  if (c == 0 || p0 >= 0) return 0;
  int lo = 1, hi = c;
  while (lo < hi) {
    const int i = (lo + hi) >> 1;
    if (path[i] < i) lo = i + 1;
    else hi = i;
  }
  return lo;
}

// The moves of c tokens of `per` values each, U values of a thread a step; place(i,
// w, to, from) finds value w of token i: nowhere if `to` is left, zero if `from` is.
template <typename V, int U, typename F>
RFX_DEV void move_accepted(int c, int up, int per, F place) {
  auto step = [&](int64_t e0, int64_t end) __attribute__((always_inline)) {
    V v[U];
    V* to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t e = e0 + u * 1024 + threadIdx.x;
      to[u] = nullptr;
      v[u] = V{};
      if (e >= end) continue;
      const int i = (int)(e / per);
      const V* from = nullptr;
      place(i, (int)(e - (int64_t)i * per), to[u], from);
      if (from) v[u] = *from;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if constexpr (sizeof(V) == 16) asm volatile("" : "+v"(v[u].x), "+v"(v[u].y), "+v"(v[u].z), "+v"(v[u].w));
      else asm volatile("" : "+v"(v[u]));
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (to[u]) *to[u] = v[u];
  };
  constexpr int kStep = 1024 * U;
  const int64_t below = (int64_t)up * per, all = (int64_t)c * per;
  for (int64_t e0 = (below - 1) / kStep * kStep; below > 0 && e0 >= 0; e0 -= kStep) step(e0, below);
  for (int64_t e0 = below; e0 < all; e0 += kStep) step(e0, all);
}

constexpr int kAcceptUnits = 4;  // 16-byte pieces of a thread and step
__global__ __launch_bounds__(1024) void paged_accept_kernel(const PagedAcceptArgs a, int row_bytes, int scaled, int per_part) {
  const int parts = (a.c.n_kv + per_part - 1) / per_part;
  const int b = blockIdx.x / parts, h0 = (blockIdx.x - b * parts) * per_part, heads = min(per_part, a.c.n_kv - h0);
  const int32_t* const path = a.path + (int64_t)b * a.max_path;
  const int p0 = a.max_path > 0 ? path[0] : 0;  // (under way with the lengths)
  const Accepted x = accepted_of(a, b);
  const int up = from_below(path, p0, x.c);
  // (page row of head 0 that accepted token i comes from, and goes to)
  auto places = [&](int i, int& src, int& dst) __attribute__((always_inline)) {
    const int p = path[i];
    dst = page_row(a.c, a.q, b, x.first + i);
    src = p < 0 || p >= x.n ? -1 : page_row(a.c, a.q, b, x.first + p);
  };
  const int per_row = row_bytes / 16, side_units = heads * per_row;  // of a token: K and V of the heads
  move_accepted<uint4, kAcceptUnits>(x.c, up, 2 * side_units, [&](int i, int w, uint4*& to, const uint4*& from)
                                     __attribute__((always_inline)) {
    const int side = w / side_units, y = w - side * side_units;
    const int h = y / per_row, piece = y - h * per_row;
    int src, dst;
    places(i, src, dst);
    if (dst < 0 || src == dst) return;
    char* const base = side ? a.c.v : a.c.k;
    const int64_t hoff = (int64_t)(h0 + h) << a.c.shift;
    to = reinterpret_cast<uint4*>(base + (dst + hoff) * row_bytes + piece * 16);
    if (src >= 0) from = reinterpret_cast<const uint4*>(base + (src + hoff) * row_bytes + piece * 16);
  });
  // the scales of K and V, and the weights: floats of every head
  const int kinds = 2 * scaled + (a.weights != nullptr);
  if (kinds) {
    move_accepted<float, 1>(x.c, up, kinds * heads, [&](int i, int w, float*& to, const float*& from)
                            __attribute__((always_inline)) {
      int src, dst;
      places(i, src, dst);
      if (dst < 0 || src == dst) return;
      const int kind = w / heads;
      float* const all = kind == 2 * scaled ? a.weights : kind ? a.c.v_scale : a.c.k_scale;
      float* const base = all + ((int64_t)(h0 + w - kind * heads) << a.c.shift);
      to = base + dst;
      if (src >= 0) from = base + src;
    });
  }
  if (a.weights) {  // the rows that were not accepted leave no weight (all that moves has been read)
    const int64_t end = min(x.first + x.n, (int64_t)a.q.max_pages << a.c.shift);
    for (int64_t j = max(x.first + x.c, (int64_t)0) + threadIdx.x; j < end; j += 1024) {
      const int r = page_row(a.c, a.q, b, j);
      if (r < 0) continue;
      for (int h = h0; h < h0 + heads; ++h) a.weights[r + ((int64_t)h << a.c.shift)] = 0.f;
    }
  }
  if (parts > 1) return;
  __syncthreads();  // every thread has read the length
  if (threadIdx.x == 0) a.lengths[b] = (int32_t)max(x.first + x.c, (int64_t)0);
}

__global__ __launch_bounds__(256) void paged_accepted_lengths_kernel(const PagedAcceptArgs a) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b >= a.q.n) return;
  const Accepted x = accepted_of(a, b);
  a.lengths[b] = (int32_t)max(x.first + x.c, (int64_t)0);
}

}  // namespace

hipError_t launch_paged_tree(const PagedTreeArgs& a, hipStream_t s) {
  RFX_LAUNCH(paged_tree_kernel, dim3((unsigned)a.q.n), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_accept(const PagedAcceptArgs& a, int elem_bytes, int scaled, hipStream_t s) {
  const int row_bytes = a.c.dh * elem_bytes;
  // a step of a workgroup is 64 KB
  const int64_t bytes = 2ll * a.max_path * a.c.n_kv * row_bytes;
  const int parts = (int)std::min<int64_t>(a.c.n_kv, std::max<int64_t>(1, std::min<int64_t>(bytes >> 16, 2048 / a.q.n)));
  const int per_part = (a.c.n_kv + parts - 1) / parts, grid = a.q.n * ((a.c.n_kv + per_part - 1) / per_part);
  RFX_LAUNCH(paged_accept_kernel, dim3((unsigned)grid), dim3(1024), 0, s, a, row_bytes, scaled, per_part);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && grid > a.q.n) {
    RFX_LAUNCH(paged_accepted_lengths_kernel, dim3((unsigned)((a.q.n + 255) / 256)), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

// Rows of a tile: as in the attention of runs, by the rows of an average sequence,
// but 16 also where there is so little to do that the shorter way of the few-row
// kernel counts more than its rate (calls with their merge, us, 16 rows against
// 128: 128 rows of 256 over 833 keys 16 against 29, 512 rows over 3,000 keys 31
// against 36, 8 times 32 rows of 128 over 8,192 keys 23 against 31; the other way
// 8 times 128 rows of 256 over 3,000 keys 47 against 35, 8 times 128 rows of 128
// over 8,192 keys 49 against 36).  Their probabilities then have 16 bits.  How
// many workgroups share the batch's work; and the splits that a tile can have at most, which the workspace has room for.
PagedTreePlan paged_tree_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q, int dtype) {
  PagedTreePlan p;
  const int group = n_q / c.n_kv_heads;
  const int64_t cap = (int64_t)b.max_pages * c.page_size;
  const int64_t len = b.max_length > 0 && b.max_length < cap ? b.max_length : cap;
  p.tile_rows = rows_of_tile(n_rows, b.n_seqs, group, c.n_kv_heads, c.head_dim, dtype);
  if (dtype == REFLEX_DTYPE_BF16 && n_rows * n_q * c.head_dim <= (1 << 29) / std::max<int64_t>(len, 1)) p.tile_rows = 16;
  const int64_t slots = p.tile_rows == 128 && c.head_dim > 128 ? 256 : 512;
  p.units = (int)std::max<int64_t>(1, slots / c.n_kv_heads);
  const int64_t tiles = (n_rows * group + p.tile_rows - 1) / p.tile_rows;
  const int64_t row = (int64_t)n_q * (c.head_dim + 2) * sizeof(float) * n_rows;  // bytes of one split of all rows
  // four times what the tiles would have if they were alike, of 128 keys at least; one
  // where there are more sequences than CUs, which are tiles enough (and every
  // workgroup looks all of them over)
  const int64_t most = b.n_seqs > 256 ? 1 : std::min<int64_t>({64, std::max<int64_t>(1, 4 * p.units / tiles), std::max<int64_t>(1, (len + 127) / 128)});
  p.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>(most, (256 << 20) / row));
  p.bytes = p.nsplit == 1 ? 0 : (size_t)(row * p.nsplit);
  return p;
}

template <typename T>
hipError_t launch_paged_tree_attention(const PagedAttnArgs& a, int store, hipStream_t s) {
  return launch_mode<kTree, T>(a, store, s);
}
template hipError_t launch_paged_tree_attention<float>(const PagedAttnArgs&, int, hipStream_t);
template hipError_t launch_paged_tree_attention<bf16_t>(const PagedAttnArgs&, int, hipStream_t);

}  // namespace reflex
