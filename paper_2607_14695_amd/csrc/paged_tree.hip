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
// are held in LDS: the walk is a chain of LDS reads, the kernel all latency.
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
// + path[i].  Both go up and path[i] >= i, so a place is never read after a
// later step has written it: the workgroup takes the moves in order, some
// thousands of bytes a step, and stores a step only when all of it was read.
// One workgroup to a sequence, which also writes its length.
constexpr int kAcceptUnits = 4;  // 16-byte pieces of a thread and step
__global__ __launch_bounds__(1024) void paged_accept_kernel(const PagedAcceptArgs a, int row_bytes, int scaled) {
  const int b = blockIdx.x;
  const int len = a.q.len[b];
  const int64_t n = max((int64_t)a.q.cu[b + 1] - a.q.cu[b], (int64_t)0);
  const int64_t first = (int64_t)len - n;
  const int c = (int)min((int64_t)max(a.counts[b], 0), min(n, (int64_t)a.max_path));
  const int32_t* const path = a.path + (int64_t)b * a.max_path;
  // (page row of head 0 that accepted token i comes from, and goes to)
  auto places = [&](int i, int& src, int& dst) __attribute__((always_inline)) {
    const int p = path[i];
    dst = page_row(a.c, a.q, b, first + i);
    src = p < 0 || p >= n ? -1 : page_row(a.c, a.q, b, first + p);
  };
  const int per_row = row_bytes / 16;
  const int units = 2 * a.c.n_kv * per_row;  // of a token: K and V of every head
  const int64_t all = (int64_t)c * units;
  for (int64_t e0 = 0; e0 < all; e0 += 1024 * kAcceptUnits) {
    uint4 v[kAcceptUnits];
    char* to[kAcceptUnits];
#pragma unroll
    for (int u = 0; u < kAcceptUnits; ++u) {
      const int64_t e = e0 + u * 1024 + threadIdx.x;
      to[u] = nullptr;
      v[u] = zero16();
      if (e >= all) continue;
      const int i = (int)(e / units), w = (int)(e - (int64_t)i * units);
      const int side = w / (units / 2), x = w - side * (units / 2);
      const int h = x / per_row, piece = x - h * per_row;
      int src, dst;
      places(i, src, dst);
      if (dst < 0 || src == dst) continue;
      char* const base = side ? a.c.v : a.c.k;
      const int64_t hoff = (int64_t)h << a.c.shift;
      to[u] = base + (dst + hoff) * row_bytes + piece * 16;
      if (src >= 0) v[u] = ld16(base + (src + hoff) * row_bytes + piece * 16);
    }
#pragma unroll
    for (int u = 0; u < kAcceptUnits; ++u) asm volatile("" : "+v"(v[u].x), "+v"(v[u].y), "+v"(v[u].z), "+v"(v[u].w));
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kAcceptUnits; ++u)
      if (to[u]) st16(to[u], v[u]);
  }
  if (scaled) {
    const int per = 2 * a.c.n_kv;
    const int64_t total = (int64_t)c * per;
    for (int64_t e0 = 0; e0 < total; e0 += 1024) {
      const int64_t e = e0 + threadIdx.x;
      float v = 0.f;
      float* to = nullptr;
      if (e < total) {
        const int i = (int)(e / per), w = (int)(e - (int64_t)i * per);
        int src, dst;
        places(i, src, dst);
        if (dst >= 0 && src != dst) {
          float* const base = (w >= a.c.n_kv ? a.c.v_scale : a.c.k_scale) + ((int64_t)(w % a.c.n_kv) << a.c.shift);
          to = base + dst;
          if (src >= 0) v = base[src];
        }
      }
      asm volatile("" : "+v"(v));
      __syncthreads();
      if (to) *to = v;
    }
  }
  __syncthreads();  // every thread has read the length
  if (threadIdx.x == 0) a.lengths[b] = (int32_t)max(first + c, (int64_t)0);
}

}  // namespace

hipError_t launch_paged_tree(const PagedTreeArgs& a, hipStream_t s) {
  RFX_LAUNCH(paged_tree_kernel, dim3((unsigned)a.q.n), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_paged_accept(const PagedAcceptArgs& a, int elem_bytes, int scaled, hipStream_t s) {
  RFX_LAUNCH(paged_accept_kernel, dim3((unsigned)a.q.n), dim3(1024), 0, s, a, a.c.dh * elem_bytes, scaled);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_paged_tree_attention(const PagedAttnArgs& a, int store, hipStream_t s) {
  return launch_mode<kTree, T>(a, store, s);
}
template hipError_t launch_paged_tree_attention<float>(const PagedAttnArgs&, int, hipStream_t);
template hipError_t launch_paged_tree_attention<bf16_t>(const PagedAttnArgs&, int, hipStream_t);

}  // namespace reflex
