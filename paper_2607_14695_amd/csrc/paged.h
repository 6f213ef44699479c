// Shared by the backbone operators (rotary positions, the paged cache and its
// attention): kernel arguments, and the way from a packed row to its slot.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/reflex.h"
#include "common.h"
#include "kernels.h"

namespace reflex {

struct Rows {
  const char* p;     // element (r, h, d) at p + (r*rs + h*hs + d) elements
  int64_t rs, hs;
};

struct Pages {
  char* k;
  char* v;
  float* k_scale;
  float* v_scale;
  int n_pages, shift, n_kv, dh;  // page_size = 1 << shift
};

struct Seqs {
  const int32_t* cu;
  const int32_t* len;
  const int32_t* table;
  int n, max_pages;
};

// Number of the sequence that holds packed row `row` (the same in every lane
// of the wave), or -1: how many of cu[0 .. n] are <= row, less one.  64 entries
// per step, so up to 63 sequences take one load and 4095 two.
RFX_DEV int seq_of_row(const Seqs& q, int64_t row, int lane) {
  int lo = 0, m = q.n + 1;
  while (m > 64) {
    const int stride = (m + 63) >> 6;
    const int at = (lane + 1) * stride - 1;
    const int v = at < m ? q.cu[lo + at] : INT32_MAX;
    const int c = __popcll(__ballot((int64_t)v <= row));
    lo += c * stride;
    m = min(stride, m - c * stride);
  }
  const int v = lane < m ? q.cu[lo + lane] : INT32_MAX;
  return lo + __popcll(__ballot(lane < m && (int64_t)v <= row)) - 1;
}

// Row index within the pages ((page * n_kv + head) * page_size + slot for head
// 0; head h lies h << shift further) of token `pos` of sequence b, or -1 where
// it is absent.  Fits 31 bits by the limit on the cache's rows.
RFX_DEV int page_row(const Pages& c, const Seqs& q, int b, int64_t pos) {
  if (pos < 0 || (pos >> c.shift) >= q.max_pages) return -1;
  const int page = q.table[(int64_t)b * q.max_pages + (pos >> c.shift)];
  if ((unsigned)page >= (unsigned)c.n_pages) return -1;
  return ((page * c.n_kv) << c.shift) + (int)(pos & ((1 << c.shift) - 1));
}

// Sum of a value over the lanes up to this one: within 16 lanes, then across them.
RFX_DEV int lanes_up_to(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// r / d for 0 <= r <= 2^30, given 1 / d rounded (and a quotient below 2^23) or to a
// unit in the last place (below 2^21): the product is off by less than one.
RFX_DEV int divided(int r, int d, float inv) {
  int q = (int)((float)r * inv);
  const int rest = r - q * d;
  q += rest >= d ? 1 : 0;
  return q - (rest < 0 ? 1 : 0);
}

struct RotaryArgs {
  const int64_t* pos;   // [axis * ps + row]; null: the token's index (writes only)
  int64_t ps;
  Rows x, y;
  int64_t n_rows;
  int n_heads, heads_per;  // heads per thread
  int inverse;
  reflex_rotary plan;
};
template <typename T> hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s);

struct PagedWriteArgs {
  Pages c;
  Seqs q;
  Rows k, v;
  int64_t n_rows;
  int heads_per;
  int rotate;
  const int64_t* pos;
  int64_t ps;
  reflex_rotary plan;
};
template <typename T> hipError_t launch_paged_write(const PagedWriteArgs& a, int store, hipStream_t s);

struct PagedReadArgs {
  Pages c;
  Seqs q;
  Rows k, v;
  int64_t n_rows;
};
template <typename T> hipError_t launch_paged_read(const PagedReadArgs& a, int store, hipStream_t s);

struct PagedAttnArgs {
  Pages c;
  Seqs q;
  Rows x, o;         // queries, result
  int64_t n_rows;
  int n_q, group;    // query heads, query heads per K/V head
  // scale * log2(e) = factor * scale2: scale2 > 0 is a normal number (a masked
  // -inf stays -inf), and factor, by which the queries enter, is 1 or -1, or
  // 2^-64 of that for a scale that scale2 alone could not hold
  float scale2, factor;
  int causal, window;
  int nsplit;        // key splits; with more than one, partials go to the workspace
  float* part_o;     // [n_rows * n_q][nsplit][dh]
  float2* part_ml;   // [n_rows * n_q][nsplit] (running maximum, sum)
  const uint64_t* tree;  // kTree: [n_rows][tree_words], which of its sequence's rows a row sees
  int tree_words;
  int units, tile_rows;  // kTree: workgroups of a K/V head that the chip holds, rows of a tile; nsplit: at most
  float2* stats;     // kWeigh: [n_rows * n_q] (maximum, 1 / sum, or 0 for a row that sees nothing)
  float* scores;     // kWeigh: [n_rows * n_q][score_pitch] in units of log2 e, if row_splits is 0; else the
                     // row splits' sums [row_splits][sequences * K/V heads][score_pitch]
  int64_t score_pitch;
  int row_splits;
  bool merge_with_sums;  // the splits are joined in the launch that sums the kept scores
};
struct PagedAttnPlan {
  int nsplit;
  size_t bytes;
};
PagedAttnPlan paged_attention_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q,
                                   int dtype, int window);
struct PagedTreePlan {
  int tile_rows, units, nsplit;
  size_t bytes;
};
PagedTreePlan paged_tree_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q, int dtype);
// How weighed attention comes to the keys' sums: from kept scores (row_splits
// 0), or from scores that are formed again by so many workgroups for the same keys.
struct PagedWeighPlan {
  int row_splits;
  int64_t pitch;  // keys that the table holds, or 0
  size_t bytes;   // of the scores or of the splits' sums
  bool few;       // so few rows that a workgroup sums 256 keys
};
PagedWeighPlan paged_weigh_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q, int dtype);
template <typename T> hipError_t launch_paged_attention(const PagedAttnArgs& a, int store, hipStream_t s);
template <typename T> hipError_t launch_paged_tree_attention(const PagedAttnArgs& a, int store, hipStream_t s);
// keys: the length that the longest sequence is expected to have
template <typename T>
hipError_t launch_paged_weighed_attention(const PagedAttnArgs& a, int store, float* weights, int64_t keys, bool few,
                                          hipStream_t s);

constexpr int kMaxTreeWords = 64, kMaxTreeRows = 64 * kMaxTreeWords;

struct PagedTreeArgs {
  Seqs q;
  const int32_t* parents;
  int64_t n_rows;
  int words;
  uint64_t* mask;  // [n_rows][words]
  int64_t* pos;    // [n_rows], or null
};
hipError_t launch_paged_tree(const PagedTreeArgs& a, hipStream_t s);

struct PagedAcceptArgs {
  Pages c;
  Seqs q;
  const int32_t* path;    // [sequences][max_path]
  const int32_t* counts;  // [sequences]
  int max_path;
  float* weights;         // [pages][heads][page size], moved too, or null
  int32_t* lengths;       // written; may be q.len
};
hipError_t launch_paged_accept(const PagedAcceptArgs& a, int elem_bytes, int scaled, hipStream_t s);

struct PagedEvictArgs {
  Pages c;
  Seqs q;
  float* weights;      // [pages][heads][page size]
  int keep, sinks, recent;
  int32_t* kept;       // [sequences][heads][keep], or null
  int32_t* lengths;    // written; may be q.len
  int32_t* from;       // workspace: [sequences][heads][keep] page rows
  int2* cut;           // workspace: [sequences][heads]
};
hipError_t launch_paged_evict(const PagedEvictArgs& a, int elem_bytes, int scaled, int64_t keys, hipStream_t s);

}  // namespace reflex
