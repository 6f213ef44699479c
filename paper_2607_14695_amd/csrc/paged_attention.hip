// Attention of a chunk of new tokens over a paged cache: its plan, and its
// kernels for rows that see a run of keys.
#include "paged_attention.h"

namespace reflex {

namespace {

// Key splits at most: a merging wave holds one in each lane.
constexpr int kMaxSplits = 64;

}  // namespace

PagedAttnPlan paged_attention_plan(const reflex_paged_cache& c, const reflex_paged_batch& b, int64_t n_rows, int n_q,
                                   int dtype, int window) {
  PagedAttnPlan p;
  const int group = n_q / c.n_kv_heads;
  const int64_t cap = (int64_t)b.max_pages * c.page_size;
  const int64_t len = b.max_length > 0 && b.max_length < cap ? b.max_length : cap;
  const int bm = rows_of_tile(n_rows, b.n_seqs, group, c.n_kv_heads, c.head_dim, dtype);
  // Workgroups without a split, were the sequences alike.  Splits make one round
  // of two workgroups to a CU of them (the widest many-row kernel: of one), each
  // with 128 keys at least: 64 single tokens over 15,409 fp8 keys took 78 us with
  // 8 splits against 88 with 11 and 87 with 6.
  const int64_t seqs = std::max<int64_t>(1, std::min<int64_t>(b.n_seqs, n_rows));
  const int64_t blocks = seqs * ((n_rows * group + seqs * bm - 1) / (seqs * bm)) * c.n_kv_heads;
  const int64_t slots = bm == 128 && c.head_dim > 128 ? 256 : 512;
  const int64_t most = std::max<int64_t>(
      1, std::min(slots / blocks, std::min<int64_t>(kMaxSplits, 65535 / c.n_kv_heads)));
  auto splits = [&](int64_t keys) {  // of a tile that sees so many
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(most, (keys + 127) / 128));
    const int64_t per = std::max<int64_t>(((keys + want - 1) / want + 127) / 128 * 128, 128);
    return (int)std::max<int64_t>(1, (keys + per - 1) / per);
  };
  p.nsplit = splits(len);
  // with a window a tile sees that and its own tokens, from a whole 128 on; the
  // workspace, which is asked for without a window, bounds the splits
  if (window > 0) p.nsplit = std::min(p.nsplit, splits(std::min<int64_t>(len, (int64_t)window + bm / group + 128)));
  p.bytes = p.nsplit == 1 ? 0 : (size_t)n_rows * n_q * p.nsplit * (c.head_dim + 2) * sizeof(float);
  return p;
}

template <typename T>
hipError_t launch_paged_attention(const PagedAttnArgs& a, int store, hipStream_t s) {
  return launch_mode<kPlain, T>(a, store, s);
}
template hipError_t launch_paged_attention<float>(const PagedAttnArgs&, int, hipStream_t);
template hipError_t launch_paged_attention<bf16_t>(const PagedAttnArgs&, int, hipStream_t);

}  // namespace reflex
