// C ABI of the operators on a replica's paged cache: its pages, attention for
// trees of drafted tokens, and attention over selected blocks.
#include "handle.h"

using namespace coco;

namespace {

int check_layers(const coco_layer* H, int first, int n) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  // (first + n could wrap)
  if (first < 0 || n < 1 || n > H->cfg.n_layers || first > H->cfg.n_layers - n)
    return fail(COCO_EINVAL, "layers [%d, %d + %d) outside [0, %d)", first, first, n,
                H->cfg.n_layers);
  return COCO_OK;
}

int check_requests(int n, int n_seqs) {
  if (n < 0) return fail(COCO_EINVAL, "negative number of requests");
  if (n > 65535) return fail(COCO_EINVAL, "%d requests in a call (at most 65535)", n);
  if (n_seqs < 1) return fail(COCO_EINVAL, "n_seqs must be >= 1");
  return COCO_OK;
}

// Key and value pools of layers first .. first + n - 1, in groups.
template <typename F>
int for_pools(const coco_layer* H, int first, int n, F launch) {
  for (int l0 = 0; l0 < n; l0 += kMaxPools / 2) {
    CachePools p;
    for (int l = l0; l < n && l < l0 + kMaxPools / 2; ++l) {
      p.p[p.n++] = (char*)H->layers[first + l].k_cache;
      p.p[p.n++] = (char*)H->layers[first + l].v_cache;
    }
    const int rc = launch(p, l0 == 0);
    if (rc) return rc;
  }
  return COCO_OK;
}

int64_t page_bytes(const coco_layer_config& c) {
  return (int64_t)c.n_kv_heads * kBlockTokens * c.head_dim * elem_bytes(c.dtype);
}

// Validation mode: each of n values of `a` in [lo, hi), named in the message.
int check_range(const char* name, const std::vector<int32_t>& a, int64_t lo, int64_t hi) {
  for (size_t i = 0; i < a.size(); ++i)
    if (a[i] < lo || a[i] >= hi)
      return fail(COCO_EINVAL, "%s[%zu] = %d out of range [%lld, %lld)", name, i, a[i],
                  (long long)lo, (long long)hi);
  return COCO_OK;
}

int check_distinct(const char* name, const std::vector<int32_t>& a, int n_ids) {
  std::vector<char> seen;
  const int rc = zeros(seen, n_ids);
  if (rc) return rc;
  for (size_t i = 0; i < a.size(); ++i) {
    if (seen[a[i]]) return fail(COCO_EINVAL, "%s[%zu] = %d is a duplicate", name, i, a[i]);
    seen[a[i]] = 1;
  }
  return COCO_OK;
}

// Validation mode: the blocks of sequence s's first `tokens` tokens.
int check_blocks(const std::vector<int32_t>& bt, int max_blocks, int s, int tokens,
                 int64_t num_blocks) {
  for (int b = 0; b < (tokens + kBlockTokens - 1) / kBlockTokens; ++b) {
    const int32_t v = bt[(size_t)s * max_blocks + b];
    if (v < 0 || v >= num_blocks)
      return fail(COCO_EINVAL, "block_table[%d][%d] = %d out of range [0, %lld)", s, b, v,
                  (long long)num_blocks);
  }
  return COCO_OK;
}

// alloc (src null) and fork.
int page_requests(coco_layer* H, int first, int nl, const int32_t* src, const int32_t* dst,
                  const int32_t* lens, int n, int32_t* table, int n_seqs, int32_t* refs,
                  int32_t* status, bool fork, hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  PageArgs a;
  a.src = src;
  a.dst = dst;
  a.lens = lens;
  a.n = n;
  a.n_seqs = n_seqs;
  a.max_blocks = c.max_blocks_per_seq;
  a.num_blocks = shared_blocks(H, 0, c.n_layers);
  a.table = table;
  a.refs = refs;
  a.status = status;
  a.list = H->page_list;
  a.off = H->page_off;
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> s, d, l, bt, rf;
    int rc;
    if ((rc = fetch(d, dst, n, st)) || (rc = fetch(l, lens, n, st)) ||
        (rc = fetch(bt, (const int32_t*)table, (size_t)n_seqs * a.max_blocks, st)) ||
        (rc = fetch(rf, (const int32_t*)refs, a.num_blocks, st)) ||
        (rc = check_range("sequence", d, 0, n_seqs)) || (rc = check_distinct("sequence", d, n_seqs)) ||
        (rc = check_range("length", l, 0, (int64_t)a.max_blocks * kBlockTokens + 1)))
      return rc;
    if (fork) {
      if ((rc = fetch(s, src, n, st)) || (rc = check_range("parent", s, 0, n_seqs))) return rc;
      std::vector<char> child;
      if ((rc = zeros(child, n_seqs))) return rc;
      for (int i = 0; i < n; ++i) child[d[i]] = 1;
      for (int i = 0; i < n; ++i) {
        if (child[s[i]])
          return fail(COCO_EINVAL, "row %d is a parent and a child of one call", s[i]);
        if ((rc = check_blocks(bt, a.max_blocks, s[i], l[i], a.num_blocks))) return rc;
        for (int b = 0; b < (l[i] + kBlockTokens - 1) / kBlockTokens; ++b)
          if (rf[bt[(size_t)s[i] * a.max_blocks + b]] < 1)
            return fail(COCO_EINVAL, "block %d of row %d has no reference",
                        bt[(size_t)s[i] * a.max_blocks + b], s[i]);
        for (int b = 0; b < a.max_blocks; ++b)
          if (bt[(size_t)d[i] * a.max_blocks + b] >= 0)
            return fail(COCO_EINVAL, "child row %d still holds blocks", d[i]);
      }
    }
  }
  CallEnd end(H, st, !fork || 2 * nl <= kMaxPools);
  HIPCHK(launch_page_plan(a, st));
  if (fork) {
    const int rc = for_pools(H, first, nl, [&](const CachePools& p, bool tables) -> int {
      HIPCHK(launch_page_fork(a, p, page_bytes(c), tables, st));
      return COCO_OK;
    });
    if (rc) return rc;
  } else {
    HIPCHK(launch_page_alloc(a, st));
  }
  return end.finish();
}

// Attention rows' shapes and pointers that the host can check.
int check_rows(const coco_layer* H, int layer, const void* q, const void* o, int n_rows,
               const int32_t* seq_starts, int n_seqs, const int32_t* bt, const int32_t* ctx) {
  const coco_layer_config& c = H->cfg;
  if (layer < 0 || layer >= c.n_layers) return fail(COCO_EINVAL, "layer %d out of range", layer);
  if (n_rows < 0) return fail(COCO_EINVAL, "n_rows < 0");
  if (n_rows == 0) return COCO_OK;
  if (!q || !o || !bt || !ctx) return fail(COCO_EINVAL, "NULL argument");
  if ((uintptr_t)q % 16 || (uintptr_t)o % 16)
    return fail(COCO_EINVAL, "q or o is not 16-byte aligned");
  if (n_seqs < 1) return fail(COCO_EINVAL, "n_seqs must be >= 1");
  if (seq_starts == nullptr && n_seqs != n_rows)
    return fail(COCO_EINVAL, "rows without seq_starts need n_seqs == n_rows");
  return COCO_OK;
}

// Validation mode: sequences' rows, lengths and blocks. Rows past the last
// sequence (a padded call) are left alone, and their arrays may hold anything.
int validate_rows(const coco_layer* H, int n_rows, const int32_t* positions,
                  const int32_t* seq_starts, int n_seqs, const int32_t* block_table,
                  const int32_t* ctx_lens, int64_t num_blocks, std::vector<int32_t>& starts,
                  std::vector<int32_t>& ctx, hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  std::vector<int32_t> pos, bt;
  int rc;
  if ((rc = fetch(ctx, ctx_lens, n_seqs, st)) ||
      (rc = fetch(bt, block_table, (size_t)n_seqs * c.max_blocks_per_seq, st)) ||
      (rc = check_range("ctx_lens", ctx, 0, (int64_t)c.max_blocks_per_seq * kBlockTokens + 1)))
    return rc;
  if (seq_starts) {
    if ((rc = fetch(starts, seq_starts, (size_t)n_seqs + 1, st))) return rc;
  } else {
    if ((rc = zeros(starts, (size_t)n_seqs + 1))) return rc;
    for (int s = 0; s <= n_seqs; ++s) starts[s] = s;
  }
  if (starts[0] != 0 || starts[n_seqs] < 0 || starts[n_seqs] > n_rows)
    return fail(COCO_EINVAL, "seq_starts must run from 0 to at most n_rows");
  if (positions && ((rc = fetch(pos, positions, starts[n_seqs], st)) ||
                    (rc = check_range("positions", pos, 0,
                                      (int64_t)c.max_blocks_per_seq * kBlockTokens))))
    return rc;
  for (int s = 0; s < n_seqs; ++s) {
    if (starts[s + 1] < starts[s]) return fail(COCO_EINVAL, "seq_starts not monotone at %d", s);
    if (starts[s + 1] > starts[s] &&
        (rc = check_blocks(bt, c.max_blocks_per_seq, s, ctx[s], num_blocks)))
      return rc;
  }
  return COCO_OK;
}

// A buffer of the handle's that grows; what it outgrows stays until destroy,
// since captured graphs may hold its address. A new one's last `zero` bytes are
// cleared for calls on any stream, before it becomes the handle's.
int grow(coco_layer* H, char** buf, size_t* have, size_t want, size_t zero = 0) {
  if (want <= *have) return COCO_OK;
  HIPCHK(hipSetDevice(H->device));
  char* p = nullptr;
  try {
    H->extra.push_back(nullptr);
  } catch (const std::exception&) {
    return fail(COCO_ENOMEM, "out of host memory");
  }
  if (hipMalloc((void**)&p, want) != hipSuccess) {
    (void)hipGetLastError();
    H->extra.pop_back();
    return fail(COCO_ENOMEM, "workspace of %zu bytes does not fit", want);
  }
  H->extra.back() = p;
  if (zero) {
    HIPCHK(hipMemset(p + want - zero, 0, zero));
    HIPCHK(hipDeviceSynchronize());
  }
  *buf = p;
  *have = want;
  return COCO_OK;
}

int check_sparse_room(const coco_layer* H, int n_rows, int n_select) {
  if (n_select < 1) return fail(COCO_EINVAL, "n_select must be >= 1");
  if (n_rows > H->sparse_rows || n_select > H->sparse_top)
    return fail(COCO_ESTATE, "%d rows of %d blocks; coco_sparse_reserve made room for %d of %d",
                n_rows, n_select, H->sparse_rows, H->sparse_top);
  return COCO_OK;
}

RowKeys row_keys(const coco_layer* H, const int32_t* seq_starts, int n_seqs, const int32_t* bt,
                 const int32_t* ctx, int64_t num_blocks) {
  RowKeys rk;
  rk.block_table = bt;
  rk.ctx_lens = ctx;
  rk.seq_starts = seq_starts;
  rk.n_seqs = n_seqs;
  rk.max_blocks = H->cfg.max_blocks_per_seq;
  rk.num_blocks = num_blocks;
  return rk;
}

}  // namespace

namespace coco {

int check_tree(const coco_layer* H, int n_rows, const int32_t* seq_starts, int n_seqs,
               const uint64_t* mask, int words) {
  if (!seq_starts || !mask) return fail(COCO_EINVAL, "NULL argument");
  if ((uintptr_t)mask % 8) return fail(COCO_EINVAL, "tree_mask is not 8-byte aligned");
  if (words < 1) return fail(COCO_EINVAL, "mask_words must be >= 1");
  if (n_rows > H->tree_rows || n_seqs > H->tree_seqs)
    return fail(COCO_ESTATE, "%d rows of %d sequences; coco_tree_reserve made room for %d of %d",
                n_rows, n_seqs, H->tree_rows, H->tree_seqs);
  return COCO_OK;
}

int validate_tree(const coco_layer* H, int n_rows, const int32_t* positions,
                  const int32_t* seq_starts, int n_seqs, const int32_t* bt, const int32_t* ctx_lens,
                  int words, int64_t num_blocks, hipStream_t st) {
  std::vector<int32_t> ss, ctx;
  int rc;
  if ((rc = validate_rows(H, n_rows, positions, seq_starts, n_seqs, bt, ctx_lens, num_blocks, ss,
                          ctx, st)))
    return rc;
  for (int s = 0; s < n_seqs; ++s) {
    if (ss[s + 1] - ss[s] > ctx[s])
      return fail(COCO_EINVAL, "sequence %d has %d nodes in %d cached tokens", s,
                  ss[s + 1] - ss[s], ctx[s]);
    if (ss[s + 1] - ss[s] > 64LL * words)
      return fail(COCO_EINVAL, "sequence %d has %d nodes for %d mask words", s,
                  ss[s + 1] - ss[s], words);
  }
  return COCO_OK;
}

int run_tree(coco_layer* H, const coco_layer_weights& w, const void* q, void* o, bool tiled,
             int n_rows, const int32_t* seq_starts, int n_seqs, const int32_t* bt,
             const int32_t* ctx, const uint64_t* mask, int words, hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  RowKeys rk = row_keys(H, seq_starts, n_seqs, bt, ctx, w.num_blocks);
  rk.mask = mask;
  rk.words = words;
  if (c.dtype == COCO_BF16)
    HIPCHK(launch_tree_attention_bf16((const bf16_t*)q, (const bf16_t*)w.k_cache,
                                      (const bf16_t*)w.v_cache, rk, n_rows, c.n_q_heads,
                                      c.n_kv_heads, (bf16_t*)o, tiled, H->tree_part_o,
                                      H->tree_part_ml, H->tree_parts, H->tree_plan, H->tree_redo,
                                      H->num_cus, st));
  else
    HIPCHK(launch_attn_rows_f32((const float*)q, (const float*)w.k_cache, (const float*)w.v_cache,
                                rk, n_rows, c.n_q_heads, c.n_kv_heads, c.head_dim, (float*)o,
                                H->num_cus, st));
  return COCO_OK;
}

int check_select(const coco_layer* H, int n_rows, const int8_t* summary, const float* scales,
                 int64_t num_blocks, int keep_first, int keep_last, const int32_t* selected,
                 int n_select) {
  if (!summary || !scales || !selected) return fail(COCO_EINVAL, "NULL argument");
  if ((uintptr_t)summary % 16) return fail(COCO_EINVAL, "summary is not 16-byte aligned");
  if (num_blocks < 1) return fail(COCO_EINVAL, "num_blocks must be >= 1");
  if (n_select < 1) return fail(COCO_EINVAL, "n_select must be >= 1");
  if (keep_first < 0 || keep_last < 0 || keep_first > n_select || keep_last > n_select - keep_first)
    return fail(COCO_EINVAL, "keep_first = %d and keep_last = %d outside n_select = %d", keep_first,
                keep_last, n_select);
  return check_sparse_room(H, n_rows, n_select);
}

int run_summarize(coco_layer* H, const coco_layer_weights& w, int8_t* summary, float* scales,
                  const int32_t* first, const int32_t* ctx, int n_seqs, const int32_t* bt,
                  hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  if (c.dtype == COCO_BF16)
    HIPCHK(launch_summarize((const bf16_t*)w.k_cache, c.n_kv_heads, c.head_dim, bt, n_seqs,
                            c.max_blocks_per_seq, w.num_blocks, first, ctx, summary, scales,
                            H->num_cus, st));
  else
    HIPCHK(launch_summarize((const float*)w.k_cache, c.n_kv_heads, c.head_dim, bt, n_seqs,
                            c.max_blocks_per_seq, w.num_blocks, first, ctx, summary, scales,
                            H->num_cus, st));
  return COCO_OK;
}

int run_select(coco_layer* H, const int8_t* summary, const float* scales, int64_t num_blocks,
               const void* q, int n_rows, const int32_t* positions, const int32_t* seq_starts,
               int n_seqs, const int32_t* bt, const int32_t* ctx, int keep_first, int keep_last,
               int32_t* selected, int n_select, hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  RowKeys rk = row_keys(H, seq_starts, n_seqs, bt, ctx, num_blocks);
  rk.positions = positions;
  rk.top = n_select;
  if (c.dtype == COCO_BF16)
    HIPCHK(launch_block_select((const bf16_t*)q, summary, scales, rk, n_rows, c.n_q_heads,
                               c.n_kv_heads, c.head_dim, keep_first, keep_last, H->sparse_keys,
                               selected, st));
  else
    HIPCHK(launch_block_select((const float*)q, summary, scales, rk, n_rows, c.n_q_heads,
                               c.n_kv_heads, c.head_dim, keep_first, keep_last, H->sparse_keys,
                               selected, st));
  return COCO_OK;
}

int run_sparse(coco_layer* H, const coco_layer_weights& w, const void* q, void* o, bool tiled,
               int n_rows, const int32_t* positions, const int32_t* seq_starts, int n_seqs,
               const int32_t* bt, const int32_t* ctx, const int32_t* selected, int n_select,
               hipStream_t st) {
  const coco_layer_config& c = H->cfg;
  RowKeys rk = row_keys(H, seq_starts, n_seqs, bt, ctx, w.num_blocks);
  rk.positions = positions;
  rk.selected = selected;
  rk.top = n_select;
  if (c.dtype == COCO_BF16)
    HIPCHK(launch_sparse_attention_bf16((const bf16_t*)q, (const bf16_t*)w.k_cache,
                                        (const bf16_t*)w.v_cache, rk, n_rows, c.n_q_heads,
                                        c.n_kv_heads, (bf16_t*)o, tiled, H->sparse_part_o,
                                        H->sparse_part_ml, st));
  else
    HIPCHK(launch_attn_rows_f32((const float*)q, (const float*)w.k_cache, (const float*)w.v_cache,
                                rk, n_rows, c.n_q_heads, c.n_kv_heads, c.head_dim, (float*)o,
                                H->num_cus, st));
  return COCO_OK;
}

}  // namespace coco

extern "C" {

int coco_kv_alloc(coco_layer_t H, const int32_t* seq_idx, const int32_t* lens, int32_t n,
                  int32_t* block_table, int32_t n_seqs, int32_t* ref_counts, int32_t* status,
                  coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  int rc = check_requests(n, n_seqs);
  if (rc || n == 0) return rc;
  if (!seq_idx || !lens || !block_table || !ref_counts || !status)
    return fail(COCO_EINVAL, "NULL argument");
  if (n > H->cfg.max_seqs)
    return fail(COCO_EINVAL, "n = %d above max_seqs = %d", n, H->cfg.max_seqs);
  return page_requests(H, 0, H->cfg.n_layers, nullptr, seq_idx, lens, n, block_table, n_seqs,
                       ref_counts, status, false, (hipStream_t)stream);
}

int coco_kv_fork(coco_layer_t H, int32_t first_layer, int32_t n_layers, const int32_t* src_seq,
                 const int32_t* dst_seq, const int32_t* lens, int32_t n, int32_t* block_table,
                 int32_t n_seqs, int32_t* ref_counts, int32_t* status, coco_stream_t stream) {
  int rc = check_layers(H, first_layer, n_layers);
  if (!rc) rc = check_requests(n, n_seqs);
  if (rc || n == 0) return rc;
  if (!src_seq || !dst_seq || !lens || !block_table || !ref_counts || !status)
    return fail(COCO_EINVAL, "NULL argument");
  if (n > H->cfg.max_seqs)
    return fail(COCO_EINVAL, "n = %d above max_seqs = %d", n, H->cfg.max_seqs);
  return page_requests(H, first_layer, n_layers, src_seq, dst_seq, lens, n, block_table, n_seqs,
                       ref_counts, status, true, (hipStream_t)stream);
}

int coco_kv_free(coco_layer_t H, const int32_t* seq_idx, const int32_t* keep_lens, int32_t n,
                 int32_t* block_table, int32_t n_seqs, int32_t* ref_counts,
                 coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  int rc = check_requests(n, n_seqs);
  if (rc || n == 0) return rc;
  if (!seq_idx || !block_table || !ref_counts) return fail(COCO_EINVAL, "NULL argument");
  const coco_layer_config& c = H->cfg;
  hipStream_t st = (hipStream_t)stream;
  const int64_t blocks = shared_blocks(H, 0, c.n_layers);
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> s, k, bt, rf;
    if ((rc = fetch(s, seq_idx, n, st)) || (rc = check_range("sequence", s, 0, n_seqs)) ||
        (keep_lens && ((rc = fetch(k, keep_lens, n, st)) ||
                       (rc = check_range("keep_lens", k, 0, INT32_MAX)))) ||
        (rc = fetch(bt, (const int32_t*)block_table, (size_t)n_seqs * c.max_blocks_per_seq, st)) ||
        (rc = fetch(rf, (const int32_t*)ref_counts, blocks, st)))
      return rc;
    for (int i = 0; i < n; ++i) {
      const int keep = keep_lens ? k[i] : 0;
      for (int b = keep / kBlockTokens + (keep % kBlockTokens > 0); b < c.max_blocks_per_seq; ++b) {
        int32_t& id = bt[(size_t)s[i] * c.max_blocks_per_seq + b];
        if (id < 0) continue;
        if (id >= blocks)
          return fail(COCO_EINVAL, "block_table[%d][%d] = %d out of range [0, %lld)", s[i], b, id,
                      (long long)blocks);
        if (--rf[id] < 0) return fail(COCO_EINVAL, "block %d has no reference to drop", id);
        id = -1;
      }
    }
  }
  CallEnd end(H, st);
  HIPCHK(launch_page_free(seq_idx, keep_lens, n, n_seqs, block_table, c.max_blocks_per_seq,
                          ref_counts, blocks, st));
  return end.finish();
}

int coco_kv_copy(coco_layer_t H, int32_t first_layer, int32_t n_layers, const int32_t* src_blocks,
                 const int32_t* dst_blocks, int32_t n, coco_stream_t stream) {
  int rc = check_layers(H, first_layer, n_layers);
  if (rc) return rc;
  if (n < 0) return fail(COCO_EINVAL, "n < 0");
  if (n == 0) return COCO_OK;
  if (!src_blocks || !dst_blocks) return fail(COCO_EINVAL, "NULL argument");
  hipStream_t st = (hipStream_t)stream;
  const int64_t blocks = shared_blocks(H, first_layer, n_layers);
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> s, d;
    if ((rc = fetch(s, src_blocks, n, st)) || (rc = fetch(d, dst_blocks, n, st)) ||
        (rc = check_range("src_blocks", s, 0, blocks)) ||
        (rc = check_range("dst_blocks", d, 0, blocks)))
      return rc;
    std::vector<char> to;
    if ((rc = zeros(to, blocks))) return rc;
    for (int i = 0; i < n; ++i) {
      if (to[d[i]]) return fail(COCO_EINVAL, "dst_blocks[%d] = %d is a duplicate", i, d[i]);
      to[d[i]] = 1;
    }
    for (int i = 0; i < n; ++i)
      if (to[s[i]] && s[i] != d[i])
        return fail(COCO_EINVAL, "block %d is copied from and to in one call", s[i]);
  }
  CallEnd end(H, st, 2 * n_layers <= kMaxPools);
  rc = for_pools(H, first_layer, n_layers, [&](const CachePools& p, bool) -> int {
    HIPCHK(launch_page_copy(src_blocks, dst_blocks, n, blocks, p, page_bytes(H->cfg), st));
    return COCO_OK;
  });
  return rc ? rc : end.finish();
}

int coco_kv_compact(coco_layer_t H, int32_t first_layer, int32_t n_layers, const int32_t* seq_idx,
                    const int32_t* base_lens, const int32_t* kept, const int32_t* kept_starts,
                    int32_t n, int32_t n_kept, const int32_t* block_table, int32_t n_seqs,
                    coco_stream_t stream) {
  int rc = check_layers(H, first_layer, n_layers);
  if (!rc) rc = check_requests(n, n_seqs);
  if (rc) return rc;
  if (n_kept < 0) return fail(COCO_EINVAL, "n_kept < 0");
  if (n == 0 || n_kept == 0) return COCO_OK;
  if (!seq_idx || !base_lens || !kept || !kept_starts || !block_table)
    return fail(COCO_EINVAL, "NULL argument");
  const coco_layer_config& c = H->cfg;
  if (c.n_kv_heads > 65535) return fail(COCO_EINVAL, "n_kv_heads above 65535");
  hipStream_t st = (hipStream_t)stream;
  const int64_t blocks = shared_blocks(H, first_layer, n_layers);
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> s, b, k, ks, bt;
    if ((rc = fetch(s, seq_idx, n, st)) || (rc = fetch(b, base_lens, n, st)) ||
        (rc = fetch(k, kept, n_kept, st)) || (rc = fetch(ks, kept_starts, (size_t)n + 1, st)) ||
        (rc = fetch(bt, block_table, (size_t)n_seqs * c.max_blocks_per_seq, st)) ||
        (rc = check_range("sequence", s, 0, n_seqs)) ||
        (rc = check_distinct("sequence", s, n_seqs)) ||
        (rc = check_range("kept", k, 0, (int64_t)c.max_blocks_per_seq * kBlockTokens)) ||
        (rc = check_range("base_lens", b, 0, (int64_t)c.max_blocks_per_seq * kBlockTokens + 1)))
      return rc;
    if (ks[0] != 0 || ks[n] != n_kept)
      return fail(COCO_EINVAL, "kept_starts must run from 0 to n_kept");
    for (int i = 0; i < n; ++i) {
      if (ks[i + 1] < ks[i]) return fail(COCO_EINVAL, "kept_starts not monotone at %d", i);
      for (int j = ks[i]; j < ks[i + 1]; ++j)
        if (k[j] < b[i] + (j - ks[i]) || (j > ks[i] && k[j] <= k[j - 1]))
          return fail(COCO_EINVAL, "kept[%d] = %d is not ascending from base_lens[%d] = %d", j,
                      k[j], i, b[i]);
      if (ks[i + 1] > ks[i]) {
        for (int e = b[i] / kBlockTokens; e <= k[ks[i + 1] - 1] / kBlockTokens; ++e) {
          const int32_t v = bt[(size_t)s[i] * c.max_blocks_per_seq + e];
          if (v < 0 || v >= blocks)
            return fail(COCO_EINVAL, "block_table[%d][%d] = %d out of range [0, %lld)", s[i], e, v,
                        (long long)blocks);
        }
      }
    }
  }
  CallEnd end(H, st, 2 * n_layers <= kMaxPools);
  rc = for_pools(H, first_layer, n_layers, [&](const CachePools& p, bool) -> int {
    if (c.dtype == COCO_BF16)
      HIPCHK(launch_page_compact<uint16_t>(seq_idx, base_lens, kept, kept_starts, n, n_kept,
                                           block_table, n_seqs, c.max_blocks_per_seq, blocks, p,
                                           c.n_kv_heads, c.head_dim, st));
    else
      HIPCHK(launch_page_compact<uint32_t>(seq_idx, base_lens, kept, kept_starts, n, n_kept,
                                           block_table, n_seqs, c.max_blocks_per_seq, blocks, p,
                                           c.n_kv_heads, c.head_dim, st));
    return COCO_OK;
  });
  return rc ? rc : end.finish();
}

int coco_tree_reserve(coco_layer_t H, int32_t max_rows, int32_t max_seqs) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  if (max_rows < 1 || max_seqs < 1) return fail(COCO_EINVAL, "sizes must be positive");
  const int rows = max_rows > H->tree_rows ? max_rows : H->tree_rows;
  const int seqs = max_seqs > H->tree_seqs ? max_seqs : H->tree_seqs;
  const coco_layer_config& c = H->cfg;
  if (c.dtype == COCO_BF16) {
    const int64_t parts =
        tree_column_parts(rows, seqs, c.n_q_heads, c.n_kv_heads, c.max_blocks_per_seq);
    if (parts > INT32_MAX)
      return fail(COCO_EINVAL, "%d rows of %d sequences: %lld partial columns exceed 2^31 - 1",
                  rows, seqs, (long long)parts);
    const size_t o = align256((size_t)parts * c.head_dim * 4), ml = align256((size_t)parts * 8);
    const size_t plan = align256((size_t)seqs * 8), redo = ((size_t)rows * c.n_q_heads + 16) * 4;
    const int rc = grow(H, &H->tree_ws, &H->tree_bytes, o + ml + plan + redo, redo);
    if (rc) return rc;
    H->tree_parts = parts;
    H->tree_part_o = (float*)H->tree_ws;
    H->tree_part_ml = (float*)(H->tree_ws + o);
    H->tree_plan = (int32_t*)(H->tree_ws + o + ml);
    H->tree_redo = (int32_t*)(H->tree_ws + o + ml + plan);
  }
  H->tree_rows = rows;
  H->tree_seqs = seqs;
  return COCO_OK;
}

int coco_tree_attention(coco_layer_t H, int32_t layer, const void* q, void* o, int32_t n_rows,
                        const int32_t* seq_starts, int32_t n_seqs, const int32_t* block_table,
                        const int32_t* ctx_lens, const uint64_t* tree_mask, int32_t mask_words,
                        coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  int rc = check_rows(H, layer, q, o, n_rows, seq_starts, n_seqs, block_table, ctx_lens);
  if (rc || n_rows == 0) return rc;
  if ((rc = check_tree(H, n_rows, seq_starts, n_seqs, tree_mask, mask_words))) return rc;
  const coco_layer_weights& w = H->layers[layer];
  hipStream_t st = (hipStream_t)stream;
  HIPCHK(hipSetDevice(H->device));
  if (H->validate && (rc = validate_tree(H, n_rows, nullptr, seq_starts, n_seqs, block_table,
                                         ctx_lens, mask_words, w.num_blocks, st)))
    return rc;
  CallEnd end(H, st, n_seqs <= kTreeLaunchSeqs);
  if ((rc = run_tree(H, w, q, o, false, n_rows, seq_starts, n_seqs, block_table, ctx_lens,
                     tree_mask, mask_words, st)))
    return rc;
  return end.finish();
}

int coco_kv_summarize(coco_layer_t H, int32_t layer, int8_t* summary, float* scales,
                      const int32_t* first_lens, const int32_t* ctx_lens, int32_t n_seqs,
                      const int32_t* block_table, coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  const coco_layer_config& c = H->cfg;
  if (layer < 0 || layer >= c.n_layers) return fail(COCO_EINVAL, "layer %d out of range", layer);
  if (n_seqs < 0 || n_seqs > 65535)
    return fail(COCO_EINVAL, "n_seqs = %d outside [0, 65535]", n_seqs);
  if (n_seqs == 0) return COCO_OK;
  if (!summary || !scales || !ctx_lens || !block_table) return fail(COCO_EINVAL, "NULL argument");
  if ((uintptr_t)summary % 16) return fail(COCO_EINVAL, "summary is not 16-byte aligned");
  const coco_layer_weights& w = H->layers[layer];
  hipStream_t st = (hipStream_t)stream;
  HIPCHK(hipSetDevice(H->device));
  int rc;
  if (H->validate) {
    std::vector<int32_t> f, ctx, bt;
    const int64_t top = (int64_t)c.max_blocks_per_seq * kBlockTokens;
    if ((first_lens && ((rc = fetch(f, first_lens, n_seqs, st)) ||
                        (rc = check_range("first_lens", f, 0, top + 1)))) ||
        (rc = fetch(ctx, ctx_lens, n_seqs, st)) ||
        (rc = check_range("ctx_lens", ctx, 0, top + 1)) ||
        (rc = fetch(bt, block_table, (size_t)n_seqs * c.max_blocks_per_seq, st)))
      return rc;
    for (int s = 0; s < n_seqs; ++s)
      if ((rc = check_blocks(bt, c.max_blocks_per_seq, s, ctx[s], w.num_blocks))) return rc;
  }
  CallEnd end(H, st);
  if ((rc = run_summarize(H, w, summary, scales, first_lens, ctx_lens, n_seqs, block_table, st)))
    return rc;
  return end.finish();
}

int coco_sparse_reserve(coco_layer_t H, int32_t max_rows, int32_t max_blocks) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  if (max_rows < 1 || max_rows > 65535 || max_blocks < 1 || max_blocks > (1 << 24))
    return fail(COCO_EINVAL, "max_rows = %d outside [1, 65535] or max_blocks = %d outside [1, 2^24]",
                max_rows, max_blocks);
  const int rows = max_rows > H->sparse_rows ? max_rows : H->sparse_rows;
  const int top = max_blocks > H->sparse_top ? max_blocks : H->sparse_top;
  const coco_layer_config& c = H->cfg;
  const size_t keys =
      align256((size_t)rows * c.n_kv_heads * select_stride(c.max_blocks_per_seq) * 4);
  // fp32 handles attend a list whole.
  const size_t parts = c.dtype == COCO_BF16 && sparse_parts(top) > 1
                           ? (size_t)rows * c.n_q_heads * sparse_parts(top)
                           : 0;
  const size_t part_o = parts * c.head_dim * 4;
  const int rc = grow(H, &H->sparse_ws, &H->sparse_bytes, keys + part_o + parts * 8);
  if (rc) return rc;
  H->sparse_keys = (uint32_t*)H->sparse_ws;
  H->sparse_part_o = (float*)(H->sparse_ws + keys);
  H->sparse_part_ml = (float*)(H->sparse_ws + keys + part_o);
  H->sparse_rows = rows;
  H->sparse_top = top;
  return COCO_OK;
}

int coco_block_select(coco_layer_t H, const int8_t* summary, const float* scales, int64_t num_blocks,
                      const void* q, int32_t n_rows, const int32_t* positions,
                      const int32_t* seq_starts, int32_t n_seqs, const int32_t* block_table,
                      const int32_t* ctx_lens, int32_t keep_first, int32_t keep_last,
                      int32_t* selected, int32_t n_select, coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  int rc = check_rows(H, 0, q, q, n_rows, seq_starts, n_seqs, block_table, ctx_lens);
  if (rc || n_rows == 0) return rc;
  if (!positions) return fail(COCO_EINVAL, "NULL argument");
  if ((rc = check_select(H, n_rows, summary, scales, num_blocks, keep_first, keep_last, selected,
                         n_select)))
    return rc;
  hipStream_t st = (hipStream_t)stream;
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> ss, ctx;
    if ((rc = validate_rows(H, n_rows, positions, seq_starts, n_seqs, block_table, ctx_lens,
                            num_blocks, ss, ctx, st)))
      return rc;
  }
  CallEnd end(H, st);
  if ((rc = run_select(H, summary, scales, num_blocks, q, n_rows, positions, seq_starts, n_seqs,
                       block_table, ctx_lens, keep_first, keep_last, selected, n_select, st)))
    return rc;
  return end.finish();
}

int coco_sparse_attention(coco_layer_t H, int32_t layer, const void* q, void* o, int32_t n_rows,
                          const int32_t* positions, const int32_t* seq_starts, int32_t n_seqs,
                          const int32_t* block_table, const int32_t* ctx_lens,
                          const int32_t* selected, int32_t n_select, coco_stream_t stream) {
  if (!H) return fail(COCO_EINVAL, "handle is NULL");
  int rc = check_rows(H, layer, q, o, n_rows, seq_starts, n_seqs, block_table, ctx_lens);
  if (rc || n_rows == 0) return rc;
  if (!positions || !selected) return fail(COCO_EINVAL, "NULL argument");
  if ((rc = check_sparse_room(H, n_rows, n_select))) return rc;
  const coco_layer_config& c = H->cfg;
  const coco_layer_weights& w = H->layers[layer];
  hipStream_t st = (hipStream_t)stream;
  HIPCHK(hipSetDevice(H->device));
  if (H->validate) {
    std::vector<int32_t> ss, ctx, sel, pos;
    if ((rc = validate_rows(H, n_rows, positions, seq_starts, n_seqs, block_table, ctx_lens,
                            w.num_blocks, ss, ctx, st)) ||
        (rc = fetch(pos, positions, n_rows, st)) ||
        (rc = fetch(sel, selected, (size_t)n_rows * c.n_kv_heads * n_select, st)))
      return rc;
    for (int s = 0; s < n_seqs; ++s)
      for (int i = ss[s]; i < ss[s + 1]; ++i) {
        const int keys = ctx[s] < pos[i] + 1 ? ctx[s] : pos[i] + 1;
        for (int g = 0; g < c.n_kv_heads; ++g) {
          int last = -1;
          for (int e = 0; e < n_select; ++e) {
            const int b = sel[((size_t)i * c.n_kv_heads + g) * n_select + e];
            if (b < 0) continue;
            if (b <= last || b > (keys - 1) / kBlockTokens || keys == 0)
              return fail(COCO_EINVAL,
                          "selected[%d][%d][%d] = %d is not ascending or past the row's keys", i, g,
                          e, b);
            last = b;
          }
        }
      }
  }
  CallEnd end(H, st);
  if ((rc = run_sparse(H, w, q, o, false, n_rows, positions, seq_starts, n_seqs, block_table,
                       ctx_lens, selected, n_select, st)))
    return rc;
  return end.finish();
}

}  // extern "C"
