/*
 * coco.h -- C ABI of the layer-replica hot path on one MI355X (gfx950).
 *
 * A layer replica (Sec. 3.1 of the paper, replication mechanism) holds a full
 * copy of the weights of one or more consecutive decoder layers plus its own
 * partition of the paged key/value cache, and runs the unchanged layer on its
 * sub-batch: the rows of the in-flight batch it was given. The library does
 * exactly that step on one GPU:
 *
 *   gather rows -> RMSNorm -> QKV projection -> RoPE + KV append ->
 *   paged GQA attention -> O projection + residual -> RMSNorm ->
 *   SwiGLU MLP + residual -> scatter rows
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * Pointers. Every data pointer is a DEVICE pointer into memory the caller
 *   owns (weights, caches, hidden buffer, index arrays). The library borrows
 *   caches, RMSNorm gains and (fp32) weight matrices for the handle's
 *   lifetime and the rest for the call. dtype COCO_BF16: coco_layer_init
 *   copies the four weight matrices of every layer into library memory in
 *   tile order (below) and never reads the caller's matrices again; the
 *   caller may free or overwrite them once init has returned.
 *   The library owns that copy and its workspace, both allocated once in
 *   coco_layer_init and sized by the config (the paper's persistent memory
 *   pool with fixed addresses, Sec. 5.2, CUDA-graph compatibility): per-row
 *   activations and split-K partials for max_rows rows, the decode attention
 *   partials, and (bf16) a RoPE cos/sin table of max_blocks_per_seq * 16
 *   positions * head_dim * 4 bytes.
 * Streams. `stream` is a hipStream_t (NULL = the null stream). Work is
 *   enqueued on it; calls return without synchronising, never allocate, and
 *   keep every address fixed, so a call can be captured in a HIP graph --
 *   except with validation switched on, which copies index arrays to the host.
 * Element types. dtype COCO_BF16: weights, hidden, caches and k/v inputs are
 *   bfloat16 (uint16 bit patterns); accumulation and softmax are fp32.
 *   dtype COCO_F32: all of those are float32.
 * Errors. A negative return is an error; coco_last_error() gives a message
 *   (thread-local). Host-checkable faults return COCO_EINVAL before anything
 *   is enqueued; a failed launch returns COCO_EHIP. Device-side contents of
 *   index arrays are checked only in validation mode (coco_layer_set_validate).
 * Threads. A handle is not thread-safe; calls that overlap on one handle
 *   (including from different streams) race on its workspace.
 *
 * Layouts
 * -------
 * Weights of one layer, nn.Linear layout ([out][in], row-major):
 *   w_qkv     [(Hq + 2*Hkv) * hd][d]   query heads, then key heads, then value
 *                                      heads, hd rows each
 *   w_o       [d][Hq * hd]
 *   w_gate_up [2*F][d]                 F gate rows, then F up rows
 *   w_down    [d][F]
 *   gamma_attn, gamma_mlp [d]          RMSNorm gains
 * (bf16) The library's copy of a weight matrix [N][K] is in tile order: the
 *   1 KB block (n / 16) * (K / 32) + k / 32 holds rows 16 (n / 16) .. + 15 and
 *   k 32 (k / 32) .. + 31 as 64 chunks of 8 consecutive k, chunk
 *   ((k % 32) / 8) * 16 + n % 16 -- one MFMA operand fragment per 16 rows x
 *   32 k, read by one contiguous 1 KB load. The copy of w_gate_up interleaves
 *   its rows: 8 gate rows, then the 8 matching up rows, in every block.
 * Paged cache of one layer, with block size B = 16 tokens:
 *   k_cache, v_cache [num_blocks][Hkv][B * hd]: one tile of B tokens x hd
 *   dimensions per (block, kv head), in MFMA operand order. Inside a tile,
 *   token slot t (0..15) and dimension h live at
 *     K: ((h/32)*64 + ((h%32)/8)*16 + t)*8 + h%8
 *     V: (((h/32)*64 + (t/4)*16 + h%16)*2 + (h/16)%2)*4 + t%4
 *   (hd must be a multiple of 32). Token t of sequence s lives in block
 *   block_table[s][t / 16], slot t % 16. Keys are stored after rotation
 *   (RoPE), values as projected.
 * Batch arrays (int32, device):
 *   row_idx[n_rows]        hidden row of each call row; distinct, < hidden_rows
 *   positions[n_rows]      absolute position of each call row's token
 *   seq_starts[n_seqs+1]   prefill: call rows of sequence s are
 *                          seq_starts[s] .. seq_starts[s+1]-1, in position
 *                          order. NULL = decode: call row i is sequence i
 *                          (then n_seqs == n_rows).
 *   block_table[n_seqs][max_blocks_per_seq]   physical block ids, -1 unused
 *   ctx_lens[n_seqs]       cached tokens of sequence s once this call's tokens
 *                          are appended (decode, normally positions[i] + 1)
 * A token whose block_table entry is no block of the pools (-1, or from
 * num_blocks on: pages that coco_kv_alloc did not serve) is not cached by any
 * call, and nothing is written in its place. A row that attends such an entry
 * reads some block of the pool instead: its output means nothing, other rows'
 * are as without it. Validation mode refuses such calls.
 * Every token attends to the cached keys of its own sequence at positions
 * 0 .. its own position (causal), its own key included: a decode row i
 * attends min(ctx_lens[i], positions[i] + 1) keys, so cached tokens past its
 * position (positions[i] < ctx_lens[i] - 1) are not read.
 */
#ifndef COCO_H
#define COCO_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct coco_layer* coco_layer_t;
typedef void* coco_stream_t; /* hipStream_t */

enum {
  COCO_OK = 0,
  COCO_EINVAL = -1, /* bad argument or unsupported configuration */
  COCO_ENOMEM = -2, /* workspace allocation failed (init only) */
  COCO_EHIP = -3,   /* a HIP runtime call or kernel launch failed */
  COCO_ESTATE = -4  /* handle unusable (e.g. destroyed, or a previous HIP fault) */
};

enum { COCO_BF16 = 0, COCO_F32 = 1 };

typedef struct {
  int32_t d_model;            /* d */
  int32_t n_q_heads;          /* Hq */
  int32_t n_kv_heads;         /* Hkv; Hq % Hkv == 0 */
  int32_t head_dim;           /* hd; 128 for COCO_BF16, multiple of 32 <= 256 for COCO_F32 */
  int32_t d_ffn;              /* F */
  int32_t n_layers;           /* layers held by this handle */
  int32_t dtype;              /* COCO_BF16 or COCO_F32 */
  int32_t block_size;         /* must be 16 */
  int32_t max_rows;           /* largest n_rows of any call (decode rows or prefill tokens) */
  int32_t max_seqs;           /* largest n_seqs of any call */
  int32_t max_blocks_per_seq; /* row stride of block_table (<= 2^24; bf16: <= 130944,
                                 the decode partition merge's limit) */
  float rope_theta;           /* RoPE base theta */
  float rms_eps;              /* RMSNorm epsilon */
} coco_layer_config;

typedef struct {
  const void* w_qkv;
  const void* w_o;
  const void* w_gate_up;
  const void* w_down;
  const void* gamma_attn;
  const void* gamma_mlp;
  void* k_cache;
  void* v_cache;
  int64_t num_blocks; /* blocks in this layer's k_cache and v_cache */
} coco_layer_weights;

/* Create a replica handle for n_layers consecutive layers (Sec. 3.1: the
 * replicated unit is a span of consecutive layers). `layers` points to
 * cfg->n_layers host structs of device pointers; they are copied. Allocates
 * the workspace on the current HIP device and, for bf16, the tile-order copy
 * of the weight matrices (the sum of their sizes over the handle's layers),
 * which it writes before returning (synchronising the device). Returns
 * COCO_EINVAL for an unsupported shape (bf16: head_dim != 128, Hq/Hkv > 16, d,
 * F or Hq*hd not multiples of 128), COCO_ENOMEM if the workspace or the
 * weight copy does not fit. */
int coco_layer_init(const coco_layer_config* cfg, const coco_layer_weights* layers,
                    coco_layer_t* out);

/* Release the workspace, the weight copy and the handle. First waits for the
 * handle's last call made outside graph capture to finish (an event recorded behind the
 * last kernel of every such call; calls on one handle are ordered, since they
 * share the workspace), not for other work on the device. A graph captured
 * from the handle's calls must not run after this. NULL is ignored. */
void coco_layer_destroy(coco_layer_t h);

/* Message of the last failed call on this thread ("" if none). */
const char* coco_last_error(void);

/* Library version as major*10000 + minor*100 + patch. */
int coco_version(void);

/* Switch device-side argument validation on (1) or off (0). When on, every
 * forward/append copies its index arrays to the host, synchronising the
 * stream, and rejects duplicate or out-of-range row_idx, non-increasing
 * positions within a sequence, positions >= ctx_lens, ctx_lens beyond the
 * block table, and block ids outside [0, num_blocks) with COCO_EINVAL before
 * launching. Off by default. */
int coco_layer_set_validate(coco_layer_t h, int32_t on);

/* Write n_tok tokens of keys and values into layer `layer`'s paged cache
 * (Sec. 3.1: each replica appends key/value entries to its own partition).
 * k, v: [n_tok][Hkv][hd] in the handle's dtype, k already rotated.
 * seq_idx[n_tok]: sequence of each token (row of block_table, < n_seqs).
 * positions[n_tok]: position of each token. A bit copy: the stored values
 * equal the inputs bit for bit. Tokens must name distinct (sequence,
 * position) pairs. */
int coco_kv_append(coco_layer_t h, int32_t layer, const void* k, const void* v,
                   const int32_t* seq_idx, const int32_t* positions, int32_t n_tok,
                   const int32_t* block_table, int32_t n_seqs, coco_stream_t stream);

/* One decoder layer on the call rows of `hidden` ([hidden_rows][d], updated
 * in place): rows named in row_idx receive the layer output, every other row
 * is left untouched (Sec. 3.1: the replica processes its sub-batch and the
 * outputs are gathered back on the batch axis). The call's keys and values
 * are appended to the layer's cache before attention. n_rows == 0 is a no-op.
 * Results do not depend on which other rows share the call: any partition of
 * a decode batch, and any request-aligned partition of a prefill batch, gives
 * output rows and cache bytes identical bit for bit to the whole batch
 * (Sec. 5.2: outputs bit-wise consistent with the baseline). */
int coco_layer_forward(coco_layer_t h, int32_t layer, void* hidden, int64_t hidden_rows,
                       const int32_t* row_idx, int32_t n_rows, const int32_t* positions,
                       const int32_t* seq_starts, int32_t n_seqs,
                       const int32_t* block_table, const int32_t* ctx_lens,
                       coco_stream_t stream);

/* Layers first_layer .. first_layer+n_layers-1 as one replicated segment
 * (Sec. 3.1: consecutive layers are replicated as a unit, activations stay in
 * local memory and transfers happen only at the segment boundaries): one
 * gather, every layer on the resident rows, one scatter. Between layers the
 * rows are held in the handle's dtype, so the result equals n_layers
 * successive coco_layer_forward calls bit for bit. */
int coco_layer_span_forward(coco_layer_t h, int32_t first_layer, int32_t n_layers,
                            void* hidden, int64_t hidden_rows, const int32_t* row_idx,
                            int32_t n_rows, const int32_t* positions,
                            const int32_t* seq_starts, int32_t n_seqs,
                            const int32_t* block_table, const int32_t* ctx_lens,
                            coco_stream_t stream);

/* For callers that cannot allocate device memory at call time (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same call as coco_layer_forward, with the same results bit for bit, but
 * its per-call buffers (activations, split-K partials, decode attention
 * partials and work list) come from a static array of 64 MiB that every GPU
 * the library runs on holds from module load until the process ends, sized
 * for this call's rows instead of the handle's max_rows. The call itself
 * allocates nothing, host or device. Its address is looked up once per
 * device by coco_layer_init. Returns COCO_EINVAL, before anything is
 * enqueued, when the call's buffers exceed 64 MiB (a batch-64 decode of the
 * 8B-shaped layer with 8k-token block tables takes about 49 MB; a
 * 2048-token prefill of the 32B-shaped layer does not fit). All such calls
 * on one GPU share the
 * array, whatever their handle: calls that overlap on one GPU (other
 * streams, other threads, other handles) race on it. The array keeps the
 * last call's contents; no part of it needs to start at zero. Validation
 * mode is not run by this entry point, and coco_layer_workspace shows the
 * handle's own workspace, not this array. */
int coco_layer_forward_noalloc(coco_layer_t h, int32_t layer, void* hidden, int64_t hidden_rows,
                               const int32_t* row_idx, int32_t n_rows, const int32_t* positions,
                               const int32_t* seq_starts, int32_t n_seqs,
                               const int32_t* block_table, const int32_t* ctx_lens,
                               coco_stream_t stream);

/* Copy an intermediate buffer of the last call into `dst` (device memory of
 * at least dst_bytes bytes), for inspection by tests. which = COCO_WS_*;
 * row i holds call row i of the last layer run, row-major. Copies
 * min(dst_bytes, buffer size) bytes on `stream`. (A bf16 prefill call keeps
 * H, O, H2 and U, the A operands of its four projections, in the tile order
 * of the weight copies, 16 rows x 32 columns per 1 KB block; this copy puts
 * the call's rows back in row-major order.) */
enum {
  COCO_WS_X = 0,  /* layer input rows, [max_rows][d], dtype (written for the
                     second and later layers of a span; the first layer reads
                     its rows from the hidden buffer) */
  COCO_WS_H = 1,  /* RMSNorm_1 output, [max_rows][d], dtype (prefill and
                     fp32 calls; bf16 decode folds RMSNorm_1 into the QKV
                     projection: not its contents) */
  COCO_WS_Q = 2,  /* rotated queries, [max_rows][Hq*hd], dtype */
  COCO_WS_O = 3,  /* attention output, [max_rows][Hq*hd], dtype */
  COCO_WS_X1 = 4, /* residual after the O projection, [max_rows][d], fp32 */
  COCO_WS_H2 = 5, /* RMSNorm_2 output, [max_rows][d], dtype (bf16 prefill
                     folds the row's 1/rms into the gate/up projection and
                     holds x1 * gamma_2 here) */
  COCO_WS_U = 6   /* SwiGLU activation, [max_rows][F], dtype */
};
int coco_layer_workspace(coco_layer_t h, int32_t which, void* dst, int64_t dst_bytes,
                         coco_stream_t stream);

/* Per-kernel timing for benchmarks (calls of any handle are unaffected while
 * it is off; kinds whose work runs inside another kernel count no launches).
 * When on, every kernel launched by coco_layer_forward and the span, tree and
 * sparse forwards on this handle is launched with a pair of HIP events
 * (hipExtLaunchKernelGGL) that the runtime timestamps at the kernel's own
 * start and end, from a pool of events created here (so switching it on
 * allocates; timed calls themselves do not). Switch it off before capturing
 * calls into a HIP graph. */
enum {
  COCO_K_GATHER_NORM = 0,    /* gather + RMSNorm_1 (or RMSNorm_1 inside a span) */
  COCO_K_GEMM_QKV = 1,       /* QKV projection */
  COCO_K_QKV_EPILOGUE = 2,   /* split-K sum + RoPE + cache append */
  COCO_K_ATTENTION = 3,      /* paged attention (decode partitions or prefill); of
                                trees and selected blocks all kernels, as one launch */
  COCO_K_ATTN_COMBINE = 4,   /* decode partition merge */
  COCO_K_GEMM_O = 5,         /* O projection */
  COCO_K_RESIDUAL_NORM = 6,  /* residual + RMSNorm_2 */
  COCO_K_GEMM_GATE_UP = 7,   /* gate/up projection */
  COCO_K_SWIGLU = 8,         /* SwiGLU */
  COCO_K_GEMM_DOWN = 9,      /* down projection */
  COCO_K_RESIDUAL_SCATTER = 10, /* residual + scatter */
  COCO_K_COUNT = 11
};
int coco_layer_set_timing(coco_layer_t h, int32_t on);

/* Sum of the event-measured durations (milliseconds) and the number of
 * launches of each kernel kind since timing was switched on or last read;
 * ms and launches hold n_kinds entries (<= COCO_K_COUNT). Synchronises with
 * the recorded events, then resets the sums. Returns COCO_ESTATE if more
 * launches were made than the pool holds (4096 per read). */
int coco_layer_read_timing(coco_layer_t h, double* ms, int64_t* launches, int32_t n_kinds);

/* ---------------------------------------------------------------------------
 * Pages of the cache. Block tables and reference counts are the caller's
 * device arrays, updated in place by the kernels in stream order, so that a
 * serving loop needs no copy to the host to know which blocks are free, and
 * the calls can be captured in a HIP graph:
 *   block_table[n_seqs][max_blocks_per_seq]  physical block ids, -1: none
 *   ref_counts[num_blocks]                   rows that hold the block, 0: free
 * (num_blocks: the smallest of the handle's layers). A block id means that
 * block in every layer. Requests take the free blocks of lowest id in the
 * order of the call; they are served in order until one does not fit, and from
 * there on only those that need no block are: status[i] = 1 where request i
 * is served, else 0 (its rows and the counts are as if it had not been made;
 * fork: the child's row is empty). A call holds at most 65535 requests
 * (alloc, fork: at most max_seqs). Rows or lengths out of range are not served
 * (status 0) or skipped; validation mode reports them.
 * ------------------------------------------------------------------------- */

/* Blocks for every empty (-1) entry of row seq_idx[i] below ceil(lens[i] / 16);
 * entries that hold a block keep it. Rows must be distinct. */
int coco_kv_alloc(coco_layer_t h, const int32_t* seq_idx, const int32_t* lens, int32_t n,
                  int32_t* block_table, int32_t n_seqs, int32_t* ref_counts, int32_t* status,
                  coco_stream_t stream);

/* Row dst_seq[i] becomes a fork of the first lens[i] tokens of row src_seq[i]:
 * it shares the parent's full blocks (counts + 1) and, where lens[i] is no
 * multiple of 16, gets a block of its own with a copy of the parent's next
 * block, keys and values of layers first_layer .. + n_layers - 1. dst_seq
 * rows must be distinct, empty, and no parent of the call; several children
 * may have one parent. A row named as its own parent is not served and keeps
 * what it holds. (Layers of another handle over the same table: pass
 * the table entries lens[i] / 16 of both rows to its coco_kv_copy.) */
int coco_kv_fork(coco_layer_t h, int32_t first_layer, int32_t n_layers, const int32_t* src_seq,
                 const int32_t* dst_seq, const int32_t* lens, int32_t n, int32_t* block_table,
                 int32_t n_seqs, int32_t* ref_counts, int32_t* status, coco_stream_t stream);

/* Row seq_idx[i] lets go of its blocks from entry ceil(keep_lens[i] / 16) on
 * (keep_lens NULL: of all): counts - 1, entries -1. A row named twice lets go
 * of a block once. */
int coco_kv_free(coco_layer_t h, const int32_t* seq_idx, const int32_t* keep_lens, int32_t n,
                 int32_t* block_table, int32_t n_seqs, int32_t* ref_counts,
                 coco_stream_t stream);

/* Copy block src_blocks[i] to dst_blocks[i], keys and values of layers
 * first_layer .. + n_layers - 1. dst_blocks must be distinct and none of them
 * a source of another pair; pairs with an id outside the pools are skipped. */
int coco_kv_copy(coco_layer_t h, int32_t first_layer, int32_t n_layers, const int32_t* src_blocks,
                 const int32_t* dst_blocks, int32_t n, coco_stream_t stream);

/* Move the tokens of row seq_idx[i] at positions kept[kept_starts[i]],
 * kept[kept_starts[i] + 1], .. (ascending) to positions base_lens[i],
 * base_lens[i] + 1, .. of the row, in layers first_layer .. + n_layers - 1: the
 * accepted path of a tree of drafted tokens moves up to its prefix, or a
 * context loses evicted tokens. A bit copy (keys keep the rotation of the
 * position they were computed at), as if every token were read before any is
 * written. kept[kept_starts[i] + k] >= base_lens[i] + k; rows distinct; the
 * blocks from base_lens[i] on must be the row's own (count 1). kept_starts
 * [n + 1] runs from 0 to n_kept. */
int coco_kv_compact(coco_layer_t h, int32_t first_layer, int32_t n_layers, const int32_t* seq_idx,
                    const int32_t* base_lens, const int32_t* kept, const int32_t* kept_starts,
                    int32_t n, int32_t n_kept, const int32_t* block_table, int32_t n_seqs,
                    coco_stream_t stream);

/* ---------------------------------------------------------------------------
 * Attention for trees of drafted tokens.
 * ------------------------------------------------------------------------- */

/* Make room for tree calls of up to max_rows rows and max_seqs sequences
 * (allocates; not under graph capture). May be called again to make more;
 * what it outgrows is kept until coco_layer_destroy, so that graphs captured
 * before stay valid. */
int coco_tree_reserve(coco_layer_t h, int32_t max_rows, int32_t max_seqs);

/* Attention of drafted tokens over layer `layer`'s cache. The call rows
 * seq_starts[s] .. seq_starts[s+1]-1 are the nodes of sequence s's tree, whose
 * keys and values are in the cache already (coco_kv_append) in its last slots:
 * node j of its N nodes at position ctx_lens[s] - N + j (ctx_lens[s] counts
 * them). Node j attends every token before the tree, and node i where bit
 * i % 64 of tree_mask[row][i / 64] is set (its path to the root and itself;
 * any other set is taken too). Bits from N on are ignored; N <= 64 mask_words.
 *   q, o [n_rows][Hq][hd], the handle's dtype, q rotated, 16-byte aligned, apart;
 *   tree_mask [n_rows][mask_words] 64-bit words
 * (bf16: the softmax weights of a tree with more than 16 nodes times query heads
 * per key/value head are rounded to bf16 for their product with the values, as in
 * the layers; smaller trees' and those of coco_sparse_attention keep 16 bits.)
 * A row that attends nothing (no prefix, no bit) gives zeros; what it does not
 * attend may hold anything. A row's result does not depend on the other
 * sequences of the call; rows from seq_starts[n_seqs] on (a padded call) are
 * left as they are. Needs coco_tree_reserve (COCO_ESTATE without). */
int coco_tree_attention(coco_layer_t h, int32_t layer, const void* q, void* o, int32_t n_rows,
                        const int32_t* seq_starts, int32_t n_seqs, const int32_t* block_table,
                        const int32_t* ctx_lens, const uint64_t* tree_mask, int32_t mask_words,
                        coco_stream_t stream);

/* Layers first_layer .. first_layer + n_layers - 1 for the nodes of drafted
 * trees, as coco_layer_span_forward for prompts, except: row i of sequence s,
 * its node j = i - seq_starts[s] of N, is cached in slot ctx_lens[s] - N + j
 * (the pages must be there: coco_kv_alloc); its position is only its rotation,
 * the number of tokens before it on its path, so that an accepted path can
 * move up to its place (coco_kv_compact) as it is; and it attends as in
 * coco_tree_attention. seq_starts[n_seqs] must be n_rows (validation mode refuses
 * other calls): a row of no sequence is not cached, but its hidden row is
 * overwritten with what means nothing. Needs coco_tree_reserve. */
int coco_layer_tree_forward(coco_layer_t h, int32_t first_layer, int32_t n_layers, void* hidden,
                            int64_t hidden_rows, const int32_t* row_idx, int32_t n_rows,
                            const int32_t* positions, const int32_t* seq_starts, int32_t n_seqs,
                            const int32_t* block_table, const int32_t* ctx_lens,
                            const uint64_t* tree_mask, int32_t mask_words, coco_stream_t stream);

/* ---------------------------------------------------------------------------
 * Attention over the blocks that a cheap score selects for each query.
 * ------------------------------------------------------------------------- */

/* Write the summaries of the blocks that hold tokens first_lens[s] (NULL: 0)
 * .. ctx_lens[s] - 1 of each sequence, from the keys in layer `layer`'s cache:
 *   summary [num_blocks][Hkv][2][hd] int8, 16-byte aligned; scales
 *   [num_blocks][Hkv] fp32 (the caller's; num_blocks as the layer's pools)
 * With hi_d, lo_d the largest and smallest of the block's cached keys in
 * dimension d (tokens below ctx_lens[s]; a non-finite element counts as 0) and
 * x in [-100, 100] the exponent with max(|hi|, |lo|) < 2^x: scale 2^(x - 7),
 * summary[0] = ceil(hi / scale), summary[1] = floor(lo / scale), held within
 * +-127. Blocks shared by several sequences of the call must be full in each. */
int coco_kv_summarize(coco_layer_t h, int32_t layer, int8_t* summary, float* scales,
                      const int32_t* first_lens, const int32_t* ctx_lens, int32_t n_seqs,
                      const int32_t* block_table, coco_stream_t stream);

/* Make room for calls that select or attend blocks of up to max_rows rows (at
 * most 65535) and max_blocks selected blocks (as coco_tree_reserve). */
int coco_sparse_reserve(coco_layer_t h, int32_t max_rows, int32_t max_blocks);

/* Choose n_select blocks of its sequence for each row and kv head. The row
 * attends min(ctx_lens, position + 1) keys; of the nb blocks that hold them
 * the first keep_first and the last keep_last are always chosen, then those
 * of the highest score, the lowest block among equals; all nb if
 * nb <= n_select. With q8 = round(q 2^(7 - x)), held within +-127, x the exponent
 * with |q| < 2^x over the head group (held within +-100, non-finite elements
 * 0), the score is the largest over the group's query heads of
 * sum_d q8_d (q8_d > 0 ? summary[0]_d : summary[1]_d), times the block's
 * scale: all in whole numbers, so equal inputs choose equal blocks.
 *   q [n_rows][Hq][hd]; positions [n_rows]; seq_starts as in
 *   coco_layer_forward (NULL: row i is sequence i);
 *   num_blocks: blocks in summary and scales (ids beyond score as block 0)
 *   selected [n_rows][Hkv][n_select] int32: blocks of the sequence (entries of
 *   its table row), ascending, then -1 */
int coco_block_select(coco_layer_t h, const int8_t* summary, const float* scales,
                      int64_t num_blocks, const void* q, int32_t n_rows, const int32_t* positions,
                      const int32_t* seq_starts, int32_t n_seqs, const int32_t* block_table,
                      const int32_t* ctx_lens, int32_t keep_first, int32_t keep_last,
                      int32_t* selected, int32_t n_select, coco_stream_t stream);

/* Attention of each row over its keys (positions 0 .. min(ctx_lens,
 * position + 1) - 1) in the blocks selected[row][kv head] lists, of
 * coco_block_select or the caller's own: distinct blocks in any order;
 * entries outside the row's blocks (-1) are skipped. (Validation mode takes
 * ascending blocks of the row and -1 only.) A row without keys gives zeros. q, o
 * and rows past the sequences as in coco_tree_attention (and so there and in
 * coco_block_select). */
int coco_sparse_attention(coco_layer_t h, int32_t layer, const void* q, void* o, int32_t n_rows,
                          const int32_t* positions, const int32_t* seq_starts, int32_t n_seqs,
                          const int32_t* block_table, const int32_t* ctx_lens,
                          const int32_t* selected, int32_t n_select, coco_stream_t stream);

/* A decode step of one layer (coco_layer_forward with seq_starts NULL: row i is
 * sequence i) whose rows attend selected blocks: once the new token is cached,
 * the summaries of its block are written (coco_kv_summarize from positions
 * on; those of the blocks before it must be there), n_select blocks chosen as by
 * coco_block_select and written to selected, and attended. summary and scales
 * cover the layer's blocks. Needs coco_sparse_reserve. */
int coco_layer_sparse_forward(coco_layer_t h, int32_t layer, void* hidden, int64_t hidden_rows,
                              const int32_t* row_idx, int32_t n_rows, const int32_t* positions,
                              const int32_t* block_table, const int32_t* ctx_lens,
                              int8_t* summary, float* scales, int32_t keep_first,
                              int32_t keep_last, int32_t* selected, int32_t n_select,
                              coco_stream_t stream);

/* Peak probes for benchmarks (not part of the layer): the rates this GPU
 * sustains, against which measured kernels are quoted next to the published
 * peaks. Both enqueue one kernel on `stream` and return COCO_EINVAL for bad
 * arguments or COCO_EHIP for a failed launch (without a coco_last_error
 * message); the caller times them with events on the same stream.
 *
 * coco_probe_read: reads `bytes` (a multiple of 16, 16-byte aligned) of device
 * memory at `buf` once, as 16-byte vector loads spread over `blocks`
 * 256-thread workgroups with a grid-wide stride; variant 0: four loads in
 * flight per thread, 1: eight, 2: eight non-temporal. Writes one 32-bit word
 * per workgroup to `out` (device, >= 4 * blocks bytes).
 *
 * coco_probe_mfma_bf16: `blocks` workgroups of four waves, each wave running
 * `iters` rounds (a multiple of 8) of `chains` (4 or 8) independent
 * v_mfma_f32_32x32x16_bf16 chains on register operands; writes one float per
 * wave to `out` (device, >= 16 * blocks bytes) and the dense flop count of
 * the launch to *flops (host). operands 0: the same small constants in every
 * instruction; 1: random bf16 values with random signs and magnitudes in
 * [0.5, 2), eight operand sets per lane taken in turn, so consecutive
 * instructions of a chain see different data (the rate under the power draw
 * of data like a GEMM's). */
int coco_probe_read(const void* buf, int64_t bytes, void* out, int32_t blocks, int32_t variant,
                    coco_stream_t stream);
int coco_probe_mfma_bf16(int64_t iters, void* out, int32_t blocks, int32_t chains,
                         int32_t operands, double* flops, coco_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* COCO_H */
