// The replica handle and the error reporting that the library's entry points
// share (internal to libcoco).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <exception>
#include <vector>

#include "../../include/coco.h"
#include "common.h"
#include "kernels.h"

namespace coco {

// Records the message of a failed call on this thread (a fixed buffer:
// reporting an error allocates nothing) and returns `code`.
__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...);

#define HIPCHK(expr)                                                                  \
  do {                                                                                \
    hipError_t e_ = (expr);                                                           \
    if (e_ != hipSuccess)                                                             \
      return ::coco::fail(COCO_EHIP, "%s: %s", #expr, hipGetErrorString(e_));         \
  } while (0)

inline size_t align256(size_t b) { return (b + 255) & ~(size_t)255; }

inline int elem_bytes(int dtype) { return dtype == COCO_BF16 ? 2 : 4; }

// n zeros: no exception leaves an entry point.
template <typename V>
int zeros(std::vector<V>& dst, size_t n) {
  try {
    dst.assign(n, V());
  } catch (const std::exception&) {
    return fail(COCO_ENOMEM, "%zu values do not fit host memory", n);
  }
  return COCO_OK;
}

// Copies n values of a device array to the host behind the stream's work
// (validation mode; synchronises).
template <typename V>
int fetch(std::vector<V>& dst, const V* src, size_t n, hipStream_t st) {
  const int rc = zeros(dst, n);
  if (rc || n == 0) return rc;
  HIPCHK(hipMemcpyAsync(dst.data(), src, n * sizeof(V), hipMemcpyDeviceToHost, st));
  HIPCHK(hipStreamSynchronize(st));
  return COCO_OK;
}

}  // namespace coco

// Per-call buffers of the launch sequence, carved out of one region (the
// handle's workspace, or the static scratch array of the no-alloc entry
// point).
struct Work {
  void *x = nullptr, *h = nullptr, *q = nullptr, *o = nullptr, *h2 = nullptr, *u = nullptr;
  float *x1 = nullptr, *part = nullptr, *attn_o = nullptr, *attn_ml = nullptr;
  // Row sums of squares per K-slice (decode QKV with RMSNorm_1 folded in). The
  // prefill O projection's, per 32 columns ([rows][d / 32]), are in `part`,
  // which prefill has no other use for.
  float* ss = nullptr;
  int32_t* split_off = nullptr;  // decode attention work list
  int32_t* row_info = nullptr;   // prefill row slots [rows][2] (RowSlotArgs)
};

struct coco_layer {
  coco_layer_config cfg;
  std::vector<coco_layer_weights> layers;
  int device = 0;
  int num_cus = 0;  // compute units of `device` (persistent grid sizes)
  bool validate = false;
  char* ws = nullptr;
  size_t ws_bytes = 0;
  // bf16: the library's tile-order copies of every layer's four weight
  // matrices (layers[l].w_* point into it after init).
  char* packed = nullptr;
  size_t packed_bytes = 0;
  Work w;  // the workspace's per-call buffers, sized for max_rows
  double* inv_freq = nullptr;
  float* rope = nullptr;  // RoPE table [rope_rows][head_dim / 2] (cos, sin)
  int rope_rows = 0;      // positions the configuration admits
  size_t act_rows_bytes[7] = {};
  int max_splits = 0;
  int dec_rows = 0;
  // Which of the last regular call's activations h, o, h2, u are in tile
  // order (act_layout), read back row-major by coco_layer_workspace, and
  // that call's rows.
  bool ws_tiled[7] = {};
  int last_rows = 0;
  // Per-kernel timing (benchmark mode).
  bool timing = false;
  std::vector<hipEvent_t> ev;  // pairs: start, stop
  std::vector<int> ev_kind;    // kind of each recorded pair
  bool ev_overflow = false;
  hipStream_t ev_stream = nullptr;
  // Recorded at the end of every call made outside graph capture.
  hipEvent_t done = nullptr;
  // Page requests: the free blocks found (one per block) and each request's
  // first place among them (max_seqs).
  int32_t *page_list = nullptr, *page_off = nullptr;
  // What coco_tree_reserve and coco_sparse_reserve made room for, and the
  // buffers (in `extra`, which keeps outgrown ones until destroy).
  int tree_rows = 0, tree_seqs = 0;
  int sparse_rows = 0, sparse_top = 0;
  char *tree_ws = nullptr, *sparse_ws = nullptr;
  size_t tree_bytes = 0, sparse_bytes = 0;
  float *tree_part_o = nullptr, *tree_part_ml = nullptr;
  int64_t tree_parts = 0;
  int32_t *tree_plan = nullptr, *tree_redo = nullptr;
  float *sparse_part_o = nullptr, *sparse_part_ml = nullptr;
  uint32_t* sparse_keys = nullptr;
  std::vector<char*> extra;
};

namespace coco {

// Blocks every layer of [first, first + n) has.
inline int64_t shared_blocks(const coco_layer* H, int first, int n) {
  int64_t nb = INT64_MAX;
  for (int l = first; l < first + n; ++l)
    if (H->layers[l].num_blocks < nb) nb = H->layers[l].num_blocks;
  return nb;
}

// Records the handle's completion event behind the call's last kernel, unless
// the stream is being captured into a graph (the event would then only fire
// on replays).
int mark_done(coco_layer* H, hipStream_t st);

// The handle's completion event for a call whose last kernel is launched with
// COCO_LAUNCH_LAST: that kernel completes it (recorded behind a kernel, the event
// costs a small call 1 to 2.5 us more). Without such a launch between, or where
// the call is captured or launches its last kernel in several groups (whole
// false), finish() is mark_done.
struct CallEnd {
  coco_layer* H;
  hipStream_t st;
  bool attached = false;
  CallEnd(coco_layer* h, hipStream_t s, bool whole = true) : H(h), st(s) {
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    attached = whole && hipStreamIsCapturing(s, &cs) == hipSuccess &&
               cs == hipStreamCaptureStatusNone;
    if (attached) launch_events().done = H->done;
  }
  ~CallEnd() { launch_events().done = nullptr; }
  int finish() { return attached && !launch_events().done ? COCO_OK : mark_done(H, st); }
};

// What the rows of a layer call attend where that is not their causal prefix.
struct LayerRows {
  // Trees.
  const uint64_t* mask = nullptr;
  int words = 0;
  // Selected blocks.
  int8_t* summary = nullptr;
  float* scales = nullptr;
  int keep_first = 0, keep_last = 0, n_select = 0;
  int32_t* selected = nullptr;
};

// The attention operators without their entry points' checks of the handle and
// batch: what the host can check, validation mode's checks of device arrays
// (positions may be null), and the launches. q, o: the handle's type; tiled: o
// of a bf16 handle in tile order.
int check_tree(const coco_layer* H, int n_rows, const int32_t* seq_starts, int n_seqs,
               const uint64_t* mask, int words);
int validate_tree(const coco_layer* H, int n_rows, const int32_t* positions,
                  const int32_t* seq_starts, int n_seqs, const int32_t* bt, const int32_t* ctx_lens,
                  int words, int64_t num_blocks, hipStream_t st);
int run_tree(coco_layer* H, const coco_layer_weights& w, const void* q, void* o, bool tiled,
             int n_rows, const int32_t* seq_starts, int n_seqs, const int32_t* bt,
             const int32_t* ctx, const uint64_t* mask, int words, hipStream_t st);
int check_select(const coco_layer* H, int n_rows, const int8_t* summary, const float* scales,
                 int64_t num_blocks, int keep_first, int keep_last, const int32_t* selected,
                 int n_select);
int run_summarize(coco_layer* H, const coco_layer_weights& w, int8_t* summary, float* scales,
                  const int32_t* first, const int32_t* ctx, int n_seqs, const int32_t* bt,
                  hipStream_t st);
int run_select(coco_layer* H, const int8_t* summary, const float* scales, int64_t num_blocks,
               const void* q, int n_rows, const int32_t* positions, const int32_t* seq_starts,
               int n_seqs, const int32_t* bt, const int32_t* ctx, int keep_first, int keep_last,
               int32_t* selected, int n_select, hipStream_t st);
int run_sparse(coco_layer* H, const coco_layer_weights& w, const void* q, void* o, bool tiled,
               int n_rows, const int32_t* positions, const int32_t* seq_starts, int n_seqs,
               const int32_t* bt, const int32_t* ctx, const int32_t* selected, int n_select,
               hipStream_t st);

}  // namespace coco
