// What the kernels of a prompts' call through a window (bf16) share: its arguments, and
// how the rows of its sequences are divided into work.
#ifndef COCO_WINDOW_PROMPT_H
#define COCO_WINDOW_PROMPT_H

#include "common.h"
#include "kernels.h"

namespace coco {

constexpr int kTileCols = 256;  // columns of a workgroup of the prompts' kernel

// Parts of a list of `entries` blocks for `cols` columns: blocks of one part (a
// multiple of a stage's two).
constexpr int kSplitCols = 512, kPartBlocks = 64, kMaxParts = 16;
constexpr int kFewCols = 64, kFewPart = 32;
__device__ __forceinline__ int window_part(int64_t cols, int entries, int few) {
  if (cols > kSplitCols) return entries > 0 ? (entries + 1) / 2 * 2 : 2;
  const int most = cols > few ? kPartBlocks : kFewPart;
  const int least = (entries + kMaxParts - 1) / kMaxParts;
  return least > most ? (least + 1) / 2 * 2 : most;
}

struct PromptArgs {
  const bf16_t* q;
  const bf16_t* k_cache;
  const bf16_t* v_cache;
  RowKeys rk;
  int Hq, Hkv;
  float scale_log2;
  bf16_t* o;
  bool tiled;        // o in tile order
  float* part_o;     // [column part][HD]
  float* part_ml;    // [column part][2]
  int64_t part_cap;  // column parts they hold
  int32_t* counts;   // [0 .. 7] items drawn, [8] workgroups that are done (not of few)
  float* stats;      // [rows][Hq][2] or null
  int few;           // sequences of so many columns at most are window_few_kernel's
};

// A sequence's rows: N of slots first .. first + N - 1, C columns per key/value
// head in `tiles` workgroup tiles (0: few), the parts of its list, and the blocks
// of the longest item. item0, part0: its first work item and column part.
struct PromptSeq {
  int row0, n, first, tiles, part, splits, longest, item0, part0;
};
// Column parts that a sequence needs, and whether the scratch has them behind those of the
// sequences before: rows of the call that several sequences claim may not fit, and the
// kernels and the merge leave the same sequences out.
__device__ __forceinline__ int column_parts(const PromptSeq& x, int Hq) {
  return x.splits > 1 ? x.n * Hq * x.splits : 0;
}
__device__ __forceinline__ bool parts_fit(const PromptArgs& a, const PromptSeq& x) {
  return (int64_t)x.part0 + column_parts(x, a.Hq) <= a.part_cap;
}
__device__ __forceinline__ PromptSeq prompt_seq(const RowKeys& rk, int s, int G, int few) {
  PromptSeq x;
  // (q, o and the scratch have room for the call's rows, whatever seq_starts says)
  x.row0 = min(max(rk.seq_starts[s], 0), rk.rows);
  x.n = max(min(rk.seq_starts[s + 1], rk.rows) - x.row0, 0);
  const int len = min(max(rk.ctx_lens[s], 0), rk.max_blocks * kBlockTokens);
  x.first = len - x.n;
  const int64_t cols = (int64_t)x.n * G;
  x.tiles = cols > few ? (int)((cols + kTileCols - 1) / kTileCols) : 0;
  const int entries = window_list(max(x.first, -1), len - 1, rk.window, rk.sinks).entries;
  x.part = window_part(cols, entries, few);
  x.splits = max(1, (entries + x.part - 1) / x.part);
  // (the last tile's)
  const int tile0 = max(max(x.first, len - kTileCols / G), -1);
  x.longest = min(window_list(tile0, len - 1, rk.window, rk.sinks).entries, x.part);
  x.item0 = x.part0 = 0;
  return x;
}

// The rows of sequences of at most kFewCols columns: their own kernel. last: of the call.
hipError_t launch_window_few(const PromptArgs& a, int num_cus, bool last, hipStream_t st);

}  // namespace coco

#endif
