// Softmax weights of window rows per key, added up over the rows of a sequence
// and its query heads: weights[s][t] += sum_{row, head} exp(s_t - m) / l, with
// each row's m and l from its attention (which must be done: a weight needs the
// row's whole sum). The scores are computed again, half of the attention's
// products, rather than kept: a prompt has rows x heads of them per key.
//
// bf16: a workgroup has 128 keys of a sequence and key/value head, 32 of them in
// the registers of each of its four waves as the operand of 32x32 products, and
// walks the columns (rows times query heads of the group) that can see them, 32
// at a time through LDS: S[32 keys][32 columns] = K Q^T. A lane then holds one
// column, whose m and 1 / l are two registers, and 16 keys, whose sums over the
// columns it keeps; the 32 lanes' sums meet once, at the end. The heads' sums are
// added by a second kernel, in order.
// fp32: a workgroup has 16 keys, its waves the key/value heads.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int HD = 128;
constexpr int kTile = kBlockTokens * HD;
constexpr int kWaves = 4;
constexpr int kTileBlocks = 2 * kWaves;  // blocks of a workgroup
constexpr int kCols = 32;                // columns of a step
constexpr float kLog2e = 1.4426950408889634f;

// A sequence's rows and cached tokens: N rows of slots first .. last (= L - 1).
struct SeqRows {
  int row0, n, first, last;
  WindowList list;
};
__device__ __forceinline__ SeqRows seq_rows(const RowKeys& rk, int s) {
  SeqRows x;
  x.row0 = rk.seq_starts ? rk.seq_starts[s] : s;
  x.n = rk.seq_starts ? max(rk.seq_starts[s + 1] - x.row0, 0) : 1;
  x.last = min(max(rk.ctx_lens[s], 0), rk.max_blocks * kBlockTokens) - 1;
  x.first = x.last + 1 - x.n;
  // (rows before the context's start see nothing)
  x.list = window_list(max(x.first, -1), x.last, rk.window, rk.sinks);
  if (x.n == 0) x.list.entries = 0;
  return x;
}
// Rows j0 .. j1 - 1 of the sequence that can see a slot of t0 .. t1.
__device__ __forceinline__ void rows_of(const RowKeys& rk, const SeqRows& x, int t0, int t1,
                                        int& j0, int& j1) {
  j0 = max(t0 - x.first, 0);
  j1 = x.n;
  // (slots above p - window, for p up to t1 + window - 1)
  if (t0 >= rk.sinks && rk.window < x.last - t1 + 1)
    j1 = min(max(t1 + rk.window - x.first, 0), x.n);
}

__global__ __launch_bounds__(64 * kWaves, 2) void window_weights_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k_cache, RowKeys rk, int Hq, int Hkv,
    float scale_log2, const float* __restrict__ stats, float* __restrict__ sums) {
  __shared__ __attribute__((aligned(16))) bf16_t qs[2][kCols * HD];
  const int g = blockIdx.x % Hkv, e0 = blockIdx.x / Hkv * kTileBlocks, s = blockIdx.y;
  const int G = Hq / Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c32 = lane & 31, hf = lane >> 5;
  const SeqRows x = seq_rows(rk, s);
  if (e0 >= x.list.entries) return;
  const int e_last = min(e0 + kTileBlocks, x.list.entries) - 1;
  int j0, j1;
  rows_of(rk, x, x.list.block(e0) * kBlockTokens,
          x.list.block(e_last) * kBlockTokens + kBlockTokens - 1, j0, j1);

  // The wave's two blocks (past the list the last one: not stored), and its keys:
  // step u holds dims 16 u + 8 hf .. + 7 of key lane % 32.
  int t[2];
  u32x4_t kf[8];
  {
    const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
    const int ea = min(e0 + 2 * wv, e_last), eb = min(e0 + 2 * wv + 1, e_last);
    t[0] = x.list.block(ea) * kBlockTokens;
    t[1] = x.list.block(eb) * kBlockTokens;
    const int id = readable_block(bt[(lane & 16 ? t[1] : t[0]) / kBlockTokens], rk.num_blocks);
    const bf16_t* kb = k_cache + ((int64_t)id * Hkv + g) * kTile;
#pragma unroll
    for (int u = 0; u < 8; ++u)
      kf[u] = *(const u32x4_t*)(kb + ((u >> 1) * 64 + (2 * (u & 1) + hf) * 16 + (lane & 15)) * 8);
  }
  const int t_low = min(t[0], t[1]), t_high = max(t[0], t[1]) + kBlockTokens - 1;

  const int c_end = j1 * G;
  // A step's columns in operand order: 1 KB pieces u of 16 dims, lane (c, hf) dims
  // 16 u + 8 hf .. + 7 of column c. Each wave brings two.
  auto issue = [&](int c0, int slot) {
    const int c = min(c0 + c32, c_end - 1);
    const bf16_t* qp =
        q + ((int64_t)(x.row0 + c / G) * Hq + g * G + c % G) * HD + 8 * hf;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int u = 2 * wv + y;
      __builtin_amdgcn_global_load_lds(qp + 16 * u, (lds_void_t*)(qs[slot] + u * 512), 16, 0, 0);
    }
  };
  float w[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) w[r] = 0.f;
  int slot = 0;
  if (j0 < j1) issue(j0 * G, 0);
  for (int c0 = j0 * G; c0 < c_end; c0 += kCols) {
    const int c = min(c0 + c32, c_end - 1), j = c / G;
    const f32x2_t st =
        *(const f32x2_t*)(stats + ((int64_t)(x.row0 + j) * Hq + g * G + c % G) * 2);
    __syncthreads();  // the step is here, and the slot of the next free
    if (c0 + kCols < c_end) issue(c0 + kCols, slot ^ 1);
    f32x16_t z = {};
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const u32x4_t b = *(const u32x4_t*)(qs[slot] + (u * 64 + lane) * 8);
      z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[u]),
                                                  __builtin_bit_cast(bf16x8_t, b), z, 0, 0, 0);
    }
    slot ^= 1;
    const int p_low = x.first + c0 / G, p_high = x.first + min(c0 + kCols, c_end) / G;
    if (!(t_high <= p_low && (t_low > p_high - rk.window || t_high < rk.sinks))) {
      const int p = max(x.first + j, -1);
      const uint32_t seen = window_bits(t[0], p, rk.window, rk.sinks) |
                            window_bits(t[1], p, rk.window, rk.sinks) << 16;
      const uint32_t mine = seen >> (4 * hf);
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = (mine >> (8 * (r / 4) + r % 4) & 1) ? z[r] : -INFINITY;
    }
    const float inv = c0 + c32 < c_end ? st[1] : 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      w[r] = fmaf(__builtin_amdgcn_exp2f(fmaf(z[r], scale_log2, -st[0])), inv, w[r]);
  }
  // Sums over the 32 columns; lane r keeps key 8 (r / 4) + 4 hf + r % 4.
  float out = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    float v = row_sum16(w[r]);
    const auto sw =
        __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (c32 == r) out = v;
  }
  if (c32 < 16) {
    const int key = 8 * (c32 / 4) + 4 * hf + c32 % 4, b = key >> 4;
    if (e0 + 2 * wv + b <= e_last)
      sums[((int64_t)s * Hkv + g) * rk.max_blocks * kBlockTokens + (b ? t[1] : t[0]) + (key & 15)] =
          out;
  }
}

// The key/value heads' sums of the blocks that a sequence's rows see, in order.
__global__ __launch_bounds__(256) void window_weights_add_kernel(RowKeys rk, int Hkv,
                                                                 const float* __restrict__ sums,
                                                                 float* __restrict__ weights) {
  const int s = blockIdx.y, at = blockIdx.x * 256 + threadIdx.x;
  const SeqRows x = seq_rows(rk, s);
  const int e = at / kBlockTokens;
  if (e >= x.list.entries) return;
  const int t = x.list.block(e) * kBlockTokens + at % kBlockTokens;
  if (t > x.last) return;
  const int64_t width = (int64_t)rk.max_blocks * kBlockTokens;
  const float* from = sums + (int64_t)s * Hkv * width + t;
  float v = 0.f;
#pragma unroll 8
  for (int g = 0; g < Hkv; ++g) v += from[g * width];
  // (a token between the first ones and every row's window is seen by none)
  if (v != 0.f) weights[s * width + t] += v;
}

constexpr int kRowsWaves = 8;

// HS: head_dim / 32. Lane (t, j4): dims 32 p + 8 j4 .. + 7 of key t.
template <int HS>
__global__ __launch_bounds__(64 * kRowsWaves) void window_weights_f32_kernel(
    const float* __restrict__ q, const float* __restrict__ k_cache, RowKeys rk, int Hq, int Hkv,
    float scale_log2, const float* __restrict__ stats, float* __restrict__ weights) {
  constexpr int hd = 32 * HS;
  __shared__ float sm[kRowsWaves][kBlockTokens];
  const int e = blockIdx.x, s = blockIdx.y, G = Hq / Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = lane & 15, j4 = lane >> 4;
  const SeqRows x = seq_rows(rk, s);
  if (e >= x.list.entries) return;
  const int b = x.list.block(e), t0 = b * kBlockTokens;
  int r0, r1;
  rows_of(rk, x, t0, t0 + kBlockTokens - 1, r0, r1);
  const int id = readable_block(rk.block_table[(int64_t)s * rk.max_blocks + b], rk.num_blocks);
  float w = 0.f;
  for (int g = wv; g < Hkv; g += kRowsWaves) {
    f32x4_t kf[HS][2];
    const float* kb = k_cache + ((int64_t)id * Hkv + g) * (kBlockTokens * hd);
#pragma unroll
    for (int p = 0; p < HS; ++p) {
      kf[p][0] = *(const f32x4_t*)(kb + (p * 64 + lane) * 8);
      kf[p][1] = *(const f32x4_t*)(kb + (p * 64 + lane) * 8 + 4);
    }
    for (int j = r0; j < r1; ++j) {
      const uint32_t seen = window_bits(t0, max(x.first + j, -1), rk.window, rk.sinks);
      const int64_t head0 = (int64_t)(x.row0 + j) * Hq + g * G;
      for (int h = 0; h < G; ++h) {
        const float* qp = q + (head0 + h) * hd + 8 * j4;
        float z = 0.f;
#pragma unroll
        for (int p = 0; p < HS; ++p)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const f32x4_t v = *(const f32x4_t*)(qp + 32 * p + 4 * y);
#pragma unroll
            for (int c = 0; c < 4; ++c) z = fmaf(v[c], kf[p][y][c], z);
          }
        z = col_sum4(z) * scale_log2;
        const f32x2_t st = *(const f32x2_t*)(stats + (head0 + h) * 2);
        if (seen >> t & 1) w = fmaf(__builtin_amdgcn_exp2f(z - st[0]), st[1], w);
      }
    }
  }
  if (lane < kBlockTokens) sm[wv][lane] = w;
  __syncthreads();
  if (threadIdx.x < kBlockTokens && t0 + (int)threadIdx.x <= x.last) {
    float v = 0.f;
#pragma unroll
    for (int u = 0; u < kRowsWaves; ++u) v += sm[u][threadIdx.x];
    if (v != 0.f) weights[((int64_t)s * rk.max_blocks) * kBlockTokens + t0 + threadIdx.x] += v;
  }
}

// The most blocks that a sequence of the call's rows can see.
int64_t most_entries(const RowKeys& rk, int n_rows) {
  const int64_t rows = rk.seq_starts ? n_rows : 1;
  const int64_t w = ((int64_t)rk.window + rows + 2 * kBlockTokens - 2) / kBlockTokens,
                s = ((int64_t)rk.sinks + kBlockTokens - 1) / kBlockTokens;
  return w + s < rk.max_blocks ? w + s : rk.max_blocks;
}

}  // namespace

hipError_t launch_window_weights_bf16(const uint16_t* q, const uint16_t* k_cache, const RowKeys& rk,
                                      int n_rows, int Hq, int Hkv, const float* stats, float* sums,
                                      float* weights, int num_cus, hipStream_t st) {
  if (n_rows <= 0 || rk.n_seqs <= 0) return hipSuccess;
  const int64_t entries = most_entries(rk, n_rows);
  const int64_t tiles = (entries + kTileBlocks - 1) / kTileBlocks * Hkv;
  if (rk.n_seqs > 65535 || tiles > 0x7fffffff || Hq > 16 * Hkv) return hipErrorInvalidValue;
  COCO_LAUNCH(window_weights_kernel, dim3((unsigned)tiles, rk.n_seqs), dim3(64 * kWaves), 0, st, q,
              k_cache, rk, Hq, Hkv, kLog2e / sqrtf((float)HD), stats, sums);
  COCO_LAUNCH_LAST(window_weights_add_kernel,
                   dim3((unsigned)((entries * kBlockTokens + 255) / 256), rk.n_seqs), dim3(256), 0,
                   st, rk, Hkv, sums, weights);
  return hipGetLastError();
}

hipError_t launch_window_weights_f32(const float* q, const float* k_cache, const RowKeys& rk,
                                     int n_rows, int Hq, int Hkv, int hd, const float* stats,
                                     float* weights, int num_cus, hipStream_t st) {
  typedef float T;
  if (n_rows <= 0 || rk.n_seqs <= 0) return hipSuccess;
  const int64_t entries = most_entries(rk, n_rows);
  if (rk.n_seqs > 65535 || hd % 32 != 0) return hipErrorInvalidValue;
  const float scale_log2 = kLog2e / sqrtf((float)hd);
#define COCO_WEIGH(HS)                                                                           \
  COCO_LAUNCH_LAST((window_weights_f32_kernel<HS>), dim3((unsigned)entries, rk.n_seqs),          \
                   dim3(64 * kRowsWaves), 0, st, q, k_cache, rk, Hq, Hkv, scale_log2, stats, weights)
  COCO_BY_HEAD_DIM(COCO_WEIGH);
#undef COCO_WEIGH
  return hipGetLastError();
}

}  // namespace coco
