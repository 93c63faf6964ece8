// fp32 attention of rows that do not see a plain causal prefix of the paged
// cache: the nodes of a tree of drafted tokens, rows that attend selected blocks,
// and single tokens that see a sliding window and a context's first tokens.
//
// One workgroup per row and GH query heads of one key/value head, eight waves
// striding over the row's blocks with an online softmax each, merged in LDS in
// wave order. Lane (t, j4) holds token t's part of a key tile and, of a value
// tile, tokens 4 j4 .. + 3 of dims 32 p + t and + 16.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

constexpr int kRowsWaves = 8;

struct F8 {
  float e[8];
};
__device__ __forceinline__ F8 load8(const float* p) {
  const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4);
  return F8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}

// Bits k0 .. k0 + 15 of what a tree node sees, k0 counted from the first node:
// set before it (the prefix), the row's mask among the n nodes, clear behind.
__device__ __forceinline__ uint32_t tree_bits(const uint64_t* mask, int words, int n, int k0) {
  if (k0 <= -16) return 0xFFFFu;
  uint64_t v;
  if (k0 >= 0) {
    const int w = k0 >> 6, sh = k0 & 63;
    v = w < words ? mask[w] >> sh : 0;
    if (sh > 48 && w + 1 < words) v |= mask[w + 1] << (64 - sh);
  } else {
    v = mask[0] << -k0 | ((1ull << -k0) - 1);
  }
  const int left = n - k0;
  if (left < 16) v &= left > 0 ? (1ull << left) - 1 : 0;
  return (uint32_t)v & 0xFFFFu;
}

enum RowsMode { kRowsTree, kRowsBlocks, kRowsWindow };

// HS: head_dim / 32.
template <int HS, int GH, RowsMode MODE>
__global__ __launch_bounds__(64 * kRowsWaves) void attn_rows_kernel(
    const float* __restrict__ q, const float* __restrict__ k_cache,
    const float* __restrict__ v_cache, RowKeys rk, int Hq, int Hkv, float* __restrict__ o,
    float* __restrict__ stats) {
  constexpr int hd = 32 * HS;
  __shared__ float sm_m[kRowsWaves][GH], sm_l[kRowsWaves][GH];
  __shared__ float sm_o[kRowsWaves][GH][hd];
  const int i = blockIdx.x, h0 = blockIdx.y * GH;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t = lane & 15, j4 = lane >> 4;
  if (row_past_seqs(rk.seq_starts, rk.n_seqs, i)) return;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int g = h0 / (Hq / Hkv);
  // Keys of the row's sequence that it may attend; tree: nodes, and the first
  // node's place among the keys.
  int n, nodes = 0, prefix = 0;
  const uint64_t* mask = nullptr;
  const int32_t* list = nullptr;
  int entries;
  WindowList win{};
  if constexpr (MODE == kRowsWindow) {
    n = min(max(rk.ctx_lens[s], 0), rk.max_blocks * kBlockTokens);  // (a row per sequence)
    win = window_list(n - 1, n - 1, rk.window, rk.sinks);
  } else if constexpr (MODE == kRowsTree) {
    n = rk.ctx_lens[s];
    nodes = rk.seq_starts[s + 1] - rk.seq_starts[s];
    prefix = n - nodes;
    mask = rk.mask + (int64_t)i * rk.words;
  } else {
    n = min(rk.ctx_lens[s] - 1, rk.positions[i]) + 1;
    list = rk.selected + ((int64_t)i * Hkv + g) * rk.top;
  }
  n = min(max(n, 0), rk.max_blocks * kBlockTokens);
  const int blocks = (n + kBlockTokens - 1) / kBlockTokens;
  entries = MODE == kRowsTree ? blocks : MODE == kRowsBlocks ? rk.top : win.entries;
  const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
  // Scores in powers of two: 2^x is one instruction, within 1 ulp.
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)hd);

  // This lane's part of the queries: dims 32 p + 8 j4 .. + 7.
  F8 qv[GH][HS];
#pragma unroll
  for (int e = 0; e < GH; ++e)
#pragma unroll
    for (int p = 0; p < HS; ++p)
      qv[e][p] = load8(q + ((int64_t)i * Hq + h0 + e) * hd + 32 * p + 8 * j4);

  float m[GH], l[GH], acc[GH][HS][2];
#pragma unroll
  for (int e = 0; e < GH; ++e) {
    m[e] = -INFINITY;
    l[e] = 0.f;
#pragma unroll
    for (int p = 0; p < HS; ++p) acc[e][p][0] = acc[e][p][1] = 0.f;
  }
  // A wave's next 64 entries in its lanes, block of the sequence and of the pool
  // (-1: nothing there), so that an entry costs one dependent read, not three.
  // (Reading a tile while the one before is attended gained nothing more: two
  // waves to a SIMD, it is the instructions that take the time.)
  int b_l = -1, blk_l = 0;
  for (int x = 0; wv + x * kRowsWaves < entries; ++x) {
    if (x % kWave == 0) {
      const int mine = wv + (x + lane) * kRowsWaves;
      b_l = -1;
      if (mine < entries)
        b_l = MODE == kRowsTree ? mine : MODE == kRowsBlocks ? list[mine] : win.block(mine);
      if (b_l >= blocks) b_l = -1;
      if (b_l >= 0) blk_l = readable_block(bt[b_l], rk.num_blocks);
    }
    const int b = __builtin_amdgcn_readlane(b_l, x % kWave);
    if (b < 0) continue;
    const int tok0 = b * kBlockTokens;
    uint32_t seen;
    if constexpr (MODE == kRowsTree) {
      seen = tree_bits(mask, rk.words, nodes, tok0 - prefix);
      if (seen == 0) continue;
    } else if constexpr (MODE == kRowsWindow) {
      seen = window_bits(tok0, n - 1, rk.window, rk.sinks);
    } else {
      seen = n - tok0 < 16 ? (1u << (n - tok0)) - 1 : 0xFFFFu;
    }
    const int64_t tile =
        ((int64_t)__builtin_amdgcn_readlane(blk_l, x % kWave) * Hkv + g) * (kBlockTokens * hd);
    F8 kf[HS], vf[HS];
#pragma unroll
    for (int p = 0; p < HS; ++p) {
      kf[p] = load8(k_cache + tile + (p * 64 + lane) * 8);
      vf[p] = load8(v_cache + tile + (p * 64 + lane) * 8);
    }
    const bool live = seen >> t & 1;
    // Values of tokens that the row does not see may be anything, NaN among it.
    if (seen != 0xFFFFu) {
#pragma unroll
      for (int p = 0; p < HS; ++p)
#pragma unroll
        for (int c = 0; c < 8; ++c)
          if (!(seen >> (4 * j4 + c % 4) & 1)) vf[p].e[c] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < GH; ++e) {
      float z = 0.f;
#pragma unroll
      for (int p = 0; p < HS; ++p)
#pragma unroll
        for (int c = 0; c < 8; ++c) z = fmaf(qv[e][p].e[c], kf[p].e[c], z);
      z = col_sum4(z);
      z = live ? z * scale_log2 : -INFINITY;
      const float m_new = fmaxf(m[e], row_max16(z));
      // A block of keys that all score -inf leaves m at -inf.
      const float m_ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m[e] - m_ref);
      const float pr = __builtin_amdgcn_exp2f(z - m_ref);
      l[e] = fmaf(l[e], alpha, row_sum16(pr));
      m[e] = m_new;
      float p4[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) p4[c] = __shfl(pr, 4 * j4 + c, kWave);
#pragma unroll
      for (int p = 0; p < HS; ++p)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          float a = acc[e][p][f] * alpha;
#pragma unroll
          for (int c = 0; c < 4; ++c) a = fmaf(p4[c], vf[p].e[4 * f + c], a);
          acc[e][p][f] = a;
        }
    }
  }
#pragma unroll
  for (int e = 0; e < GH; ++e) {
    if (lane == 0) {
      sm_m[wv][e] = m[e];
      sm_l[wv][e] = l[e];
    }
#pragma unroll
    for (int p = 0; p < HS; ++p)
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        float a = acc[e][p][f];  // dim 32 p + 16 f + lane % 16, tokens 4 j4 ..
        a = col_sum4(a);
        if (j4 == 0) sm_o[wv][e][32 * p + 16 * f + t] = a;
      }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < GH * hd; x += 64 * kRowsWaves) {
    const int e = x / hd, dim = x - e * hd;
    float mx = sm_m[0][e];
#pragma unroll
    for (int w = 1; w < kRowsWaves; ++w) mx = fmaxf(mx, sm_m[w][e]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float a = 0.f, L = 0.f;
#pragma unroll
    for (int w = 0; w < kRowsWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_m[w][e] - ref);
      a = fmaf(f, sm_o[w][e][dim], a);
      L = fmaf(f, sm_l[w][e], L);
    }
    o[((int64_t)i * Hq + h0 + e) * hd + dim] = L == 0.f ? 0.f : a / L;
    if (MODE == kRowsWindow && stats != nullptr && dim == 0) {
      float* to = stats + ((int64_t)i * Hq + h0 + e) * 2;
      to[0] = ref;
      to[1] = L == 0.f ? 0.f : 1.0f / L;
    }
  }
}

}  // namespace

hipError_t launch_attn_rows_f32(const float* q, const float* k_cache, const float* v_cache,
                                const RowKeys& rk, int n_rows, int Hq, int Hkv, int hd, float* o,
                                int num_cus, hipStream_t st, float* stats) {
  if (n_rows <= 0) return hipSuccess;
  // Heads per workgroup: they share the key/value loads; the queries they
  // keep in registers (hd / 4 floats per lane each) bound their number. Fewer of
  // them while the call leaves CUs without a workgroup (a head's bits are its own):
  // 5 rows of 16 heads over 16k keys 85 us with one head, 169 with four; 5 rows of
  // 24 blocks 4.4 and 7.8.
  const int G = Hq / Hkv;
  int gh = (G % 4 == 0 && hd <= 64) ? 4 : (G % 2 == 0 && hd <= 128) ? 2 : 1;
  while (gh > 1 && (int64_t)n_rows * (Hq / gh) < num_cus) gh /= 2;
  const dim3 grid(n_rows, Hq / gh), block(64 * kRowsWaves);
#define COCO_ROWS_MODE(HS, GH, MODE)                                                            \
  COCO_LAUNCH_LAST((attn_rows_kernel<HS, GH, MODE>), grid, block, 0, st, q, k_cache, v_cache,   \
                   rk, Hq, Hkv, o, stats)
#define COCO_ROWS(HS, GH)                                                                       \
  do {                                                                                          \
    if (rk.mask)                                                                                \
      COCO_ROWS_MODE(HS, GH, kRowsTree);                                                        \
    else if (rk.window > 0)                                                                     \
      COCO_ROWS_MODE(HS, GH, kRowsWindow);                                                      \
    else                                                                                        \
      COCO_ROWS_MODE(HS, GH, kRowsBlocks);                                                      \
  } while (0)
#define COCO_ROWS4(HS) \
  if (gh == 4) COCO_ROWS(HS, 4); else if (gh == 2) COCO_ROWS(HS, 2); else COCO_ROWS(HS, 1)
#define COCO_ROWS2(HS) \
  if (gh == 2) COCO_ROWS(HS, 2); else COCO_ROWS(HS, 1)
  switch (hd) {
    case 32: COCO_ROWS4(1); break;
    case 64: COCO_ROWS4(2); break;
    case 96: COCO_ROWS2(3); break;
    case 128: COCO_ROWS2(4); break;
    case 160: COCO_ROWS(5, 1); break;
    case 192: COCO_ROWS(6, 1); break;
    case 224: COCO_ROWS(7, 1); break;
    case 256: COCO_ROWS(8, 1); break;
    default: return hipErrorInvalidValue;
  }
#undef COCO_ROWS4
#undef COCO_ROWS2
#undef COCO_ROWS
#undef COCO_ROWS_MODE
  return hipGetLastError();
}

}  // namespace coco
