// Attention of prompts' rows through a sliding window and a context's first tokens
// (fp32).
//
// The 16 columns of a workgroup are rows times query heads of a key/value head; its
// waves (eight, four for wide heads) take every eighth block of the cache, by its place
// in the sequence, with an online softmax each, merged in LDS in wave order:
//   S^T[16 keys][16 cols] = K Q^T               8 HS x mfma 16x16x4
//   O^T[hd][16 cols] += V^T[hd][16] P^T[16][16] 8 HS x mfma 16x16x4
// with HS = hd / 32. K and V go in as they lie in their tiles, P as it comes out of
// the first product. A block that a column does not see leaves it as it is, bit for
// bit, so a row's result does not depend on the rows beside it.
//
// A product of 2048 operations takes 32 cycles, as many operations a cycle as in the
// vector unit, which is free for the softmax then: 4000 tokens of 16 heads of 64 on 4
// take 413 us (80 TFLOP/s, where a large product of matrices reaches 154) and 1366 with
// a workgroup of eight waves per row and vector instructions. (Two tiles of columns that
// share the loads of a block: 475 us, and half the workgroups for short calls.)
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

constexpr float kLazy = 8.f;  // a maximum is followed once it is 2^8 behind

struct F8 {
  float e[8];
};
__device__ __forceinline__ F8 load8(const float* p) {
  const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4);
  return F8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ bool odd(float v) {  // infinite or NaN
  return (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u;
}
// What a value that is not finite adds to a sum, as a count: 1 for an infinity, 64 for
// a negative one, 4096 for NaN.
__device__ __forceinline__ float odd_count(float v) {
  return !odd(v) ? 0.f : v != v ? 4096.f : v < 0.f ? 64.f : 1.f;
}

// (Four waves have 512 registers each.)
constexpr int waves_of(int HS) { return HS <= 5 ? 8 : 4; }

template <int HS>
__global__ __launch_bounds__(64 * waves_of(HS),
                             HS <= 2 ? 4 : HS <= 5 ? 2 : 1) void window_prompt_f32_kernel(
    const float* __restrict__ q, const float* __restrict__ k_cache,
    const float* __restrict__ v_cache, RowKeys rk, int Hq, int Hkv, int chunks,
    float scale_log2, float* __restrict__ o, float* __restrict__ stats) {
  constexpr int hd = 32 * HS, TC = 16, kPitch = hd + 4, kWaves = waves_of(HS);
  __shared__ __attribute__((aligned(16))) float sm_o[kWaves][TC][kPitch];
  __shared__ float sm_m[kWaves][TC], sm_l[kWaves][TC];
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  // Rows times `heads` query heads from head0 on, of key/value head g.
  const int G = Hq / Hkv, heads = min(G, TC), rows = TC / heads;
  const int g = blockIdx.y / chunks, head0 = blockIdx.y % chunks * heads;
  const int left = min(G - head0, heads);
  const int row_end = min(min((int)blockIdx.x * rows + rows, rk.rows), rk.seq_starts[rk.n_seqs]);
  // (A workgroup's rows may be of several sequences: one after the other.)
  for (int row0 = blockIdx.x * rows; row0 < row_end;) {
    const int s = row_to_seq(rk.seq_starts, rk.n_seqs, row0);
    const int seq_end = min(rk.seq_starts[s + 1], rk.rows);
    const int row1 = min(row_end, seq_end);
    if (row1 <= row0) break;
    const int len = min(max(rk.ctx_lens[s], 0), rk.max_blocks * kBlockTokens);
    const int p_low = len - seq_end + row0, p_high = len - seq_end + row1 - 1;
    const WindowList list = window_list(max(p_low, -1), p_high, rk.window, rk.sinks);
    const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;

    // This lane's column (one that is none repeats the last row or head).
    const int j = c16 / heads, row = min(row0 + j, row1 - 1);
    const int head = g * G + head0 + min(c16 - j * heads, left - 1);
    const int p = max(len - seq_end + row, -1);
    F8 qf[HS];
#pragma unroll
    for (int y = 0; y < HS; ++y)
      qf[y] = load8(q + ((int64_t)row * Hq + head) * hd + 32 * y + 8 * j4);
    float m = -INFINITY, l = 0.f;
    f32x4_t acc[HS][2];
#pragma unroll
    for (int y = 0; y < HS; ++y) acc[y][0] = acc[y][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // The wave's blocks wv, wv + 8, .. : `n_head` of the first tokens', then the window's.
    const int n_head = max(list.head - wv + kWaves - 1, 0) / kWaves;
    const int first = list.first + ((wv - list.first) & (kWaves - 1));
    const int n_all = n_head + max(list.first + list.entries - list.head - first + kWaves - 1, 0) /
                                   kWaves;
    const auto block = [&](int x) {
      return x < n_head ? wv + kWaves * x : first + kWaves * (x - n_head);
    };
    int ids = 0;
    for (int x = 0; x < n_all; ++x) {
      if (x % kWave == 0)
        ids = readable_block(bt[block(min(x + lane, n_all - 1))], rk.num_blocks);
      const int64_t tile =
          ((int64_t)__builtin_amdgcn_readlane(ids, x % kWave) * Hkv + g) * (kBlockTokens * hd);
      F8 kf[HS], vf[HS];
#pragma unroll
      for (int y = 0; y < HS; ++y) {
        kf[y] = load8(k_cache + tile + (y * 64 + lane) * 8);
        vf[y] = load8(v_cache + tile + (y * 64 + lane) * 8);
      }
      const int t0 = block(x) * kBlockTokens;
      // Whether every column sees all of it; if not, a value that is not finite may be
      // one that a column does not see, and stays apart.
      const bool whole = t0 + kBlockTokens - 1 <= p_low &&
                         (t0 > p_high - rk.window || t0 + kBlockTokens - 1 < rk.sinks);
      f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < HS; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          z = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[y].e[e], qf[y].e[e], z, 0, 0, 0);
      bool apart = false;
      if (!whole) {
        bool any = false;
#pragma unroll
        for (int y = 0; y < HS; ++y)
#pragma unroll
          for (int e = 0; e < 8; ++e) any = any || odd(vf[y].e[e]);
        apart = __ballot(any) != 0;
      }
      uint32_t seen = 15;  // bit r: key 4 j4 + r
      if (!whole) {
        seen = window_bits(t0, p, rk.window, rk.sinks) >> (4 * j4) & 15;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!(seen >> r & 1)) z[r] = -INFINITY;
      }
      const float top = col_max4(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) * scale_log2;
      const float m_new = top > m + kLazy ? top : m;
      if (__ballot(m_new != m) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
        for (int y = 0; y < HS; ++y) {
          acc[y][0] *= alpha;
          acc[y][1] *= alpha;
        }
        l *= alpha;
        m = m_new;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      f32x4_t w;
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(fmaf(z[r], scale_log2, -ref));
      l += (w[0] + w[1]) + (w[2] + w[3]);
      if (apart) {
        // The odd values by their counts, 4096 times as many where the weight is 0
        // (infinity times 0), for the columns that see their keys.
#pragma unroll
        for (int y = 0; y < HS; ++y)
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            f32x4_t n = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < 4; ++r)
              n = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  odd_count(vf[y].e[4 * f + r]),
                  seen >> r & 1 ? (w[r] != 0.f ? 1.f : 4096.f) : 0.f, n, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int count = (int)fminf(n[r], 8192.f);
              const float up = count & 63 ? INFINITY : 0.f,
                          down = count >> 6 & 63 ? -INFINITY : 0.f;
              acc[y][f][r] += count >= 4096 ? NAN : up + down;
            }
          }
#pragma unroll
        for (int y = 0; y < HS; ++y)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (odd(vf[y].e[e])) vf[y].e[e] = 0.f;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int y = 0; y < HS; ++y)
#pragma unroll
          for (int f = 0; f < 2; ++f)
            acc[y][f] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[y].e[4 * f + r], w[r], acc[y][f], 0,
                                                             0, 0);
    }
    l = col_sum4(l);
    if (j4 == 0) {
      sm_m[wv][c16] = m;
      sm_l[wv][c16] = l;
    }
#pragma unroll
    for (int y = 0; y < HS; ++y)
#pragma unroll
      for (int f = 0; f < 2; ++f)
        *(f32x4_t*)&sm_o[wv][c16][32 * y + 16 * f + 4 * j4] = acc[y][f];
    __syncthreads();
    for (int x = threadIdx.x; x < TC * (hd / 4); x += 64 * kWaves) {
      const int c = x / (hd / 4), dim = x % (hd / 4) * 4, r0 = c / heads, h = c - r0 * heads;
      if (row0 + r0 >= row1 || h >= left) continue;
      float M = sm_m[0][c];
#pragma unroll
      for (int u = 1; u < kWaves; ++u) M = fmaxf(M, sm_m[u][c]);
      const float ref = M == -INFINITY ? 0.f : M;
      f32x4_t y = {0.f, 0.f, 0.f, 0.f};
      float L = 0.f;
#pragma unroll
      for (int u = 0; u < kWaves; ++u) {
        const float f = __builtin_amdgcn_exp2f(sm_m[u][c] - ref);
        const f32x4_t v = *(const f32x4_t*)&sm_o[u][c][dim];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
        L = fmaf(f, sm_l[u][c], L);
      }
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      const int64_t at = (int64_t)(row0 + r0) * Hq + g * G + head0 + h;
      *(f32x4_t*)(o + at * hd + dim) = y * inv;
      if (stats != nullptr && dim == 0) *(f32x2_t*)(stats + at * 2) = f32x2_t{ref, inv};
    }
    __syncthreads();  // the next sequence's rows go where these were
    row0 = row1;
  }
}

}  // namespace

hipError_t launch_window_prompt_f32(const float* q, const float* k_cache, const float* v_cache,
                                    const RowKeys& rk, int n_rows, int Hq, int Hkv, int hd,
                                    float* o, float* stats, hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  typedef float T;
  const int G = Hq / Hkv, heads = G < 16 ? G : 16, rows = 16 / heads;
  const int chunks = (G + heads - 1) / heads;
  if ((int64_t)Hkv * chunks > 65535) return hipErrorInvalidValue;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)hd);
#define COCO_PROMPT(HS)                                                                         \
  COCO_LAUNCH_LAST((window_prompt_f32_kernel<HS>),                                              \
                   dim3((n_rows + rows - 1) / rows, Hkv * chunks), dim3(64 * waves_of(HS)), 0,  \
                   st, q, k_cache, v_cache, rk, Hq, Hkv, chunks, scale_log2, o, stats)
  COCO_BY_HEAD_DIM(COCO_PROMPT);
#undef COCO_PROMPT
  return hipGetLastError();
}

}  // namespace coco
