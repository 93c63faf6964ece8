// Attention through a sliding window and a context's first tokens of sequences with a
// few rows (bf16, hd = 128): at most kFewCols columns, rows times query heads of a
// key/value head.
//
// As single tokens: the cache's bytes bound them, and go from the cache straight to
// registers. A workgroup has 16 columns and one part of the sequence's list, its four
// waves every fourth block with an online softmax each, merged in LDS in wave order; the
// parts are merged by the prompts' second kernel. S = K Q^T and O^T += V^T P^T by 16x16
// products with K and V as they lie in their tiles, P in two bf16 parts (2^-16 of a
// weight off). Workgroups take such items in turn.
//
// 8 rows of 32 heads on 8 over 2000 tokens take 15.8 us and 16 sequences of 8 over 4000
// 59.7 (of which the cache's bytes are 50), in the prompts' kernel 38 and 75.6: its item
// is 256 columns whatever there are. At 64 columns it is 16 and 88 for 39 and 78.
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "window_prompt.h"

namespace coco {

namespace {

constexpr int HD = 128;
constexpr int kTile = kBlockTokens * HD;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kWorkgroups = 2;  // of a CU
constexpr int kCols = 16;
constexpr int kPitch = HD + 4;  // floats between columns in LDS: 4 banks on
constexpr float kLazy = 8.f;    // a maximum is followed once it is 2^8 behind

struct Tile {
  u32x4_t k[4], v[4];
};

// Of two bf16 values: what those that are not finite add to a sum, as counts (1 for an
// infinity, 64 for a negative one, 4096 for NaN).
__device__ __forceinline__ uint32_t odd_count(uint32_t h) {
  if ((h & 0x7F80u) != 0x7F80u) return 0;
  return h & 0x7Fu ? 0x4580u : h & 0x8000u ? 0x4280u : 0x3F80u;
}
__device__ __forceinline__ uint32_t odd_counts(uint32_t w) {
  return odd_count(w & 0xFFFFu) | odd_count(w >> 16) << 16;
}
// The signs of the halves where their exponents are all ones.
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {
  return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
}

__global__ __launch_bounds__(kThreads, kWorkgroups) void window_few_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) float sm_o[kWaves][kCols][kPitch];
  __shared__ float sm_m[kWaves][kCols], sm_l[kWaves][kCols];
  __shared__ PromptSeq seqs_s[kWindowLaunchSeqs];
  __shared__ int red[kWaves];
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63, G = a.Hq / a.Hkv;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  const uint32_t inv_G = small_inv(G);
  // Items: per sequence parts, tiles of columns and key/value heads, innermost last.
  int total = 0, n_parts = 0;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    PromptSeq x{};
    if (s < rk.n_seqs) x = prompt_seq(rk, s, G, a.few);
    const int np = column_parts(x, a.Hq);
    x.part0 = block_prefix<kWaves>(np, red, n_parts) - np;
    const int ni = x.tiles == 0 && parts_fit(a, x)
                       ? (x.n * G + kCols - 1) / kCols * x.splits * a.Hkv
                       : 0;
    x.item0 = block_prefix<kWaves>(ni, red, total) - ni;
    if (s < rk.n_seqs) seqs_s[s] = x;
  }
  __syncthreads();

  const auto one = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
#pragma unroll 1
  for (int item = blockIdx.x; item < total; item += gridDim.x) {
    int lo = 0, hi = rk.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (seqs_s[mid].item0 <= item) lo = mid; else hi = mid - 1;
    }
    const int s = one(lo);
    const PromptSeq& sq = seqs_s[s];
    const int row0 = one(sq.row0), first = one(sq.first), splits = one(sq.splits),
              part = one(sq.part), part0 = one(sq.part0), cols = one(sq.n) * G;
    const int at = one(item - sq.item0), tiles = (cols + kCols - 1) / kCols;
    const int g = at % a.Hkv, r = at / a.Hkv, c0 = r % tiles * kCols, sp = r / tiles;
    const int last = min(cols - c0, kCols) - 1;  // column of the tile
    const WindowList list =
        window_list(max(first, -1), first + one(sq.n) - 1, rk.window, rk.sinks);
    const int e0 = sp * part, e1 = min(list.entries, e0 + part);
    const int n_all = max(e1 - e0 - wv + kWaves - 1, 0) / kWaves;  // the wave's blocks
    const int p_low = max(first + small_div(c0, inv_G), -1),
              p_high = first + small_div(c0 + last, inv_G);

    // This lane's column (one past the last repeats it).
    const int c = c0 + min(c16, last), j = small_div(c, inv_G);
    const int p = max(first + j, -1);
    const bf16_t* qp = a.q + ((int64_t)(row0 + j) * a.Hq + g * G + (c - j * G)) * HD + 8 * j4;
    bf16x8_t qf[4];
#pragma unroll
    for (int x = 0; x < 4; ++x)
      qf[x] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(qp + 32 * x));
    float m = -INFINITY, l = 0.f;
    f32x4_t acc[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // Block x of the wave's: of the sequence, and, 64 at a time in the lanes, of the pool.
    const auto block = [&](int x) { return list.block(e0 + wv + kWaves * x); };
    const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
    int ids = 0;
    const auto load = [&](Tile& t, int x) {
      if (x % kWave == 0)
        ids = readable_block(bt[block(min(x + lane, n_all - 1))], rk.num_blocks);
      const int64_t tile = ((int64_t)__builtin_amdgcn_readlane(ids, x % kWave) * a.Hkv + g) * kTile;
      const u32x4_t* kp = (const u32x4_t*)(a.k_cache + tile);
      const u32x4_t* vp = (const u32x4_t*)(a.v_cache + tile);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        t.k[u] = kp[64 * u + lane];
        t.v[u] = vp[64 * u + lane];
      }
    };
    const auto attend = [&](Tile& t, int x) {
      f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, t.k[u]), qf[u], z,
                                                    0, 0, 0);
      const int t0 = block(x) * kBlockTokens;
      const bool whole = t0 + kBlockTokens - 1 <= p_low &&
                         (t0 > p_high - rk.window || t0 + kBlockTokens - 1 < rk.sinks);
      // Where a column does not see all of it, a value that is not finite may be one that
      // it does not see, and stays apart.
      uint32_t seen = 15;  // bit r: key 4 j4 + r
      bool apart = false;
      if (!whole) {
        seen = window_bits(t0, p, rk.window, rk.sinks) >> (4 * j4) & 15;
        uint32_t odd = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) odd |= odd_halves(t.v[u][e]);
        apart = __ballot(odd != 0) != 0;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (!(seen >> r & 1)) z[r] = -INFINITY;
      }
      const float top = col_max4(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) * a.scale_log2;
      const float m_new = top > m + kLazy ? top : m;
      if (__ballot(m_new != m) != 0) {
        const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[u] *= alpha;
        l *= alpha;
        m = m_new;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      float pr[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) pr[r] = __builtin_amdgcn_exp2f(fmaf(z[r], a.scale_log2, -ref));
      l += (pr[0] + pr[1]) + (pr[2] + pr[3]);
      if (apart) {
        // The odd values by their counts, 4096 times as many where the weight is 0
        // (infinity times 0), for the columns that see their keys.
        uint32_t n[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) n[r] = seen >> r & 1 ? (pr[r] != 0.f ? 0x3F80u : 0x4580u) : 0u;
        const s16x4_t nb =
            __builtin_bit_cast(s16x4_t, u32x2_t{n[0] | n[1] << 16, n[2] | n[3] << 16});
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t w0 = t.v[u / 2][u % 2 * 2], w1 = t.v[u / 2][u % 2 * 2 + 1];
          const f32x4_t counts = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
              __builtin_bit_cast(s16x4_t, u32x2_t{odd_counts(w0), odd_counts(w1)}), nb,
              f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int count = (int)fminf(counts[r], 8192.f);
            const float up = count & 63 ? INFINITY : 0.f, down = count >> 6 & 63 ? -INFINITY : 0.f;
            acc[u][r] += count >= 4096 ? NAN : up + down;
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t odd = odd_halves(t.v[u][e]);
            t.v[u][e] &= ~(odd | (odd - (odd >> 15)));
          }
      }
      const u32x2_t p01 = pack_two_parts(pr[0], pr[1]), p23 = pack_two_parts(pr[2], pr[3]);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const s16x4_t pb = __builtin_bit_cast(s16x4_t, u32x2_t{p01[y], p23[y]});
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const u32x2_t v = {t.v[u / 2][u % 2 * 2], t.v[u / 2][u % 2 * 2 + 1]};
          acc[u] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4_t, v), pb,
                                                             acc[u], 0, 0, 0);
        }
      }
    };
    Tile ta, tb;
    if (n_all > 0) load(ta, 0);
#pragma unroll 1
    for (int x = 0; x < n_all; x += 2) {
      if (x + 1 < n_all) load(tb, x + 1);
      attend(ta, x);
      if (x + 1 >= n_all) break;
      if (x + 2 < n_all) load(ta, x + 2);
      attend(tb, x + 1);
    }
    l = col_sum4(l);
    if (j4 == 0) {
      sm_m[wv][c16] = m;
      sm_l[wv][c16] = l;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) *(f32x4_t*)&sm_o[wv][c16][16 * u + 4 * j4] = acc[u];
    __syncthreads();
    for (int x = tid; x < (last + 1) * (HD / 4); x += kThreads) {
      const int col = x / (HD / 4), dim = x % (HD / 4) * 4;
      float M = sm_m[0][col];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_m[w][col]);
      const float ref = M == -INFINITY ? 0.f : M;
      f32x4_t y = {0.f, 0.f, 0.f, 0.f};
      float L = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm_m[w][col] - ref);
        const f32x4_t v = *(const f32x4_t*)&sm_o[w][col][dim];
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
        L = fmaf(f, sm_l[w][col], L);
      }
      const int jj = small_div(c0 + col, inv_G), head = g * G + (c0 + col - jj * G);
      if (splits > 1) {
        const int64_t to = part0 + ((int64_t)jj * a.Hq + head) * splits + sp;
        *(f32x4_t*)(a.part_o + to * HD + dim) = y;
        if (dim == 0) *(f32x2_t*)(a.part_ml + 2 * to) = f32x2_t{M, L};
      } else {
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        const int cc = head * HD + dim, row = row0 + jj;
        store4(a.o + (a.tiled ? tile_off(row, cc, a.Hq * HD) : (int64_t)row * a.Hq * HD + cc),
               y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
        if (a.stats != nullptr && dim == 0)
          *(f32x2_t*)(a.stats + ((int64_t)row * a.Hq + head) * 2) = f32x2_t{ref, inv};
      }
    }
    __syncthreads();  // the next item's go where these were
  }
}

}  // namespace

hipError_t launch_window_few(const PromptArgs& a, int num_cus, bool last, hipStream_t st) {
  if (last)
    COCO_LAUNCH_LAST(window_few_kernel, dim3(kWorkgroups * num_cus), dim3(kThreads), 0, st, a);
  else
    COCO_LAUNCH(window_few_kernel, dim3(kWorkgroups * num_cus), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace coco
