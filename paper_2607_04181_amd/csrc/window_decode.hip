// Attention of single tokens through a sliding window and a context's first
// tokens (bf16, hd = 128), and the sums of its softmax weights per key.
//
// O = sum_t exp(s_t - m) v_t / sum_t exp(s_t - m) over the slots t that the row
// sees, s_t = q . k_t / sqrt(hd), m the largest. One workgroup per row,
// key/value head and kWindowPart blocks of those that it sees, its four waves
// taking every fourth block with an online softmax each; merged in LDS in wave
// order, and the parts by a second kernel in order, so that a row's bits depend
// on its own length, the window and the first tokens alone.
//
// The query heads of the group are the columns of a 16x16 tile: S = K Q^T with K
// as it lies in the cache tile, O^T += V^T P^T with V as it lies and P^T as S
// leaves it in the registers. P goes in as the sum of two bf16 parts (2^-16 of a
// weight off): the cache's bytes bound the kernel.
//
// Weights: a key's weight needs the row's final maximum and sum, so the scores
// are kept (4 bytes per key and query head beside the 512 of a key and value)
// and the second kernel's other workgroups add them up: head by head in order.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

constexpr int HD = 128;
constexpr int kTile = kBlockTokens * HD;
constexpr int kWaves = 4;
constexpr int kPitch = HD + 4;   // floats between heads in LDS: 4 banks on
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.f;     // a maximum is followed once it is 2^8 behind

struct DecodeArgs {
  const bf16_t* q;
  const bf16_t* k_cache;
  const bf16_t* v_cache;
  RowKeys rk;
  int Hq, Hkv, parts;
  float scale_log2;
  bf16_t* o;
  bool tiled;      // o in tile order
  float* part_o;   // [rows][Hkv][parts][G][128]; null: one part, and no weights
  float* part_ml;  // [rows][Hkv][parts][G][2]
  float* scores;   // [rows][Hkv][parts * kWindowPart][G][16]
  float* weights;  // [rows][max_blocks * 16]
};

__device__ __forceinline__ bf16_t* out_at(const DecodeArgs& a, int i, int head, int dim) {
  const int c = head * HD + dim;
  return a.o + (a.tiled ? tile_off(i, c, a.Hq * HD) : (int64_t)i * a.Hq * HD + c);
}

// The slot of row i, the newest of its sequence (-1: it sees nothing).
__device__ __forceinline__ int row_slot(const RowKeys& rk, int i) {
  return min(max(rk.ctx_lens[i], 0), rk.max_blocks * kBlockTokens) - 1;
}

struct Tile {
  u32x4_t k[4], v[4];
};

__global__ __launch_bounds__(64 * kWaves, 3) void window_decode_kernel(DecodeArgs a) {
  __shared__ __attribute__((aligned(16))) float sm_o[kWaves][16][kPitch];
  __shared__ float sm_m[kWaves][16], sm_l[kWaves][16];
  const int part = blockIdx.y, g = blockIdx.x % a.Hkv, i = blockIdx.x / a.Hkv, G = a.Hq / a.Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  const RowKeys& rk = a.rk;
  const int p = row_slot(rk, i);
  const WindowList list = window_list(p, p, rk.window, rk.sinks);
  const int e0 = part * kWindowPart;
  if (part > 0 && e0 >= list.entries) return;

  // Lane x holds the wave's entry 4 x + wv of the part: its block of the sequence,
  // and its tiles.
  int b = -1, blk = 0;
  {
    const int e = e0 + kWaves * lane + wv;
    if (lane < kWindowPart / kWaves && e < list.entries) b = list.block(e);
  }
  if (b >= 0) blk = readable_block(rk.block_table[(int64_t)i * rk.max_blocks + b], rk.num_blocks);
  const int mine = __popcll(__ballot(b >= 0));  // (the first ones)

  // Operands of the queries: columns past the group are zero.
  bf16x8_t qf[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    u32x4_t w = {0, 0, 0, 0};
    if (c16 < G)
      w = *(const u32x4_t*)(a.q + ((int64_t)i * a.Hq + g * G + c16) * HD + 32 * x + 8 * j4);
    qf[x] = __builtin_bit_cast(bf16x8_t, w);
  }

  float m = -INFINITY, l = 0.f;
  f32x4_t acc[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto load = [&](Tile& t, int x) {
    const int64_t at = ((int64_t)__builtin_amdgcn_readlane(blk, x) * a.Hkv + g) * kTile;
    const u32x4_t* kp = (const u32x4_t*)(a.k_cache + at);
    const u32x4_t* vp = (const u32x4_t*)(a.v_cache + at);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      t.k[u] = kp[64 * u + lane];
      t.v[u] = vp[64 * u + lane];
    }
  };
  auto attend = [&](Tile& t, int x) {
    f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = 0; u < 4; ++u)
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, t.k[u]), qf[u], z,
                                                  0, 0, 0);
    const uint32_t seen =
        window_bits(__builtin_amdgcn_readlane(b, x) * kBlockTokens, p, rk.window, rk.sinks);
    if (seen != 0xFFFFu) {
      // Slots that the row does not see may hold anything, NaN among it.
      const uint32_t s4 = seen >> (4 * j4);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!(s4 >> r & 1)) z[r] = -INFINITY;
      const uint32_t m0 = (s4 & 1 ? 0xFFFFu : 0) | (s4 & 2 ? 0xFFFF0000u : 0);
      const uint32_t m1 = (s4 & 4 ? 0xFFFFu : 0) | (s4 & 8 ? 0xFFFF0000u : 0);
#pragma unroll
      for (int u = 0; u < 4; ++u) t.v[u] &= u32x4_t{m0, m1, m0, m1};
    }
    if (a.scores != nullptr && c16 < G) {
      const int64_t e = ((int64_t)i * a.Hkv + g) * ((int64_t)a.parts * kWindowPart) + e0 +
                        kWaves * x + wv;
      *(f32x4_t*)(a.scores + (e * G + c16) * kBlockTokens + 4 * j4) = z;
    }
    const float top =
        col_max4(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) * a.scale_log2;
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
    const u32x2_t p01 = pack_two_parts(pr[0], pr[1]), p23 = pack_two_parts(pr[2], pr[3]);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const s16x4_t pb = __builtin_bit_cast(s16x4_t, u32x2_t{p01[y], p23[y]});
#pragma unroll
      for (int u = 0; u < 8; ++u)
        acc[u] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            __builtin_bit_cast(s16x4_t, u32x2_t{t.v[u / 2][u % 2 * 2], t.v[u / 2][u % 2 * 2 + 1]}),
            pb, acc[u], 0, 0, 0);
    }
  };

  Tile ta, tb;
  if (mine > 0) load(ta, 0);
#pragma unroll 1
  for (int x = 0; x < mine; x += 2) {
    if (x + 1 < mine) load(tb, x + 1);
    attend(ta, x);
    if (x + 1 >= mine) break;
    if (x + 2 < mine) load(ta, x + 2);
    attend(tb, x + 1);
  }
  l = col_sum4(l);
  if (c16 < G) {
    if (j4 == 0) {
      sm_m[wv][c16] = m;
      sm_l[wv][c16] = l;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) *(f32x4_t*)&sm_o[wv][c16][16 * u + 4 * j4] = acc[u];
  }
  __syncthreads();
  const int64_t at = (((int64_t)i * a.Hkv + g) * a.parts + part) * G;
  for (int x = threadIdx.x; x < G * (HD / 4); x += 64 * kWaves) {
    const int h = x / (HD / 4), dim = x % (HD / 4) * 4;
    float M = sm_m[0][h];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_m[w][h]);
    const float ref = M == -INFINITY ? 0.f : M;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_m[w][h] - ref);
      const f32x4_t v = *(const f32x4_t*)&sm_o[w][h][dim];
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
      L = fmaf(f, sm_l[w][h], L);
    }
    if (a.part_o == nullptr) {
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      store4(out_at(a, i, g * G + h, dim), y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    } else {
      *(f32x4_t*)(a.part_o + (at + h) * HD + dim) = y;
      if (dim == 0) {
        a.part_ml[2 * (at + h)] = M;
        a.part_ml[2 * (at + h) + 1] = L;
      }
    }
  }
}

// Two partial softmaxes in one: the maximum and sum of (M, L) and (m, l).
__device__ __forceinline__ f32x2_t merge_stats(f32x2_t a, f32x2_t b) {
  const float m = fmaxf(a[0], b[0]), ref = m == -INFINITY ? 0.f : m;
  return f32x2_t{m, fmaf(a[1], __builtin_amdgcn_exp2f(a[0] - ref),
                         b[1] * __builtin_amdgcn_exp2f(b[0] - ref))};
}

constexpr int kGroups = 8;        // of 32 threads, four dims a thread
constexpr int kSumEntries = 16;   // blocks of a workgroup that adds up weights
constexpr int kStatHeads = 32;    // heads whose maxima and sums it holds at a time
constexpr int kStatThreads = 8;   // threads to one of those

// Workgroups below `merges` (query heads) of a row put a head's parts together: each
// group every eighth part, the groups in order. (One group to a head, four loads at a
// time: 12.5 us for 4 rows of 32 parts on 64 heads, where this takes 5.0.) The others
// add up the weights of kSumEntries of its blocks, a lane four keys, each wave every
// fourth key/value head of kStatHeads query heads, in wave order.
__global__ __launch_bounds__(256) void window_merge_kernel(DecodeArgs a, int merges) {
  __shared__ f32x2_t sm_ml[kStatHeads];
  __shared__ __attribute__((aligned(16))) f32x4_t sm_w[kGroups][32];
  const int i = blockIdx.y, G = a.Hq / a.Hkv, tid = threadIdx.x;
  const RowKeys& rk = a.rk;
  const int p = row_slot(rk, i);
  const WindowList list = window_list(p, p, rk.window, rk.sinks);
  const int parts = max(1, (list.entries + kWindowPart - 1) / kWindowPart);
  if ((int)blockIdx.x < merges) {
    const int head = blockIdx.x, group = tid >> 5, dim = (tid & 31) * 4;
    const int64_t at = ((int64_t)i * a.Hkv + head / G) * a.parts * G + head % G;
    f32x2_t ml = {-INFINITY, 0.f};
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = group; p0 < parts; p0 += 4 * kGroups) {
      f32x4_t v[4];
      f32x2_t x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t y0 = at + (int64_t)min(p0 + u * kGroups, parts - 1) * G;
        x[u] = *(const f32x2_t*)(a.part_ml + 2 * y0);
        v[u] = *(const f32x4_t*)(a.part_o + y0 * HD + dim);
      }
      float m = ml[0];
#pragma unroll
      for (int u = 0; u < 4; ++u) m = fmaxf(m, x[u][0]);
      const float ref = m == -INFINITY ? 0.f : m, alpha = __builtin_amdgcn_exp2f(ml[0] - ref);
      y *= alpha;
      ml[1] *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (p0 + u * kGroups >= parts) break;
        const float f = __builtin_amdgcn_exp2f(x[u][0] - ref);
        ml[1] = fmaf(f, x[u][1], ml[1]);
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[u][r], y[r]);
      }
      ml[0] = m;
    }
    sm_w[group][tid & 31] = y;
    if ((tid & 31) == 0) sm_ml[group] = ml;
    __syncthreads();
    if (group != 0) return;
    const int groups = min(parts, kGroups);
    float M = sm_ml[0][0], L = 0.f;
    for (int u = 1; u < groups; ++u) M = fmaxf(M, sm_ml[u][0]);
    const float ref = M == -INFINITY ? 0.f : M;
    y = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int u = 0; u < groups; ++u) {
      const float f = __builtin_amdgcn_exp2f(sm_ml[u][0] - ref);
      const f32x4_t v = sm_w[u][tid];
      L = fmaf(f, sm_ml[u][1], L);
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
    }
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    store4(out_at(a, i, head, dim), y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    return;
  }
  const int e0 = ((int)blockIdx.x - merges) * kSumEntries;
  if (e0 >= list.entries) return;
  const int lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int e = e0 + lane / 4, t4 = lane % 4 * 4;
  const bool live = e < list.entries;
  const int step = kStatHeads / G;  // (G <= 16)
  f32x4_t w = {0.f, 0.f, 0.f, 0.f};
  for (int g0 = 0; g0 < a.Hkv; g0 += step) {
    // The heads' maxima and 1 / sums from their parts, eight threads to one.
    const int h = tid / kStatThreads, g1 = min(step, a.Hkv - g0);
    f32x2_t ml = {-INFINITY, 0.f};
    if (h < g1 * G) {
      const int64_t at = ((int64_t)i * a.Hkv + g0 + h / G) * a.parts * G + h % G;
      for (int p0 = tid % kStatThreads; p0 < parts; p0 += kStatThreads)
        ml = merge_stats(ml, *(const f32x2_t*)(a.part_ml + 2 * (at + (int64_t)p0 * G)));
    }
    ml = merge_stats(ml, f32x2_t{row_swap<0xB1>(ml[0]), row_swap<0xB1>(ml[1])});
    ml = merge_stats(ml, f32x2_t{row_swap<0x4E>(ml[0]), row_swap<0x4E>(ml[1])});
    ml = merge_stats(ml, f32x2_t{row_swap<0x141>(ml[0]), row_swap<0x141>(ml[1])});
    if (g0 > 0) __syncthreads();  // every wave is done with the heads before
    if (tid % kStatThreads == 0)
      sm_ml[h] = f32x2_t{ml[0] == -INFINITY ? 0.f : ml[0], ml[1] == 0.f ? 0.f : 1.0f / ml[1]};
    __syncthreads();
    for (int g = wv; g < g1; g += kWaves) {
      const int64_t row = ((int64_t)i * a.Hkv + g0 + g) * ((int64_t)a.parts * kWindowPart);
      const float* z0 = a.scores + (row + (live ? e : e0)) * G * kBlockTokens + t4;
      for (int h0 = 0; h0 < G; h0 += 4) {
        f32x4_t z[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          z[u] = *(const f32x4_t*)(z0 + min(h0 + u, G - 1) * kBlockTokens);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (h0 + u >= G) break;
          const f32x2_t x = sm_ml[g * G + h0 + u];
#pragma unroll
          for (int r = 0; r < 4; ++r)
            w[r] = fmaf(__builtin_amdgcn_exp2f(fmaf(z[u][r], a.scale_log2, -x[0])), x[1], w[r]);
        }
      }
    }
  }
  f32x4_t* const sums = &sm_w[0][0];
  sums[wv * kWave + lane] = w;
  __syncthreads();
  if (wv != 0 || !live) return;
  f32x4_t sum = sums[lane];
#pragma unroll
  for (int u = 1; u < kWaves; ++u) sum += sums[u * kWave + lane];
  const int t0 = list.block(e) * kBlockTokens;
  const uint32_t seen = window_bits(t0, p, rk.window, rk.sinks) >> t4;
  float* to = a.weights + (int64_t)i * rk.max_blocks * kBlockTokens + t0 + t4;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (seen >> r & 1) to[r] += sum[r];
}

}  // namespace

// The most parts of any row: its list is as long as the table, or the blocks that
// the window and the first tokens can touch.
int window_parts(int window, int sinks, int max_blocks) {
  const int64_t w = ((int64_t)window + 2 * kBlockTokens - 2) / kBlockTokens,
                s = ((int64_t)sinks + kBlockTokens - 1) / kBlockTokens;
  const int64_t blocks = w + s < max_blocks ? w + s : max_blocks;
  return (int)((blocks + kWindowPart - 1) / kWindowPart);
}

hipError_t launch_window_decode_bf16(const uint16_t* q, const uint16_t* k_cache,
                                     const uint16_t* v_cache, const RowKeys& rk, int n_rows, int Hq,
                                     int Hkv, uint16_t* o, bool tiled, int parts, float* part_o,
                                     float* part_ml, float* scores, float* weights,
                                     hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  if (Hq > 16 * Hkv || n_rows > 65535 || parts > 65535 ||
      (int64_t)n_rows * Hkv > 0x7fffffff)
    return hipErrorInvalidValue;
  const bool merged = parts > 1 || weights != nullptr;
  DecodeArgs a;
  a.q = q;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.rk = rk;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.parts = parts;
  a.scale_log2 = kLog2e / sqrtf((float)HD);
  a.o = o;
  a.tiled = tiled;
  a.part_o = merged ? part_o : nullptr;
  a.part_ml = merged ? part_ml : nullptr;
  a.scores = weights != nullptr ? scores : nullptr;
  a.weights = weights;
  const dim3 grid(n_rows * Hkv, parts);
  if (!merged) {
    COCO_LAUNCH_LAST(window_decode_kernel, grid, dim3(64 * kWaves), 0, st, a);
    return hipGetLastError();
  }
  COCO_LAUNCH(window_decode_kernel, grid, dim3(64 * kWaves), 0, st, a);
  const int sums = weights != nullptr ? parts * (kWindowPart / kSumEntries) : 0;
  COCO_LAUNCH_LAST(window_merge_kernel, dim3(Hq + sums, n_rows), dim3(256), 0, st, a, Hq);
  return hipGetLastError();
}

}  // namespace coco
