// Attention of bf16 rows over the blocks that a list selects, on the matrix
// cores.
//
// O = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) over the keys of the listed
// blocks, s_j = q . k_j / sqrt(hd), m the largest. One workgroup per row,
// key/value head and kSparsePart list entries, its four waves taking every
// fourth entry with an online softmax each; merged in LDS in wave order, and
// the parts of a longer list by a second kernel in list order, so that a row's
// bits depend on its list alone.
//
// A (block, head) tile of the cache is read once, for all query heads of the
// group: they are the 16 columns of a 16x16 tile (up to 16 - G of them idle),
// S = K Q^T with K as it lies in the tile, and O^T += V^T P^T with V as it lies
// and P^T as S leaves it in the registers (lane (c, j) holds head c's tokens
// 4 j .. + 3). P goes in as the sum of two bf16 parts, 2^-16 of a weight off: the
// cache's bytes bound the kernel, and the second product costs 0.4% (96 rows of
// 128 blocks, summaries and choice included: 208.4 and 209.2 us; error against 64
// bits 2.3e-3 with one part, 1.7e-3 with two, which is the output's rounding).
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

struct SparseArgs {
  const bf16_t* q;
  const bf16_t* k_cache;
  const bf16_t* v_cache;
  RowKeys rk;
  int Hq, Hkv, parts;
  float scale_log2;
  bf16_t* o;
  bool tiled;      // o in tile order
  float* part_o;   // [rows][Hkv][parts][G][128]
  float* part_ml;  // [rows][Hkv][parts][G][2]
};

__device__ __forceinline__ bf16_t* out_at(const SparseArgs& a, int i, int head, int dim) {
  const int c = head * HD + dim;
  return a.o + (a.tiled ? tile_off(i, c, a.Hq * HD) : (int64_t)i * a.Hq * HD + c);
}

struct Tile {
  u32x4_t k[4], v[4];
};

__global__ __launch_bounds__(64 * kWaves, 3) void sparse_attention_kernel(SparseArgs a) {
  __shared__ __attribute__((aligned(16))) float sm_o[kWaves][16][kPitch];
  __shared__ float sm_m[kWaves][16], sm_l[kWaves][16];
  const int part = blockIdx.x, g = blockIdx.y, i = blockIdx.z, G = a.Hq / a.Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  const RowKeys& rk = a.rk;
  if (row_past_seqs(rk.seq_starts, rk.n_seqs, i)) return;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int n = min(max(min(rk.ctx_lens[s] - 1, rk.positions[i]) + 1, 0),
                    rk.max_blocks * kBlockTokens);
  const int blocks = (n + kBlockTokens - 1) / kBlockTokens;

  // Lane e holds the wave's entry e: its block of the sequence, and its tiles.
  int b = -1;
  {
    const int e = part * kSparsePart + kWaves * lane + wv;
    if (lane < kSparsePart / kWaves && e < rk.top)
      b = rk.selected[((int64_t)i * a.Hkv + g) * rk.top + e];
    if (b >= blocks) b = -1;
  }
  int blk = 0;
  if (b >= 0) blk = readable_block(rk.block_table[(int64_t)s * rk.max_blocks + b], rk.num_blocks);
  uint64_t left = __ballot(b >= 0);

  // Operands of the queries: columns past the group are zero.
  bf16x8_t qf[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    u32x4_t x = {0, 0, 0, 0};
    if (c16 < G) x = *(const u32x4_t*)(a.q + ((int64_t)i * a.Hq + g * G + c16) * HD + 32 * p + 8 * j4);
    qf[p] = __builtin_bit_cast(bf16x8_t, x);
  }

  float m = -INFINITY, l = 0.f;
  f32x4_t acc[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto load = [&](Tile& t) {  // the next entry, which it returns
    const int e = __builtin_ctzll(left);
    left &= left - 1;
    const int64_t at = ((int64_t)__builtin_amdgcn_readlane(blk, e) * a.Hkv + g) * kTile;
    const u32x4_t* kp = (const u32x4_t*)(a.k_cache + at);
    const u32x4_t* vp = (const u32x4_t*)(a.v_cache + at);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      t.k[p] = kp[64 * p + lane];
      t.v[p] = vp[64 * p + lane];
    }
    return e;
  };
  auto attend = [&](Tile& t, int e) {
    f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < 4; ++p)
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, t.k[p]), qf[p], z,
                                                  0, 0, 0);
    const int tokens = n - __builtin_amdgcn_readlane(b, e) * kBlockTokens;
    if (tokens < kBlockTokens) {
      // The row's last block: what lies behind may be anything, NaN among it.
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * j4 + r >= tokens) z[r] = -INFINITY;
      const uint32_t m0 = (4 * j4 < tokens ? 0xFFFFu : 0) | (4 * j4 + 1 < tokens ? 0xFFFF0000u : 0);
      const uint32_t m1 =
          (4 * j4 + 2 < tokens ? 0xFFFFu : 0) | (4 * j4 + 3 < tokens ? 0xFFFF0000u : 0);
#pragma unroll
      for (int p = 0; p < 4; ++p) t.v[p] &= u32x4_t{m0, m1, m0, m1};
    }
    const float top =
        col_max4(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) * a.scale_log2;
    const float m_new = top > m + kLazy ? top : m;
    if (__ballot(m_new != m) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
      for (int x = 0; x < 8; ++x) acc[x] *= alpha;
      l *= alpha;
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.f : m;
    float p[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(fmaf(z[r], a.scale_log2, -ref));
    l += (p[0] + p[1]) + (p[2] + p[3]);
    const u32x2_t p01 = pack_two_parts(p[0], p[1]), p23 = pack_two_parts(p[2], p[3]);
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const s16x4_t pb = __builtin_bit_cast(s16x4_t, u32x2_t{p01[part], p23[part]});
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        acc[2 * x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            __builtin_bit_cast(s16x4_t, u32x2_t{t.v[x][0], t.v[x][1]}), pb, acc[2 * x], 0, 0, 0);
        acc[2 * x + 1] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            __builtin_bit_cast(s16x4_t, u32x2_t{t.v[x][2], t.v[x][3]}), pb, acc[2 * x + 1], 0, 0,
            0);
      }
    }
  };

  Tile ta, tb;
  if (left) {
    int ea = load(ta);
    while (true) {
      const bool second = left != 0;
      int eb = 0;
      if (second) eb = load(tb);
      attend(ta, ea);
      if (!second) break;
      const bool third = left != 0;
      if (third) ea = load(ta);
      attend(tb, eb);
      if (!third) break;
    }
  }
  l = col_sum4(l);
  if (c16 < G) {
    if (j4 == 0) {
      sm_m[wv][c16] = m;
      sm_l[wv][c16] = l;
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) *(f32x4_t*)&sm_o[wv][c16][16 * x + 4 * j4] = acc[x];
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
    if (a.parts == 1) {
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

// A row's parts, four loads at a time, for eight heads per workgroup.
__global__ __launch_bounds__(256) void sparse_combine_kernel(SparseArgs a) {
  const int i = blockIdx.x, head = blockIdx.y * 8 + (threadIdx.x >> 5);
  const int dim = (threadIdx.x & 31) * 4, G = a.Hq / a.Hkv;
  if (head >= a.Hq || row_past_seqs(a.rk.seq_starts, a.rk.n_seqs, i)) return;
  const int64_t at = ((int64_t)i * a.Hkv + head / G) * a.parts * G + head % G;
  float M = -INFINITY, L = 0.f;
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < a.parts; p0 += 4) {
    f32x4_t v[4];
    float m[4], l[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t x = at + (int64_t)min(p0 + u, a.parts - 1) * G;
      m[u] = a.part_ml[2 * x];
      l[u] = a.part_ml[2 * x + 1];
      v[u] = *(const f32x4_t*)(a.part_o + x * HD + dim);
    }
    float m_new = M;
#pragma unroll
    for (int u = 0; u < 4; ++u) m_new = fmaxf(m_new, m[u]);
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(M - ref);
    y *= alpha;
    L *= alpha;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (p0 + u >= a.parts) break;
      const float f = __builtin_amdgcn_exp2f(m[u] - ref);
      L = fmaf(f, l[u], L);
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[u][r], y[r]);
    }
    M = m_new;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  store4(out_at(a, i, head, dim), y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

}  // namespace

hipError_t launch_sparse_attention_bf16(const uint16_t* q, const uint16_t* k_cache,
                                        const uint16_t* v_cache, const RowKeys& rk, int n_rows,
                                        int Hq, int Hkv, uint16_t* o, bool tiled, float* part_o,
                                        float* part_ml, hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  if (Hq > 16 * Hkv || n_rows > 65535 || Hkv > 65535) return hipErrorInvalidValue;
  SparseArgs a;
  a.q = q;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.rk = rk;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.parts = sparse_parts(rk.top);
  a.scale_log2 = kLog2e / sqrtf((float)HD);
  a.o = o;
  a.tiled = tiled;
  a.part_o = part_o;
  a.part_ml = part_ml;
  const dim3 grid(a.parts, Hkv, n_rows), block(64 * kWaves);
  if (a.parts == 1) {
    COCO_LAUNCH_LAST(sparse_attention_kernel, grid, block, 0, st, a);
  } else {
    COCO_LAUNCH(sparse_attention_kernel, grid, block, 0, st, a);
    COCO_LAUNCH_LAST(sparse_combine_kernel, dim3(n_rows, (Hq + 7) / 8), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace coco
