// Block summaries of the paged cache's keys, and the blocks that a cheap score
// selects for each query.
//
// The summary of a (block, kv head) is the largest and the smallest value of
// its keys in every dimension, as bytes against a power of two 2^(x - 7) with
// max(|hi|, |lo|) < 2^x (x held within +-100): hi rounded up, lo down, so that
// the bytes still enclose the keys, but for what is held within +-127: elements
// above 127/128 of 2^x (or of 2^100), by less than a step of the bytes (below 2^100).
// For a query q, sum_d max(q_d hi_d, q_d lo_d) then bounds q . k over the block's
// keys, or falls short of it by that little, and is the inner product of
// [max(q, 0), min(q, 0)] with [hi, lo]: with q in bytes of its own power of two,
// one int8 matrix product of 2 hd terms per block and head. A sum is a whole
// number below 2^23, times 2^(x - 7) exactly a float: the scores, and with them
// the choice, do not depend on the order of any sum.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float elem(const float* p) { return *p; }
__device__ __forceinline__ float elem(const bf16_t* p) { return bf16_to_f32(*p); }

__device__ __forceinline__ float finite_or_0(float x) { return __builtin_isfinite(x) ? x : 0.f; }

// x with a < 2^x, within [-100, 100] (a >= 0 and finite).
__device__ __forceinline__ int exponent_of(float a) {
  int x = 0;
  (void)frexpf(a, &x);
  return min(100, max(-100, x));
}

// The value of the lane whose index differs in bit BIT, and for 4 in bits 2 to 0
// (a mirror of eight lanes).
template <int BIT>
__device__ __forceinline__ float swap_lanes(float x) {
  constexpr int ctrl = BIT == 8 ? 0x128 : BIT == 4 ? 0x141 : BIT == 2 ? 0x4E : 0xB1;
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xF, 0xF, false));
}

// One step of the largest and smallest of N values over 16 lanes: a lane gives
// one half of its values away and keeps the other (N even), or keeps all.
// Pairs of lanes hold the same values up to here. FIRST: hi and lo are one.
template <int BIT, int N, bool FIRST>
__device__ __forceinline__ void spread_step(float* hi, float* lo, int lane, int& base) {
  if constexpr (N % 2 != 0) {
#pragma unroll
    for (int v = 0; v < N; ++v) {
      hi[v] = fmaxf(hi[v], swap_lanes<BIT>(hi[v]));
      lo[v] = fminf(lo[v], swap_lanes<BIT>(lo[v]));
    }
  } else {
    const bool up = lane & BIT;
    base += up ? N / 2 : 0;
#pragma unroll
    for (int v = 0; v < N / 2; ++v) {
      const float got = swap_lanes<BIT>(up ? hi[v] : hi[v + N / 2]);
      const float own = up ? hi[v + N / 2] : hi[v];
      if constexpr (FIRST) {
        hi[v] = fmaxf(own, got);
        lo[v] = fminf(own, got);
      } else {
        const float got2 = swap_lanes<BIT>(up ? lo[v] : lo[v + N / 2]);
        const float own2 = up ? lo[v + N / 2] : lo[v];
        hi[v] = fmaxf(own, got);
        lo[v] = fminf(own2, got2);
      }
    }
  }
}

__device__ __forceinline__ void load8(const float* p, float* x) {
  const f32x4_t a = *(const f32x4_t*)p, b = *(const f32x4_t*)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = finite_or_0(a[i]);
    x[4 + i] = finite_or_0(b[i]);
  }
}
__device__ __forceinline__ void load8(const bf16_t* p, float* x) {
  const u32x4_t a = *(const u32x4_t*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = finite_or_0(bf16_to_f32(a[i] & 0xFFFFu));
    x[2 * i + 1] = finite_or_0(__uint_as_float(a[i] & 0xFFFF0000u));
  }
}

// A tile's summary by one wave: lane (t, j4) reads token t's dims 32 p + 8 j4 ..
// + 7 as they lie, and the 16 lanes of a j4 halve what they hold in each step of
// the reduction over tokens. HS: head_dim / 32.
template <typename T, int HS>
__global__ __launch_bounds__(256) void summarize_kernel(
    const T* __restrict__ k_cache, int Hkv, const int32_t* __restrict__ block_table,
    int max_blocks, int64_t num_blocks, const int32_t* __restrict__ first,
    const int32_t* __restrict__ ctx_lens, int8_t* __restrict__ summary,
    float* __restrict__ scales) {
  constexpr int hd = 32 * HS, V = 8 * HS;
  constexpr int V1 = V / 2, V2 = V1 / 2, V3 = V2 / 2, V4 = V3 % 2 ? V3 : V3 / 2;
  const int s = blockIdx.y;
  const int lane = threadIdx.x & 63, j4 = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = min(ctx_lens[s], max_blocks * kBlockTokens);
  const int b0 = first ? max(first[s], 0) / kBlockTokens : 0;
  const int items = ((n + kBlockTokens - 1) / kBlockTokens - b0) * Hkv;
  for (int it = blockIdx.x * 4 + wv; it < items; it += gridDim.x * 4) {
    const int b = b0 + it / Hkv, g = it % Hkv;
    const int64_t blk = block_table[(int64_t)s * max_blocks + b];
    if (blk < 0 || blk >= num_blocks) continue;
    // Lanes past the last token repeat it.
    const int t = min(lane & 15, n - b * kBlockTokens - 1);
    const T* tile = k_cache + (blk * Hkv + g) * (int64_t)(kBlockTokens * hd) + (j4 * 16 + t) * 8;
    float hi[V], lo[V1];
#pragma unroll
    for (int p = 0; p < HS; ++p) load8(tile + 512 * p, hi + 8 * p);
    int base = 0;  // the lane's values are V4 from here on, value 8 p + e dim 32 p + 8 j4 + e
    spread_step<8, V, true>(hi, lo, lane, base);
    spread_step<4, V1, false>(hi, lo, lane, base);
    spread_step<2, V2, false>(hi, lo, lane, base);
    spread_step<1, V3, false>(hi, lo, lane, base);
    float a = 0.f;
#pragma unroll
    for (int v = 0; v < V4; ++v) a = fmaxf(a, fmaxf(fabsf(hi[v]), fabsf(lo[v])));
    const int x = exponent_of(wave_max(a));
    const float up = ldexpf(1.f, 7 - x);
    int8_t* out = summary + (blk * Hkv + g) * 2 * hd;
    int bh[V4], bl[V4];
#pragma unroll
    for (int v = 0; v < V4; ++v) {
      bh[v] = (int)fminf(fmaxf(ceilf(hi[v] * up), -127.f), 127.f);
      bl[v] = (int)fminf(fmaxf(floorf(lo[v] * up), -127.f), 127.f);
    }
    const int d0 = 8 * j4 + (base >> 3) * 32 + (base & 7);
    if constexpr (V4 == 2) {
      *(uint16_t*)(out + d0) = (uint16_t)((bh[0] & 0xFF) | (bh[1] & 0xFF) << 8);
      *(uint16_t*)(out + hd + d0) = (uint16_t)((bl[0] & 0xFF) | (bl[1] & 0xFF) << 8);
    } else {
#pragma unroll
      for (int v = 0; v < V4; ++v) {
        const int d = 8 * j4 + ((base + v) >> 3) * 32 + ((base + v) & 7);
        out[d] = (int8_t)bh[v];
        out[hd + d] = (int8_t)bl[v];
      }
    }
    if (lane == 0) scales[blk * Hkv + g] = ldexpf(1.f, x - 7);
  }
}

// Floats as unsigned integers of the same order.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int row_keys(const RowKeys& rk, int s, int i) {
  return min(max(min(rk.ctx_lens[s] - 1, rk.positions[i]) + 1, 0), rk.max_blocks * kBlockTokens);
}

constexpr int kScoreWaves = 4;
constexpr int kScoreHeads = 64;  // query heads of a group at a time

// Scores of a row's blocks for one kv head, in a grid of their own: scored and
// chosen by one workgroup per row and head, a row of 1900 blocks takes 10 us
// longer and 96 rows of 640 2 us less. Bound by the summaries' bytes in pieces of
// 256 (those rows: 141 MB in 42 us; loading a step ahead, with fewer workgroups
// and more steps of each, changes nothing). 64 blocks per wave and step, all
// loads of the first step issued before the queries are turned into bytes: lane
// (c, j4) holds bytes 16 j4 .. of each 64-byte piece of the summaries of blocks
// c, 16 + c, ..; the product with the same bytes of query head c leaves heads
// 4 j4 .. + 3 of block c. HS: head_dim / 32 (the pieces unrolled: behind a loop over
// them the compiler read the first sum after two wait states in place of eight;
// tests/test_mfma_waits.py looks for that in the assembly of every kernel).
template <typename T, int HS>
__global__ __launch_bounds__(64 * kScoreWaves) void block_score_kernel(
    const T* __restrict__ q, const int8_t* __restrict__ summary, const float* __restrict__ scales,
    RowKeys rk, int n_rows, int chunks, int Hq, int Hkv, int64_t stride,
    uint32_t* __restrict__ keys) {
  constexpr int hd = 32 * HS;
  __shared__ __attribute__((aligned(16))) int8_t q8[kScoreHeads][2 * hd + 16];
  __shared__ float red[kScoreWaves];
  // The heads of a (row, chunk) run on one XCD (blockIdx % 8): they share the
  // lines of the scales and of the block table.
  const int at8 = blockIdx.x / 8, g = at8 % Hkv, unit = at8 / Hkv * 8 + blockIdx.x % 8;
  const int i = unit / chunks, chunk = unit - i * chunks;
  if (i >= n_rows) return;
  const int G = Hq / Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  if (row_past_seqs(rk.seq_starts, rk.n_seqs, i)) return;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int nb = (row_keys(rk, s, i) + kBlockTokens - 1) / kBlockTokens;
  // Rows that choose all their blocks need no scores.
  if (nb <= rk.top || chunk * 64 * kScoreWaves >= nb) return;
  const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;

  i32x4_t sv[4][HS];
  float sc = 0.f;
  auto load = [&](int b0) {  // blocks b0 .. + 63 (past the end: the last)
    int blk = bt[min(b0 + lane, nb - 1)];
    if (blk < 0 || blk >= rk.num_blocks) blk = 0;
    sc = scales[(int64_t)blk * Hkv + g];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t at = __shfl(blk, 16 * u + c16, kWave);
      const int8_t* sp = summary + (at * Hkv + g) * 2 * hd + 16 * j4;
#pragma unroll
      for (int k = 0; k < HS; ++k) sv[u][k] = *(const i32x4_t*)(sp + 64 * k);
    }
  };
  const int first = (chunk * kScoreWaves + wv) * 64;
  if (first < nb) load(first);

  const T* qp = q + ((int64_t)i * Hq + g * G) * hd;
  float a = 0.f;
  for (int x = threadIdx.x; x < G * hd; x += 64 * kScoreWaves)
    a = fmaxf(a, fabsf(finite_or_0(elem(qp + x))));
  a = wave_max(a);
  if (lane == 0) red[wv] = a;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kScoreWaves; ++w) a = fmaxf(a, red[w]);
  const float up = ldexpf(1.f, 7 - exponent_of(a));
  uint32_t* out = keys + ((int64_t)i * Hkv + g) * stride;
  for (int h0 = 0; h0 < G; h0 += kScoreHeads) {
    const int heads = min(G - h0, kScoreHeads);
    const int padded = (heads + 15) / 16 * 16;
    __syncthreads();
    for (int x = threadIdx.x; x < padded * hd; x += 64 * kScoreWaves) {
      const int h = x / hd, d = x - h * hd;
      // Rows past the group repeat its last head.
      const float v = finite_or_0(elem(qp + (int64_t)(h0 + min(h, heads - 1)) * hd + d));
      const int b = (int)fminf(fmaxf(rintf(v * up), -127.f), 127.f);
      q8[h][d] = (int8_t)max(b, 0);
      q8[h][hd + d] = (int8_t)min(b, 0);
    }
    __syncthreads();
    for (int b0 = first; b0 < nb; b0 += chunks * kScoreWaves * 64) {
      if (h0 != 0 || b0 != first) load(b0);
      int best[4] = {INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
      for (int ht = 0; ht < padded; ht += 16) {
        i32x4_t qv[HS];
#pragma unroll
        for (int k = 0; k < HS; ++k) qv[k] = *(const i32x4_t*)&q8[ht + c16][64 * k + 16 * j4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          i32x4_t acc = {0, 0, 0, 0};
#pragma unroll
          for (int k = 0; k < HS; ++k)
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(qv[k], sv[u][k], acc, 0, 0, 0);
          best[u] = max(best[u], max(max(acc[0], acc[1]), max(acc[2], acc[3])));
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        best[u] = max(best[u], __shfl_xor(best[u], 16, kWave));
        best[u] = max(best[u], __shfl_xor(best[u], 32, kWave));
      }
      const int x = j4 == 0 ? best[0] : j4 == 1 ? best[1] : j4 == 2 ? best[2] : best[3];
      const int b = b0 + lane;
      if (b < nb) {
        const uint32_t key = order_key((float)x * sc);
        out[b] = h0 == 0 ? key : max(out[b], key);
      }
    }
  }
}

constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kSelKeys = 8;  // of a thread, consecutive
constexpr int kSelChunk = kSelThreads * kSelKeys;

// Inclusive sum over the workgroup's threads; red: one int per wave, free again
// once every thread has passed the next barrier.
__device__ __forceinline__ int sel_scan(int x, int* red, int& all) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  x = wave_scan(x);
  if (lane == kWave - 1) red[wv] = x;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < kSelWaves; ++w) {
    if (w < wv) x += red[w];
    all += red[w];
  }
  return x;
}

// The choice of one (row, kv head): the always attended blocks, then the
// highest keys, ties to the lowest block; ids ascending, then -1. The lowest
// chosen key is found digit by digit, 8 bits at a time from the highest bit in
// which the keys differ, until all keys that share the digits so far are chosen;
// a thread's consecutive keys stay in its registers where a row has no more
// than 2048 blocks.
__global__ __launch_bounds__(kSelThreads) void block_choose_kernel(
    RowKeys rk, int Hkv, int keep_first, int keep_last, int64_t stride,
    const uint32_t* __restrict__ keys, int32_t* __restrict__ selected) {
  __shared__ int hist[256], red[2][kSelWaves], digit_s, above_s, count_s;
  __shared__ uint32_t ends[2][kSelWaves];
  const int i = blockIdx.y, g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (row_past_seqs(rk.seq_starts, rk.n_seqs, i)) return;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int nb = (row_keys(rk, s, i) + kBlockTokens - 1) / kBlockTokens;
  const uint32_t* kp = keys + ((int64_t)i * Hkv + g) * stride;
  int32_t* out = selected + ((int64_t)i * Hkv + g) * rk.top;
  if (nb <= rk.top) {
    for (int x = tid; x < rk.top; x += kSelThreads) out[x] = x < nb ? x : -1;
    return;
  }
  // nb > top >= keep_first + keep_last: the two do not meet. What the search
  // still has to choose among the blocks between them:
  const int lo = keep_first, hi = nb - keep_last;
  int want = rk.top - keep_first - keep_last;
  uint32_t k[kSelKeys];
  int held = -1;
  auto fetch = [&](int c0) {  // the thread's keys of the chunk at block c0
    if (held == c0) return;
    held = c0;
#pragma unroll
    for (int e = 0; e < kSelKeys; e += 4) {
      const int b = c0 + tid * kSelKeys + e;
      u32x4_t v = {0, 0, 0, 0};
      if (b < nb) v = *(const u32x4_t*)(kp + b);  // (rows are padded to 4 keys)
#pragma unroll
      for (int r = 0; r < 4; ++r) k[e + r] = v[r];
    }
  };
  uint32_t prefix = 0;
  int shift = 32;
  if (want > 0) {
    uint32_t least = ~0u, most = 0;
    for (int c0 = 0; c0 < nb; c0 += kSelChunk) {
      fetch(c0);
#pragma unroll
      for (int e = 0; e < kSelKeys; ++e) {
        const int b = c0 + tid * kSelKeys + e;
        if (b >= lo && b < hi) {
          least = min(least, k[e]);
          most = max(most, k[e]);
        }
      }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      least = min(least, (uint32_t)__shfl_xor((int)least, d, kWave));
      most = max(most, (uint32_t)__shfl_xor((int)most, d, kWave));
    }
    if (lane == 0) {
      ends[0][wv] = least;
      ends[1][wv] = most;
    }
    hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
      least = min(least, ends[0][w]);
      most = max(most, ends[1][w]);
    }
    // Digits below `shift` are open; all keys agree above it.
    shift = least == most ? 0 : 32 - __builtin_clz(least ^ most);
    prefix = shift >= 32 ? 0 : most >> shift << shift;
    while (shift > 0) {
      const int top_bits = shift;
      shift = max(shift - 8, 0);
      for (int c0 = 0; c0 < nb; c0 += kSelChunk) {
        fetch(c0);
#pragma unroll
        for (int e = 0; e < kSelKeys; ++e) {
          const int b = c0 + tid * kSelKeys + e;
          if (b >= lo && b < hi && (uint64_t)k[e] >> top_bits == (uint64_t)prefix >> top_bits)
            atomicAdd(&hist[(k[e] >> shift) & ((1u << (top_bits - shift)) - 1)], 1);
        }
      }
      __syncthreads();
      // From the highest digit down: the one that the last wanted key has.
      const int mine = hist[255 - tid];
      hist[255 - tid] = 0;
      int all;
      const int upto = sel_scan(mine, red[0], all);
      if (upto >= want && upto - mine < want) {
        digit_s = 255 - tid;
        above_s = upto - mine;
        count_s = mine;
      }
      __syncthreads();
      prefix |= (uint32_t)digit_s << shift;
      want -= above_s;
      if (count_s == want) break;
    }
  }
  // Keys above prefix from bit `shift` on are chosen, and the first `want` of
  // the blocks that equal it there.
  int placed = 0, ties = 0;
  for (int c0 = 0; c0 < nb; c0 += kSelChunk) {
    fetch(c0);
    uint32_t over = 0, tie = 0, always = 0;
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e) {
      const int b = c0 + tid * kSelKeys + e;
      if (b >= nb) continue;
      if (b < lo || b >= hi) {
        always |= 1u << e;
      } else if (shift < 32) {
        over |= (uint32_t)(k[e] >> shift > prefix >> shift) << e;
        tie |= (uint32_t)(k[e] >> shift == prefix >> shift) << e;
      }
    }
    int all;
    int rank = ties + sel_scan(__popc(tie), red[0], all) - __popc(tie);
    ties += all;
    uint32_t take = always | over;
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e)
      if (tie >> e & 1) {
        if (rank < want) take |= 1u << e;
        ++rank;
      }
    int at = placed + sel_scan(__popc(take), red[1], all) - __popc(take);
    placed += all;
#pragma unroll
    for (int e = 0; e < kSelKeys; ++e)
      if (take >> e & 1) {
        if (at < rk.top) out[at] = c0 + tid * kSelKeys + e;
        ++at;
      }
  }
}

}  // namespace

template <typename T>
hipError_t launch_summarize(const T* k_cache, int Hkv, int hd, const int32_t* block_table,
                            int n_seqs, int max_blocks, int64_t num_blocks, const int32_t* first,
                            const int32_t* ctx_lens, int8_t* summary, float* scales, int num_cus,
                            hipStream_t st) {
  if (n_seqs <= 0) return hipSuccess;
  if (hd % 32 != 0 || hd > 256 || n_seqs > 65535) return hipErrorInvalidValue;
  const int64_t most = ((int64_t)max_blocks * Hkv + 3) / 4;
  const int64_t fill = (16LL * num_cus + n_seqs - 1) / n_seqs;
  const dim3 grid((unsigned)(most < fill ? most : fill), n_seqs);
#define COCO_SUMMARY(HS)                                                                    \
  COCO_LAUNCH_LAST((summarize_kernel<T, HS>), grid, dim3(256), 0, st, k_cache, Hkv,         \
                   block_table, max_blocks, num_blocks, first, ctx_lens, summary, scales)
  COCO_BY_HEAD_DIM(COCO_SUMMARY);
#undef COCO_SUMMARY
  return hipGetLastError();
}

template <typename T>
hipError_t launch_block_select(const T* q, const int8_t* summary, const float* scales,
                               const RowKeys& rk, int n_rows, int Hq, int Hkv, int hd,
                               int keep_first, int keep_last, uint32_t* keys, int32_t* selected,
                               hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  if (hd % 32 != 0 || hd > 256 || n_rows > 65535 || Hkv > 65535) return hipErrorInvalidValue;
  int chunks = (rk.max_blocks + 64 * kScoreWaves - 1) / (64 * kScoreWaves);
  if (chunks > 16) chunks = 16;
  const int64_t wgs = ((int64_t)chunks * n_rows + 7) / 8 * 8 * Hkv;
  if (wgs > INT32_MAX) return hipErrorInvalidValue;
  const dim3 grid((unsigned)wgs);
  const int64_t stride = select_stride(rk.max_blocks);
#define COCO_SCORE(HS)                                                                       \
  COCO_LAUNCH((block_score_kernel<T, HS>), grid, dim3(64 * kScoreWaves), 0, st, q, summary, \
              scales, rk, n_rows, chunks, Hq, Hkv, stride, keys)
  COCO_BY_HEAD_DIM(COCO_SCORE);
#undef COCO_SCORE
  RowKeys chosen = rk;
  chosen.selected = nullptr;
  COCO_LAUNCH_LAST(block_choose_kernel, dim3(Hkv, n_rows), dim3(kSelThreads), 0, st, chosen, Hkv,
                   keep_first, keep_last, stride, keys, selected);
  return hipGetLastError();
}

#define COCO_INST(T)                                                                          \
  template hipError_t launch_summarize<T>(const T*, int, int, const int32_t*, int, int,       \
                                          int64_t, const int32_t*, const int32_t*, int8_t*,   \
                                          float*, int, hipStream_t);                          \
  template hipError_t launch_block_select<T>(const T*, const int8_t*, const float*,           \
                                             const RowKeys&, int, int, int, int, int, int,    \
                                             uint32_t*, int32_t*, hipStream_t);
COCO_INST(bf16_t)
COCO_INST(float)
#undef COCO_INST

}  // namespace coco
