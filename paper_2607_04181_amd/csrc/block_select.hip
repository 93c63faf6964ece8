// Block summaries of the paged cache's keys, and the blocks that a cheap score
// selects for each query.
//
// The summary of a (block, kv head) is the largest and the smallest value of
// its keys in every dimension, as bytes against a power of two 2^(x - 7) with
// max(|hi|, |lo|) < 2^x (x held within +-100): hi rounded up, lo down, so that
// the bytes still enclose the keys. For a query q, sum_d max(q_d hi_d, q_d
// lo_d) bounds q . k over the block's keys, and is the inner product of
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

// Bytes of one wave's summary: lane l holds dims l, l + 64, ..
template <typename T>
__global__ __launch_bounds__(256) void summarize_kernel(
    const T* __restrict__ k_cache, int Hkv, int hd, const int32_t* __restrict__ block_table,
    int max_blocks, int64_t num_blocks, const int32_t* __restrict__ first,
    const int32_t* __restrict__ ctx_lens, int8_t* __restrict__ summary,
    float* __restrict__ scales) {
  const int s = blockIdx.y;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = min(ctx_lens[s], max_blocks * kBlockTokens);
  const int b0 = first ? max(first[s], 0) / kBlockTokens : 0;
  const int items = ((n + kBlockTokens - 1) / kBlockTokens - b0) * Hkv;
  for (int it = blockIdx.x * 4 + wv; it < items; it += gridDim.x * 4) {
    const int b = b0 + it / Hkv, g = it % Hkv;
    const int64_t blk = block_table[(int64_t)s * max_blocks + b];
    if (blk < 0 || blk >= num_blocks) continue;
    const int left = min(n - b * kBlockTokens, kBlockTokens);
    const T* tile = k_cache + (blk * Hkv + g) * (int64_t)(kBlockTokens * hd);
    float hi[4], lo[4], a = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int h = lane + 64 * u;
      hi[u] = -INFINITY;
      lo[u] = INFINITY;
      if (h >= hd) continue;
      for (int t = 0; t < left; ++t) {
        const float x = finite_or_0(elem(tile + k_tile_offset(t, h)));
        hi[u] = fmaxf(hi[u], x);
        lo[u] = fminf(lo[u], x);
      }
      a = fmaxf(a, fmaxf(fabsf(hi[u]), fabsf(lo[u])));
    }
    const int x = exponent_of(wave_max(a));
    const float up = ldexpf(1.f, 7 - x);
    int8_t* out = summary + (blk * Hkv + g) * 2 * hd;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int h = lane + 64 * u;
      if (h >= hd) continue;
      out[h] = (int8_t)fminf(fmaxf(ceilf(hi[u] * up), -127.f), 127.f);
      out[hd + h] = (int8_t)fminf(fmaxf(floorf(lo[u] * up), -127.f), 127.f);
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
  return min(max(min(rk.ctx_lens[s], rk.positions[i] + 1), 0), rk.max_blocks * kBlockTokens);
}

constexpr int kScoreWaves = 4;
constexpr int kScoreHeads = 64;  // query heads of a group at a time

// Scores of a row's blocks for one kv head, 16 blocks per wave and step: lane
// (c, j4) holds bytes 16 j4 .. of a 64-byte step of block c's summary and of
// query head c's bytes; the product leaves blocks 4 j4 .. + 3 of head c. HS:
// head_dim / 32 (the steps unrolled: with the sums of a loop over them read in
// the block behind it, the compiler left too few wait states before the first).
template <typename T, int HS>
__global__ __launch_bounds__(64 * kScoreWaves) void block_score_kernel(
    const T* __restrict__ q, const int8_t* __restrict__ summary, const float* __restrict__ scales,
    RowKeys rk, int Hq, int Hkv, uint32_t* __restrict__ keys) {
  constexpr int hd = 32 * HS;
  __shared__ __attribute__((aligned(16))) int8_t q8[kScoreHeads][2 * hd + 16];
  __shared__ float red[kScoreWaves];
  const int i = blockIdx.z, g = blockIdx.y, G = Hq / Hkv;
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, j4 = lane >> 4;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int nb = (row_keys(rk, s, i) + kBlockTokens - 1) / kBlockTokens;
  if ((int)blockIdx.x * 16 * kScoreWaves >= nb) return;
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
  const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
  uint32_t* out = keys + ((int64_t)i * Hkv + g) * rk.max_blocks;
  for (int h0 = 0; h0 < G; h0 += kScoreHeads) {
    const int heads = min(G - h0, kScoreHeads);
    const int padded = (heads + 15) / 16 * 16;
    __syncthreads();
    for (int x = threadIdx.x; x < padded * hd; x += 64 * kScoreWaves) {
      const int h = x / hd, d = x - h * hd;
      // Columns past the group repeat its last head.
      const float v = finite_or_0(elem(qp + (int64_t)(h0 + min(h, heads - 1)) * hd + d));
      const int b = (int)fminf(fmaxf(rintf(v * up), -127.f), 127.f);
      q8[h][d] = (int8_t)max(b, 0);
      q8[h][hd + d] = (int8_t)min(b, 0);
    }
    __syncthreads();
    for (int b0 = (blockIdx.x * kScoreWaves + wv) * 16; b0 < nb;
         b0 += gridDim.x * kScoreWaves * 16) {
      int64_t blk = bt[min(b0 + c16, nb - 1)];
      if (blk < 0 || blk >= rk.num_blocks) blk = 0;
      const int8_t* sp = summary + (blk * Hkv + g) * 2 * hd + 16 * j4;
      i32x4_t sv[HS];
#pragma unroll
      for (int k = 0; k < HS; ++k) sv[k] = *(const i32x4_t*)(sp + 64 * k);
      int best[4] = {INT32_MIN, INT32_MIN, INT32_MIN, INT32_MIN};
      for (int ht = 0; ht < padded; ht += 16) {
        i32x4_t acc = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < HS; ++k)
          acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(
              sv[k], *(const i32x4_t*)&q8[ht + c16][64 * k + 16 * j4], acc, 0, 0, 0);
#pragma unroll
        for (int r = 0; r < 4; ++r) best[r] = max(best[r], acc[r]);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) best[r] = max(best[r], __shfl_xor(best[r], d, kWave));
      if (c16 < 4) {
        const int b = b0 + 4 * j4 + c16;
        if (b < nb) {
          int64_t pb = bt[b];
          if (pb < 0 || pb >= rk.num_blocks) pb = 0;
          const int x = c16 == 0 ? best[0] : c16 == 1 ? best[1] : c16 == 2 ? best[2] : best[3];
          const uint32_t key = order_key((float)x * scales[pb * Hkv + g]);
          out[b] = h0 == 0 ? key : max(out[b], key);
        }
      }
    }
  }
}

constexpr int kSelThreads = 256;
constexpr int kSelWaves = kSelThreads / kWave;

// The choice of one (row, kv head): the always attended blocks, then the
// highest keys, ties to the lowest block; ids ascending, then -1. A radix
// search over four bytes finds the lowest chosen key.
__global__ __launch_bounds__(kSelThreads) void block_choose_kernel(
    RowKeys rk, int Hkv, int keep_first, int keep_last, const uint32_t* __restrict__ keys,
    int32_t* __restrict__ selected) {
  __shared__ int hist[256], digit_s, above_s, sums[2 * kSelWaves];
  const int i = blockIdx.y, g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int s = row_to_seq(rk.seq_starts, rk.n_seqs, i);
  const int nb = (row_keys(rk, s, i) + kBlockTokens - 1) / kBlockTokens;
  const uint32_t* kp = keys + ((int64_t)i * Hkv + g) * rk.max_blocks;
  int32_t* out = selected + ((int64_t)i * Hkv + g) * rk.top;
  if (nb <= rk.top) {
    for (int x = tid; x < rk.top; x += kSelThreads) out[x] = x < nb ? x : -1;
    return;
  }
  // nb > top >= keep_first + keep_last: the two do not meet. What the search
  // still has to choose among the blocks between them:
  const int lo = keep_first, hi = nb - keep_last;
  int want = rk.top - keep_first - keep_last;
  uint32_t prefix = 0;
  if (want > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      hist[tid] = 0;
      __syncthreads();
      for (int b = lo + tid; b < hi; b += kSelThreads) {
        const uint32_t k = kp[b];
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))
          atomicAdd(&hist[(k >> shift) & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int above = 0, d = 255;
        for (; d > 0 && above + hist[d] < want; --d) above += hist[d];
        digit_s = d;
        above_s = above;
      }
      __syncthreads();
      prefix |= (uint32_t)digit_s << shift;
      want -= above_s;
      __syncthreads();
    }
  }
  // prefix: the lowest chosen key; want: how many of the blocks that have it.
  const bool search = rk.top > keep_first + keep_last;
  int placed = 0, ties = 0;
  for (int b0 = 0; b0 < nb; b0 += kSelThreads) {
    const int b = b0 + tid;
    const bool always = b < lo || (b >= hi && b < nb);
    const uint32_t k = (!always && b < nb) ? kp[b] : 0;
    const bool tie = search && !always && b < nb && k == prefix;
    const uint64_t tv = __ballot(tie);
    if (lane == 0) sums[wv] = __popcll(tv);
    __syncthreads();
    int tr = ties;
    for (int w = 0; w < kSelWaves; ++w) {
      if (w < wv) tr += sums[w];
      ties += sums[w];
    }
    tr += __popcll(tv & ((1ull << lane) - 1));
    const bool take =
        always || (search && b < nb && (k > prefix || (tie && tr < want)));
    const uint64_t cv = __ballot(take);
    if (lane == 0) sums[kSelWaves + wv] = __popcll(cv);
    __syncthreads();
    int at = placed;
    for (int w = 0; w < kSelWaves; ++w) {
      const int c = sums[kSelWaves + w];
      if (w < wv) at += c;
      placed += c;
    }
    at += __popcll(cv & ((1ull << lane) - 1));
    if (take && at < rk.top) out[at] = b;
    __syncthreads();
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
  COCO_LAUNCH((summarize_kernel<T>), dim3((unsigned)(most < fill ? most : fill), n_seqs),
              dim3(256), 0, st, k_cache, Hkv, hd, block_table, max_blocks, num_blocks, first,
              ctx_lens, summary, scales);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_block_select(const T* q, const int8_t* summary, const float* scales,
                               const RowKeys& rk, int n_rows, int Hq, int Hkv, int hd,
                               int keep_first, int keep_last, uint32_t* keys, int32_t* selected,
                               hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  if (hd % 32 != 0 || hd > 256 || n_rows > 65535 || Hkv > 65535) return hipErrorInvalidValue;
  const int chunks = (rk.max_blocks + 16 * kScoreWaves - 1) / (16 * kScoreWaves);
  const dim3 grid(chunks < 64 ? chunks : 64, Hkv, n_rows);
#define COCO_SCORE(HS)                                                                       \
  COCO_LAUNCH((block_score_kernel<T, HS>), grid, dim3(64 * kScoreWaves), 0, st, q, summary, \
              scales, rk, Hq, Hkv, keys)
  if constexpr (sizeof(T) == 2) {
    if (hd != 128) return hipErrorInvalidValue;
    COCO_SCORE(4);
  } else {
    switch (hd) {
      case 32: COCO_SCORE(1); break;
      case 64: COCO_SCORE(2); break;
      case 96: COCO_SCORE(3); break;
      case 128: COCO_SCORE(4); break;
      case 160: COCO_SCORE(5); break;
      case 192: COCO_SCORE(6); break;
      case 224: COCO_SCORE(7); break;
      case 256: COCO_SCORE(8); break;
      default: return hipErrorInvalidValue;
    }
  }
#undef COCO_SCORE
  RowKeys chosen = rk;
  chosen.selected = nullptr;
  COCO_LAUNCH(block_choose_kernel, dim3(Hkv, n_rows), dim3(kSelThreads), 0, st, chosen, Hkv,
              keep_first, keep_last, keys, selected);
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
