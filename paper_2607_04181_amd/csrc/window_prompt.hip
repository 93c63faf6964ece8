// Attention of prompts' rows through a sliding window and a context's first
// tokens (bf16, hd = 128).
//
// The columns of a sequence and key/value head are its rows times the group's
// query heads, C = N G (column c: row c / G, head c % G), so that the heads of a
// group share every key and value that is read. A wave owns 64 columns, as two
// tiles of 32, and walks 32 keys (two blocks) at a time:
//   S^T[32 keys][32 cols] = K[32][hd] Q^T[hd][32]    8 x mfma 32x32x16
//   online softmax per column, 16 keys in each of its two lanes
//   O^T[hd][32 cols] += V^T[hd][32] P^T[32][32]      8 x mfma 32x32x16
// P comes out of the first product in the operand layout of the second: lane
// (c, hf) holds keys 8 q + 4 hf + r of column c.
//
// Why 64 columns: a 32x32x16 product takes 32 cycles and an operand of 1 KB from
// LDS, so one tile per wave would ask LDS for all of its 128 bytes per cycle; two
// tiles share each key and value operand. One wave to a SIMD then, with its 512
// registers (accumulators 128, queries 64, operands 64, scores 32), and nothing
// but its own instructions to fill the pipes: the two tiles are half a step apart,
// so that the vector work of one tile's softmax stands beside the products of the
// other (step st: scores of tile 0 for st + 1 and values of tile 0, softmax of
// tile 1; then scores and values of tile 1, softmax of tile 0 for st + 1).
//
// A workgroup is four waves with 256 columns of one sequence and key/value head.
// They share the keys through LDS in a ring of eight stages of 32. Its list of blocks
// is what its rows see between them; a stage that every column of a wave sees whole
// takes no mask. Values that are not finite are looked for once, at the end: where a
// sum is NaN, the item is done again with such values held apart.
//
// What bounds it: at 8000 tokens, 32 heads on 8 and a window of 4096, 400 GFLOP in 409
// us (0.98 PFLOP/s, where a large product of matrices reaches 1.57). A step of 32 keys
// is 1024 cycles of products for each SIMD and 1136 with the softmax beside them, and
// with every CU at it the clock is at 1.6 to 1.7 GHz: 0.70 us, for 0.85 in the kernel.
// Left out one by one, the operands from LDS are 9% of its time, the loads into LDS 6%
// and the barriers 4%; 10 us of an item are its start and its end.
//
// The list of a sequence with at most kSplitCols columns is split into parts by a
// rule on the sequence's own columns and list, merged by another kernel in order:
// a row's bits depend on its sequence's rows and length alone. (Those with at most
// kFewCols are not of this kernel.)
#include <math.h>

#include "common.h"
#include "kernels.h"
#include "window_prompt.h"

namespace coco {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) bf16_t lds_bf16_t;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;

constexpr int HD = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kCols = 64;                   // columns of a wave
static_assert(kTileCols == kWaves * kCols, "columns of a workgroup");
constexpr int kTile = kBlockTokens * HD;
constexpr int kRing = 8;                    // stages in LDS
constexpr int kStage = 4 * kTile;           // elements: keys and values of two blocks
constexpr int kXCDs = 8;
constexpr int kMaxSeqs = kWindowLaunchSeqs;
static_assert(kMaxSeqs == 512, "a sequence's place among them takes 9 bits");
constexpr float kLazy = 8.f;                // log2 units a running max may lag

// Piece i of four, 1 KB each, of a cache tile into LDS at byte `to`.
template <int I>
__device__ __forceinline__ void load_tile(const bf16_t* from, uint32_t to) {
  __builtin_amdgcn_global_load_lds(from, (lds_void_t*)(uintptr_t)to, 16, I * 1024, 0);
}

// Key fragments of two blocks: step s holds dims 16 s + 8 hf .. + 7 of key m.
__device__ __forceinline__ int k_frag_off(int lane, int s) {
  const int hf = lane >> 5, t = lane & 15;
  return ((s >> 1) * 64 + (2 * (s & 1) + hf) * 16 + t) * 8;
}
// Value operand (pair d, half y) of lane (m, hf): dim value_dim(2 d + y, m), keys
// 4 hf .. + 3 and 8 + 4 hf .. + 3 of a block. A lane's 16-byte chunk of a value
// tile holds two dims 16 apart; which of them is the first operand's alternates
// with the lanes, or eight-byte reads 16 bytes apart would meet in half the banks.
__device__ __forceinline__ int value_swap(int m) { return (m >> 3 ^ m >> 4) & 1; }
__device__ __forceinline__ int value_dim(int i, int m) {
  return 32 * (i & 2) + 32 * (m >> 4) + 16 * ((i & 1) ^ value_swap(m)) + (m & 15);
}

// A column's running maximum before it has seen a key: below every score, and finite,
// so that differences need no test.
constexpr float kNoMax = -3.402823466e38f;

// Largest of 16 values (NaN loses). Three at a time: a maximum of two quiets its
// operands first.
__device__ __forceinline__ float max16(const f32x16_t& s) {
  float m = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
  for (int r = 3; r + 1 < 16; r += 2) m = fmaxf(fmaxf(m, s[r]), s[r + 1]);
  return fmaxf(fmaxf(m, s[15]), kNoMax);
}

// -inf where the column does not see the key. Bit k of seen: key k of the 32.
__device__ __forceinline__ void mask_scores(f32x16_t& s, uint32_t seen, int hf) {
  const uint32_t mine = seen >> (4 * hf);
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    // (a bit spread over a word: comparisons would take 32 scalar registers)
    const uint32_t m = (uint32_t)((int32_t)(mine << (31 - (8 * (r / 4) + r % 4))) >> 31);
    s[r] = __uint_as_float((m & __float_as_uint(s[r])) | (~m & 0xFF800000u));
  }
}

// A product with a weight of 0 would let a non-finite value of a key that some
// columns do not see, or of a slot that holds anything, reach them. Whether any of
// the wave's values is one: their exponents' bits, plus one, carry.
__device__ __forceinline__ bool any_odd(const u32x4_t v[2][2][2]) {
  uint32_t odd = 0;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= (v[j][i >> 1][i & 1][e] & 0x7F807F80u) + 0x00800080u;
  return __ballot((odd & 0x80008000u) != 0) != 0;
}
// Whether any of a tile's sums is not a number, or infinities of both signs.
__device__ __forceinline__ bool any_nan(const f32x16_t acc[4]) {
  f32x4_t t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] += acc[i][r];
  const float sum = (t[0] + t[1]) + (t[2] + t[3]);
  return sum != sum;
}
// Such values are left out (add_odd gives them to the columns that see the key).
__device__ __forceinline__ void drop_odd(u32x4_t v[2][2][2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = v[j][i >> 1][i & 1][e];
        const uint32_t x = ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
        v[j][i >> 1][i & 1][e] = w & ~(x | (x - (x >> 15)));
      }
}

// One tile's columns: running softmax and O^T. acc[i][r]: dim value_dim(i, m), m =
// 8 (r / 4) + 4 hf + r % 4.
struct Cols {
  float m, l;
  f32x16_t acc[4];
};

// The largest score of a column's 32 keys (this lane's 16: mx), in powers of two.
__device__ __forceinline__ float column_top(float mx, float scale_log2) {
  const auto sw =
      __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  return fmaxf(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), kNoMax) * scale_log2;
}
// The running max of a column moves only when a step's largest score exceeds it by
// kLazy: to m_new, where any column's moves.
__device__ __forceinline__ float next_max(const Cols& c, float top) {
  return top > c.m + kLazy ? top : c.m;
}
__device__ __forceinline__ void rescale_if(bool moved, Cols& c, float m_new) {
  if (__builtin_expect(moved, 0)) {
    const float alpha = __builtin_amdgcn_exp2f(c.m - m_new);
#pragma unroll
    for (int i = 0; i < 4; ++i) c.acc[i] *= alpha;
    c.l *= alpha;
    c.m = m_new;
  }
}
__device__ __forceinline__ void rescale(Cols& c, float m_new) {
  rescale_if(__ballot(m_new != c.m) != 0, c, m_new);
}
// Weights of 32 keys as operands of two products: rounded to bf16 once (2^-8 of a weight at
// most, and as the layers' attention does), where single tokens and few rows hold two parts.
// Those are bound by the cache's bytes; here a second part would be 24 products for 16 in a
// half step, whose products bound it, and 16 registers of a wave that uses 510 of its 512.
__device__ __forceinline__ void weights_of(Cols& c, const f32x16_t& z, float scale_log2,
                                           u32x4_t p[2]) {
  float pr[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) pr[r] = __builtin_amdgcn_exp2f(fmaf(z[r], scale_log2, -c.m));
  // (in half_step's order: an item that is done again has the same bits)
  float ls = pr[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) ls += pr[r];
  c.l += ls;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) p[j][e] = pack_bf16x2(pr[8 * j + 2 * e], pr[8 * j + 2 * e + 1]);
}

__device__ __forceinline__ f32x16_t scores_of(const u32x4_t k[8], const bf16x8_t q[8]) {
  f32x16_t z = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[i]), q[i], z, 0, 0,
                                                0);
  return z;
}
// O^T += V^T P^T.
__device__ __forceinline__ void add_values(Cols& c, const u32x4_t v[2][2][2], const u32x4_t p[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c.acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8_t, v[j][i >> 1][i & 1]), __builtin_bit_cast(bf16x8_t, p[j]),
          c.acc[i], 0, 0, 0);
}

// Half a step: sixteen products, and beside each a sixteenth of the other tile's
// softmax. The products: scores z of the next stage (k, q), then values v with
// weights p for cv's columns. The softmax: weights w of scores zs for cs's columns.
// m_now: cs's running max with its scores; m_next: cv's with the next ones. `lds(i)`:
// operand reads that go out behind product i.
// Nothing is moved from one sixteenth to another: left to itself, the compiler puts
// the products back to back and the exponentials behind them, and a wave that is
// alone on its SIMD then has one pipe idle at a time. A product takes 33 cycles and
// lets 28 cycles of other instructions by, an exponential 8 and any other 4 to 5
// (timed one by one), so every sixteenth has an exponential and about four others; a
// result is used a sixteenth after it was asked for, or its latency would show.
template <typename F>
__device__ __forceinline__ void half_step(const u32x4_t k[8], const bf16x8_t q[8], f32x16_t& z,
                                          Cols& cv, const u32x4_t v[2][2][2], const u32x4_t p[2],
                                          Cols& cs, const f32x16_t& zs, u32x4_t w[2], float m_now,
                                          float& m_next, float scale_log2, F lds) {
  z = f32x16_t{};
  const bool moved = __ballot(m_now != cs.m) != 0;
  float pr[16], ls = 0.f, mx = 0.f, top = 0.f;
  float x = fmaf(zs[0], scale_log2, -m_now);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (i < 8)
      z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[i]), q[i], z, 0, 0,
                                                  0);
    else
      cv.acc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8_t, v[i >> 2 & 1][i >> 1 & 1][i & 1]),
          __builtin_bit_cast(bf16x8_t, p[i >> 2 & 1]), cv.acc[i & 3], 0, 0, 0);
    lds(i);
    pr[i] = __builtin_amdgcn_exp2f(x);
    if (i < 15) x = fmaf(zs[i + 1], scale_log2, -m_now);
    if (i == 7) rescale_if(moved, cs, m_now);  // (at the start, its branch waited: 571 us for 558)
    if (i >= 1) ls = i == 1 ? pr[0] : ls + pr[i - 1];
    if (i >= 2 && i % 2 == 0) w[i - 2 >> 3][i - 2 >> 1 & 3] = pack_bf16x2(pr[i - 2], pr[i - 1]);
    if (i == 9) mx = fmaxf(fmaxf(z[0], z[1]), z[2]);
    if (i == 10) mx = fmaxf(fmaxf(mx, z[3]), z[4]);
    if (i == 11) mx = fmaxf(fmaxf(fmaxf(fmaxf(mx, z[5]), z[6]), z[7]), z[8]);
    if (i == 12) mx = fmaxf(fmaxf(mx, z[9]), z[10]);
    if (i == 13)
      mx = fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(mx, z[11]), z[12]), z[13]), z[14]), z[15]), kNoMax);
    if (i == 14) top = column_top(mx, scale_log2);
    // (here, not where they are used)
    asm volatile("" : "+v"(pr[i]), "+v"(x), "+v"(ls), "+v"(mx));
    if (i >= 2 && i % 2 == 0) asm volatile("" : "+v"(w[i - 2 >> 3][i - 2 >> 1 & 3]));
    __builtin_amdgcn_sched_barrier(0);
  }
  cs.l += ls + pr[15];
  w[1][3] = pack_bf16x2(pr[14], pr[15]);
  m_next = next_max(cv, top);
}

// The non-finite values of a stage for the columns that see their keys (seen). A
// product counts them: 1 for each infinity, 64 for each negative one, 4096 for each
// NaN, times 1, or 4096 where the weight is 0 (times infinity: NaN).
__device__ __forceinline__ uint32_t odd_count(uint32_t h) {  // of a value, as bf16
  if ((h & 0x7F80u) != 0x7F80u) return 0;
  return h & 0x7Fu ? 0x4580u : h & 0x8000u ? 0x4280u : 0x3F80u;
}
__device__ __forceinline__ void add_odd(Cols& c, const u32x4_t v[2][2][2], const u32x4_t p[2],
                                        uint32_t seen, int hf) {
  const uint32_t mine = seen >> (4 * hf);
  u32x4_t n[2];
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    const uint32_t w = p[r >> 3][r >> 1 & 3];
    const int key = 8 * (r / 4) + r % 4;
    n[r >> 3][r >> 1 & 3] = (mine >> key & 1 ? (w & 0xFFFFu ? 0x3F80u : 0x4580u) : 0u) |
                            (mine >> key & 2 ? (w >> 16 ? 0x3F80u : 0x4580u) : 0u) << 16;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x16_t t = {};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4_t k;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = v[j][i >> 1][i & 1][e];
        k[e] = odd_count(w & 0xFFFFu) | odd_count(w >> 16) << 16;
      }
      t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k),
                                                  __builtin_bit_cast(bf16x8_t, n[j]), t, 0, 0, 0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      // (whole numbers, exact as far as they are told apart; no branches: 128 of them)
      const int count = (int)fminf(t[r], 8192.f);
      const float one = count & 63 ? INFINITY : 0.f, other = count >> 6 & 63 ? -INFINITY : 0.f;
      c.acc[i][r] += count >= 4096 ? NAN : one + other;
    }
  }
}

__global__ __launch_bounds__(kThreads, 1) void window_prompt_kernel(PromptArgs a) {
  __shared__ __attribute__((aligned(16))) bf16_t ring[kRing * kStage];
  __shared__ PromptSeq seqs_s[kMaxSeqs];
  __shared__ __attribute__((aligned(16))) int order_s[kMaxSeqs], items_s[kMaxSeqs];
  __shared__ int red[kWaves], next_s[2], bad_s[2];
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5, G = a.Hq / a.Hkv;
  const uint32_t inv_G = small_inv(G);

  // Items: per sequence (tile, part) times key/value heads, the heads innermost:
  // item % 8 is the XCD, so that the tiles of a head share that L2's keys where the
  // heads are a multiple of 8. Sequences of the longest items first (order_s, and the
  // first items of each in items_s): the last round of the CUs is of short ones (4 prompts of
  // 340 to 512 tokens on 40 heads of 8, window 1000: 88 us in the call's order, 70).
  int total = 0, n_parts = 0;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    PromptSeq x{};
    if (s < rk.n_seqs) x = prompt_seq(rk, s, G, a.few);
    const int np = column_parts(x, a.Hq);
    x.part0 = block_prefix<kWaves>(np, red, n_parts) - np;
    if (!parts_fit(a, x)) x.tiles = 0;
    // (unlike keys: of equal lengths the first in the call; behind the last none)
    if (s < rk.n_seqs) seqs_s[s] = x;
    if (s < (rk.n_seqs + 3) / 4 * 4)
      items_s[s] = s < rk.n_seqs ? min(x.longest, 0x3FFFFF) << 9 | (511 - s) : -1;
  }
  __syncthreads();
  for (int s = tid; s < rk.n_seqs; s += kThreads) {
    const int mine = items_s[s];
    int before = 0;
#pragma unroll 4
    for (int t = 0; t < rk.n_seqs; t += 4) {
      const i32x4_t v = *(const i32x4_t*)&items_s[t];
      before += (v[0] > mine) + (v[1] > mine) + (v[2] > mine) + (v[3] > mine);
    }
    order_s[before] = s;
  }
  __syncthreads();
  for (int r0 = 0; r0 < rk.n_seqs; r0 += kThreads) {
    int ni = 0;
    if (r0 + tid < rk.n_seqs) {
      const PromptSeq& x = seqs_s[order_s[r0 + tid]];
      ni = x.tiles * x.splits * a.Hkv;
    }
    const int item0 = block_prefix<kWaves>(ni, red, total) - ni;
    if (r0 + tid < rk.n_seqs) items_s[r0 + tid] = item0;
  }
  __syncthreads();

  // (The ring's address goes through a register of its own: the compiler would
  // otherwise wait for every load in flight before each operand read.)
  uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  asm volatile("" : "+s"(ring_at));

  // Workgroups draw the items of their XCD in order.
  const int queues = gridDim.x % kXCDs == 0 ? kXCDs : 1;
  const int queue = blockIdx.x % queues, per_queue = (int)gridDim.x / queues;
  if (tid < 2) bad_s[tid] = 0;

  // An item: one tile of one sequence and key/value head, and one part of its list.
  struct Item {
    int row0, first, splits, part0, sp, g;
    int j_tile, r_tile;  // row of the tile's first column, and its head
    int last;            // its last column
    int64_t rowhead;     // row * Hq + head of a first column of head 0
    int e0, e1, stages;  // of its list
    WindowList list;
    const int32_t* bt;
  };
  Item it{};
  auto one = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  auto describe = [&](int item) {
    int lo = 0, hi = rk.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (items_s[mid] <= item) lo = mid; else hi = mid - 1;
    }
    const int s = one(order_s[lo]);
    const PromptSeq& sq = seqs_s[s];
    it.row0 = one(sq.row0);
    it.first = one(sq.first);
    it.splits = one(sq.splits);
    it.part0 = one(sq.part0);
    it.bt = rk.block_table + (int64_t)s * rk.max_blocks;
    const int part = one(sq.part), at = one(item - items_s[lo]), at_head = at / a.Hkv;
    it.g = at - at_head * a.Hkv;
    const int later = at_head / it.splits;
    it.sp = at_head - later * it.splits;
    // Later rows see more: their tiles first.
    const int tile0 = (one(sq.tiles) - 1 - later) * kTileCols;
    it.j_tile = tile0 / G;
    it.r_tile = tile0 - it.j_tile * G;
    it.last = min(one(sq.n) * G - tile0, kTileCols) - 1;
    it.rowhead = (int64_t)(it.row0 + it.j_tile) * a.Hq + it.g * G;
    it.list = window_list(max(it.first + it.j_tile, -1),
                          it.first + it.j_tile + small_div(it.r_tile + it.last, inv_G), rk.window,
                          rk.sinks);
    it.e0 = it.sp * part;
    it.e1 = min(it.list.entries, it.e0 + part);
    it.stages = it.e1 > it.e0 ? (it.e1 - it.e0 + 1) / 2 : 0;
  };
  // A wave brings one tile of each stage, keys (waves 0, 2) or values of one of
  // its two blocks; past the list the last block again, whose keys count as
  // unseen. Called with st = 0, 1, ..: the blocks of 64 stages at a time in a
  // register's lanes.
  int ids = 0;
  auto refill = [&](int st) {
    const int e = min(it.e0 + (st + lane) * 2 + (wv >> 1), it.e1 - 1);
    ids = readable_block(it.bt[it.list.block(e)], rk.num_blocks);
  };
  auto source = [&](int st) {
    return (wv & 1 ? a.v_cache : a.k_cache) +
           ((int64_t)__builtin_amdgcn_readlane(ids, st & 63) * a.Hkv + it.g) * kTile;
  };
  auto place = [&](int st) { return ring_at + ((st % kRing) * kStage + wv * kTile) * 2; };
  auto issue = [&](int st) {
    if ((st & 63) == 0) refill(st);
    const bf16_t* src = source(st) + lane * 8;
    load_tile<0>(src, place(st));
    load_tile<1>(src, place(st));
    load_tile<2>(src, place(st));
    load_tile<3>(src, place(st));
  };
  // This lane's columns (columns past the last repeat it): their rows' slots, their queries.
  const int wave0 = wv * kCols;
  int p[2];
  bf16x8_t qf[2][8];
  auto begin_item = [&](int item) {
    describe(item);
#pragma unroll 1
    for (int st = 0; st < kRing - 1 && st < it.stages; ++st) issue(st);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int x = it.r_tile + min(wave0 + 32 * t + (lane & 31), it.last), j = small_div(x, inv_G);
      p[t] = max(it.first + it.j_tile + j, -1);
      const bf16_t* qp = a.q + it.rowhead * HD + (x + j * (a.Hq - G)) * HD + 8 * hf;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        qf[t][i] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(qp + 16 * i));
    }
  };

  int drawn_k = blockIdx.x / queues;
  int drawn = 0;
  bool careful = false;  // an item that is done again
  if (drawn_k * queues + queue < total) begin_item(drawn_k * queues + queue);
#pragma unroll 1
  for (int k = 0; drawn_k * queues + queue < total; ++k) {
    if (tid == 0 && !careful) drawn = atomicAdd(a.counts + queue, 1);
    const int stages = it.stages, last = it.last;
    const bool idle = wave0 > last;
    const int fast_end = careful ? 0 : stages - 1;

    // Stages that every column of the wave sees whole: from..to. (Among the window's
    // blocks only; slots above p - window for the latest row, up to p for the first.)
    const int p_low = max(it.first + it.j_tile + small_div(it.r_tile + wave0, inv_G), -1),
              p_high = max(it.first + it.j_tile +
                               small_div(it.r_tile + min(wave0 + kCols - 1, last), inv_G),
                           -1);  // (p_high - window does not overflow)
    const int b_low = max(p_high - rk.window + kBlockTokens, 0) / kBlockTokens,
              b_high = (p_low + 1) / kBlockTokens - 1;
    const int from = (it.list.head + max(b_low - it.list.first, 0) - it.e0 + 1) >> 1,
              to = ((min(it.list.head + b_high - it.list.first, it.e1 - 1) - it.e0 + 1) >> 1) - 1;
    auto whole = [&](int st) { return st >= from && st <= to; };

    Cols c[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      c[t].m = kNoMax;
      c[t].l = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) c[t].acc[i] = f32x16_t{};
    }

    // Step st reads the keys of stage st + 2 and brings stage st + 7 to the place of
    // st - 1. Every second one waits first, until this wave's shares of stages st + 2
    // and st + 3 are here, with three later ones on their way, and until every wave's
    // are: all are done with stage st then. (Past the end the last stage again, so that
    // the loads on their way are always as many. The first kRing - 1 are waited for
    // below. A barrier in every step took 8000 tokens with a window of 4096 439 us, this 434.)
    auto arrive = [&](int st) {
      if (st & 1) {
        wait_vmcnt<4 * (kRing - 5)>();
        stage_barrier();
      }
    };
    auto begin = [&](int st) {
      arrive(st);
      issue(st + kRing - 1);
    };
    uint32_t k_lane = ring_at + ((lane & 16 ? 2 * kTile : 0) + k_frag_off(lane, 0)) * 2;
    asm volatile("" : "+v"(k_lane));
    auto read_k_part = [&](uint32_t at, int i) {
      return *(const lds_u32x4_t*)((const lds_bf16_t*)(uintptr_t)at + k_frag_off(lane, i) -
                                   k_frag_off(lane, 0));
    };
    auto read_k = [&](int st, u32x4_t kf[8]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) kf[i] = read_k_part(k_lane + (st % kRing) * (kStage * 2), i);
    };
    // Operand i (block i / 4, pair i / 2 % 2, half i % 2): two runs of four keys 512
    // bytes apart by one read. (From an address that the compiler does not see
    // through, or it would read the 16 bytes of both halves and move them.)
    uint32_t v_lane = ring_at + (kTile + ((lane >> 4 & 1) * 64 + hf * 16 + (lane & 15)) * 8) * 2 +
                      8 * value_swap(lane & 31);
    asm volatile("" : "+v"(v_lane));
    auto read_v_part = [&](uint32_t at, int i, u32x4_t vf[2][2][2]) {
      const lds_bf16_t* x = (const lds_bf16_t*)(uintptr_t)(at ^ (i & 1) * 8) +
                            (i >> 2) * 2 * kTile + (i >> 1 & 1) * 1024;
      const u32x2_t a0 = *(const lds_u32x2_t*)x, a1 = *(const lds_u32x2_t*)(x + 256);
      vf[i >> 2][i >> 1 & 1][i & 1] = u32x4_t{a0.x, a0.y, a1.x, a1.y};
    };
    auto read_v = [&](int st, u32x4_t vf[2][2][2]) {
#pragma unroll
      for (int i = 0; i < 8; ++i) read_v_part(v_lane + (st % kRing) * (kStage * 2), i, vf);
    };
    // The keys of stage st that a row of slot p sees, as bits.
    auto stage_bits = [&](int st, int p) {
      const int e = it.e0 + 2 * st;
      if (e >= it.list.head && e + 1 < it.e1) {  // two blocks in a row
        const int t0 = it.list.block(e) * kBlockTokens;
        const int hi = min(p + 1 - t0, 32), lo = min(max(p - rk.window + 1, 0) - t0, 32);
        const auto below = [](int n) { return n <= 0 ? 0u : 0xFFFFFFFFu >> (32 - n); };
        if (t0 >= rk.sinks) return below(hi) & ~below(lo);
      }
      uint32_t seen = window_bits(it.list.block(e) * kBlockTokens, p, rk.window, rk.sinks);
      if (e + 1 < it.e1)
        seen |= window_bits(it.list.block(e + 1) * kBlockTokens, p, rk.window, rk.sinks) << 16;
      return seen;
    };

    // (The queries are here: a wait for them inside the walk would be for every load.)
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 8; ++i) asm volatile("" : "+a"(qf[t][i]));
    wait_vmcnt<0>();
    stage_barrier();  // the first stages are here
    // (Every wave passes as many barriers: those of begin(0) .. begin(stages - 2).)
    if (idle) {
#pragma unroll 1
      for (int st = 0; st + 1 < stages; ++st) begin(st);
    } else if (stages > 0) {
      u32x4_t kf[8], vf[2][2][2], pw[2][2];
      f32x16_t z0, z1;
      float m0, m1;
      // Scores of stage st where not every column sees all of it; m: the running max
      // with them.
      auto mask = [&](f32x16_t& z, float& m, int t, int st) {
        mask_scores(z, stage_bits(st, p[t]), hf);
        m = next_max(c[t], column_top(max16(z), a.scale_log2));
      };
      auto scores = [&](f32x16_t& z, float& m, int t, int st) {
        z = scores_of(kf, qf[t]);
        if (whole(st))
          m = next_max(c[t], column_top(max16(z), a.scale_log2));
        else
          mask(z, m, t, st);
      };
      read_k(0, kf);
      scores(z0, m0, 0, 0);
      scores(z1, m1, 1, 0);
      rescale(c[0], m0);
      weights_of(c[0], z0, a.scale_log2, pw[0]);
      if (stages > 1) read_k(1, kf);
      // Here and at the start of each step: tile 0's weights of stage st, tile 1's
      // scores of it (m1 with them), the keys of st + 1. masked: steps to stages that
      // not every column sees whole. (A loop for each kind spilled registers.)
      int st = 0;
      auto steps = [&](bool masked, int end) {
#pragma unroll 1
        while (__builtin_expect_with_probability(st < end, 1, 0.99)) {
          const uint32_t v_at = v_lane + (st % kRing) * (kStage * 2);
          const auto values = [&](int i) {
            if (i < 4) {
              read_v_part(v_at, 2 * i, vf);
              read_v_part(v_at, 2 * i + 1, vf);
            }
          };
          half_step(kf, qf[0], z0, c[0], vf, pw[0], c[1], z1, pw[1], m1, m0, a.scale_log2, values);
          if (__builtin_expect(masked, 0)) mask(z0, m0, 0, st + 1);
          // begin(st), its loads beside the first products.
          arrive(st);
          const bf16_t* src = source(st + kRing - 1) + lane * 8;
          const uint32_t dst = place(st + kRing - 1);
          const uint32_t k_at = k_lane + (st + 2) % kRing * (kStage * 2);
          const auto stage_and_keys = [&](int i) {
            if (i == 0) load_tile<0>(src, dst);
            if (i == 1) load_tile<1>(src, dst);
            if (i == 2) load_tile<2>(src, dst);
            if (i == 3) load_tile<3>(src, dst);
            if (i >= 2 && i < 10) kf[i - 2] = read_k_part(k_at, i - 2);
          };
          half_step(kf, qf[1], z1, c[1], vf, pw[1], c[0], z0, pw[0], m0, m1, a.scale_log2,
                    stage_and_keys);
          ++st;
          if (__builtin_expect(masked, 0)) mask(z1, m1, 1, st);
        }
      };
#pragma unroll 1
      while (st < fast_end) {
        // (up to the next step whose stage st + kRing - 1 starts another 64 table entries)
        if ((st + kRing - 1 & 63) == 0) refill(st + kRing - 1);
        const int end = min(fast_end, (st + kRing - 1 & ~63) + 65 - kRing);
        const bool all = whole(st + 1);
        steps(!all, all ? min(end, to) : st + 1 < from ? min(end, from - 1) : end);
      }
      // The last stage; and all of an item that is done again, since a sum was not a
      // number: one thing after the other, with the values that not every column may
      // meet held apart. (In one loop with the steps above it spilled registers.)
#pragma unroll 1
      do {
        read_v(st, vf);
        const bool odd = careful && !whole(st) && any_odd(vf);
        if (odd) drop_odd(vf);
        rescale(c[1], m1);
        weights_of(c[1], z1, a.scale_log2, pw[1]);
        add_values(c[0], vf, pw[0]);
        add_values(c[1], vf, pw[1]);
        if (odd) {
          read_v(st, vf);
          add_odd(c[0], vf, pw[0], stage_bits(st, p[0]), hf);
          add_odd(c[1], vf, pw[1], stage_bits(st, p[1]), hf);
        }
        if (++st >= stages) break;
        scores(z0, m0, 0, st);
        scores(z1, m1, 1, st);
        rescale(c[0], m0);
        weights_of(c[0], z0, a.scale_log2, pw[0]);
        begin(st - 1);
        read_k(st + 1, kf);
      } while (true);
    }
    if (!careful && (any_nan(c[0].acc) || any_nan(c[1].acc))) bad_s[k & 1] = 1;
    if (tid == 0) {
      next_s[k & 1] = per_queue + drawn;
      bad_s[(k & 1) ^ 1] = 0;
    }
    wait_vmcnt<0>();  // (the stages past the end)
    __syncthreads();  // every wave is done with the ring
    // A value that is not finite, of a key that some of the columns do not see, made
    // sums of others NaN (as a NaN that they do see does): the item once more.
    careful = !careful && one(bad_s[k & 1]) != 0;
    if (careful) {
#pragma unroll 1
      for (int st = 0; st < kRing - 1 && st < it.stages; ++st) issue(st);
      continue;
    }
    // The next item's first stages are on their way while this one's rows are written:
    // through a place of the ring that they leave free, 4 KB of it per wave, so that a
    // row goes out in whole lines. (Straight from the accumulators, 8 bytes a lane,
    // they took 8 us of an item.)
    const Item was = it;
    drawn_k = one(next_s[k & 1]);
    if (drawn_k * queues + queue < total) begin_item(drawn_k * queues + queue);
    char* const sp = (char*)(ring + (kRing - 1) * kStage) + wv * 4096;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int c32 = lane & 31;
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(c[t].l),
                                                       __float_as_uint(c[t].l), false, false);
      const float L = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      // Column x of the wave's 64: row * Hq + head, from the tile's first row on.
      const auto rowhead_of = [&](int x) {
        const int y = was.r_tile + wave0 + x;
        return y + small_div(y, inv_G) * (a.Hq - G);
      };
      const auto part_of = [&](int rowhead) {
        return was.part0 + (was.rowhead + rowhead - (int64_t)was.row0 * a.Hq) * was.splits + was.sp;
      };
      if (hf == 0 && wave0 + 32 * t + c32 <= last) {
        const int rowhead = rowhead_of(32 * t + c32);
        if (was.splits > 1)
          *(f32x2_t*)(a.part_ml + 2 * part_of(rowhead)) = f32x2_t{c[t].m, L};
        else if (a.stats != nullptr)
          *(f32x2_t*)(a.stats + 2 * (was.rowhead + rowhead)) =
              f32x2_t{c[t].m == kNoMax ? 0.f : c[t].m, inv};
      }
      // Runs of four dims from the first of value_dim(i, m), m = 8 (r / 4) + 4 hf ..
#pragma unroll
      for (int dh = 0; dh < 2; ++dh) {  // dims 64 dh ..
        if (was.splits == 1) {
          // 32 columns of 128 bytes in 16-byte pieces, piece u at u ^ (column % 8).
#pragma unroll
          for (int i = 2 * dh; i < 2 * dh + 2; ++i)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
              const f32x16_t& o = c[t].acc[i];
              const int u = value_dim(i, 2 * r) % 64 / 8;
              *(u32x2_t*)(sp + c32 * 128 + ((u ^ (c32 & 7)) << 4) + 8 * hf) =
                  u32x2_t{pack_bf16x2(o[r] * inv, o[r + 1] * inv),
                          pack_bf16x2(o[r + 2] * inv, o[r + 3] * inv)};
            }
          wave_lds_order();
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int col = 8 * y + (lane >> 3), u = lane & 7;
            const u32x4_t v = *(const u32x4_t*)(sp + col * 128 + ((u ^ (col & 7)) << 4));
            if (wave0 + 32 * t + col > last) continue;
            const int rowhead = rowhead_of(32 * t + col), d = 64 * dh + 8 * u;
            bf16_t* out = a.o + was.rowhead * HD + rowhead * HD + d;
            if (a.tiled) {
              const int x = was.r_tile + wave0 + 32 * t + col, j = small_div(x, inv_G);
              out = a.o + tile_off(was.row0 + was.j_tile + j, (was.g * G + x - j * G) * HD + d,
                                   a.Hq * HD);
            }
            *(u32x4_t*)out = v;
          }
          wave_lds_order();
        } else {
          // 16 columns of 256 bytes at a time.
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            if (c32 >> 4 == ch) {
#pragma unroll
              for (int i = 2 * dh; i < 2 * dh + 2; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                  const f32x16_t& o = c[t].acc[i];
                  const int u = value_dim(i, 2 * r) % 64 / 4 + hf;
                  *(f32x4_t*)(sp + (c32 & 15) * 256 + ((u ^ (c32 & 15)) << 4)) =
                      f32x4_t{o[r], o[r + 1], o[r + 2], o[r + 3]};
                }
            }
            wave_lds_order();
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int col = 4 * y + (lane >> 4), u = lane & 15;
              const f32x4_t v = *(const f32x4_t*)(sp + col * 256 + ((u ^ col) << 4));
              if (wave0 + 32 * t + 16 * ch + col > last) continue;
              *(f32x4_t*)(a.part_o + part_of(rowhead_of(32 * t + 16 * ch + col)) * HD + 64 * dh +
                          4 * u) = v;
            }
            wave_lds_order();
          }
        }
      }
    }
  }
  // The last workgroup leaves the counts as it found them.
  if (tid == 0 && atomicAdd(a.counts + kXCDs, 1) == (int)gridDim.x - 1)
    for (int i = 0; i <= kXCDs; ++i) atomicExch(a.counts + i, 0);
}

// The parts of a row's heads, in order: four dims per thread, 32 threads per head.
// Workgroup b has the b-th row of those of sequences in parts.
constexpr int kMergeHeads = 4, kMergeThreads = 32 * kMergeHeads;
__global__ __launch_bounds__(kMergeThreads) void window_prompt_merge_kernel(PromptArgs a) {
  __shared__ int rows_s[kMergeThreads / kWave], parts_s[kMergeThreads / kWave], found[3];
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, G = a.Hq / a.Hkv;
  if (tid == 0) found[0] = -1;
  int rows = 0, parts = 0;  // of the sequences so far
  for (int s0 = 0; s0 < rk.n_seqs && rows <= (int)blockIdx.x; s0 += kMergeThreads) {
    int n = 0, np = 0;
    if (s0 + tid < rk.n_seqs) {
      const PromptSeq y = prompt_seq(rk, s0 + tid, G, a.few);
      n = y.splits > 1 ? y.n : 0;
      np = column_parts(y, a.Hq);
    }
    int row1 = wave_scan(n), part1 = wave_scan(np);
    if (lane == kWave - 1) {
      rows_s[wv] = row1;
      parts_s[wv] = part1;
    }
    __syncthreads();
    row1 += rows;
    part1 += parts;
    for (int w = 0; w < kMergeThreads / kWave; ++w) {
      if (w < wv) {
        row1 += rows_s[w];
        part1 += parts_s[w];
      }
      rows += rows_s[w];
      parts += parts_s[w];
    }
    if (row1 - n <= (int)blockIdx.x && (int)blockIdx.x < row1) {
      found[0] = s0 + tid;
      found[1] = (int)blockIdx.x - (row1 - n);
      found[2] = part1 - np;
    }
    __syncthreads();
  }
  __syncthreads();
  const int s = found[0];
  if (s < 0) return;
  PromptSeq x = prompt_seq(rk, s, G, a.few);
  x.part0 = found[2];
  if (!parts_fit(a, x)) return;
  const int row = x.row0 + found[1];
  const int head = blockIdx.y * kMergeHeads + tid / 32, dim = tid % 32 * 4;
  if (head >= a.Hq) return;
  const int64_t idx = (int64_t)x.part0 + ((int64_t)found[1] * a.Hq + head) * x.splits;
  float M = -INFINITY, L = 0.f;
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  for (int p0 = 0; p0 < x.splits; p0 += 4) {
    f32x4_t v[4];
    f32x2_t ml[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = idx + min(p0 + u, x.splits - 1);
      ml[u] = *(const f32x2_t*)(a.part_ml + 2 * i);
      v[u] = *(const f32x4_t*)(a.part_o + i * HD + dim);
    }
    float m_new = M;
#pragma unroll
    for (int u = 0; u < 4; ++u) m_new = fmaxf(m_new, ml[u][0]);
    const float ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(M - ref);
    y *= alpha;
    L *= alpha;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (p0 + u >= x.splits) break;
      const float f = __builtin_amdgcn_exp2f(ml[u][0] - ref);
      L = fmaf(f, ml[u][1], L);
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[u][r], y[r]);
    }
    M = m_new;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  const int cc = head * HD + dim;
  store4(a.o + (a.tiled ? tile_off(row, cc, a.Hq * HD) : (int64_t)row * a.Hq * HD + cc), y[0] * inv,
         y[1] * inv, y[2] * inv, y[3] * inv);
  if (a.stats != nullptr && dim == 0)
    *(f32x2_t*)(a.stats + ((int64_t)row * a.Hq + head) * 2) =
        f32x2_t{M == -INFINITY ? 0.f : M, inv};
}

}  // namespace

// The most that any call of so many rows and sequences can need: columns of sequences of
// few rows in parts of kFewPart blocks at least, those of the others of kPartBlocks.
int64_t window_column_parts(int64_t max_rows, int64_t max_seqs, int max_blocks, int Hq, int Hkv) {
  const auto columns = [&](int64_t most) {
    const int64_t cols = max_seqs * Hkv * most;
    return cols < max_rows * Hq ? cols : max_rows * Hq;
  };
  const auto parts = [&](int blocks) {
    const int n = (max_blocks + blocks - 1) / blocks;
    return n < kMaxParts ? n : kMaxParts;
  };
  const int64_t few = columns(kFewCols);
  return few * parts(kFewPart) + (columns(kSplitCols) - few) * parts(kPartBlocks);
}

hipError_t launch_window_prompt_bf16(const uint16_t* q, const uint16_t* k_cache,
                                     const uint16_t* v_cache, const RowKeys& rk, int n_rows, int Hq,
                                     int Hkv, uint16_t* o, bool tiled, float* part_o,
                                     float* part_ml, int64_t part_cap, int32_t* counts,
                                     float* stats, int num_cus, hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  if (Hq > 16 * Hkv || num_cus <= 0) return hipErrorInvalidValue;
  PromptArgs a;
  a.q = q;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.rk = rk;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.scale_log2 = kLog2e / sqrtf((float)HD);
  a.o = o;
  a.tiled = tiled;
  a.part_o = part_o;
  a.part_ml = part_ml;
  a.part_cap = part_cap;
  a.counts = counts;
  a.stats = stats;
  // A sequence alone in its call (padding aside) is of one kind by the call's rows, and
  // takes one kernel: the other costs 4 us to find nothing.
  const bool many = (int64_t)n_rows * (Hq / Hkv) > kFewCols;
  a.few = many && rk.n_seqs == 1 ? 0 : kFewCols;
  // Whether any sequence's list can be in parts.
  const int64_t w = ((int64_t)rk.window + n_rows + 2 * kBlockTokens - 2) / kBlockTokens +
                    ((int64_t)rk.sinks + kBlockTokens - 1) / kBlockTokens;
  const bool parts = w > kFewPart && rk.max_blocks > kFewPart;
  // One workgroup per CU; batches of more than kMaxSeqs sequences in several
  // launches, which share the partial buffers in turn.
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kMaxSeqs) {
    a.rk.seq_starts = rk.seq_starts + s0;
    a.rk.ctx_lens = rk.ctx_lens + s0;
    a.rk.block_table = rk.block_table + (int64_t)s0 * rk.max_blocks;
    a.rk.n_seqs = rk.n_seqs - s0 < kMaxSeqs ? rk.n_seqs - s0 : kMaxSeqs;
    if (a.few > 0) {
      const hipError_t e = launch_window_few(a, num_cus, !many && !parts, st);
      if (e != hipSuccess) return e;
    }
    if (many && parts)
      COCO_LAUNCH(window_prompt_kernel, dim3(num_cus), dim3(kThreads), 0, st, a);
    else if (many)
      COCO_LAUNCH_LAST(window_prompt_kernel, dim3(num_cus), dim3(kThreads), 0, st, a);
    if (parts) {
      const int64_t most = (int64_t)a.rk.n_seqs * (kSplitCols / (Hq / Hkv));
      COCO_LAUNCH_LAST(window_prompt_merge_kernel,
                       dim3(most < n_rows ? (int)most : n_rows,
                            (Hq + kMergeHeads - 1) / kMergeHeads),
                       dim3(kMergeThreads), 0, st, a);
    }
  }
  return hipGetLastError();
}

}  // namespace coco
