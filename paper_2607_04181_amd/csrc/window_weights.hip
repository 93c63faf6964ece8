// Softmax weights of window rows per key, added up over the rows of a sequence
// and its query heads: weights[s][t] += sum_{row, head} exp(s_t - m) / l, with
// each row's m and l from its attention (which must be done: a weight needs the
// row's whole sum). The scores are computed again, half of the attention's
// products, rather than kept: a prompt has rows x heads of them per key.
//
// bf16: a workgroup has 256 keys of a sequence and key/value head, 64 of them in
// the registers of each of its four waves as the operands of 32x32 products, and
// walks the columns (rows times query heads of the group) that can see them, 32
// at a time through LDS: S[32 keys][32 columns] = K Q^T. A lane then holds one
// column, whose m and 1 / l are two registers, and 16 keys of each tile, whose sums
// over the columns it keeps; the 32 lanes' sums meet once, at the end, and the sums of
// the heads, and of the parts of many columns, in a second kernel, in order. Three
// workgroups to a CU take such pieces in turn, one's products (16 of 33 cycles a step)
// beside the others' exponentials and multiply-adds (32 of 8 and 64 of 4), as long.
// 16 sequences of 36 to 64 rows (32 heads on 8, 58500 cached tokens between them) take
// 46 us, 4000 rows of a prompt 102: with 32 keys to a wave and all columns in one item
// 57 and 393. Of the 46, the products are 10 and the vector instructions 20. What bounds
// it is the rest: starts of items (tables, then keys, then the first columns, with nothing
// of the next item ahead) and the last round, when some CUs have none.
// fp32: the same of 64 keys, 16 of them in a wave's registers; single tokens without a
// second kernel.
#include <limits.h>
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) bf16_t lds_bf16_t;
typedef __attribute__((address_space(3))) f32x2_t lds_f32x2_t;
typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;

constexpr int HD = 128;
constexpr int kTile = kBlockTokens * HD;
constexpr int kWaves = 4;
constexpr int kTileBlocks = 4 * kWaves;  // blocks of a workgroup
constexpr int kTileBlocksF32 = kWaves;
constexpr int kCols = 32;                // columns of a step
// Columns of an item, by the blocks of its tile. bf16: 497 rows of 32 heads on 8 over 1300
// tokens take 39 us with 1024, 25 with 512 and 20 with 256, 4000 rows 117, 105 and 102, 8000
// with a window of 1024 103, 111 and 112; fp32: 135 rows of 16 heads of 64 on 4 in each of two
// sequences 28 us with 1024, 19.5 with 256, 14.5 with 128. Scratch is 4 bytes a key for each
// item and key/value head.
template <int TB>
constexpr int kPartCols = TB == kTileBlocks ? 256 : 128;
constexpr int kTurn = 8 * 37;
constexpr int kRing = 3;                 // steps in LDS
constexpr int kSlot = kCols * HD + kCols * 16;  // elements of one: queries, then statistics
constexpr int kWorkgroups = 3;           // of a CU
constexpr float kLog2e = 1.4426950408889634f;

// A sequence's rows and cached tokens: N rows of slots first .. last (= L - 1).
struct SeqRows {
  int row0, n, first, last;
  WindowList list;
};
__device__ __forceinline__ SeqRows seq_rows(const RowKeys& rk, int s) {
  SeqRows x;
  x.row0 = rk.seq_starts ? min(max(rk.seq_starts[s], 0), rk.rows) : s;
  x.n = rk.seq_starts ? max(min(rk.seq_starts[s + 1], rk.rows) - x.row0, 0) : 1;
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

// Sums of 16 values over the 32 columns of a tile: lane (c, hf) returns that of value
// c / 2. Half of the values go to the other half of the lanes at a time (37
// instructions; value by value they are 145).
__device__ __forceinline__ float column_sums(const float w[16], int lane) {
  float x[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(w[r]),
                                                     __float_as_uint(w[r + 8]), false, false);
    x[r] = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)  // rotated by 8 lanes of 16
    x[r] = (lane & 8 ? x[r + 4] : x[r]) + row_swap<0x128>(lane & 8 ? x[r] : x[r + 4]);
#pragma unroll
  for (int r = 0; r < 2; ++r)  // 8 lanes mirrored
    x[r] = (lane & 4 ? x[r + 2] : x[r]) + row_swap<0x141>(lane & 4 ? x[r] : x[r + 2]);
  x[0] = (lane & 2 ? x[1] : x[0]) + row_swap<0x4E>(lane & 2 ? x[0] : x[1]);  // lane ^ 2
  return x[0] + row_swap<0xB1>(x[0]);                                        // lane ^ 1
}

// A sequence's work: tile k, blocks k TB .. of its list, in parts of kPartCols<TB>
// of the columns that can see it; key/value heads innermost. Tiles below `many` (those
// with first tokens, which every row sees) have `most` parts at most, the others `few`.
// A part past a tile's columns has no work and leaves no sums.
struct SeqItems {
  int row0, n, last, item0;
};
struct Parts {
  int tiles, many, most, few;
};
template <int TB>
__device__ __forceinline__ int parts_of(int64_t rows, int G) {
  return (int)((rows * G + kPartCols<TB> - 1) / kPartCols<TB>);
}
template <int TB>
__device__ __forceinline__ Parts seq_parts(const RowKeys& rk, const SeqRows& x, int G) {
  Parts y;
  y.tiles = (x.list.entries + TB - 1) / TB;
  const int first = min(rk.sinks / kBlockTokens + (rk.sinks % kBlockTokens != 0), x.list.entries);
  y.many = (first + TB - 1) / TB;
  y.most = parts_of<TB>(x.n, G);
  // (slots t .. t + 16 TB - 1: rows of slots t .. t + 16 TB - 2 + window)
  const int64_t rows = (int64_t)rk.window + TB * kBlockTokens - 1;
  y.few = parts_of<TB>(rows < x.n ? rows : x.n, G);
  return y;
}
// The rows j0 .. j1 - 1 that can see tile k, blocks e0 .. e_last of the list.
template <int TB>
__device__ __forceinline__ void tile_rows(const RowKeys& rk, const SeqRows& x, int k, int& e_last,
                                          int& j0, int& j1) {
  const int e0 = k * TB;
  e_last = min(e0 + TB, x.list.entries) - 1;
  rows_of(rk, x, x.list.block(e0) * kBlockTokens,
          x.list.block(e_last) * kBlockTokens + kBlockTokens - 1, j0, j1);
}

// The sequences' items into seqs, and their first ones into items0 for the sums' kernel;
// all of them. More than `cap` (rows that several sequences claim: no room for their
// sums): none, for it too. red: one int per wave.
template <int TB>
__device__ __forceinline__ int plan_items(const RowKeys& rk, int G, int Hkv, int64_t cap,
                                          SeqItems* seqs, int* red, int32_t* items0) {
  const int tid = threadIdx.x;
  int total = 0;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += 64 * kWaves) {
    SeqRows x{};
    if (s0 + tid < rk.n_seqs) x = seq_rows(rk, s0 + tid);
    const Parts y = seq_parts<TB>(rk, x, G);
    const int items = (y.many * y.most + (y.tiles - y.many) * y.few) * Hkv;
    const int item0 = block_prefix<kWaves>(items, red, total) - items;
    if (s0 + tid < rk.n_seqs) seqs[s0 + tid] = SeqItems{x.row0, x.n, x.last, item0};
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int s = tid; s < rk.n_seqs; s += 64 * kWaves)
      items0[s] = total > cap ? INT_MAX : seqs[s].item0;
  return total > cap ? 0 : total;
}
// An item: blocks e0 .. e_last of sequence s's list for key/value head g, columns c0 ..
// of the `cols` from row j0 on. False: no work.
struct Item {
  int s, g, e0, e_last, j0, c0, cols;
  SeqRows x;
};
template <int TB>
__device__ __forceinline__ bool find_item(const RowKeys& rk, const SeqItems* seqs, int item, int G,
                                          int Hkv, Item& it) {
  const auto one = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  int lo = 0, hi = rk.n_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (seqs[mid].item0 <= item) lo = mid; else hi = mid - 1;
  }
  it.s = one(lo);
  SeqRows& x = it.x;
  x.row0 = one(seqs[it.s].row0);
  x.n = one(seqs[it.s].n);
  x.last = one(seqs[it.s].last);
  x.first = x.last + 1 - x.n;
  x.list = window_list(max(x.first, -1), x.last, rk.window, rk.sinks);
  const Parts y = seq_parts<TB>(rk, x, G);
  const int at = one(item - seqs[it.s].item0), later = at / Hkv - y.many * y.most;
  it.g = at % Hkv;
  const int tile = later < 0 ? at / Hkv / y.most : y.many + later / y.few;
  const int part = later < 0 ? at / Hkv % y.most : later % y.few;
  int j1;
  it.e0 = tile * TB;
  tile_rows<TB>(rk, x, tile, it.e_last, it.j0, j1);
  it.cols = max(j1 - it.j0, 0) * G;
  it.c0 = part * kPartCols<TB>;
  return it.c0 < it.cols;
}

__global__ __launch_bounds__(64 * kWaves, kWorkgroups) void window_weights_kernel(
    const bf16_t* __restrict__ q, const bf16_t* __restrict__ k_cache, RowKeys rk, int Hq, int Hkv,
    float scale_log2, const float* __restrict__ stats, float* __restrict__ sums, int64_t sums_cap,
    int32_t* __restrict__ items0) {
  __shared__ __attribute__((aligned(128))) bf16_t ring[kRing * kSlot];
  __shared__ SeqItems seqs_s[kWindowLaunchSeqs];
  __shared__ int red[kWaves];
  const int G = Hq / Hkv;
  const uint32_t inv_G = small_inv(G);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c32 = lane & 31, hf = lane >> 5;
  const int total = plan_items<kTileBlocks>(rk, G, Hkv, sums_cap, seqs_s, red, items0);
  // (The ring's address goes through a register of its own: the compiler would
  // otherwise wait for every load in flight before each operand read.)
  uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  asm volatile("" : "+s"(ring_at));
  // Dims 16 u + 8 hf .. of column c32: chunk 2 u + hf of its halves.
  const uint32_t q_at = ring_at + (c32 >> 3) * 2048 + (c32 & 7) * 128 + (hf ^ (c32 & 7)) * 16;

#pragma unroll 1
  for (int item0 = 0, turn = blockIdx.x; item0 < total; item0 += gridDim.x) {
    // (Turned from round to round, by a multiple of the XCDs: a tile's later parts are the
    // ones without work, and a workgroup would get the same ones of several tiles.)
    const int item = item0 + turn;
    turn = (turn + kTurn) % gridDim.x;
    Item it;
    if (item >= total || !find_item<kTileBlocks>(rk, seqs_s, item, G, Hkv, it)) continue;
    const SeqRows& x = it.x;
    const int s = it.s, g = it.g, e0 = it.e0, e_last = it.e_last, j0 = it.j0, c0 = it.c0;

    // A step's columns, from row j's head r on, of `left`. Wave w brings columns 8 w .. + 7
    // as two halves of their dims, 128 bytes a column, so that a load is of whole lines
    // (in operand order, 32 bytes of a line at a time, 51 us for 48). Chunk x of a half at
    // x ^ (column % 8): rows of 128 bytes would meet in the same banks. Then the columns'
    // statistics, two floats in each 32 bytes.
    struct Step {
      int j, r, left;
    };
    const auto next = [&](Step& y) {
      const int r = y.r + kCols, d = small_div(r, inv_G);
      y = Step{y.j + d, r - d * G, y.left - kCols};
    };
    const bf16_t* const q_seq = q + ((int64_t)x.row0 * Hq + g * G) * HD;
    const float* const stats_seq = stats + ((int64_t)x.row0 * Hq + g * G) * 2;
    const auto issue = [&](const Step& y, int slot) {
      // (row * Hq + head of this lane's column)
      const int h = y.r + min(8 * wv + (lane >> 3), y.left - 1);
      const int64_t head = (int64_t)y.j * Hq + (h + small_div(h, inv_G) * (Hq - G));
      const bf16_t* qp = q_seq + head * HD + (lane & 7 ^ lane >> 3) * 8;
      const uint32_t to = ring_at + slot * (kSlot * 2) + wv * 2048;
      __builtin_amdgcn_global_load_lds(qp, (lds_void_t*)(uintptr_t)to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds(qp + 64, (lds_void_t*)(uintptr_t)(to + 1024), 16, 0, 0);
      const uint32_t to_stats = ring_at + slot * (kSlot * 2) + kCols * HD * 2 + wv * 256;
      __builtin_amdgcn_global_load_lds(stats_seq + head * 2 + (lane & 1),
                                       (lds_void_t*)(uintptr_t)to_stats, 4, 0, 0);
    };
    Step now{j0 + c0 / G, c0 % G, min(it.cols - c0, kPartCols<kTileBlocks>)}, ahead = now;
    for (int i = 0; i < kRing - 1; ++i) {
      issue(ahead, i);
      if (ahead.left > kCols) next(ahead);
    }

    // The wave's four blocks (past the list the last one: not stored), and its keys:
    // step u holds dims 16 u + 8 hf .. + 7 of key lane % 32 of two blocks.
    int t[2][2];
    u32x4_t kf[2][8];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
      const int e = e0 + 4 * wv + 2 * y;
      t[y][0] = x.list.block(min(e, e_last)) * kBlockTokens;
      t[y][1] = x.list.block(min(e + 1, e_last)) * kBlockTokens;
      const int id =
          readable_block(bt[(lane & 16 ? t[y][1] : t[y][0]) / kBlockTokens], rk.num_blocks);
      const bf16_t* kb = k_cache + ((int64_t)id * Hkv + g) * kTile;
#pragma unroll
      for (int u = 0; u < 8; ++u)
        kf[y][u] =
            *(const u32x4_t*)(kb + ((u >> 1) * 64 + (2 * (u & 1) + hf) * 16 + (lane & 15)) * 8);
    }
    const int t_low = min(min(t[0][0], t[0][1]), min(t[1][0], t[1][1])),
              t_high = max(max(t[0][0], t[0][1]), max(t[1][0], t[1][1])) + kBlockTokens - 1;
    float w[2][16];
#pragma unroll
    for (int r = 0; r < 16; ++r) w[0][r] = w[1][r] = 0.f;
    int slot = 0;
#pragma unroll 1
    while (now.left > 0) {
      wait_vmcnt<3 * (kRing - 2)>();
      stage_barrier();  // the step is here, and the slot of the one before free
      const lds_bf16_t* from = (const lds_bf16_t*)(uintptr_t)(ring_at + slot * (kSlot * 2));
      const f32x2_t st = *(const lds_f32x2_t*)(from + kCols * HD + c32 * 16);
      float inv = c32 < now.left ? st[1] : 0.f;
      issue(ahead, slot == 0 ? kRing - 1 : slot - 1);
      if (ahead.left > kCols) next(ahead);
      f32x16_t z[2] = {};
#pragma unroll
      for (int u0 = 0; u0 < 8; u0 += 4) {
        u32x4_t b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          b[u] = *(const lds_u32x4_t*)(uintptr_t)((q_at + slot * (kSlot * 2) + u0 * 256) ^ u * 32);
        // (four at once: one by one, each product waited for its own)
#pragma unroll
        for (int u = 0; u < 4; ++u) asm volatile("" : "+v"(b[u]));
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            z[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                __builtin_bit_cast(bf16x8_t, kf[y][u0 + u]), __builtin_bit_cast(bf16x8_t, b[u]),
                z[y], 0, 0, 0);
      }
      slot = slot == kRing - 1 ? 0 : slot + 1;
      const int p_low = x.first + now.j,
                p_high = p_low + small_div(now.r + min(now.left, kCols) - 1, inv_G);
      if (!(t_high <= p_low && (t_low > p_high - rk.window || t_high < rk.sinks))) {
        const int p = max(p_low + small_div(now.r + min(c32, now.left - 1), inv_G), -1);
        // A row whose sum is NaN (a score of NaN or +inf) has an inverse of NaN, and 0 times
        // it would reach the keys that it does not see: its seen scores carry the NaN.
        const float odd = inv == inv ? 0.f : inv;
        inv = inv == inv ? inv : 1.f;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t seen = window_bits(t[y][0], p, rk.window, rk.sinks) |
                                window_bits(t[y][1], p, rk.window, rk.sinks) << 16;
          const uint32_t mine = seen >> (4 * hf);
#pragma unroll
          for (int r = 0; r < 16; ++r)
            z[y][r] = (mine >> (8 * (r / 4) + r % 4) & 1) ? z[y][r] + odd : -INFINITY;
        }
      }
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          w[y][r] =
              fmaf(__builtin_amdgcn_exp2f(fmaf(z[y][r], scale_log2, -st[0])), inv, w[y][r]);
      next(now);
    }
    // (a tile's keys in the order of its list)
    float* const to = sums + (int64_t)item * (kTileBlocks * kBlockTokens) + 64 * wv;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const float out = column_sums(w[y], lane);
      const int r = c32 >> 1;
      if (!(lane & 1)) to[32 * y + 8 * (r / 4) + 4 * hf + r % 4] = out;
    }
    wait_vmcnt<0>();  // (the steps past the end)
    __syncthreads();  // every wave is done with the ring
  }
}

// fp32: a workgroup's waves have a block of 16 keys each, and walk the item's columns 16
// at a time, the keys' and the columns' operands from memory: S[16 keys][16 columns] =
// K Q^T, 8 HS x mfma 16x16x4 of 32 cycles each. 2000 rows of a prompt, 16 heads of 64 on
// 4, take 84 to 89 us (2680 with a workgroup that walked them for its 16 keys). The matrix
// units are busy for 31% of it; the waves wait for half of their time: at the items' starts,
// and for columns that are asked for one step, 16 products on one accumulator, ahead.
template <int HS>
__global__ __launch_bounds__(64 * kWaves, 2) void window_weights_rows_f32_kernel(
    const float* __restrict__ q, const float* __restrict__ k_cache, RowKeys rk, int Hq, int Hkv,
    float scale_log2, const float* __restrict__ stats, float* __restrict__ sums, int64_t sums_cap,
    int32_t* __restrict__ items0) {
  constexpr int hd = 32 * HS;
  __shared__ SeqItems seqs_s[kWindowLaunchSeqs];
  __shared__ int red[kWaves];
  const int G = Hq / Hkv, lane = threadIdx.x & 63, c16 = lane & 15, j4 = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int total = plan_items<kTileBlocksF32>(rk, G, Hkv, sums_cap, seqs_s, red, items0);
#pragma unroll 1
  for (int item0 = 0, turn = blockIdx.x; item0 < total; item0 += gridDim.x) {
    const int item = item0 + turn;
    turn = (turn + kTurn) % gridDim.x;
    Item it;
    if (item >= total || !find_item<kTileBlocksF32>(rk, seqs_s, item, G, Hkv, it)) continue;
    const int b = it.x.list.block(min(it.e0 + wv, it.e_last)), t0 = b * kBlockTokens;
    const int id = readable_block(rk.block_table[(int64_t)it.s * rk.max_blocks + b], rk.num_blocks);
    const float* kb = k_cache + ((int64_t)id * Hkv + it.g) * (kBlockTokens * hd) + lane * 8;
    f32x4_t kf[HS][2];
#pragma unroll
    for (int y = 0; y < HS; ++y) {
      kf[y][0] = *(const f32x4_t*)(kb + y * 512);
      kf[y][1] = *(const f32x4_t*)(kb + y * 512 + 4);
    }
    const int end = min(it.c0 + kPartCols<kTileBlocksF32>, it.cols);
    f32x4_t w = {0.f, 0.f, 0.f, 0.f}, qf[HS][2];
    f32x2_t st;
    int p;
    const auto load = [&](int c0) {
      const int c = min(c0 + c16, end - 1), j = it.j0 + c / G;
      const int64_t head = (int64_t)(it.x.row0 + j) * Hq + it.g * G + c % G;
      const float* qp = q + head * hd + 8 * j4;
#pragma unroll
      for (int y = 0; y < HS; ++y) {
        qf[y][0] = *(const f32x4_t*)(qp + 32 * y);
        qf[y][1] = *(const f32x4_t*)(qp + 32 * y + 4);
      }
      st = *(const f32x2_t*)(stats + head * 2);
      if (c0 + c16 >= end) st[1] = 0.f;
      p = max(it.x.first + j, -1);
    };
    load(it.c0);
    for (int c0 = it.c0; c0 < end; c0 += 16) {
      f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < HS; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          z = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[y][e / 4][e % 4], qf[y][e / 4][e % 4], z, 0,
                                                   0, 0);
      const f32x2_t now = st;
      const uint32_t seen = window_bits(t0, p, rk.window, rk.sinks) >> (4 * j4);
      if (c0 + 16 < end) load(c0 + 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // (0 of 1 / sum, which may be NaN, for a key that the row does not see)
        const bool sees = seen >> r & 1;
        const float x = sees ? fmaf(z[r], scale_log2, -now[0]) : -INFINITY;
        w[r] = fmaf(__builtin_amdgcn_exp2f(x), sees ? now[1] : 0.f, w[r]);
      }
    }
    float out = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float v = row_sum16(w[r]);
      if (c16 == r) out = v;
    }
    float* const to = sums + (int64_t)item * (kTileBlocksF32 * kBlockTokens) + kBlockTokens * wv;
    if (c16 < 4) to[4 * j4 + c16] = out;
  }
}

// A key's sums of the parts and key/value heads, each wave every fourth in order, the
// waves in order: a lane a key, 64 keys to a workgroup.
template <int TB>
__global__ __launch_bounds__(64 * kWaves) void window_weights_add_kernel(
    RowKeys rk, int G, int Hkv, const float* __restrict__ sums, int64_t sums_cap,
    const int32_t* __restrict__ items0, float* __restrict__ weights) {
  constexpr int kTileKeys = TB * kBlockTokens;
  __shared__ float sm[kWaves][64];
  const int s = blockIdx.y, lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRows x = seq_rows(rk, s);
  const int e = blockIdx.x * (64 / kBlockTokens) + lane / kBlockTokens;
  const int tile = blockIdx.x / (kTileKeys / 64);
  if ((int)blockIdx.x * (64 / kBlockTokens) >= x.list.entries) return;
  const Parts y = seq_parts<TB>(rk, x, G);
  int e_last, j0, j1;
  tile_rows<TB>(rk, x, tile, e_last, j0, j1);
  const int64_t item = items0[s] + (int64_t)Hkv * (tile < y.many
                                                       ? tile * y.most
                                                       : y.many * y.most + (tile - y.many) * y.few);
  const int n = parts_of<TB>(max(j1 - j0, 0), G) * Hkv;
  if (item + n > sums_cap) return;
  const float* from = sums + item * kTileKeys + blockIdx.x % (kTileKeys / 64) * 64 + lane;
  float v = 0.f;
#pragma unroll 8
  for (int i = wv; i < n; i += kWaves) v += from[(int64_t)i * kTileKeys];
  sm[wv][lane] = v;
  __syncthreads();
  if (wv != 0 || e >= x.list.entries) return;
#pragma unroll
  for (int u = 1; u < kWaves; ++u) v += sm[u][lane];
  const int t = x.list.block(e) * kBlockTokens + lane % kBlockTokens;
  // (a token between the first ones and every row's window is seen by none)
  if (t <= x.last && v != 0.f) weights[(int64_t)s * rk.max_blocks * kBlockTokens + t] += v;
}

// fp32, single tokens: a workgroup has 16 keys, its waves the key/value heads.
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

// The most items of any launch of a call of so many rows and sequences.
int64_t window_weight_items(int64_t max_rows, int64_t max_seqs, int max_blocks, int Hq, int Hkv,
                            bool bf16) {
  int64_t seqs = max_seqs < kWindowLaunchSeqs ? max_seqs : kWindowLaunchSeqs;
  if (max_rows < seqs) seqs = max_rows;
  const int tb = bf16 ? kTileBlocks : kTileBlocksF32;
  const int part = bf16 ? kPartCols<kTileBlocks> : kPartCols<kTileBlocksF32>;
  const int64_t tiles = (max_blocks + tb - 1) / tb;
  const int64_t items = tiles * Hkv * (seqs + max_rows * (Hq / Hkv) / part);
  return items < 0x7fffffff ? items : 0x7fffffff;
}
int64_t window_sums_bytes(int64_t items, bool bf16) {
  return items * (bf16 ? kTileBlocks : kTileBlocksF32) * kBlockTokens * 4 + kWindowLaunchSeqs * 4;
}

namespace {

// run(the sequences' arrays, their number, items0, their weights) for each launch's
// sequences, then their sums.
template <int TB, typename F>
hipError_t weigh_prompts(const RowKeys& rk, int n_rows, int Hq, int Hkv, float* sums,
                         int64_t items_cap, float* weights, hipStream_t st, F run) {
  const int64_t entries = most_entries(rk, n_rows), width = (int64_t)rk.max_blocks * kBlockTokens;
  int32_t* items0 = (int32_t*)(sums + items_cap * (TB * kBlockTokens));
  RowKeys part = rk;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kWindowLaunchSeqs) {
    part.seq_starts = rk.seq_starts + s0;
    part.ctx_lens = rk.ctx_lens + s0;
    part.block_table = rk.block_table + (int64_t)s0 * rk.max_blocks;
    part.n_seqs = rk.n_seqs - s0 < kWindowLaunchSeqs ? rk.n_seqs - s0 : kWindowLaunchSeqs;
    run(part, items0);
    COCO_LAUNCH_LAST(window_weights_add_kernel<TB>,
                     dim3((unsigned)((entries * kBlockTokens + 63) / 64), part.n_seqs),
                     dim3(64 * kWaves), 0, st, part, Hq / Hkv, Hkv, sums, items_cap, items0,
                     weights + s0 * width);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_window_weights_bf16(const uint16_t* q, const uint16_t* k_cache, const RowKeys& rk,
                                      int n_rows, int Hq, int Hkv, const float* stats, float* sums,
                                      int64_t items_cap, float* weights, int num_cus,
                                      hipStream_t st) {
  if (n_rows <= 0 || rk.n_seqs <= 0) return hipSuccess;
  if (Hq > 16 * Hkv || num_cus <= 0) return hipErrorInvalidValue;
  return weigh_prompts<kTileBlocks>(
      rk, n_rows, Hq, Hkv, sums, items_cap, weights, st, [&](const RowKeys& part, int32_t* items0) {
        COCO_LAUNCH(window_weights_kernel, dim3(kWorkgroups * num_cus), dim3(64 * kWaves), 0, st, q,
                    k_cache, part, Hq, Hkv, kLog2e / sqrtf((float)HD), stats, sums, items_cap,
                    items0);
      });
}

hipError_t launch_window_weights_f32(const float* q, const float* k_cache, const RowKeys& rk,
                                     int n_rows, int Hq, int Hkv, int hd, const float* stats,
                                     float* sums, int64_t items_cap, float* weights, int num_cus,
                                     hipStream_t st) {
  typedef float T;
  if (n_rows <= 0 || rk.n_seqs <= 0) return hipSuccess;
  if (rk.n_seqs > 65535 || hd % 32 != 0 || num_cus <= 0) return hipErrorInvalidValue;
  const float scale_log2 = kLog2e / sqrtf((float)hd);
#define COCO_WEIGH(HS)                                                                           \
  if (rk.seq_starts != nullptr)                                                                  \
    return weigh_prompts<kTileBlocksF32>(                                                        \
        rk, n_rows, Hq, Hkv, sums, items_cap, weights, st,                                       \
        [&](const RowKeys& part, int32_t* items0) {                                              \
          COCO_LAUNCH((window_weights_rows_f32_kernel<HS>), dim3(kWorkgroups * num_cus),         \
                      dim3(64 * kWaves), 0, st, q, k_cache, part, Hq, Hkv, scale_log2, stats,    \
                      sums, items_cap, items0);                                                  \
        });                                                                                      \
  COCO_LAUNCH_LAST((window_weights_f32_kernel<HS>),                                              \
                   dim3((unsigned)most_entries(rk, n_rows), rk.n_seqs), dim3(64 * kRowsWaves),   \
                   0, st, q, k_cache, rk, Hq, Hkv, scale_log2, stats, weights)
  COCO_BY_HEAD_DIM(COCO_WEIGH);
#undef COCO_WEIGH
  return hipGetLastError();
}

}  // namespace coco
