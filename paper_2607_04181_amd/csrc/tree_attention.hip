// Attention of trees of drafted tokens over the paged cache (bf16, hd = 128).
//
// The columns of a sequence and key/value head are its nodes times the group's
// query heads, C = N G (column c: node c / G, head c % G). Every wave owns 32 of
// them and walks 32 keys (two blocks) at a time:
//   S^T[32 keys][32 cols] = K[32][hd] Q^T[hd][32]    8 x mfma 32x32x16
//   online softmax per column, 16 keys in each of its two lanes
//   O^T[hd][32 cols] += V^T[hd][32] P^T[32][32]      8 x mfma 32x32x16
// P comes out of the first product in the operand layout of the second: lane
// (c, hf) holds keys 8 q + 4 hf + r of column c, and the value tiles hold runs
// of four keys, two dims side by side, so that two 16-byte reads give the
// operands of two products (dims h and h + 16) for 16 keys.
//
// P is rounded to bf16 for the second product, as the layers' attention does: half
// a step of a weight (2^-9 on average), its sums in fp32. A second product with
// what that leaves (as trees of few columns have it below) takes the error against
// 64 bits from 2.3e-3 to the plain form's 1.7e-3, and 32 trees of up to 64 nodes on
// 64 query heads from 353 us to 412, one of 61 from 98 to 118, 64 of 26 from 207 to
// 212: many columns are bound by products.
//
// A workgroup is four waves with 128 columns (a column tile); two workgroups
// per CU. They share the keys through LDS, 32 at a time, in a ring of four
// stages with three on their way: what a tile of few columns is bound by is the
// bytes in flight. (Eight waves of 256 columns and stages of 128 keys, two in
// LDS, reached 2.7 TB/s on 64 sequences of 4 nodes and 4k keys; this 4.2, of the
// 4.9 of a large copy.) Many columns are bound by products and softmax, which
// take about as long each and of which the two waves of a SIMD, in different
// workgroups, overlap about a third: 555 TFLOP/s for 32 trees of up to 64
// nodes, merge included, of the 1650 of a large bf16 product. (Scheduling by
// hand or priorities around the products changed it by less than 3%. 64 columns
// per wave, one wave to a SIMD, would halve the operand reads; as written once, the
// compiler took all 512 registers and spilled 63 of them and 313 scalar ones, and
// it was not taken further. This kernel spills 191 scalar registers to lanes of
// vector ones, none of them between the products of a stage that every column
// sees whole.) The column tiles of the same keys run at the same time on one XCD
// and read them from its L2.
//
// The keys of a sequence are split into parts (tree_part) that depend on its
// own length and columns only, merged by a second kernel in order: a row's
// bits do not depend on the rest of the call.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void_t;
typedef __attribute__((address_space(3))) bf16_t lds_bf16_t;
typedef __attribute__((address_space(3))) u32x2_t lds_u32x2_t;

constexpr int HD = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * kWave;
constexpr int kCols = 32;   // columns of a wave
constexpr int kTileCols = kWaves * kCols;
constexpr int kStKeys = 32;  // keys of a stage
constexpr int kTile = kBlockTokens * HD;
constexpr int kRing = 4;    // stages in LDS
constexpr int kStage = 4 * kTile;  // elements: keys and values of two blocks
constexpr int kFewCols = 16;  // most columns of a sequence without the ring
constexpr int kXCDs = 8;
constexpr int kMaxSeqs = kTreeLaunchSeqs;
constexpr float kLazy = 8.f;  // log2 units a running max may lag

struct TreeSeq {
  int nodes, len;   // nodes, cached tokens (nodes included)
  int tiles;        // column tiles per key/value head
  int splits, part; // parts of the keys, and keys of one
};

// Keys of one of the parts that `len` keys of a sequence with `cols` columns
// are split into: so many parts that one sequence fills the chip, but more
// columns make a part's partial result (512 bytes per column) dear next to its
// keys (512 bytes each), so parts grow with them, and their number is bounded by
// what the merge of one row takes. Measured: with up to 16 columns, parts of
// 128 keys instead of 512 gain one token over 1k keys 3% and cost eight of them
// 44 and 64 trees of 4 nodes 7, and 32 parts instead of 16 cost one token over 16k
// 17; with 104 columns, parts of 512 keys instead of 1024 gain one or eight
// trees over 2k keys 16 and 12% and cost 64 of them 6, and 32 trees of 64 nodes
// 13; parts of 2048 above 256 columns gain the latter 9% and cost one of them 28.
__host__ __device__ __forceinline__ int tree_part(int64_t cols, int len) {
  const int least = cols <= 64 ? 512 : 1024;
  const int most = cols <= kFewCols || cols > 128 ? kTreeSplits : kTreeSplitsFew;
  int want = (len + least - 1) / least;
  want = want < 1 ? 1 : want > most ? most : want;
  const int part = ((len + want - 1) / want + 127) / 128 * 128;
  return part > 128 ? part : 128;
}
__host__ __device__ __forceinline__ int tree_splits(int64_t cols, int len) {
  const int part = tree_part(cols, len);
  return len > part ? (len + part - 1) / part : 1;
}

__device__ __forceinline__ TreeSeq tree_plan(const int32_t* seq_starts, const int32_t* ctx_lens,
                                             int s, int G, int max_blocks) {
  TreeSeq t;
  t.nodes = max(seq_starts[s + 1] - seq_starts[s], 0);
  t.len = min(max(ctx_lens[s], 0), max_blocks * kBlockTokens);
  const int64_t cols = (int64_t)t.nodes * G;
  t.tiles = (int)((cols + kTileCols - 1) / kTileCols);
  t.part = tree_part(cols, t.len);
  t.splits = tree_splits(cols, t.len);
  return t;
}

// Bits of keys k0 .. k0 + 31 that a node sees, k0 counted from the first node.
__device__ __forceinline__ uint32_t tree_bits32(const uint64_t* mask, int words, int n, int k0) {
  if (k0 <= -32) return 0xFFFFFFFFu;
  uint64_t v;
  if (k0 >= 0) {
    const int w = k0 >> 6, sh = k0 & 63;
    v = w < words ? mask[w] >> sh : 0;
    if (sh > 32 && w + 1 < words) v |= mask[w + 1] << (64 - sh);
  } else {
    v = mask[0] << -k0 | ((1ull << -k0) - 1);
  }
  const int left = n - k0;
  if (left < 32) v &= left > 0 ? (1ull << left) - 1 : 0;
  return (uint32_t)v;
}

struct TreeArgs {
  const bf16_t* q;
  const bf16_t* k_cache;
  const bf16_t* v_cache;
  RowKeys rk;
  int Hq, Hkv;
  float scale_log2;
  bf16_t* o;
  bool tiled;
  float* part_o;    // [column part][HD]
  float* part_ml;   // [column part][2]
  int64_t part_cap; // column parts they hold
  int32_t* plan;    // [n_seqs][2]: first column part, parts
  int32_t* drawn;   // items drawn (zero between calls)
  int32_t* redo;    // [rows * Hq]: rows with non-finite values to add (zero between calls)
};

// Where a lane's run of four dims goes that starts at value v (a multiple of 4)
// of its 64: dims D + 4 hf .. + 3 with D from v alone; and, in tile order, the
// run's place from its head's first.
__device__ __forceinline__ int run_dim(int v) {
  return 64 * (v >> 5) + 16 * (v >> 4 & 1) + 32 * (v >> 3 & 1) + 8 * (v >> 2 & 1);
}
__device__ __forceinline__ int run_tiled(int v) {
  const int d = run_dim(v);
  return (d >> 5) * 512 + (d >> 3 & 3) * 128;
}

// Key fragments of two blocks: step s holds dims 16 s + 8 hf .. + 7 of key m.
// kb[i]: the tile of block i.
__device__ __forceinline__ int k_frag_off(int lane, int s) {
  const int hf = lane >> 5, t = lane & 15;
  return ((s >> 1) * 64 + (2 * (s & 1) + hf) * 16 + t) * 8;
}
__device__ __forceinline__ int v_frag_off(int lane, int p) {
  const int hf = lane >> 5;
  return ((2 * p + ((lane >> 4) & 1)) * 64 + hf * 16 + (lane & 15)) * 8;
}

// Largest of 16 values (NaN loses).
__device__ __forceinline__ float max16(const f32x16_t& s) {
  float m = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
  for (int r = 3; r + 1 < 16; r += 2) m = fmaxf(fmaxf(m, s[r]), s[r + 1]);
  return fmaxf(m, s[15]);
}

// Scores of keys among or behind the nodes: -inf where the column does not see
// the key. Bit k of seen: key 4 hf + k of the 32 (a lane holds 8 q + 4 hf + r).
__device__ __forceinline__ void mask_scores(f32x16_t& s, uint32_t seen) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (seen >> (8 * (r / 4) + r % 4) & 1) ? s[r] : -INFINITY;
}

// Values of such keys: those from key `left` on are dropped (their slots may
// hold anything). A product with a probability of 0 would let a non-finite value
// of a node reach the columns that do not see it: such elements are left out.
// Returns the keys (as bits of `seen`) that held one.
__device__ __forceinline__ uint32_t mask_values(u32x4_t v[2][2][2], int hf, int left) {
  uint32_t odd = 0;  // bit 8 j + 4 u + k: key 16 j + 8 u + 4 hf + k, in any of this lane's dims
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int u = e >> 1, k = 16 * j + 8 * u + 4 * hf + 2 * (e & 1);
          uint32_t w = v[j][d][y][e];
          w &= (k < left ? 0xFFFFu : 0u) | (k + 1 < left ? 0xFFFF0000u : 0u);
          const bool lo = (w & 0x7F80u) == 0x7F80u, hi = (w & 0x7F800000u) == 0x7F800000u;
          if (lo) w &= 0xFFFF0000u;
          if (hi) w &= 0xFFFFu;
          odd |= ((lo ? 1u : 0u) | (hi ? 2u : 0u)) << (8 * j + 4 * u + 2 * (e & 1));
          v[j][d][y][e] = w;
        }
  if (__ballot(odd != 0) == 0) return 0;
  uint32_t mine = 0;  // this half of the lanes' keys
#pragma unroll 1
  for (int i = 0; i < 16; ++i) {
    const uint64_t any = __ballot(odd >> i & 1);
    const uint32_t here = hf == 0 ? (uint32_t)any : (uint32_t)(any >> 32);
    mine |= (here != 0 ? 1u : 0u) << (8 * (i >> 2) + (i & 3));
  }
  return mine;
}

// One wave's columns: running softmax and O^T. acc[2 p + y]: dims 32 (2 p +
// m / 16) + 16 y + m % 16, m = 8 (r / 4) + 4 hf + r % 4.
struct Cols {
  float m, l;
  f32x16_t acc[4];
};

// The running max of a column moves only when a step's largest score (of this
// lane's 16 keys: mx) exceeds it by kLazy.
__device__ __forceinline__ void tree_rescale(Cols& c, float mx, float scale_log2) {
  const auto sw =
      __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  const float top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2;
  const float m_new = top > c.m + kLazy ? top : c.m;
  if (__ballot(m_new != c.m) != 0) {
    const float alpha = __builtin_amdgcn_exp2f(c.m - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
    for (int i = 0; i < 4; ++i) c.acc[i] *= alpha;
    c.l *= alpha;
    c.m = m_new;
  }
}

// Probabilities of 32 keys as operands of two products.
__device__ __forceinline__ void tree_probs(Cols& c, const f32x16_t& s, float scale_log2,
                                           u32x4_t p[2]) {
  const float m_ref = c.m == -INFINITY ? 0.f : c.m;
  float pr[16];
#pragma unroll
  for (int r = 0; r < 16; ++r) pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale_log2, -m_ref));
  float ls = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 4) ls += (pr[r] + pr[r + 1]) + (pr[r + 2] + pr[r + 3]);
  c.l += ls;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) p[j][e] = pack_bf16x2(pr[8 * j + 2 * e], pr[8 * j + 2 * e + 1]);
}

// O^T += V^T P^T. v[j][d][y]: block j's operand of dims 32 (2 d + m / 16) + 16 y
// + m % 16: keys 4 hf .. + 3, then 8 + 4 hf .. + 3.
__device__ __forceinline__ void tree_values(Cols& c, const u32x4_t v[2][2][2],
                                            const u32x4_t p[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c.acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          __builtin_bit_cast(bf16x8_t, v[j][i >> 1][i & 1]), __builtin_bit_cast(bf16x8_t, p[j]),
          c.acc[i], 0, 0, 0);
}

// ---- Few columns (up to 16): they share their operands with too few others to
// pay for LDS. Each wave takes every fourth block of the part straight into
// registers, three blocks on their way, with 16x16 tiles of the columns:
//   S[16 keys][16 cols] = K Q^T    4 x mfma 16x16x32
//   O^T[hd][16 cols] += V^T P^T    8 x mfma 16x16x16
// P comes out as the operand of the second (lane (c, j4): keys 4 j4 .. + 3 of
// column c), in two bf16 parts; the waves' results meet in LDS in wave order. One token over 1k keys
// takes 10.9 us with the merge (calls replayed from a graph), through the ring
// 15.8; over 16k 24.1 and 33.5; 64 trees of 4 nodes over 4k keys 225 (4.8 TB/s) and
// 226. (32 columns, two tiles, spill registers in this kernel and lose at 64
// trees what they gain at one.)
struct FewTile {
  u32x4_t k[4], v[4];
};

// As mask_values for one block: lane (m, j4) holds keys 4 j4 .. + 3 of dims
// 32 x + m and + 16. Returns the block's keys that held a non-finite value.
__device__ __forceinline__ uint32_t few_mask_values(u32x4_t v[4], int j4, int left) {
  uint32_t odd = 0;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = 2 * (e & 1), k = 4 * j4 + c;
      uint32_t w = v[x][e];
      w &= (k < left ? 0xFFFFu : 0u) | (k + 1 < left ? 0xFFFF0000u : 0u);
      const bool lo = (w & 0x7F80u) == 0x7F80u, hi = (w & 0x7F800000u) == 0x7F800000u;
      if (lo) w &= 0xFFFF0000u;
      if (hi) w &= 0xFFFFu;
      odd |= ((lo ? 1u : 0u) | (hi ? 2u : 0u)) << c;
      v[x][e] = w;
    }
  if (__ballot(odd != 0) == 0) return 0;
  uint32_t keys = 0;
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    const uint64_t any = __ballot(odd >> c & 1);
    for (int j = 0; j < 4; ++j) keys |= (any >> (16 * j) & 0xFFFFu ? 1u : 0u) << (4 * j + c);
  }
  return keys;
}

// Part sp of sequence s for kv head g; part0: the sequence's first column part.
// sm_o: [4][16][128], the 16-byte pieces of column c at place ^ c.
__device__ __forceinline__ void few_columns(const TreeArgs& a, const TreeSeq& ts, int s, int g,
                                            int sp, int64_t part0, float* sm_o,
                                            float (*sm_ml)[kFewCols][2]) {
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63, c16 = lane & 15, j4 = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int G = a.Hq / a.Hkv, cols = ts.nodes * G, row0 = rk.seq_starts[s];
  const int prefix = ts.len - ts.nodes;
  const int t0 = sp * ts.part, t1 = min(ts.len, t0 + ts.part);
  const int b0 = t0 / kBlockTokens + wv;
  const int left_blocks = (t1 + kBlockTokens - 1) / kBlockTokens - b0;
  const int mine = left_blocks > 0 ? (left_blocks + kWaves - 1) / kWaves : 0;
  const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;

  int ids = 0;
  auto load = [&](FewTile& t, int j) {  // with j = 0, 1, ..
    if ((j & 63) == 0) {
      const int64_t id = bt[min(b0 + (j + lane) * kWaves, rk.max_blocks - 1)];
      ids = (int)(id < 0 ? 0 : id >= rk.num_blocks ? rk.num_blocks - 1 : id);
    }
    const int64_t at = ((int64_t)__builtin_amdgcn_readlane(ids, j & 63) * a.Hkv + g) * kTile;
    const u32x4_t* kp = (const u32x4_t*)(a.k_cache + at);
    const u32x4_t* vp = (const u32x4_t*)(a.v_cache + at);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      t.k[p] = kp[64 * p + lane];
      t.v[p] = vp[64 * p + lane];
    }
  };
  FewTile ta, tb, tc;
  if (mine > 0) load(ta, 0);
  if (mine > 1) load(tb, 1);
  if (mine > 2) load(tc, 2);

  // This lane's column (past the last: the last).
  const int c = min(c16, cols - 1), row = row0 + c / G;
  const int64_t rowhead = (int64_t)row * a.Hq + g * G + c % G;
  const uint64_t* mask = rk.mask + (int64_t)row * rk.words;
  bf16x8_t qf[4];
#pragma unroll
  for (int p = 0; p < 4; ++p)
    qf[p] = __builtin_bit_cast(bf16x8_t,
                               *(const u32x4_t*)(a.q + rowhead * HD + 32 * p + 8 * j4));
  float m = -INFINITY, l = 0.f;
  f32x4_t acc[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) acc[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto attend = [&](FewTile& t, int j) {
    f32x4_t z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int p = 0; p < 4; ++p)
      z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, t.k[p]), qf[p], z,
                                                  0, 0, 0);
    const int tok0 = (b0 + j * kWaves) * kBlockTokens;
    if (tok0 + kBlockTokens > prefix) {
      const uint32_t odd = few_mask_values(t.v, j4, t1 - tok0);
      const uint32_t seen = tree_bits32(mask, rk.words, ts.nodes, tok0 - prefix);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!(seen >> (4 * j4 + r) & 1)) z[r] = -INFINITY;
      if (odd & seen) a.redo[rowhead] = 1;
    }
    const float top = col_max4(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]))) * a.scale_log2;
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
      for (int x = 0; x < 8; ++x)
        acc[x] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(
            __builtin_bit_cast(s16x4_t, u32x2_t{t.v[x / 2][x % 2 * 2], t.v[x / 2][x % 2 * 2 + 1]}),
            pb, acc[x], 0, 0, 0);
    }
  };
#pragma unroll 1
  for (int j = 0; j < mine; j += 3) {
    attend(ta, j);
    if (j + 3 < mine) load(ta, j + 3);
    if (j + 1 >= mine) break;
    attend(tb, j + 1);
    if (j + 4 < mine) load(tb, j + 4);
    if (j + 2 >= mine) break;
    attend(tc, j + 2);
    if (j + 5 < mine) load(tc, j + 5);
  }

  l = col_sum4(l);
  if (j4 == 0) {
    sm_ml[wv][c16][0] = m;
    sm_ml[wv][c16][1] = l;
  }
#pragma unroll
  for (int x = 0; x < 8; ++x)
    *(f32x4_t*)(sm_o + (wv * kFewCols + c16) * HD + (((4 * x + j4) ^ c16) << 2)) = acc[x];
  __syncthreads();
  for (int i = tid; i < cols * (HD / 4); i += kThreads) {
    const int c = i / (HD / 4), q4 = i % (HD / 4);
    float M = sm_ml[0][c][0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_ml[w][c][0]);
    const float ref = M == -INFINITY ? 0.f : M;
    f32x4_t y = {0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm_ml[w][c][0] - ref);
      const f32x4_t v = *(const f32x4_t*)(sm_o + (w * kFewCols + c) * HD + ((q4 ^ c) << 2));
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
      L = fmaf(f, sm_ml[w][c][1], L);
    }
    const int n = c / G, head = g * G + c % G;
    if (ts.splits > 1) {
      const int64_t idx = part0 + ((int64_t)n * a.Hq + head) * ts.splits + sp;
      *(f32x4_t*)(a.part_o + idx * HD + 4 * q4) = y;
      if (q4 == 0) {
        a.part_ml[2 * idx] = M;
        a.part_ml[2 * idx + 1] = L;
      }
    } else {
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      const int col = head * HD + 4 * q4;
      store4(a.o + (a.tiled ? tile_off(row0 + n, col, a.Hq * HD)
                            : (int64_t)(row0 + n) * a.Hq * HD + col),
             y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
    }
  }
}

// Inclusive sum of x over the workgroup's threads so far: `carry` before, the
// whole added to it. red: one int per wave.
__device__ __forceinline__ int block_scan(int x, int* red, int& carry) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  x = wave_scan(x);
  if (lane == kWave - 1) red[wv] = x;
  __syncthreads();
  x += carry;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wv) x += red[w];
    carry += red[w];
  }
  __syncthreads();
  return x;
}

__global__ __launch_bounds__(kThreads, 2) void tree_attention_kernel(TreeArgs a) {
  __shared__ __attribute__((aligned(16))) bf16_t ring[kRing * kStage];
  __shared__ int units_s[kMaxSeqs], base_s[kMaxSeqs], items_s[kMaxSeqs], few_s[kMaxSeqs];
  __shared__ int red[kWaves], next_s[2];
  __shared__ float few_ml[kWaves][kFewCols][2];
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5;
  const int G = a.Hq / a.Hkv;

  // Units (part, kv head) of all sequences in order go round the XCDs (blockIdx
  // % 8); an XCD's list of items is its units' column tiles.
  const int queues = gridDim.x % kXCDs == 0 ? kXCDs : 1;
  const int queue = blockIdx.x % queues;
  int n_units = 0, n_parts = 0, total = 0, total_few = 0;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    int nu = 0, np = 0, tiles = 0;
    bool few = false;
    if (s < rk.n_seqs) {
      const TreeSeq t = tree_plan(rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
      tiles = t.tiles;
      few = t.nodes * G <= kFewCols;
      nu = t.tiles > 0 ? t.splits * a.Hkv : 0;
      np = t.splits > 1 ? t.nodes * a.Hq * t.splits : 0;
      if (blockIdx.x == 0) a.plan[2 * s + 1] = t.splits;
    }
    const int u1 = block_scan(nu, red, n_units), u0 = u1 - nu;
    const int p0 = block_scan(np, red, n_parts) - np;
    // The queue's units among u0 .. u1 - 1.
    const int mine = ((u1 - queue + queues - 1) / queues - (u0 - queue + queues - 1) / queues);
    const int ni = few ? 0 : mine * tiles, nf = few ? mine : 0;
    const int i0 = block_scan(ni, red, total) - ni;
    const int f0 = block_scan(nf, red, total_few) - nf;
    if (s < rk.n_seqs) {
      units_s[s] = u0;
      base_s[s] = p0;
      items_s[s] = i0;
      few_s[s] = f0;
      if (blockIdx.x == 0) a.plan[2 * s] = p0;
    }
  }
  __syncthreads();
  if (n_parts > a.part_cap) return;  // more rows than the call named: no room for their parts

  // Workgroups draw items in order, each its next one while it works (the merge
  // kernel sets the counts back to zero). A fixed share of the items left a
  // quarter of the chip idle at the end.
  const int first = blockIdx.x / queues, per_queue = (int)gridDim.x / queues;
  auto seq_of = [&](const int* starts, int item) {
    int lo = 0, hi = rk.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (starts[mid] <= item) lo = mid; else hi = mid - 1;
    }
    return __builtin_amdgcn_readfirstlane(lo);
  };
  // The sequences of few columns.
  int item = first;
#pragma unroll 1
  for (int k = 0; item < total_few; ++k) {
    int drawn = 0;
    if (tid == 0) drawn = per_queue + atomicAdd(a.drawn + kXCDs + queue, 1);
    const int s = seq_of(few_s, item);
    const TreeSeq ts = tree_plan(rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
    const int x = __builtin_amdgcn_readfirstlane(item - few_s[s]);
    const int u0 = __builtin_amdgcn_readfirstlane(units_s[s]);
    const int u = (queue - u0 % queues + queues) % queues + x * queues;
    const int g = u % a.Hkv, sp = u / a.Hkv;
    const int base = __builtin_amdgcn_readfirstlane(base_s[s]);
    few_columns(a, ts, s, g, sp, base, (float*)ring, few_ml);
    if (tid == 0) next_s[k & 1] = drawn;
    __syncthreads();
    item = __builtin_amdgcn_readfirstlane(next_s[k & 1]);
  }
  __syncthreads();

  // (The ring's address goes through a register of its own: the compiler would
  // otherwise wait for every load in flight before each operand read.)
  uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  asm volatile("" : "+s"(ring_at));

  item = first;
#pragma unroll 1
  for (int k = 0; item < total; ++k) {
    int drawn = 0;
    if (tid == 0) drawn = per_queue + atomicAdd(a.drawn + queue, 1);
    const int s = seq_of(items_s, item);
    const TreeSeq ts = tree_plan(rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
    const int x = __builtin_amdgcn_readfirstlane(item - items_s[s]);
    const int u0 = __builtin_amdgcn_readfirstlane(units_s[s]);
    // The sequence's unit: the queue's (x / tiles)-th from u0 on.
    const int u = (queue - u0 % queues + queues) % queues + x / ts.tiles * queues;
    const int g = u % a.Hkv, sp = u / a.Hkv;
    const int cols = ts.nodes * G, row0 = rk.seq_starts[s];
    const int col0 = x % ts.tiles * kTileCols + wv * kCols;
    const bool idle = col0 >= cols;
    const int prefix = ts.len - ts.nodes;
    const int t0 = sp * ts.part, t1 = min(ts.len, t0 + ts.part);
    const int stages = (t1 - t0 + kStKeys - 1) / kStKeys;

    // A wave brings one tile of each stage, keys (waves 0, 2) or values of one
    // of its two blocks; past the last key the last block again, whose scores
    // count as unseen. Called with st = 0, 1, ..: the blocks of 64 stages at a
    // time in a register's lanes.
    const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
    const bf16_t* cache = (wv & 1 ? a.v_cache : a.k_cache) + g * kTile + lane * 8;
    const int b_last = (t1 - 1) / kBlockTokens;
    int ids = 0;
    auto issue = [&](int st) {
      if ((st & 63) == 0) {
        const int b = t0 / kBlockTokens + (st + lane) * 2 + (wv >> 1);
        const int64_t id = bt[min(b, b_last)];
        ids = (int)(id < 0 ? 0 : id >= rk.num_blocks ? rk.num_blocks - 1 : id);
      }
      const bf16_t* src =
          cache + (int64_t)__builtin_amdgcn_readlane(ids, st & 63) * (a.Hkv * kTile);
      const uint32_t dst = ring_at + ((st % kRing) * kStage + wv * kTile) * 2;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        __builtin_amdgcn_global_load_lds(src + i * 512, (lds_void_t*)(uintptr_t)(dst + i * 1024),
                                         16, 0, 0);
    };
    if (stages > 0) issue(0);
    if (stages > 1) issue(1);
    if (stages > 2) issue(2);

    // This lane's column; columns past the last repeat it.
    const int col = col0 + (lane & 31);
    const int colc = min(col, cols - 1);
    const int row = row0 + colc / G, head = g * G + colc % G;
    const uint64_t* mask = rk.mask + (int64_t)row * rk.words;
    bf16x8_t qf[8];
    const bf16_t* qp = a.q + ((int64_t)row * a.Hq + head) * HD + 8 * hf;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      qf[i] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(qp + 16 * i));
    Cols c;
    c.m = -INFINITY;
    c.l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) c.acc[i] = f32x16_t{};

    auto begin = [&](int st) {
      // This wave's tile of stage st + 1, with one later on its way.
      if (st + 2 < stages)
        wait_vmcnt<4>();
      else
        wait_vmcnt<0>();
      stage_barrier();  // every wave's; and all are done with stage st - 1
      if (st + 3 < stages) issue(st + 3);
    };
    auto read_k = [&](int st, u32x4_t kf[8]) {
      const bf16_t* kb = ring + (st % kRing) * kStage + (lane & 16 ? 2 * kTile : 0);
#pragma unroll
      for (int i = 0; i < 8; ++i) kf[i] = *(const u32x4_t*)(kb + k_frag_off(lane, i));
    };
    auto scores = [&](const u32x4_t kf[8]) {
      f32x16_t z = {};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), qf[i], z,
                                                    0, 0, 0);
      return z;
    };
    // Value operands of block j: per dim pair d, dims h and h + 16, as two runs
    // of four keys 512 bytes apart (one read of two 8-byte halves each; the
    // second address is hidden, or the compiler would read 16 bytes at a time
    // and move the halves).
    auto read_v = [&](int st, u32x4_t vf[2][2][2]) {
      const bf16_t* lo = ring + (st % kRing) * kStage + kTile + v_frag_off(lane, 0);
      uint32_t at = (uint32_t)(uintptr_t)(lds_bf16_t*)lo + 8;
      asm volatile("" : "+v"(at));
      const lds_bf16_t* hi = (const lds_bf16_t*)(uintptr_t)at;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          const int off = j * 2 * kTile + d * 1024;
          const u32x2_t a = *(const u32x2_t*)(lo + off), b = *(const u32x2_t*)(lo + off + 256);
          const u32x2_t e = *(const lds_u32x2_t*)(hi + off),
                        f = *(const lds_u32x2_t*)(hi + off + 256);
          vf[j][d][0] = u32x4_t{a.x, a.y, b.x, b.y};
          vf[j][d][1] = u32x4_t{e.x, e.y, f.x, f.y};
        }
    };
    if (stages > 2)
      wait_vmcnt<8>();
    else
      wait_vmcnt<0>();
    stage_barrier();  // stage 0 is here
    if (idle) {
#pragma unroll 1
      for (int st = 0; st < stages; ++st) begin(st);
    } else if (stages > 0) {
      // Scores of a stage are computed while the one before goes through softmax
      // and its values. z, mx: those of the next stage.
      f32x16_t z;
      float mx;
      auto next_scores = [&](int st) {
        u32x4_t kf[8];
        read_k(st, kf);
        z = scores(kf);
        const int tok0 = t0 + st * kStKeys;
        if (tok0 + kStKeys > prefix)
          mask_scores(z, tree_bits32(mask, rk.words, ts.nodes, tok0 - prefix) >> (4 * hf));
        mx = max16(z);
      };
      next_scores(0);
      // Stages that, with their next, every column sees whole; then the others.
      const int clear = min(stages, max(prefix - t0, 0) / kStKeys) - 1;
      int st = 0;
      auto step = [&](const f32x16_t& now, f32x16_t& next) {
        begin(st);
        tree_rescale(c, mx, a.scale_log2);
        u32x4_t kf[8], vf[2][2][2], p[2];
        read_k(st + 1, kf);
        read_v(st, vf);
        next = scores(kf);
        tree_probs(c, now, a.scale_log2, p);
        tree_values(c, vf, p);
        mx = max16(next);
        ++st;
      };
      f32x16_t z2;  // two steps a turn: the scores change places without moves
#pragma unroll 1
      while (st + 1 < clear) {
        step(z, z2);
        step(z2, z);
      }
      if (st < clear) {
        step(z, z2);
        z = z2;
      }
#pragma unroll 1
      for (; st < stages; ++st) {
        begin(st);
        tree_rescale(c, mx, a.scale_log2);
        const int tok0 = t0 + st * kStKeys;
        u32x4_t vf[2][2][2], p[2];
        read_v(st, vf);
        if (tok0 + kStKeys > prefix) {
          const uint32_t seen = tree_bits32(mask, rk.words, ts.nodes, tok0 - prefix) >> (4 * hf);
          if (mask_values(vf, hf, t1 - tok0) & seen) a.redo[(int64_t)row * a.Hq + head] = 1;
        }
        tree_probs(c, z, a.scale_log2, p);
        tree_values(c, vf, p);
        if (st + 1 < stages) next_scores(st + 1);
      }
    }
    if (tid == 0) next_s[k & 1] = drawn;
    __syncthreads();  // every wave is done with the ring
    item = next_s[k & 1];

    if (col < cols) {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(c.l),
                                                       __float_as_uint(c.l), false, false);
      const float L = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      if (ts.splits > 1) {
        const int64_t idx = base_s[s] + ((int64_t)(row - row0) * a.Hq + head) * ts.splits + sp;
        float* part = a.part_o + idx * HD + 4 * hf;
#pragma unroll
        for (int v = 0; v < 64; v += 4) {
          const f32x16_t& o = c.acc[v >> 4];
          *(f32x4_t*)(part + run_dim(v)) =
              f32x4_t{o[v & 15], o[(v & 15) + 1], o[(v & 15) + 2], o[(v & 15) + 3]};
        }
        if (hf == 0) {
          a.part_ml[2 * idx] = c.m;
          a.part_ml[2 * idx + 1] = L;
        }
      } else {
        const float inv = L == 0.f ? 0.f : 1.0f / L;
        bf16_t* out = a.o + 4 * hf + (a.tiled ? tile_off(row, head * HD, a.Hq * HD)
                                              : ((int64_t)row * a.Hq + head) * HD);
#pragma unroll
        for (int v = 0; v < 64; v += 4) {
          const f32x16_t& o = c.acc[v >> 4];
          store4(out + (a.tiled ? run_tiled(v) : run_dim(v)), o[v & 15] * inv,
                 o[(v & 15) + 1] * inv, o[(v & 15) + 2] * inv, o[(v & 15) + 3] * inv);
        }
      }
    }
  }
}

// The parts of a row's heads, in order: four dims per thread, 32 threads per
// head, four heads per workgroup (eight: one token 1.6 us more, 32 trees of 64
// nodes 13).
constexpr int kMergeHeads = 4;
__global__ __launch_bounds__(32 * kMergeHeads) void tree_combine_kernel(TreeArgs a) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 2 * kXCDs) a.drawn[threadIdx.x] = 0;
  const int row = blockIdx.x + a.rk.seq_starts[0];
  if (row >= a.rk.seq_starts[a.rk.n_seqs]) return;
  // The row's sequence: the starts after the first that are not behind it, read
  // side by side (a search's dependent reads: 31 us instead of 26 for the 64 trees
  // of 26 nodes).
  int s = 0;
  for (int s0 = 1; s0 < a.rk.n_seqs; s0 += kWave) {
    const int at = s0 + (threadIdx.x & 63);
    s += __popcll(__ballot(at < a.rk.n_seqs && a.rk.seq_starts[at] <= row));
  }
  const int splits = a.plan[2 * s + 1];
  const int head = blockIdx.y * kMergeHeads + threadIdx.x / 32, dim = threadIdx.x % 32 * 4;
  if (head >= a.Hq) return;
  int32_t* redo = a.redo + (int64_t)row * a.Hq + head;
  const bool again = *redo != 0;
  if (splits <= 1 && !again) return;
  const int cc = head * HD + dim;
  bf16_t* out = a.o + (a.tiled ? tile_off(row, cc, a.Hq * HD) : (int64_t)row * a.Hq * HD + cc);
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  if (splits > 1) {
    float M = -INFINITY, L = 0.f;
    const int64_t idx =
        a.plan[2 * s] + ((int64_t)(row - a.rk.seq_starts[s]) * a.Hq + head) * splits;
    if (idx + splits > a.part_cap) return;  // (as the parts' kernel)
    // Four parts at a time, all their loads together.
    for (int p0 = 0; p0 < splits; p0 += 4) {
      f32x4_t v[4];
      f32x2_t ml[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t i = idx + min(p0 + u, splits - 1);
        ml[u] = *(const f32x2_t*)(a.part_ml + 2 * i);
        v[u] = *(const f32x4_t*)(a.part_o + i * HD + dim);
      }
      float m_new = M;
#pragma unroll
      for (int u = 0; u < 4; ++u) m_new = fmaxf(m_new, ml[u][0]);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(M - ref);
      L *= alpha;
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] *= alpha;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (p0 + u >= splits) break;
        const float f = __builtin_amdgcn_exp2f(ml[u][0] - ref);
        L = fmaf(f, ml[u][1], L);
#pragma unroll
        for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[u][r], y[r]);
      }
      M = m_new;
    }
    y *= L == 0.f ? 0.f : 1.0f / L;
  } else {  // (again: the parts' kernel wrote the row)
    const u32x2_t w = *(const u32x2_t*)out;
    y = f32x4_t{bf16_to_f32(w.x & 0xFFFFu), bf16_to_f32(w.x >> 16), bf16_to_f32(w.y & 0xFFFFu),
                bf16_to_f32(w.y >> 16)};
  }
  if (again) {
    // The row sees non-finite values in the stages that hold nodes, which left
    // them out for the sake of the columns that do not see their key. Whatever
    // its weight, such a value is the sum; a weight of 0 (a score of -inf) times
    // it is NaN.
    const TreeSeq ts = tree_plan(a.rk.seq_starts, a.rk.ctx_lens, s, a.Hq / a.Hkv, a.rk.max_blocks);
    const int g = head / (a.Hq / a.Hkv), prefix = ts.len - ts.nodes;
    const int32_t* bt = a.rk.block_table + (int64_t)s * a.rk.max_blocks;
    const uint64_t* mask = a.rk.mask + (int64_t)row * a.rk.words;
    for (int t = max(prefix, 0) / kStKeys * kStKeys; t < ts.len; ++t) {
      if (!(tree_bits32(mask, a.rk.words, ts.nodes, t - prefix) & 1)) continue;
      const int64_t id = bt[t / kBlockTokens];
      const int64_t blk = id < 0 ? 0 : id >= a.rk.num_blocks ? a.rk.num_blocks - 1 : id;
      const int64_t tile = (blk * a.Hkv + g) * kTile;
      float v[4];
      bool odd = false;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        v[r] = bf16_to_f32(a.v_cache[tile + v_tile_offset(t % kBlockTokens, dim + r)]);
        odd |= !__builtin_isfinite(v[r]);
      }
      if ((uint32_t)(__ballot(odd) >> (threadIdx.x & 32)) == 0) continue;  // (this head's lanes)
      float z = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        z = fmaf(bf16_to_f32(a.q[((int64_t)row * a.Hq + head) * HD + dim + r]),
                 bf16_to_f32(a.k_cache[tile + k_tile_offset(t % kBlockTokens, dim + r)]), z);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) z += __shfl_xor(z, d, kWave);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (!__builtin_isfinite(v[r])) y[r] += z == -INFINITY ? 0.f * v[r] : v[r];
    }
    if (dim == 0) *redo = 0;
  }
  store4(out, y[0], y[1], y[2], y[3]);
}

}  // namespace

// The most that any call of so many rows and sequences can need. A sequence of
// len keys has tree_splits(cols, len) parts: at most `few` where it has up to 128
// columns per key/value head, `many` above (a part holds at least 512 or 1024
// keys before it is rounded up).
int64_t tree_column_parts(int64_t max_rows, int64_t max_seqs, int Hq, int Hkv, int max_blocks) {
  const int64_t len = (int64_t)max_blocks * kBlockTokens;
  const int64_t few = len / 512 + 1 < kTreeSplitsFew ? len / 512 + 1 : kTreeSplitsFew;
  const int64_t many = len / 1024 + 1 < kTreeSplits ? len / 1024 + 1 : kTreeSplits;
  const int64_t cols = max_seqs * Hkv * 128 < max_rows * Hq ? max_seqs * Hkv * 128 : max_rows * Hq;
  return cols * few + (max_rows * Hq - cols) * many;
}

hipError_t launch_tree_attention_bf16(const uint16_t* q, const uint16_t* k_cache,
                                      const uint16_t* v_cache, const RowKeys& rk, int n_rows,
                                      int Hq, int Hkv, uint16_t* o, bool tiled, float* part_o,
                                      float* part_ml, int64_t part_cap, int32_t* plan,
                                      int32_t* redo, int num_cus, hipStream_t st) {
  if (n_rows <= 0) return hipSuccess;
  TreeArgs a;
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
  a.plan = plan;
  a.drawn = redo;
  a.redo = redo + 2 * kXCDs;
  // Two workgroups per CU (LDS, registers); batches of more than kMaxSeqs sequences
  // in several launches, which share the partial buffers in turn.
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kMaxSeqs) {
    a.rk.seq_starts = rk.seq_starts + s0;
    a.rk.ctx_lens = rk.ctx_lens + s0;
    a.rk.block_table = rk.block_table + (int64_t)s0 * rk.max_blocks;
    a.rk.n_seqs = rk.n_seqs - s0 < kMaxSeqs ? rk.n_seqs - s0 : kMaxSeqs;
    COCO_LAUNCH(tree_attention_kernel, dim3(2 * num_cus), dim3(kThreads), 0, st, a);
    COCO_LAUNCH_LAST(tree_combine_kernel, dim3(n_rows, (Hq + kMergeHeads - 1) / kMergeHeads),
                     dim3(32 * kMergeHeads), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace coco
