// Attention of trees of drafted tokens over the paged cache (bf16, hd = 128).
//
// The columns of a sequence and key/value head are its nodes times the group's
// query heads, C = N G (column c: node c / G, head c % G). Every wave owns 32
// of them and walks 32 keys (two blocks) at a time:
//   S^T[32 keys][32 cols] = K[32][hd] Q^T[hd][32]    8 x mfma 32x32x16
//   online softmax per column, 16 keys in each of its two lanes
//   O^T[hd][32 cols] += V^T[hd][32] P^T[32][32]      8 x mfma 32x32x16
// P comes out of the first product in the operand layout of the second: lane
// (c, hf) holds keys 8 q + 4 hf + r of column c, and the value tiles hold runs
// of four keys, two dims side by side, so that two 16-byte reads give the
// operands of two products (dims h and h + 16) for 16 keys.
//
// What is read: keys and values once per column tile, so a tile takes as many
// columns as its eight waves hold: 32 RG columns with RG in {2, 4, 8} groups, the
// other 8 / RG waves of a group taking other keys. The waves share the keys
// through LDS, 128 at a time, double-buffered. Few columns are bound by the
// cache's bytes; from RG = 4 on matrix products and softmax bound it. (A path
// of its own for up to 32 columns, keys straight to registers, cost registers
// the other one needs and was no faster.)
//
// The keys of a sequence are split into parts (tree_plan) that depend on its
// own length and columns only, merged by a second kernel in order: a row's
// bits do not depend on the rest of the call.
#include <math.h>

#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int HD = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kCols = 32;   // columns of a wave
constexpr int kChunk = 32;  // keys of a step
constexpr int kTile = kBlockTokens * HD;
constexpr int kStBlk = 8;   // blocks of a stage (128 keys)
constexpr int kMaxSeqs = 1024;  // sequences of a launch
constexpr int kXCDs = 8;
constexpr float kLazy = 8.f;  // log2 units a running max may lag

// Column tiles of a sequence with `groups` 32-column groups: full tiles of 8,
// then the rest as tiles of 2, 4 (3 groups, or 5 with a 2), 6 as 4 and 2, 7 as 8:
// an idle group costs less than reading the keys again.
__device__ __forceinline__ int tree_tiles(int groups) {
  const int r = groups & 7;
  return (groups >> 3) + (r == 0 ? 0 : r == 5 || r == 6 ? 2 : 1);
}
// Tile t's first group, and its width.
__device__ __forceinline__ int tree_tile(int groups, int t, int* rg) {
  const int full = groups >> 3, r = groups & 7;
  if (t < full) {
    *rg = 8;
    return 8 * t;
  }
  if (t > full) {
    *rg = 2;
    return 8 * full + 4;
  }
  *rg = r == 7 ? 8 : r >= 3 ? 4 : 2;
  return 8 * full;
}

struct TreeSeq {
  int nodes, len;   // nodes, cached tokens (nodes included)
  int tiles;        // column tiles per key/value head
  int splits, part; // parts of the keys, and keys of one
};

// Keys of one of the parts that `len` keys of a sequence with `cols` columns
// are split into. Few columns: one stage (128 keys), so that one sequence fills
// the chip; more columns make a part's partial result (512 bytes per column)
// dear next to its keys (512 bytes each), so parts grow with them. The number
// of parts falls with cols and grows with len (tree_column_parts counts on it).
__host__ __device__ __forceinline__ int tree_part(int64_t cols, int len) {
  const int least = cols <= 16 ? 128 : cols <= 64 ? 512 : 1024;
  const int most = cols <= 128 ? kTreeSplitsFew : kTreeSplits;
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
  t.tiles = tree_tiles((int)((cols + kCols - 1) / kCols));
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

// One wave's columns: running softmax and O^T. acc[2 p + y]: dims 32 (2 p +
// m / 16) + 16 y + m % 16, m = 8 (r / 4) + 4 hf + r % 4.
struct Cols {
  float m, l;
  f32x16_t acc[4];
};

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
  int32_t* redo;    // [rows * Hq]: rows to compute again (zero between calls)
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

__device__ __forceinline__ f32x16_t tree_scores(const u32x4_t kf[8], const bf16x8_t qf[8]) {
  f32x16_t s = {};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), qf[i], s, 0,
                                                0, 0);
  return s;
}

// Softmax step of 32 keys; p: the probabilities as operands of two products.
__device__ __forceinline__ void tree_softmax(Cols& c, const f32x16_t& s, float scale_log2,
                                             u32x4_t p[2]) {
  float mx = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
  const auto sw =
      __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2;
  // The running max moves only when a step exceeds it by kLazy.
  const float m_new = mx > c.m + kLazy ? mx : c.m;
  const float m_ref = m_new == -INFINITY ? 0.f : m_new;
  const float alpha = __builtin_amdgcn_exp2f(c.m - m_ref);
  float pr[16];
#pragma unroll
  for (int r = 0; r < 16; ++r)
    pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale_log2, -m_ref));
  float ls = 0.f;
#pragma unroll
  for (int r = 0; r < 16; r += 4) ls += (pr[r] + pr[r + 1]) + (pr[r + 2] + pr[r + 3]);
  if (__ballot(m_new != c.m) != 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c.acc[i] *= alpha;
    c.l *= alpha;
  }
  c.m = m_new;
  c.l += ls;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) p[j][e] = pack_bf16x2(pr[8 * j + 2 * e], pr[8 * j + 2 * e + 1]);
}

__device__ __forceinline__ f32x16_t pv_step(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1,
                                            u32x4_t p, f32x16_t acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
      __builtin_bit_cast(bf16x8_t, u32x4_t{a0, a1, b0, b1}), __builtin_bit_cast(bf16x8_t, p), acc,
      0, 0, 0);
}

// O^T += V^T P^T. v[j][p]: the two chunks (keys 4 hf .. and 8 + 4 hf ..) of
// block j, dim pair p.
__device__ __forceinline__ void tree_pv(Cols& c, const u32x4_t v[2][2][2], const u32x4_t p[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const u32x4_t a = v[j][d][0], b = v[j][d][1];
      c.acc[2 * d] = pv_step(a.x, a.y, b.x, b.y, p[j], c.acc[2 * d]);
      c.acc[2 * d + 1] = pv_step(a.z, a.w, b.z, b.w, p[j], c.acc[2 * d + 1]);
    }
}

// Keys among or behind the nodes: scores that the column does not see count as
// -inf, and values from key `left` on are dropped (their slots may hold
// anything). A product with a probability of 0 would let a non-finite value of a
// node reach the columns that do not see it: such elements are left out, and the
// result is whether this lane's column sees one (the merge kernel then computes
// its row again, key by key).
__device__ __forceinline__ bool tree_mask(f32x16_t& s, u32x4_t v[2][2][2], int hf, int left,
                                          uint32_t seen) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (seen >> (8 * (r / 4) + r % 4) & 1) ? s[r] : -INFINITY;
  uint32_t odd = 0;  // bit 8 j + 4 u + k: key 16 j + 8 u + 4 hf + k, in any of this lane's dims
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int d = 0; d < 2; ++d)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = 16 * j + 8 * u + 4 * hf + 2 * (e & 1);
          uint32_t w = v[j][d][u][e];
          w &= (k < left ? 0xFFFFu : 0u) | (k + 1 < left ? 0xFFFF0000u : 0u);
          const bool lo = (w & 0x7F80u) == 0x7F80u, hi = (w & 0x7F800000u) == 0x7F800000u;
          if (lo) w &= 0xFFFF0000u;
          if (hi) w &= 0xFFFFu;
          odd |= ((lo ? 1u : 0u) | (hi ? 2u : 0u)) << (8 * j + 4 * u + 2 * (e & 1));
          v[j][d][u][e] = w;
        }
  if (__ballot(odd != 0) == 0) return false;
  uint32_t mine = 0;  // this half's keys of the chunk that hold one in any lane's dims
#pragma unroll 1
  for (int i = 0; i < 16; ++i) {
    const uint64_t any = __ballot(odd >> i & 1);
    const uint32_t here = hf == 0 ? (uint32_t)any : (uint32_t)(any >> 32);
    mine |= (here != 0 ? 1u : 0u) << (8 * (i >> 2) + (i & 3));  // its place in `seen`
  }
  return (mine & seen) != 0;
}

__global__ __launch_bounds__(kThreads, 2) void tree_attention_kernel(TreeArgs a) {
  // Two stages of eight blocks' key and value tiles; at the end the waves'
  // O^T ([wave][64 values][64 lanes] floats), 128 KB either way.
  __shared__ __attribute__((aligned(16))) bf16_t kv[2 * kStBlk * 2 * kTile];
  __shared__ int items_s[kMaxSeqs + 1], base_s[kMaxSeqs];
  __shared__ int wsum[2][kWaves];
  __shared__ float sm_m[kWaves][kCols], sm_l[kWaves][kCols];
  const RowKeys& rk = a.rk;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5;
  const int G = a.Hq / a.Hkv;

  // The work list: sequences' items (part, kv head, column tile) in order, and
  // where their column parts start.
  int carry_i = 0, carry_b = 0;
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kThreads) {
    const int s = s0 + tid;
    int ni = 0, nb = 0;
    TreeSeq t{};
    if (s < rk.n_seqs) {
      t = tree_plan(rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
      ni = t.tiles * t.splits * a.Hkv;
      nb = t.splits > 1 ? t.nodes * a.Hq * t.splits : 0;
    }
    int si = ni, sb = nb;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const int x = __shfl_up(si, d, kWave), y = __shfl_up(sb, d, kWave);
      if (lane >= d) {
        si += x;
        sb += y;
      }
    }
    if (lane == kWave - 1) {
      wsum[0][wv] = si;
      wsum[1][wv] = sb;
    }
    __syncthreads();
    int bi = carry_i, bb = carry_b;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wv) {
        bi += wsum[0][w];
        bb += wsum[1][w];
      }
      carry_i += wsum[0][w];
      carry_b += wsum[1][w];
    }
    if (s < rk.n_seqs) {
      items_s[s] = bi + si - ni;
      base_s[s] = bb + sb - nb;
      if (blockIdx.x == 0) {
        a.plan[2 * s] = bb + sb - nb;
        a.plan[2 * s + 1] = t.splits;
      }
    }
    __syncthreads();
  }
  if (tid == 0) items_s[rk.n_seqs] = carry_i;
  __syncthreads();
  const int total = carry_i;
  if (carry_b > a.part_cap) return;  // more rows than the call named: no room for their parts

  // Consecutive items on one XCD (blockIdx % 8), so that the column tiles of
  // the same keys read them from its L2.
  const int grid = gridDim.x;
  const int per = grid / kXCDs;
  const int me = grid % kXCDs == 0 ? (blockIdx.x % kXCDs) * per + blockIdx.x / kXCDs : blockIdx.x;

  for (int item = me; item < total; item += grid) {
    int lo = 0, hi = rk.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (items_s[mid] <= item) lo = mid; else hi = mid - 1;
    }
    const int s = lo;
    const TreeSeq ts = tree_plan(rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
    int x = item - items_s[s];
    const int tile_i = x % ts.tiles;
    x /= ts.tiles;
    const int g = x % a.Hkv, sp = x / a.Hkv;
    const int cols = ts.nodes * G, row0 = rk.seq_starts[s];
    int rgs;
    const int group0 = tree_tile((cols + kCols - 1) / kCols, tile_i, &rgs);
    const int kss = kWaves / rgs;              // key sets
    const int rg = wv % rgs, ks = wv / rgs;    // this wave's columns and keys
    const int prefix = ts.len - ts.nodes;
    const int t0 = sp * ts.part, t1 = min(ts.len, t0 + ts.part);
    const int32_t* bt = rk.block_table + (int64_t)s * rk.max_blocks;
    const int b_last = (max(t1, 1) - 1) / kBlockTokens;
    auto block_of = [&](int b) -> int64_t {
      const int64_t id = bt[min(b, b_last)];
      return id < 0 ? 0 : id >= rk.num_blocks ? rk.num_blocks - 1 : id;
    };

    // This wave's column in this lane; columns past the last repeat it.
    const int col = (group0 + rg) * kCols + (lane & 31);
    const int colc = min(col, cols - 1);
    const int row = row0 + colc / G, head = g * G + colc % G;
    const uint64_t* mask = rk.mask + (int64_t)row * rk.words;
    const bool idle = (group0 + rg) * kCols >= cols;
    bf16x8_t qf[8];
    {
      const bf16_t* qp = a.q + ((int64_t)row * a.Hq + head) * HD + 8 * hf;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        qf[i] = __builtin_bit_cast(bf16x8_t, *(const u32x4_t*)(qp + 16 * i));
    }
    Cols c;
    c.m = -INFINITY;
    c.l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) c.acc[i] = f32x16_t{};

    // Softmax and values of the 32 keys from tok0 on.
    auto finish = [&](f32x16_t& sc, u32x4_t v[2][2][2], int tok0) {
      if (tok0 + kChunk > prefix) {
        // Bit k: key tok0 + 4 hf + k (a lane's keys are 8 q + 4 hf + r).
        const uint32_t seen = tree_bits32(mask, rk.words, ts.nodes, tok0 - prefix) >> (4 * hf);
        if (tree_mask(sc, v, hf, t1 - tok0, seen)) a.redo[(int64_t)row * a.Hq + head] = 1;
      }
      u32x4_t p[2];
      tree_softmax(c, sc, a.scale_log2, p);
      tree_pv(c, v, p);
    };

    const int stages = (t1 - t0 + kStBlk * kBlockTokens - 1) / (kStBlk * kBlockTokens);
    auto issue = [&](int st) {
      const int64_t b = block_of(t0 / kBlockTokens + st * kStBlk + wv);
      bf16_t* dst = kv + ((st & 1) * kStBlk + wv) * 2 * kTile;
      const bf16_t* src[2] = {a.k_cache + (b * a.Hkv + g) * kTile + lane * 8,
                              a.v_cache + (b * a.Hkv + g) * kTile + lane * 8};
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int pc = 0; pc < 4; ++pc)
          __builtin_amdgcn_global_load_lds(src[w] + pc * 512,
                                           (lds_void_t*)(dst + w * kTile + pc * 512), 16, 0, 0);
    };
    issue(0);
    __syncthreads();
    for (int st = 0; st < stages; ++st) {
      if (st + 1 < stages) issue(st + 1);
      for (int ch = ks; ch < kStBlk / 2; ch += kss) {
        const int tok0 = t0 + (st * kStBlk + 2 * ch) * kBlockTokens;
        if (idle || tok0 >= t1) continue;
        const bf16_t* kb = kv + ((st & 1) * kStBlk + 2 * ch) * 2 * kTile;
        const bf16_t* kl = kb + (lane & 16 ? 2 * kTile : 0);
        u32x4_t kf[8], vf[2][2][2];
#pragma unroll
        for (int i = 0; i < 8; ++i) kf[i] = *(const u32x4_t*)(kl + k_frag_off(lane, i));
        f32x16_t sc = tree_scores(kf, qf);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u)
              vf[j][d][u] = *(const u32x4_t*)(kb + (2 * j + 1) * kTile + v_frag_off(lane, d) +
                                              u * 256);
        finish(sc, vf, tok0);
      }
      __syncthreads();  // stage st + 1 landed; stage st's buffer is free
    }

    // Merge the key sets of each column group: weights from the sets' maxima,
    // sums in set order, wave (rg, ks) adding values 64 ks / kss .. of all sets.
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(c.l), __float_as_uint(c.l),
                                                       false, false);
      c.l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    float M = c.m, L = c.l;
    // Where this lane's column goes: a part, or the output row.
    const bool live = !idle && col < cols;
    const int64_t idx = base_s[s] + ((int64_t)(row - row0) * a.Hq + head) * ts.splits + sp;
    float* const part = ts.splits > 1 ? a.part_o + idx * HD + 4 * hf : nullptr;
    bf16_t* const out = a.o + 4 * hf + (a.tiled ? tile_off(row, head * HD, a.Hq * HD)
                                                : ((int64_t)row * a.Hq + head) * HD);
    float* xs = reinterpret_cast<float*>(kv);
    if (kss > 1) {
      __syncthreads();  // every wave is done with kv (register path: with the last merge)
      if (hf == 0) {
        sm_m[wv][lane] = c.m;
        sm_l[wv][lane] = c.l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) xs[(wv * 64 + i * 16 + r) * 64 + lane] = c.acc[i][r];
      __syncthreads();
      M = -INFINITY;
      for (int k = 0; k < kss; ++k) M = fmaxf(M, sm_m[k * rgs + rg][lane & 31]);
      const float ref = M == -INFINITY ? 0.f : M;
      L = 0.f;
      float f[kWaves];
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        f[k] = 0.f;
        if (k < kss) {
          f[k] = __builtin_amdgcn_exp2f(sm_m[k * rgs + rg][lane & 31] - ref);
          L = fmaf(f[k], sm_l[k * rgs + rg][lane & 31], L);
        }
      }
      const int per_w = 64 / kss;
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      for (int v4 = ks * per_w; v4 < (ks + 1) * per_w; v4 += 4) {
        f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k)
          if (k < kss) {
            const float* w = xs + ((k * rgs + rg) * 64 + v4) * 64 + lane;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = fmaf(f[k], w[r * 64], y[r]);
          }
        if (!live) continue;
        if (part)
          *(f32x4_t*)(part + run_dim(v4)) = y;
        else
          store4(out + (a.tiled ? run_tiled(v4) : run_dim(v4)), y[0] * inv, y[1] * inv, y[2] * inv,
                 y[3] * inv);
      }
      __syncthreads();  // LDS is free for the next item
    } else if (live) {
      const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          const f32x4_t y = {c.acc[i][r], c.acc[i][r + 1], c.acc[i][r + 2], c.acc[i][r + 3]};
          const int v4 = 16 * i + r;
          if (part)
            *(f32x4_t*)(part + run_dim(v4)) = y;
          else
            store4(out + (a.tiled ? run_tiled(v4) : run_dim(v4)), y[0] * inv, y[1] * inv,
                   y[2] * inv, y[3] * inv);
        }
    }
    if (part && live && ks == 0 && hf == 0) {
      a.part_ml[2 * idx] = M;
      a.part_ml[2 * idx + 1] = L;
    }
  }
}

// The parts of a row's heads, in order: four dims per thread, 32 threads per
// head, eight heads per workgroup.
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
  const int row = blockIdx.x + a.rk.seq_starts[0];
  if (row >= a.rk.seq_starts[a.rk.n_seqs]) return;
  const int s = row_to_seq(a.rk.seq_starts, a.rk.n_seqs, row);
  const int splits = a.plan[2 * s + 1];
  const int head = blockIdx.y * 8 + threadIdx.x / 32, dim = threadIdx.x % 32 * 4;
  if (head >= a.Hq) return;
  int32_t* redo = a.redo + (int64_t)row * a.Hq + head;
  const bool again = *redo != 0;
  if (splits <= 1 && !again) return;
  float M = -INFINITY, L = 0.f;
  f32x4_t y = {0.f, 0.f, 0.f, 0.f};
  if (!again) {
    const int64_t idx =
        a.plan[2 * s] + ((int64_t)(row - a.rk.seq_starts[s]) * a.Hq + head) * splits;
    for (int p = 0; p < splits; ++p) M = fmaxf(M, a.part_ml[2 * (idx + p)]);
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 4
    for (int p = 0; p < splits; ++p) {
      const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * (idx + p)] - ref);
      L = fmaf(f, a.part_ml[2 * (idx + p) + 1], L);
      const f32x4_t v = *(const f32x4_t*)(a.part_o + (idx + p) * HD + dim);
#pragma unroll
      for (int r = 0; r < 4; ++r) y[r] = fmaf(f, v[r], y[r]);
    }
  } else {
    // A row that sees a non-finite value among the nodes: key by key.
    const TreeSeq ts = tree_plan(a.rk.seq_starts, a.rk.ctx_lens, s, a.Hq / a.Hkv, a.rk.max_blocks);
    const int g = head / (a.Hq / a.Hkv), prefix = ts.len - ts.nodes;
    const int32_t* bt = a.rk.block_table + (int64_t)s * a.rk.max_blocks;
    const uint64_t* mask = a.rk.mask + (int64_t)row * a.rk.words;
    float qv[4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
      qv[r] = bf16_to_f32(a.q[((int64_t)row * a.Hq + head) * HD + dim + r]);
    for (int t = 0; t < ts.len; ++t) {
      if (!(tree_bits32(mask, a.rk.words, ts.nodes, t - prefix) & 1)) continue;
      const int64_t id = bt[t / kBlockTokens];
      const int64_t blk = id < 0 ? 0 : id >= a.rk.num_blocks ? a.rk.num_blocks - 1 : id;
      const int64_t tile = (blk * a.Hkv + g) * kTile;
      float z = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        z = fmaf(qv[r], bf16_to_f32(a.k_cache[tile + k_tile_offset(t % kBlockTokens, dim + r)]), z);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) z += __shfl_xor(z, d, kWave);
      z *= a.scale_log2;
      const float m_new = fmaxf(M, z);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(M - ref), p = __builtin_amdgcn_exp2f(z - ref);
      L = fmaf(L, alpha, p);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        y[r] = fmaf(p, bf16_to_f32(a.v_cache[tile + v_tile_offset(t % kBlockTokens, dim + r)]),
                    y[r] * alpha);
      M = m_new;
    }
    if (dim == 0) *redo = 0;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
  const int cc = head * HD + dim;
  bf16_t* out = a.o + (a.tiled ? tile_off(row, cc, a.Hq * HD) : (int64_t)row * a.Hq * HD + cc);
  store4(out, y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
}

}  // namespace

// The most that any call of so many rows and sequences can need. A sequence of
// len keys has tree_splits(cols, len) parts: at most `few` of kTreeSplitsFew where
// it has up to 128 columns per key/value head, `many` above. (Part sizes are
// rounded up to 128 keys, which is why a shorter sequence may have more parts
// than a longer one: the bounds are those of any length up to the longest.)
int64_t tree_column_parts(int64_t max_rows, int64_t max_seqs, int Hq, int Hkv, int max_blocks) {
  const int64_t len = (int64_t)max_blocks * kBlockTokens;
  // A part holds at least 128 keys (few columns), 1024 before rounding (many).
  const int64_t few = len / 128 + 1 < kTreeSplitsFew ? len / 128 + 1 : kTreeSplitsFew;
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
  a.redo = redo;
  // One workgroup per CU (its LDS); batches of more than kMaxSeqs sequences
  // in several launches, which share the partial buffers in turn.
  for (int s0 = 0; s0 < rk.n_seqs; s0 += kMaxSeqs) {
    a.rk.seq_starts = rk.seq_starts + s0;
    a.rk.ctx_lens = rk.ctx_lens + s0;
    a.rk.block_table = rk.block_table + (int64_t)s0 * rk.max_blocks;
    a.rk.n_seqs = rk.n_seqs - s0 < kMaxSeqs ? rk.n_seqs - s0 : kMaxSeqs;
    COCO_LAUNCH(tree_attention_kernel, dim3(num_cus), dim3(kThreads), 0, st, a);
    COCO_LAUNCH(tree_combine_kernel, dim3(n_rows, (Hq + 7) / 8), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace coco
