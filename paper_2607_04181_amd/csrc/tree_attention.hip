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
// A workgroup is eight waves that take 64, 128 or 256 columns (RG = 2, 4, 8
// column groups) and KS = 8 / RG sets of keys; one workgroup per CU. Keys and
// values go through LDS in stages of 128 keys, double-buffered, one barrier
// each. Within a stage a wave takes its 4 / KS steps of 32 keys alone: the next
// step's key operands are read while this one's go through softmax, so that of
// the two waves of a SIMD one can multiply while the other does vector work.
// Few columns are bound by the cache's bytes, many by products and softmax,
// which take about as long each.
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

constexpr int HD = 128;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kCols = 32;   // columns of a wave
constexpr int kChunk = 32;  // keys of a step
constexpr int kTile = kBlockTokens * HD;
constexpr int kStBlk = 8;   // blocks of a stage
constexpr int kStKeys = kStBlk * kBlockTokens;
constexpr int kMaxSeqs = 1024;  // sequences of a launch
constexpr float kLazy = 8.f;  // log2 units a running max may lag

// Column tiles of a sequence with `groups` 32-column groups: full tiles of 8,
// then the rest as a tile of 2, of 4 (3 or 4 groups), of 4 and 2 (5, 6) or of 8
// (7): an idle group costs less than reading the keys again.
__device__ __forceinline__ int tree_tiles(int groups) {
  const int r = groups & 7;
  return (groups >> 3) + (r == 0 ? 0 : r == 5 || r == 6 ? 2 : 1);
}
// Tile t's first group, and its width.
__device__ __forceinline__ int tree_tile(int groups, int t, int* rg) {
  const int full = groups >> 3, r = groups & 7;
  *rg = t < full || (t == full && r == 7) ? 8 : t == full && r >= 3 ? 4 : 2;
  return t <= full ? 8 * t : 8 * full + 4;
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

// Largest of 16 values (NaN loses).
__device__ __forceinline__ float max16(const f32x16_t& s) {
  float m = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
  for (int r = 3; r + 1 < 16; r += 2) m = fmaxf(fmaxf(m, s[r]), s[r + 1]);
  return fmaxf(m, s[15]);
}

__device__ __forceinline__ f32x16_t pv_step(uint32_t a0, uint32_t a1, uint32_t b0, uint32_t b1,
                                            u32x4_t p, f32x16_t acc) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
      __builtin_bit_cast(bf16x8_t, u32x4_t{a0, a1, b0, b1}), __builtin_bit_cast(bf16x8_t, p), acc,
      0, 0, 0);
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

// What a wave needs of its item.
struct Walk {
  const bf16_t *k_cache, *v_cache;  // of the kv head: block b's tile at b * stride
  int stride, last_block;
  const int32_t* bt;
  const uint64_t* mask;
  int words, nodes, prefix;
  int t0, t1;
  int ks;
  bool idle;
  float scale_log2;
  int32_t* redo;
};

// The keys t0 .. t1 - 1 in stages of 128, of which this wave takes every
// KS-th 32. kv: two stages of eight blocks' key and value tiles.
template <int KS>
__device__ __forceinline__ void tree_walk(const Walk& w, const bf16x8_t qf[8], bf16_t* kv,
                                          int lane, int wv, Cols& c) {
  const int hf = lane >> 5;
  const int stages = (w.t1 - w.t0 + kStKeys - 1) / kStKeys;
  const int b_last = (w.t1 - 1) / kBlockTokens;

  // A wave brings one block of each stage (past the last key: the last block
  // again, whose scores count as unseen). Called with st = 0, 1, ..: the blocks
  // of 64 stages at a time in a register's lanes.
  int ids = 0;
  // (The address goes through a register of its own: the compiler would
  // otherwise wait for every load in flight before each operand read.)
  uint32_t kv_at = (uint32_t)(uintptr_t)(lds_void_t*)kv;
  asm volatile("" : "+s"(kv_at));
  auto issue = [&](int st) {
    if ((st & 63) == 0) {
      const int b = w.t0 / kBlockTokens + (st + lane) * kStBlk + wv;
      ids = min(max(w.bt[min(b, b_last)], 0), w.last_block);
    }
    const int64_t at = (int64_t)__builtin_amdgcn_readlane(ids, st & 63) * w.stride + lane * 8;
    const uint32_t dst = kv_at + ((st & 1) * kStBlk + wv) * (2 * kTile * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_global_load_lds(w.k_cache + at + i * 512,
                                       (lds_void_t*)(uintptr_t)(dst + i * 1024), 16, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      __builtin_amdgcn_global_load_lds(w.v_cache + at + i * 512,
                                       (lds_void_t*)(uintptr_t)(dst + kTile * 2 + i * 1024), 16, 0,
                                       0);
  };
  // Operands of the 32 keys of step ch of a stage.
  auto read_k = [&](int st, int ch, u32x4_t kf[8]) {
    const bf16_t* kb =
        kv + ((st & 1) * kStBlk + 2 * ch) * 2 * kTile + (lane & 16 ? 2 * kTile : 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) kf[i] = *(const u32x4_t*)(kb + k_frag_off(lane, i));
  };
  auto read_v = [&](int st, int ch, u32x4_t vf[2][2][2]) {
    const bf16_t* vb = kv + ((st & 1) * kStBlk + 2 * ch) * 2 * kTile + kTile;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          vf[j][d][u] = *(const u32x4_t*)(vb + 2 * j * kTile + v_frag_off(lane, d) + u * 256);
  };
  auto scores = [&](const u32x4_t kf[8]) {
    f32x16_t s = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kf[i]), qf[i], s,
                                                  0, 0, 0);
    return s;
  };
  // Probabilities of 32 keys as operands of two products. The running max of a
  // column moves only when a step exceeds it by kLazy.
  auto softmax = [&](const f32x16_t& s, u32x4_t p[2]) {
    const float mx = max16(s);
    const auto sw =
        __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    const float top = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * w.scale_log2;
    const float m_new = top > c.m + kLazy ? top : c.m;
    if (__ballot(m_new != c.m) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(c.m - (m_new == -INFINITY ? 0.f : m_new));
#pragma unroll
      for (int i = 0; i < 4; ++i) c.acc[i] *= alpha;
      c.l *= alpha;
      c.m = m_new;
    }
    const float m_ref = c.m == -INFINITY ? 0.f : c.m;
    float pr[16];
#pragma unroll
    for (int r = 0; r < 16; ++r)
      pr[r] = __builtin_amdgcn_exp2f(fmaf(s[r], w.scale_log2, -m_ref));
    float ls = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 4) ls += (pr[r] + pr[r + 1]) + (pr[r + 2] + pr[r + 3]);
    c.l += ls;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) p[j][e] = pack_bf16x2(pr[8 * j + 2 * e], pr[8 * j + 2 * e + 1]);
  };
  auto values = [&](const u32x4_t v[2][2][2], const u32x4_t p[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const u32x4_t a = v[j][d][0], b = v[j][d][1];
        c.acc[2 * d] = pv_step(a.x, a.y, b.x, b.y, p[j], c.acc[2 * d]);
        c.acc[2 * d + 1] = pv_step(a.z, a.w, b.z, b.w, p[j], c.acc[2 * d + 1]);
      }
  };
  auto begin = [&](int st) {
    wait_vmcnt<0>();  // this wave's block of stage st
    stage_barrier();  // every wave's; and all are done with stage st - 1
    if (st + 1 < stages) issue(st + 1);
  };

  issue(0);
  if (w.idle) {
#pragma unroll 1
    for (int st = 0; st < stages; ++st) begin(st);
    return;
  }
  // Stages that every column sees whole; then the others.
  const int clear = min(stages, max(w.prefix - w.t0, 0) / kStKeys);
  int st = 0;
#pragma unroll 1
  for (; st < clear; ++st) {
    begin(st);
    u32x4_t kf[8];
    read_k(st, w.ks, kf);
#pragma unroll 1
    for (int ch = w.ks; ch < 4; ch += KS) {
      u32x4_t vf[2][2][2], p[2];
      const f32x16_t s = scores(kf);
      read_v(st, ch, vf);
      if (KS < 4) read_k(st, min(ch + KS, 3), kf);
      softmax(s, p);
      values(vf, p);
    }
  }
#pragma unroll 1
  for (; st < stages; ++st) {
    begin(st);
#pragma unroll 1
    for (int ch = w.ks; ch < 4; ch += KS) {
      const int tok0 = w.t0 + st * kStKeys + ch * kChunk;
      if (tok0 >= w.t1) continue;
      u32x4_t kf[8], vf[2][2][2], p[2];
      read_k(st, ch, kf);
      f32x16_t s = scores(kf);
      read_v(st, ch, vf);
      if (tok0 + kChunk > w.prefix) {
        const uint32_t seen =
            tree_bits32(w.mask, w.words, w.nodes, tok0 - w.prefix) >> (4 * hf);
        mask_scores(s, seen);
        if (mask_values(vf, hf, w.t1 - tok0) & seen) *w.redo = 1;
      }
      softmax(s, p);
      values(vf, p);
    }
  }
}

__global__ __launch_bounds__(kThreads, 2) void tree_attention_kernel(TreeArgs a) {
  // Two stages of keys and values; at the end the waves' O^T ([wave][64
  // values][64 lanes] floats), 128 KB either way.
  __shared__ __attribute__((aligned(16))) bf16_t kv[2 * kStBlk * 2 * kTile];
  __shared__ int items_s[kMaxSeqs + 1], base_s[kMaxSeqs];
  __shared__ int wsum[2][kWaves], next_s[2];
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
  const int total = carry_i;
  if (carry_b > a.part_cap) return;  // more rows than the call named: no room for their parts

  // Workgroups draw items in order, each its next one while it works (the merge
  // kernel sets the count back to zero). A fixed share of the items left a
  // quarter of the chip idle at the end.
  int item = blockIdx.x;
#pragma unroll 1
  for (int k = 0; item < total; ++k) {
    int drawn = 0;
    if (tid == 0) drawn = (int)gridDim.x + atomicAdd(a.drawn, 1);
    int lo = 0, hi = rk.n_seqs - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (items_s[mid] <= item) lo = mid; else hi = mid - 1;
    }
    const int s = __builtin_amdgcn_readfirstlane(lo);
    const TreeSeq ts = tree_plan((const int32_t*)rk.seq_starts, rk.ctx_lens, s, G, rk.max_blocks);
    int x = __builtin_amdgcn_readfirstlane(item - items_s[s]);
    const int tile_i = x % ts.tiles;
    x /= ts.tiles;
    const int g = x % a.Hkv, sp = x / a.Hkv;
    const int cols = ts.nodes * G, row0 = rk.seq_starts[s];
    int rgs;
    const int group0 = tree_tile((cols + kCols - 1) / kCols, tile_i, &rgs);
    const int kss = kWaves / rgs;  // key sets
    Walk w;
    const int rg = wv & (rgs - 1);  // this wave's columns; and keys:
    w.ks = rgs == 8 ? 0 : rgs == 4 ? wv >> 2 : wv >> 1;
    w.stride = a.Hkv * kTile;
    w.k_cache = a.k_cache + g * kTile;
    w.v_cache = a.v_cache + g * kTile;
    w.last_block = (int)min(rk.num_blocks, (int64_t)INT32_MAX) - 1;
    w.bt = rk.block_table + (int64_t)s * rk.max_blocks;
    w.words = rk.words;
    w.nodes = ts.nodes;
    w.prefix = ts.len - ts.nodes;
    w.t0 = sp * ts.part;
    w.t1 = min(ts.len, w.t0 + ts.part);
    w.scale_log2 = a.scale_log2;
    w.idle = (group0 + rg) * kCols >= cols;

    // This lane's column; columns past the last repeat it.
    const int col = (group0 + rg) * kCols + (lane & 31);
    const int colc = min(col, cols - 1);
    const bool live = col < cols;
    const int row = row0 + colc / G, head = g * G + colc % G;
    w.mask = rk.mask + (int64_t)row * rk.words;
    w.redo = a.redo + (int64_t)row * a.Hq + head;
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
    if (ts.len > 0) {
      if (kss == 4)
        tree_walk<4>(w, qf, kv, lane, wv, c);
      else if (kss == 2)
        tree_walk<2>(w, qf, kv, lane, wv, c);
      else
        tree_walk<1>(w, qf, kv, lane, wv, c);
    }
    if (tid == 0) next_s[k & 1] = drawn;
    __syncthreads();  // every wave is done with kv
    item = next_s[k & 1];

    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(c.l), __float_as_uint(c.l),
                                                     false, false);
    float M = c.m, L = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    // Where this lane's column goes: a part, or the output row.
    const int64_t idx = base_s[s] + ((int64_t)(row - row0) * a.Hq + head) * ts.splits + sp;
    float* const part = ts.splits > 1 ? a.part_o + idx * HD + 4 * hf : nullptr;
    bf16_t* const out = a.o + 4 * hf + (a.tiled ? tile_off(row, head * HD, a.Hq * HD)
                                                : ((int64_t)row * a.Hq + head) * HD);
    auto put = [&](int v4, f32x4_t y, float inv) {
      if (part)
        *(f32x4_t*)(part + run_dim(v4)) = y;
      else
        store4(out + (a.tiled ? run_tiled(v4) : run_dim(v4)), y[0] * inv, y[1] * inv, y[2] * inv,
               y[3] * inv);
    };
    if (kss > 1) {
      // Merge the key sets of each column group: weights from the sets' maxima,
      // sums in set order, wave (rg, ks) adding values 64 ks / kss .. of all.
      float* xs = reinterpret_cast<float*>(kv);
      if (hf == 0) {
        sm_m[wv][lane] = M;
        sm_l[wv][lane] = L;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) xs[(wv * 64 + i * 16 + r) * 64 + lane] = c.acc[i][r];
      __syncthreads();
      const int lc = lane & 31;
      float f[4];
      M = -INFINITY;
      L = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (k < kss) M = fmaxf(M, sm_m[k * rgs + rg][lc]);
      const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[k] = 0.f;
        if (k < kss) {
          f[k] = __builtin_amdgcn_exp2f(sm_m[k * rgs + rg][lc] - ref);
          L = fmaf(f[k], sm_l[k * rgs + rg][lc], L);
        }
      }
      const int per_w = kss == 4 ? 16 : 32;
      const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll 1
      for (int v4 = w.ks * per_w; v4 < (w.ks + 1) * per_w; v4 += 4) {
        f32x4_t y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (k < kss) {
            const float* z = xs + ((k * rgs + rg) * 64 + v4) * 64 + lane;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] = fmaf(f[k], z[r * 64], y[r]);
          }
        if (live) put(v4, y, inv);
      }
      __syncthreads();  // LDS is free for the next item
    } else if (live) {
      const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          put(16 * i + r,
              f32x4_t{c.acc[i][r], c.acc[i][r + 1], c.acc[i][r + 2], c.acc[i][r + 3]}, inv);
    }
    if (part && live && w.ks == 0 && hf == 0) {
      a.part_ml[2 * idx] = M;
      a.part_ml[2 * idx + 1] = L;
    }
  }
}

// The parts of a row's heads, in order: four dims per thread, 32 threads per
// head, eight heads per workgroup.
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.drawn = 0;
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
  a.drawn = redo;
  a.redo = redo + 1;
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
