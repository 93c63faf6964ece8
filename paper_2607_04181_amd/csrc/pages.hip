// The cache's pages: allocating and forking blocks, dropping references,
// copying blocks, and moving the tokens that stay to the front.
//
// A block is free when its reference count is 0. Requests take the free blocks
// of lowest id in the order of the call, so the ids depend on the counts alone.
// Allocation runs in two kernels: one workgroup counts what each request needs
// and lists that many free blocks (page_plan_kernel); the second, with a
// workgroup per request or per block copied, writes tables, counts and pages
// from that list. All of it is bound by the bytes moved and, in small calls,
// by the two launches and the plan's chain of dependent reads.
#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanIds = 16;      // consecutive blocks a thread looks at per round
constexpr int kAllocEntries = 8;
constexpr int kPlanEntries = 8;   // table entries a lane reads at a time

// Blocks that request i needs; -1: it names no valid row or length.
//   alloc: its row's empty entries below ceil(len / 16);
//   fork: one, where the shared length ends inside a block.
__device__ __forceinline__ bool page_request_ok(const PageArgs& a, int i) {
  const int len = a.lens[i], row = a.dst[i];
  if (row < 0 || row >= a.n_seqs || len < 0 || len > a.max_blocks * kBlockTokens) return false;
  if (a.src == nullptr) return true;
  const int src = a.src[i];
  return src >= 0 && src < a.n_seqs && src != row;
}

// Exclusive sum over the workgroup's threads, and the whole (a wave's of up to 2^24
// each, a row's entries, fits 32 bits). Its barriers also keep one call's sums
// from the next's.
template <typename SUM>
__device__ __forceinline__ SUM plan_scan(int x, int* sums, SUM& all) {
  const int lane = threadIdx.x & 63;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int upto = wave_scan(x);
  __syncthreads();
  if (lane == kWave - 1) sums[wv] = upto;
  __syncthreads();
  SUM before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) {
    const int c = sums[w];
    if (w < wv) before += c;
    all += c;
  }
  return before + upto - x;
}

// SUM: holds what all requests can need. (64-bit in every call: 256 forks 5.9 us
// instead of 5.2.)
template <typename SUM>
__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PageArgs a) {
  __shared__ int sums[kPlanWaves];
  const int tid = threadIdx.x;
  // Counts of the first round of the search below, read while the needs are
  // found.
  int32_t r[kPlanIds];
  auto counts = [&](int64_t base) {
    const int64_t first = base + tid * kPlanIds;
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u)
      r[u] = a.refs[first + u < a.num_blocks ? first + u : a.num_blocks - 1];
  };
  counts(0);
  if (a.src == nullptr) {
    // What each request needs, into off[]: a wave per request, or 16 lanes
    // where there are more requests than waves (reads in flight, not lanes, are
    // what the scan of a table row lacks).
    const int lanes = a.n > kPlanWaves ? 16 : kWave;
    const int at = tid & (lanes - 1);
    for (int i = tid / lanes; i < a.n; i += kPlanThreads / lanes) {
      const bool ok = page_request_ok(a, i);
      int c = 0;
      if (ok) {
        const int nb = (a.lens[i] + kBlockTokens - 1) / kBlockTokens;
        const int32_t* bt = a.table + (int64_t)a.dst[i] * a.max_blocks;
        for (int b0 = at; b0 < nb; b0 += lanes * kPlanEntries) {
          int e[kPlanEntries];
#pragma unroll
          for (int u = 0; u < kPlanEntries; ++u) e[u] = bt[min(b0 + u * lanes, nb - 1)];
#pragma unroll
          for (int u = 0; u < kPlanEntries; ++u) c += b0 + u * lanes < nb && e[u] < 0;
        }
      }
      for (int d = 1; d < lanes; d <<= 1) c += __shfl_xor(c, d, kWave);
      if (at == 0) a.off[i] = ok ? c : -1;
    }
    __syncthreads();
  }
  // Their places in the list, in request order (off[] becomes the exclusive
  // sum), and in status[] what each needs. A place past 2^31 is held there, where
  // nothing fits either.
  SUM total = 0;
  int need = 0, at = 0;  // (of the thread's last request)
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    need = 0;
    if (i < a.n) {
      if (a.src == nullptr)
        need = a.off[i];
      else
        need = page_request_ok(a, i) ? (a.lens[i] % kBlockTokens != 0) : -1;
    }
    SUM all;
    const SUM before = plan_scan(max(need, 0), sums, all);
    at = (int)min(total + before, (SUM)INT32_MAX);
    if (i < a.n) {
      a.off[i] = at;
      a.status[i] = need;
    }
    total += all;
  }
  // The free blocks of lowest id, as many as are needed.
  int found = 0;
  for (int64_t base = 0; base < a.num_blocks && found < total;
       base += kPlanThreads * kPlanIds) {
    const int64_t first = base + tid * kPlanIds;
    if (base > 0) counts(base);
    uint32_t free_ids = 0;
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u)
      free_ids |= (uint32_t)(first + u < a.num_blocks && r[u] == 0) << u;
    int all;
    int place = found + plan_scan(__popc(free_ids), sums, all);
    for (; free_ids && place < total; free_ids &= free_ids - 1)
      a.list[place++] = (int)(first + __builtin_ctz(free_ids));
    found += all;
  }
  // A request is served while those up to it fit.
  const int last = (a.n - 1) / kPlanThreads * kPlanThreads + tid;
  if (last < a.n) a.status[last] = need >= 0 && (need == 0 || need <= found - at);
  for (int i = tid; i < last && i < a.n; i += kPlanThreads) {
    const int n = a.status[i];
    a.status[i] = n >= 0 && (n == 0 || n <= found - a.off[i]);
  }
}

// One wave per request: its row's empty entries get their blocks.
__global__ __launch_bounds__(kWave) void page_alloc_kernel(PageArgs a) {
  const int i = blockIdx.x, lane = threadIdx.x;
  if (a.status[i] == 0) return;
  const int nb = (a.lens[i] + kBlockTokens - 1) / kBlockTokens;
  int32_t* bt = a.table + (int64_t)a.dst[i] * a.max_blocks;
  int at = a.off[i];
  for (int b0 = 0; b0 < nb; b0 += kWave * kAllocEntries) {
    int e[kAllocEntries];
#pragma unroll
    for (int u = 0; u < kAllocEntries; ++u) e[u] = bt[min(b0 + u * kWave + lane, nb - 1)];
#pragma unroll
    for (int u = 0; u < kAllocEntries; ++u) {
      const int b = b0 + u * kWave + lane;
      const bool empty = b < nb && e[u] < 0;
      const uint64_t votes = __ballot(empty);
      if (empty) {
        const int id = a.list[at + __popcll(votes & ((1ull << lane) - 1))];
        bt[b] = id;
        a.refs[id] = 1;
      }
      at += __popcll(votes);
    }
  }
}

__device__ __forceinline__ void copy_page(char* pool, int64_t bytes, int64_t src, int64_t dst) {
  const u32x4_t* s = (const u32x4_t*)(pool + src * bytes);
  u32x4_t* d = (u32x4_t*)(pool + dst * bytes);
  for (int64_t x = threadIdx.x; x < bytes / 16; x += blockDim.x) d[x] = s[x];
}

// Workgroup (fork, 0): the child's table row and the counts; (fork, 1 + p):
// pool p's copy of the partial last block.
__global__ __launch_bounds__(256) void page_fork_kernel(PageArgs a, CachePools pools,
                                                        int64_t bytes, bool tables) {
  const int i = blockIdx.x;
  const int src = a.src[i], dst = a.dst[i], len = a.lens[i];
  const bool served = a.status[i] != 0;
  const int full = len / kBlockTokens;
  const bool tail = served && len % kBlockTokens != 0;
  const int p = (int)blockIdx.y - (tables ? 1 : 0);
  if (p >= 0) {
    if (!tail) return;
    const int from = a.table[(int64_t)src * a.max_blocks + full];
    if (from >= 0 && from < a.num_blocks) copy_page(pools.p[p], bytes, from, a.list[a.off[i]]);
    return;
  }
  // A row named as its own parent keeps what it holds.
  if (dst < 0 || dst >= a.n_seqs || dst == src) return;
  for (int b = threadIdx.x; b < a.max_blocks; b += blockDim.x) {
    int id = -1;
    if (served && b < full) {
      id = a.table[(int64_t)src * a.max_blocks + b];
      if (id >= 0 && id < a.num_blocks) atomicAdd(&a.refs[id], 1);
    } else if (tail && b == full) {
      id = a.list[a.off[i]];
      a.refs[id] = 1;
    }
    a.table[(int64_t)dst * a.max_blocks + b] = id;
  }
}

// Entries from ceil(keep / 16) on lose their block. The exchange makes a row
// that the call names twice lose it once.
__global__ __launch_bounds__(256) void page_free_kernel(const int32_t* __restrict__ seq,
                                                        const int32_t* __restrict__ keep,
                                                        int n_seqs, int32_t* table,
                                                        int max_blocks, int32_t* refs,
                                                        int64_t num_blocks) {
  const int row = seq[blockIdx.y];
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (row < 0 || row >= n_seqs || b >= max_blocks) return;
  const int k = keep ? keep[blockIdx.y] : 0;
  if (b < k / kBlockTokens + (k % kBlockTokens > 0)) return;
  int32_t* e = table + (int64_t)row * max_blocks + b;
  if (*e < 0) return;
  const int id = atomicExch(e, -1);
  if (id >= 0 && id < num_blocks) atomicSub(&refs[id], 1);
}

__global__ __launch_bounds__(256) void page_copy_kernel(const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst,
                                                        int64_t num_blocks, CachePools pools,
                                                        int64_t bytes) {
  const int s = src[blockIdx.x], d = dst[blockIdx.x];
  if (s < 0 || d < 0 || s >= num_blocks || d >= num_blocks || s == d) return;
  copy_page(pools.p[blockIdx.y], bytes, s, d);
}

// Tokens kept[starts[i] ..] of row seq[i] to positions base[i], base[i] + 1,
// ... of it, for one head of one pool: 16 at a time through registers. A token
// never moves up (kept[k] >= base + k, ascending), so no group writes where a
// later one still reads. A key tile holds 8 dims of a token together and moves
// in 16-byte pieces; a value tile has its tokens innermost, four by four, so a
// token moves by elements, 32 of a half wave 4 elements apart. HS: head_dim / 32.
template <typename T, int HS>
__global__ __launch_bounds__(256) void page_compact_kernel(
    const int32_t* __restrict__ seq, const int32_t* __restrict__ base,
    const int32_t* __restrict__ kept, const int32_t* __restrict__ starts, int n_kept,
    const int32_t* __restrict__ table, int n_seqs, int max_blocks, int64_t num_blocks,
    CachePools pools, int Hkv) {
  constexpr int kTok = 16, kTile = kBlockTokens * 32 * HS;
  constexpr int kPer = 16 / sizeof(T);                    // elements of a piece
  constexpr int kPieces = kTok * 32 * HS / kPer;          // of 16 tokens
  constexpr int kKeys = (kPieces + 255) / 256, kVals = 2 * HS;
  __shared__ int64_t from_s[kTok], to_s[kTok];  // tile << 4 | slot; -1: nothing moves
  const int i = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  T* pool = (T*)pools.p[blockIdx.z];
  const int row = seq[i];
  const int k0 = max(starts[i], 0), k1 = min(starts[i + 1], n_kept), b0 = base[i];
  if (row < 0 || row >= n_seqs) return;
  const int32_t* bt = table + (int64_t)row * max_blocks;
  const int last = max_blocks * kBlockTokens;
  auto place = [&](int pos) -> int64_t {
    if (pos < 0 || pos >= last) return -1;
    const int blk = bt[pos / kBlockTokens];
    return blk < 0 || blk >= num_blocks
               ? -1
               : (((int64_t)blk * Hkv + g) << 4 | (pos % kBlockTokens));
  };
  for (int k = k0; k < k1; k += kTok) {
    if (tid < kTok) {
      const bool live = k + tid < k1;
      const int pos = live ? kept[k + tid] : -1;
      const int to = b0 + (k - k0) + tid;
      const bool moves = live && pos != to;
      const int64_t f = moves ? place(pos) : -1, t = moves ? place(to) : -1;
      from_s[tid] = t < 0 ? -1 : f;
      to_s[tid] = f < 0 ? -1 : t;
    }
    __syncthreads();
    if (blockIdx.z & 1) {
      const int w = tid & 31;
      T r[kVals];
#pragma unroll
      for (int u = 0; u < kVals; ++u) {  // unit (token, 32 dims) of a half wave
        const int unit = (tid >> 5) + 8 * u;
        const int64_t f = from_s[unit & 15];
        if (f >= 0)
          r[u] = pool[(f >> 4) * kTile + (unit >> 4) * 512 + ((int)f & 12) * 32 + w * 4 +
                      ((int)f & 3)];
      }
      wait_vmcnt<0>();  // every value is here before any is overwritten
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kVals; ++u) {
        const int unit = (tid >> 5) + 8 * u;
        const int64_t t = to_s[unit & 15];
        if (t >= 0)
          pool[(t >> 4) * kTile + (unit >> 4) * 512 + ((int)t & 12) * 32 + w * 4 + ((int)t & 3)] =
              r[u];
      }
    } else {
      // Piece c of a token: elements c kPer .. of it.
      u32x4_t r[kKeys];
      const auto at = [&](int64_t x, int c) -> u32x4_t* {
        const int h = c * kPer;
        return (u32x4_t*)(pool + (x >> 4) * kTile + (h >> 3) * 128 + ((int)x & 15) * 8 + (h & 7));
      };
#pragma unroll
      for (int u = 0; u < kKeys; ++u) {
        const int x = tid + 256 * u;
        const int64_t f = from_s[x & 15];
        if (x < kPieces && f >= 0) r[u] = *at(f, x >> 4);
      }
      wait_vmcnt<0>();
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kKeys; ++u) {
        const int x = tid + 256 * u;
        const int64_t t = to_s[x & 15];
        if (x < kPieces && t >= 0) *at(t, x >> 4) = r[u];
      }
    }
    __syncthreads();  // the places are read, and the group is written
  }
}

// The same for long lists: the tokens of 64 positions (32 where one takes more than 512
// bytes of a head) at a time. A lane puts four tokens' elements of a dim of a value tile
// together and stores them as one, where all four move (at a list's ends one by one).
// What bounds it is a group's chain: list, table, tokens, their stores; the places of
// a group are looked up while the tokens of the one before are on their way. 64 lists of
// 2000 tokens out of 2200, 8 heads of 128 dims, 8 pools take 1087 us (3.9 TB/s; 16 at a
// time 1852), one list of 4000 177 (867), but 64 of 6 tokens 41 in place of 19. The two
// meet at 32 tokens (46 us for 64 lists): the room that a call has per list decides.
constexpr int kFewKept = 32;  // tokens a list, on average
template <typename T>
constexpr int compact_tokens(int HS) {  // (held in registers)
  return HS * sizeof(T) <= 16 ? 4 * kBlockTokens : 2 * kBlockTokens;
}
template <typename T, int HS>
__global__ __launch_bounds__(256) void page_compact_long_kernel(
    const int32_t* __restrict__ seq, const int32_t* __restrict__ base,
    const int32_t* __restrict__ kept, const int32_t* __restrict__ starts, int n_kept,
    const int32_t* __restrict__ table, int n_seqs, int max_blocks, int64_t num_blocks,
    CachePools pools, int Hkv) {
  constexpr int kTok = compact_tokens<T>(HS), kTile = kBlockTokens * 32 * HS;
  constexpr int kPer = 16 / sizeof(T);                // elements of a piece
  constexpr int kKeys = kTok * 32 * HS / kPer / 256;  // pieces of a thread
  constexpr int kVals = kTok / 4 * HS / 8;            // its (four tokens, 32 dims) of a half wave
  typedef T quad_t __attribute__((ext_vector_type(4)));
  __shared__ int64_t from_s[2][kTok], to_s[2][kTok];  // tile << 4 | slot; -1: nothing moves
  const int i = blockIdx.x, g = blockIdx.y, tid = threadIdx.x;
  T* pool = (T*)pools.p[blockIdx.z];
  const int row = seq[i];
  const int k0 = max(starts[i], 0), k1 = min(starts[i + 1], n_kept), b0 = base[i];
  if (row < 0 || row >= n_seqs || k0 >= k1) return;
  const int32_t* bt = table + (int64_t)row * max_blocks;
  const int last = max_blocks * kBlockTokens;
  auto place = [&](int pos) -> int64_t {
    if (pos < 0 || pos >= last) return -1;
    const int blk = bt[pos / kBlockTokens];
    return blk < 0 || blk >= num_blocks
               ? -1
               : (((int64_t)blk * Hkv + g) << 4 | (pos % kBlockTokens));
  };
  // Places of the group whose first position is d0 (of a block's start, or below the base).
  auto look_up = [&](int64_t d0, int half) {
    if (tid >= kTok) return;
    const int64_t k = k0 + (d0 - b0) + tid;
    const bool live = k >= k0 && k < k1;
    const int pos = live ? kept[k] : -1, to = (int)(d0 + tid);
    const bool moves = live && pos != to;
    const int64_t f = moves ? place(pos) : -1, t = moves ? place(to) : -1;
    from_s[half][tid] = t < 0 ? -1 : f;
    to_s[half][tid] = f < 0 ? -1 : t;
  };
  const int64_t first = b0 & ~(kBlockTokens - 1), end = (int64_t)b0 + (k1 - k0);
  look_up(first, 0);
  __syncthreads();
  int half = 0;
  for (int64_t d0 = first; d0 < end; d0 += kTok, half ^= 1) {
    const int64_t *from = from_s[half], *to = to_s[half];
    if (blockIdx.z & 1) {
      const int w = tid & 31;
      quad_t r[kVals];
#pragma unroll
      for (int u = 0; u < kVals; ++u) {
        const int unit = (tid >> 5) + 8 * u, t4 = unit % (kTok / 4) * 4, dims = unit / (kTok / 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int64_t f = max(from[t4 + e], (int64_t)0);  // (any place: not stored)
          r[u][e] = pool[(f >> 4) * kTile + dims * 512 + ((int)f & 12) * 32 + w * 4 + ((int)f & 3)];
        }
      }
      if (d0 + kTok < end) look_up(d0 + kTok, half ^ 1);
      wait_vmcnt<0>();  // every value is here before any is overwritten
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kVals; ++u) {
        const int unit = (tid >> 5) + 8 * u, t4 = unit % (kTok / 4) * 4, dims = unit / (kTok / 4);
        int64_t t[4];
        bool all = true;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          t[e] = to[t4 + e];
          all = all && t[e] >= 0;
        }
        T* const x = pool + (int64_t)dims * 512 + w * 4;
        if (all) {
          *(quad_t*)(x + (t[0] >> 4) * kTile + ((int)t[0] & 12) * 32) = r[u];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (t[e] >= 0)
              x[(t[e] >> 4) * kTile + ((int)t[e] & 12) * 32 + ((int)t[e] & 3)] = r[u][e];
        }
      }
    } else {
      // Piece c of a token: elements c kPer .. of it.
      u32x4_t r[kKeys];
      const auto at = [&](int64_t x, int c) -> u32x4_t* {
        const int h = c * kPer;
        return (u32x4_t*)(pool + (x >> 4) * kTile + (h >> 3) * 128 + ((int)x & 15) * 8 + (h & 7));
      };
#pragma unroll
      for (int u = 0; u < kKeys; ++u) {
        const int x = tid + 256 * u;
        r[u] = *at(max(from[x % kTok], (int64_t)0), x / kTok);
      }
      if (d0 + kTok < end) look_up(d0 + kTok, half ^ 1);
      wait_vmcnt<0>();
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kKeys; ++u) {
        const int x = tid + 256 * u;
        const int64_t t = to[x % kTok];
        if (t >= 0) *at(t, x / kTok) = r[u];
      }
    }
    // (The next group reads above everything that this one writes; the places of the
    // one after it go where this one's were.)
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_page_plan(const PageArgs& a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  if ((int64_t)a.n * a.max_blocks <= INT32_MAX)
    COCO_LAUNCH(page_plan_kernel<int>, dim3(1), dim3(kPlanThreads), 0, st, a);
  else
    COCO_LAUNCH(page_plan_kernel<int64_t>, dim3(1), dim3(kPlanThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_alloc(const PageArgs& a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH_LAST(page_alloc_kernel, dim3(a.n), dim3(kWave), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_fork(const PageArgs& a, const CachePools& pools, int64_t bytes,
                            bool tables, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH_LAST(page_fork_kernel, dim3(a.n, pools.n + (tables ? 1 : 0)), dim3(256), 0, st, a,
                   pools, bytes, tables);
  return hipGetLastError();
}

hipError_t launch_page_free(const int32_t* seq, const int32_t* keep, int n, int n_seqs,
                            int32_t* table, int max_blocks, int32_t* refs, int64_t num_blocks,
                            hipStream_t st) {
  if (n <= 0) return hipSuccess;
  COCO_LAUNCH_LAST(page_free_kernel, dim3((max_blocks + 255) / 256, n), dim3(256), 0, st, seq,
                   keep, n_seqs, table, max_blocks, refs, num_blocks);
  return hipGetLastError();
}

hipError_t launch_page_copy(const int32_t* src, const int32_t* dst, int n, int64_t num_blocks,
                            const CachePools& pools, int64_t bytes, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  COCO_LAUNCH_LAST(page_copy_kernel, dim3(n, pools.n), dim3(256), 0, st, src, dst, num_blocks,
                   pools, bytes);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_page_compact(const int32_t* seq, const int32_t* base, const int32_t* kept,
                               const int32_t* starts, int n, int n_kept, const int32_t* table,
                               int n_seqs, int max_blocks, int64_t num_blocks,
                               const CachePools& pools, int Hkv, int hd, hipStream_t st) {
  if (n <= 0 || n_kept <= 0) return hipSuccess;
  if (hd % 32 != 0 || hd > 256 || Hkv > 65535) return hipErrorInvalidValue;
  const bool few = n_kept <= (int64_t)n * kFewKept;
#define COCO_COMPACT(HS)                                                                        \
  COCO_LAUNCH_LAST((few ? page_compact_kernel<T, HS> : page_compact_long_kernel<T, HS>),        \
                   dim3(n, Hkv, pools.n), dim3(256), 0, st, seq, base, kept, starts, n_kept,    \
                   table, n_seqs, max_blocks, num_blocks, pools, Hkv)
  COCO_BY_HEAD_DIM(COCO_COMPACT);
#undef COCO_COMPACT
  return hipGetLastError();
}

template hipError_t launch_page_compact<uint16_t>(const int32_t*, const int32_t*, const int32_t*,
                                                  const int32_t*, int, int, const int32_t*, int,
                                                  int, int64_t, const CachePools&, int, int,
                                                  hipStream_t);
template hipError_t launch_page_compact<uint32_t>(const int32_t*, const int32_t*, const int32_t*,
                                                  const int32_t*, int, int, const int32_t*, int,
                                                  int, int64_t, const CachePools&, int, int,
                                                  hipStream_t);

}  // namespace coco
