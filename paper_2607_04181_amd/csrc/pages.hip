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
constexpr int kPlanIds = 8;  // blocks a thread looks at per round

// Inclusive sum over a wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(x, d, kWave);
    if (lane >= d) x += y;
  }
  return x;
}

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

__global__ __launch_bounds__(kPlanThreads) void page_plan_kernel(PageArgs a) {
  __shared__ int sums[kPlanIds * kPlanWaves];
  __shared__ int carry;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  // What each request needs, into off[].
  if (a.src != nullptr) {
    for (int i = tid; i < a.n; i += kPlanThreads)
      a.off[i] = page_request_ok(a, i) ? (a.lens[i] % kBlockTokens != 0) : -1;
  } else {
    for (int i = wv; i < a.n; i += kPlanWaves) {
      int need = -1;
      if (page_request_ok(a, i)) {
        const int nb = (a.lens[i] + kBlockTokens - 1) / kBlockTokens;
        const int32_t* bt = a.table + (int64_t)a.dst[i] * a.max_blocks;
        int c = 0;
        for (int b = lane; b < nb; b += kWave) c += bt[b] < 0;
        need = __shfl(wave_scan(c), kWave - 1, kWave);
      }
      if (lane == 0) a.off[i] = need;
    }
  }
  if (tid == 0) carry = 0;
  __syncthreads();
  // Their places in the list, in request order (off[] becomes the exclusive
  // sum, off[n] the whole), and in status[] what each needs.
  for (int i0 = 0; i0 < a.n; i0 += kPlanThreads) {
    const int i = i0 + tid;
    const int need = i < a.n ? a.off[i] : 0;
    const int x = need > 0 ? need : 0;
    const int s = wave_scan(x);
    if (lane == kWave - 1) sums[wv] = s;
    __syncthreads();
    int before = carry;
    for (int w = 0; w < wv; ++w) before += sums[w];
    if (i < a.n) {
      a.off[i] = before + s - x;
      a.status[i] = need;
    }
    __syncthreads();
    if (tid == kPlanThreads - 1) carry = before + s;
    __syncthreads();
  }
  const int total = carry;
  // The free blocks of lowest id, as many as are needed.
  int found = 0;
  for (int64_t base = 0; base < a.num_blocks && found < total;
       base += kPlanThreads * kPlanIds) {
    bool free_blk[kPlanIds];
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u) {
      const int64_t id = base + u * kPlanThreads + tid;
      free_blk[u] = id < a.num_blocks && a.refs[id] == 0;
    }
    uint64_t votes[kPlanIds];
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u) {
      votes[u] = __ballot(free_blk[u]);
      if (lane == 0) sums[u * kPlanWaves + wv] = __popcll(votes[u]);
    }
    __syncthreads();
    // Each thread sums what lies before its own eight places.
    int place[kPlanIds], at = found;
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u) {
      place[u] = at;
      for (int w = 0; w < kPlanWaves; ++w) {
        const int c = sums[u * kPlanWaves + w];
        if (w < wv) place[u] += c;
        at += c;
      }
    }
#pragma unroll
    for (int u = 0; u < kPlanIds; ++u) {
      const int p = place[u] + __popcll(votes[u] & ((1ull << lane) - 1));
      if (free_blk[u] && p < total) a.list[p] = (int)(base + u * kPlanThreads + tid);
    }
    found = at;
    __syncthreads();
  }
  // A request is served while those up to it fit.
  for (int i = tid; i < a.n; i += kPlanThreads) {
    const int need = a.status[i];
    a.status[i] = need >= 0 && (need == 0 || a.off[i] + need <= found);
  }
}

// One wave per request: its row's empty entries get their blocks.
__global__ __launch_bounds__(kWave) void page_alloc_kernel(PageArgs a) {
  const int i = blockIdx.x, lane = threadIdx.x;
  if (a.status[i] == 0) return;
  const int nb = (a.lens[i] + kBlockTokens - 1) / kBlockTokens;
  int32_t* bt = a.table + (int64_t)a.dst[i] * a.max_blocks;
  int at = a.off[i];
  for (int b0 = 0; b0 < nb; b0 += kWave) {
    const int b = b0 + lane;
    const bool empty = b < nb && bt[b] < 0;
    const uint64_t votes = __ballot(empty);
    if (empty) {
      const int id = a.list[at + __popcll(votes & ((1ull << lane) - 1))];
      bt[b] = id;
      a.refs[id] = 1;
    }
    at += __popcll(votes);
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
  if (dst < 0 || dst >= a.n_seqs) return;
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
// later one still reads.
template <typename T>
__global__ __launch_bounds__(256) void page_compact_kernel(
    const int32_t* __restrict__ seq, const int32_t* __restrict__ base,
    const int32_t* __restrict__ kept, const int32_t* __restrict__ starts, int n_kept,
    const int32_t* __restrict__ table, int n_seqs, int max_blocks, int64_t num_blocks,
    CachePools pools, int Hkv, int hd) {
  constexpr int kTok = 16, kMaxPer = kTok * 256 / 256;
  __shared__ int64_t from_s[kTok], to_s[kTok];  // tile << 4 | slot; -1: nothing moves
  const int i = blockIdx.x, g = blockIdx.y;
  T* pool = (T*)pools.p[blockIdx.z];
  const bool values = blockIdx.z & 1;
  const int row = seq[i];
  if (row < 0 || row >= n_seqs) return;
  const int32_t* bt = table + (int64_t)row * max_blocks;
  const int k0 = max(starts[i], 0), k1 = min(starts[i + 1], n_kept), b0 = base[i];
  const int last = max_blocks * kBlockTokens;
  auto place = [&](int pos) -> int64_t {
    if (pos < 0 || pos >= last) return -1;
    const int blk = bt[pos / kBlockTokens];
    return blk < 0 || blk >= num_blocks
               ? -1
               : (((int64_t)blk * Hkv + g) << 4 | (pos % kBlockTokens));
  };
  const int tile = kBlockTokens * hd;
  for (int k = k0; k < k1; k += kTok) {
    if (threadIdx.x < kTok) {
      const bool live = k + (int)threadIdx.x < k1;
      const int pos = live ? kept[k + threadIdx.x] : -1;
      const int to = b0 + (k - k0) + (int)threadIdx.x;
      const bool moves = live && pos != to;
      from_s[threadIdx.x] = moves ? place(pos) : -1;
      to_s[threadIdx.x] = moves ? place(to) : -1;
    }
    __syncthreads();
    T r[kMaxPer];
    const int n = kTok * hd;
#pragma unroll
    for (int u = 0; u < kMaxPer; ++u) {
      const int x = threadIdx.x + u * 256;
      if (x >= n) break;
      const int t = x / hd, h = x - t * hd;
      const int64_t f = from_s[t];
      if (f < 0 || to_s[t] < 0) continue;
      const int slot = (int)(f & 15);
      r[u] = pool[(f >> 4) * tile + (values ? v_tile_offset(slot, h) : k_tile_offset(slot, h))];
    }
    wait_vmcnt<0>();  // every value is here before any is overwritten
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kMaxPer; ++u) {
      const int x = threadIdx.x + u * 256;
      if (x >= n) break;
      const int t = x / hd, h = x - t * hd;
      const int64_t f = to_s[t];
      if (f < 0 || from_s[t] < 0) continue;
      const int slot = (int)(f & 15);
      pool[(f >> 4) * tile + (values ? v_tile_offset(slot, h) : k_tile_offset(slot, h))] = r[u];
    }
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_page_plan(const PageArgs& a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH(page_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_alloc(const PageArgs& a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH(page_alloc_kernel, dim3(a.n), dim3(kWave), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_fork(const PageArgs& a, const CachePools& pools, int64_t bytes,
                            bool tables, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH(page_fork_kernel, dim3(a.n, pools.n + (tables ? 1 : 0)), dim3(256), 0, st, a, pools,
              bytes, tables);
  return hipGetLastError();
}

hipError_t launch_page_free(const int32_t* seq, const int32_t* keep, int n, int n_seqs,
                            int32_t* table, int max_blocks, int32_t* refs, int64_t num_blocks,
                            hipStream_t st) {
  if (n <= 0) return hipSuccess;
  COCO_LAUNCH(page_free_kernel, dim3((max_blocks + 255) / 256, n), dim3(256), 0, st, seq, keep,
              n_seqs, table, max_blocks, refs, num_blocks);
  return hipGetLastError();
}

hipError_t launch_page_copy(const int32_t* src, const int32_t* dst, int n, int64_t num_blocks,
                            const CachePools& pools, int64_t bytes, hipStream_t st) {
  if (n <= 0) return hipSuccess;
  COCO_LAUNCH(page_copy_kernel, dim3(n, pools.n), dim3(256), 0, st, src, dst, num_blocks, pools,
              bytes);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_page_compact(const int32_t* seq, const int32_t* base, const int32_t* kept,
                               const int32_t* starts, int n, int n_kept, const int32_t* table,
                               int n_seqs, int max_blocks, int64_t num_blocks,
                               const CachePools& pools, int Hkv, int hd, hipStream_t st) {
  if (n <= 0 || n_kept <= 0) return hipSuccess;
  if (hd % 32 != 0 || hd > 256 || Hkv > 65535) return hipErrorInvalidValue;
  COCO_LAUNCH((page_compact_kernel<T>), dim3(n, Hkv, pools.n), dim3(256), 0, st, seq, base, kept,
              starts, n_kept, table, n_seqs, max_blocks, num_blocks, pools, Hkv, hd);
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
