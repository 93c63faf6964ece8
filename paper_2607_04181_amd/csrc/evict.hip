// Eviction by accumulated attention weight: which tokens a row of the cache keeps.
//
// Of the L tokens of a row with budget B < L, the first f and the last l stay, and
// of the rest the B - f - l of the largest weights, the lowest slot among equals.
// Weights are compared as 32-bit keys in their order (NaN lowest), so the choice is
// in whole numbers. One workgroup per row finds the key T of the last token taken,
// eight bits at a time from counts of the candidates' digits, and how many of
// those with key T are taken; a second one per row writes the list, each after a
// sum over the counts of the requests before its own, and moves the weights.
// The first holds a row of up to 32768 tokens in registers, read once; what both take
// is launches, barriers and one read of a few KB per row, not its bytes.
#include "common.h"
#include "kernels.h"

namespace coco {

namespace {

constexpr int kAllThreads = 1024;
// Rows of at most kFewTokens go on with 256 threads, whose barriers are shorter (64 rows of
// 280 tokens 9.1 us for both kernels, with 1024 threads 12.8; of 1000 9.3 and 12.9; of 2200, in
// steps, 15.2 and 13.0).
constexpr int kFewTokens = 1024, kFewThreads = 256;

// Larger weight, larger key; both zeros alike, NaN lowest.
__device__ __forceinline__ uint32_t weight_key(float w) {
  const uint32_t u = __float_as_uint(w + 0.0f);
  return w != w ? 0u : u >> 31 ? ~u : u | 0x80000000u;
}

struct Row {
  int row, len, keep, first, last;  // row -1: not served
  const f32x4_t* weights;           // null: all alike
};
__device__ __forceinline__ Row evict_row(const EvictArgs& a, int i) {
  Row r;
  r.row = a.seq[i];
  if (r.row < 0 || r.row >= a.n_seqs) r.row = -1;
  const int width = a.max_blocks * kBlockTokens;
  r.len = r.row < 0 ? 0 : min(max(a.ctx[r.row], 0), width);
  r.keep = min(max(a.keep[i], 0), r.len);
  r.first = min(a.keep_first, r.keep);
  r.last = min(a.keep_last, r.keep - r.first);
  r.weights = a.weights == nullptr || r.row < 0
                  ? nullptr
                  : (const f32x4_t*)(a.weights + (int64_t)r.row * width);
  return r;
}
__device__ __forceinline__ f32x4_t load_weights(const Row& r, int t) {
  return r.weights != nullptr && t < r.len ? r.weights[t / 4] : f32x4_t{0.f, 0.f, 0.f, 0.f};
}

// plan[i]: T, how many of key T stay, base, tokens listed.
template <int kThreads>
__device__ __forceinline__ void plan_row(const EvictArgs& a, const Row& r) {
  constexpr int kHeld = kThreads == kAllThreads ? 8 : 1;  // steps whose keys stay in registers
  constexpr int kWaves = kThreads / kWave, kStep = 4 * kThreads;  // slots: four per thread
  __shared__ int hist[256];
  __shared__ int found[2], base_s, red[kWaves];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  uint32_t* plan = a.plan + 4 * (int64_t)i;
  if (r.keep >= r.len) {
    if (tid == 0) {
      plan[0] = plan[1] = plan[3] = 0;
      plan[2] = r.len;
    }
    return;
  }
  const int lo = r.first, hi = r.len - r.last;  // candidates
  int left = r.keep - r.first - r.last;         // of which as many stay
  uint32_t held[kHeld][4];
#pragma unroll
  for (int c = 0; c < kHeld; ++c) {
    if (c * kStep >= r.len) break;
    const f32x4_t w = load_weights(r, c * kStep + 4 * tid);
#pragma unroll
    for (int u = 0; u < 4; ++u) held[c][u] = weight_key(w[u]);
  }
  // f(key, slot) of every candidate; all lanes of a wave take part in each.
  auto each = [&](auto f) {
#pragma unroll
    for (int c = 0; c < kHeld; ++c) {
      if (c * kStep >= r.len) break;
#pragma unroll
      for (int u = 0; u < 4; ++u) f(held[c][u], c * kStep + 4 * tid + u);
    }
#pragma unroll 1
    for (int t0 = kHeld * kStep; t0 < r.len; t0 += kStep) {
      const f32x4_t w = load_weights(r, t0 + 4 * tid);
#pragma unroll
      for (int u = 0; u < 4; ++u) f(weight_key(w[u]), t0 + 4 * tid + u);
    }
  };

  // The left-th largest key, a digit at a time. left == 0: none stays, T above all.
  uint32_t T = 0xFFFFFFFFu;
  int take = 0;
  if (left > 0) {
    T = 0;
#pragma unroll 1
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t above = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
      each([&](uint32_t key, int t) {
        const bool in = t >= lo && t < hi && (key & above) == T;
        const uint64_t lanes = __ballot(in);
        if (lanes == 0) return;
        const uint32_t d = key >> shift & 255;
        // (weights of 0: one count for the wave instead of 64 to one place)
        const uint32_t d0 = __builtin_amdgcn_readlane(d, __builtin_ctzll(lanes));
        if (__ballot(in && d == d0) == lanes) {
          if (lane == 0) atomicAdd(&hist[d0], __popcll(lanes));
        } else if (in) {
          atomicAdd(&hist[d], 1);
        }
      });
      __syncthreads();
      if (wv == 0) {
        // Digits from the largest: lane x has 255 - 4 x .. 252 - 4 x.
        int n[4], sum = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) sum += n[u] = hist[255 - 4 * lane - u];
        int before = wave_scan(sum) - sum;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (before < left && left <= before + n[u]) {
            found[0] = 255 - 4 * lane - u;
            found[1] = left - before;
          }
          before += n[u];
        }
      }
      __syncthreads();
      T |= (uint32_t)found[0] << shift;
      left = found[1];
    }
    take = left;
  }
  // The first slot that does not stay: one below T, or of key T past the take-th.
  if (tid == 0) base_s = hi;
  __syncthreads();
  int below = hi, ties = 0;  // ties: of key T in the steps so far
  each([&](uint32_t key, int t) {
    if (t >= lo && t < hi && key < T) below = min(below, t);
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) below = min(below, __shfl_xor(below, o, kWave));
  if (lane == 0) atomicMin(&base_s, below);
#pragma unroll 1
  for (int t0 = 0; t0 < r.len && ties <= take; t0 += kStep) {
    uint32_t key[4];
    const f32x4_t w = load_weights(r, t0 + 4 * tid);
    int n = 0, t = t0 + 4 * tid;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      key[u] = weight_key(w[u]);
      n += t + u >= lo && t + u < hi && key[u] == T;
    }
    const int incl = wave_scan(n);
    if (lane == kWave - 1) red[wv] = incl;
    __syncthreads();
    int before = ties + incl - n;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wv) before += red[v];
      ties += red[v];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (t + u >= lo && t + u < hi && key[u] == T && before++ == take) atomicMin(&base_s, t + u);
    __syncthreads();
  }
  __syncthreads();
  if (tid == 0) {
    const int base = min(base_s, r.keep);
    plan[0] = T;
    plan[1] = (uint32_t)take;
    plan[2] = (uint32_t)base;
    plan[3] = (uint32_t)(r.keep - base);
  }
}

__global__ __launch_bounds__(kAllThreads) void evict_plan_kernel(EvictArgs a) {
  const Row r = evict_row(a, blockIdx.x);
  if (r.len > kFewTokens)
    plan_row<kAllThreads>(a, r);
  else if (threadIdx.x < kFewThreads)  // (the other waves end, and no barrier counts them)
    plan_row<kFewThreads>(a, r);
}

// Sum over the workgroup's threads.
template <int kWaves>
__device__ __forceinline__ int64_t block_total(int64_t x, int64_t* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  int64_t sum = 0;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) sum += red[v];
  __syncthreads();
  return sum;
}

template <int kThreads>
__device__ __forceinline__ void list_row(const EvictArgs& a, const Row& r) {
  constexpr int kWaves = kThreads / kWave, kStep = 4 * kThreads;  // slots: four per thread
  __shared__ int64_t red64[kWaves];
  __shared__ int red[2][kWaves];
  const int i = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t T = a.plan[4 * (int64_t)i];
  const int take = a.plan[4 * (int64_t)i + 1], base = a.plan[4 * (int64_t)i + 2],
            count = a.plan[4 * (int64_t)i + 3];
  // The tokens listed before: those of the requests up to the first whose own do not fit.
  int64_t mine = 0;
  for (int j0 = 0; j0 < i; j0 += kThreads)
    mine += j0 + tid < i ? (int64_t)a.plan[4 * (int64_t)(j0 + tid) + 3] : 0;
  int64_t start = block_total<kWaves>(mine, red64);
  bool served = start + count <= a.n_kept;
  if (start > a.n_kept) {
    // Some request before does not fit: the list ends where it would begin. (Sums
    // of counts only grow; rare, so one thread walks them.)
    if (tid == 0) {
      int64_t at = 0;
      int j = 0;
      for (; j < i && at + a.plan[4 * (int64_t)j + 3] <= a.n_kept; ++j)
        at += a.plan[4 * (int64_t)j + 3];
      red64[0] = at;
    }
    __syncthreads();
    start = red64[0];
    served = count == 0;
  }
  if (tid == 0) {
    a.kept_starts[i] = (int)start;
    if (i == a.n - 1) a.kept_starts[a.n] = (int)(served ? start + count : start);
    a.new_lens[i] = served ? r.keep : r.len;
    a.base_lens[i] = served ? base : r.len;
  }
  if (!served || r.keep >= r.len) return;

  // Slots from base on in order; a step's weights are read before any is written
  // (no token moves up).
  const int lo = r.first, hi = r.len - r.last;
  float* w_out = r.weights != nullptr ? (float*)r.weights : nullptr;
  int ties = 0, done = 0;
#pragma unroll 1
  for (int t0 = 0; t0 < r.len; t0 += kStep) {
    const int t = t0 + 4 * tid;
    const f32x4_t w = load_weights(r, t);
    bool tie[4], stays[4];
    int n_tie = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bool candidate = t + u >= lo && t + u < hi;
      const uint32_t key = weight_key(w[u]);
      tie[u] = candidate && key == T;
      stays[u] = t + u < r.len && (!candidate || key > T);
      n_tie += tie[u];
    }
    int incl = wave_scan(n_tie);
    if (lane == kWave - 1) red[0][wv] = incl;
    __syncthreads();
    int before = ties + incl - n_tie;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wv) before += red[0][v];
      ties += red[0][v];
    }
    int n = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (tie[u]) stays[u] = before++ < take;
      stays[u] = stays[u] && t + u >= base;
      n += stays[u];
    }
    incl = wave_scan(n);
    if (lane == kWave - 1) red[1][wv] = incl;
    __syncthreads();
    int at = done + incl - n;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      if (v < wv) at += red[1][v];
      done += red[1][v];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      // (at < count but for a row that another request of the call has moved meanwhile)
      if (stays[u] && at < count) {
        a.kept[start + at] = t + u;
        if (w_out != nullptr) w_out[base + at] = w[u];
        ++at;
      }
    __syncthreads();  // the counts are read
  }
  if (w_out != nullptr)
    for (int t = r.keep + tid; t < r.len; t += kThreads) w_out[t] = 0.f;
}

__global__ __launch_bounds__(kAllThreads) void evict_list_kernel(EvictArgs a) {
  const Row r = evict_row(a, blockIdx.x);
  if (r.len > kFewTokens)
    list_row<kAllThreads>(a, r);
  else if (threadIdx.x < kFewThreads)
    list_row<kFewThreads>(a, r);
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  if (a.n <= 0) return hipSuccess;
  COCO_LAUNCH(evict_plan_kernel, dim3(a.n), dim3(kAllThreads), 0, st, a);
  COCO_LAUNCH_LAST(evict_list_kernel, dim3(a.n), dim3(kAllThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace coco
