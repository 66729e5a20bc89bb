// Eviction from the paged cache by accumulated attention weight.
//
// evict_select: one workgroup per (sequence, key head) finds the weight of the
// last token kept by a radix selection over its order-preserving integer, four
// passes of 8 bits, and writes the kept tokens in order. evict_move copies their
// vectors to the new pages.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kSelThreads = 1024;
constexpr int kMoveThreads = 256;

// Integer with the order of the weights: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (w != w) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kSelThreads) void evict_select(
    CacheParams c, const int32_t* __restrict__ lens, const float* __restrict__ weights, int budget,
    int recent, int new_capacity, int32_t* __restrict__ kept, int32_t* __restrict__ new_lens,
    float* __restrict__ new_weights) {
  __shared__ int hist[256];
  __shared__ int found[2];  // the digit, and how many are wanted within it
  __shared__ int above[kSelThreads / kWave], equal[kSelThreads / kWave];
  const int b = blockIdx.x / c.hkv, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int capacity = c.capacity(), n = clamp_len(lens[b], capacity);
  const float* w = weights + (long long)blockIdx.x * capacity;
  kept += (long long)blockIdx.x * budget;
  new_weights += (long long)blockIdx.x * new_capacity;
  const int m = n < budget ? n : budget;
  if (blockIdx.x % c.hkv == 0 && tid == 0) new_lens[b] = m;

  const bool all = n <= budget;
  const int old = all ? 0 : n - recent;  // tokens that compete
  uint32_t last = 0;                     // the rank of the last one kept
  int take = all ? 0 : budget - recent;
  const int wanted = take;
  if (wanted > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int t = tid; t < old; t += kSelThreads) {
        const uint32_t r = rank_of(w[t]);
        if (shift == 24 || (r ^ last) >> (shift + 8) == 0) atomicAdd(&hist[r >> shift & 255], 1);
      }
      __syncthreads();
      if (tid == 0) {
        int left = take, d = 255;
        for (; d > 0 && hist[d] < left; --d) left -= hist[d];
        found[0] = d;
        found[1] = left;
      }
      __syncthreads();
      last |= (uint32_t)found[0] << shift;
      take = found[1];
      __syncthreads();
    }
  }
  // `take` tokens of rank `last` are kept, the first ones, and every token above
  int base = 0, ties = 0;
  for (int t0 = 0; t0 < n; t0 += kSelThreads) {
    const int t = t0 + tid;
    const float x = t < n ? w[t] : 0.f;
    const uint32_t r = rank_of(x);
    const bool in = t < n, must = in && (t >= old || (wanted > 0 && r > last));
    const bool tie = in && t < old && wanted > 0 && r == last;
    const uint64_t mm = __ballot(must), mt = __ballot(tie);
    if (lane == 0) {
      above[wave] = __popcll(mm);
      equal[wave] = __popcll(mt);
    }
    __syncthreads();
    const uint64_t before = ((uint64_t)1 << lane) - 1;
    int must_before = __popcll(mm & before), tie_before = ties + __popcll(mt & before);
    int must_all = 0, tie_all = 0;
    for (int i = 0; i < kSelThreads / kWave; ++i) {
      if (i < wave) {
        must_before += above[i];
        tie_before += equal[i];
      }
      must_all += above[i];
      tie_all += equal[i];
    }
    // kept ties before this one: the first `take` of the row
    const int ties_kept = min(tie_before, take) - min(ties, take);
    if (must || (tie && tie_before < take)) {
      const int at = base + must_before + ties_kept;
      kept[at] = t;
      new_weights[at] = x;
    }
    base += must_all + min(ties + tie_all, take) - min(ties, take);
    ties += tie_all;
    __syncthreads();
  }
  for (int i = m + tid; i < budget; i += kSelThreads) kept[i] = -1;
  for (int i = m + tid; i < new_capacity; i += kSelThreads) new_weights[i] = 0.f;
}

// 16 lanes a token for bf16, 8 for e4m3: a 16-byte piece of its key and value each.
template <bool E4M3>
__global__ __launch_bounds__(kMoveThreads) void evict_move(CacheParams c,
                                                           const int32_t* __restrict__ lens,
                                                           int budget,
                                                           const int32_t* __restrict__ new_table,
                                                           int new_pages,
                                                           const int32_t* __restrict__ kept) {
  constexpr int kBytes = E4M3 ? kHeadDim : 2 * kHeadDim, kPer = kBytes / 16;
  constexpr int kRows = kMoveThreads / kPer;
  const int chunks = (budget + kRows - 1) / kRows;
  const int row = blockIdx.x / chunks, b = row / c.hkv, h = row % c.hkv;
  const int i = blockIdx.x % chunks * kRows + threadIdx.x / kPer, piece = threadIdx.x % kPer;
  if (i >= budget || i >= clamp_len(lens[b], c.capacity())) return;
  const int t = kept[(long long)row * budget + i];
  const int slot = (1 << c.shift) - 1;
  const long long from = page_row(c.table[(long long)b * c.table_pages + (t >> c.shift)], c.pages,
                                  c.hkv, h, c.shift, t & slot);
  const long long to = page_row(new_table[(long long)b * new_pages + (i >> c.shift)], c.pages,
                                c.hkv, h, c.shift, i & slot);
  if (from < 0 || to < 0) return;
  char *k = (char*)c.k + piece * 16, *v = (char*)c.v + piece * 16;
  const u32x4 x = *(const u32x4*)(k + from * kBytes), y = *(const u32x4*)(v + from * kBytes);
  *(u32x4*)(k + to * kBytes) = x;
  *(u32x4*)(v + to * kBytes) = y;
  if (E4M3 && piece == 0) {
    c.k_scale[to] = c.k_scale[from];
    c.v_scale[to] = c.v_scale[from];
  }
}

}  // namespace

hipError_t launch_evict(const CacheParams& c, bool e4m3, int batch, const int32_t* lens,
                        const float* weights, int budget, int recent, const int32_t* new_table,
                        int new_pages, int32_t* kept, int32_t* new_lens, float* new_weights,
                        hipStream_t st) {
  const int rows = batch * c.hkv;
  hipLaunchKernelGGL(evict_select, dim3(rows), dim3(kSelThreads), 0, st, c, lens, weights, budget,
                     recent, new_pages << c.shift, kept, new_lens, new_weights);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int per = kMoveThreads / (e4m3 ? 8 : 16), chunks = (budget + per - 1) / per;
  auto* kernel = e4m3 ? evict_move<true> : evict_move<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)rows * chunks)), dim3(kMoveThreads), 0, st,
                     c, lens, budget, new_table, new_pages, kept);
  return hipGetLastError();
}
