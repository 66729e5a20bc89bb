// Eviction from the paged cache by accumulated attention weight.
//
// evict_select: one workgroup per (sequence, key head) finds the weight of the
// last token kept and writes the kept tokens in order. A wave has a run of the
// tokens. The weight is found over its order-preserving integer: a histogram of
// the upper 11 bits; the tokens of the digit that holds the last place, collected
// in LDS (in memory again where they are too many); two histograms of theirs for
// the other 21 bits. The places of a wave's tokens follow from the counts of the
// waves before it, so the last pass needs no barrier. evict_move copies the
// tokens' vectors to the new pages.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kStep = 4 * kWave;      // tokens of a wave's step, four a lane
constexpr int kBins = 2048;           // of a histogram
constexpr int kCopies = 4;            // of it: one for the waves of a SIMD
constexpr int kListed = 1536;         // tokens that a wave can collect
constexpr int kHeld = 4;              // steps whose weights stay in registers
constexpr int kMoveThreads = 256;

// Integer with the order of the weights: NaN lowest, -0 equal to 0.
__device__ __forceinline__ uint32_t rank_of(float w) {
  if (w != w) return 0;
  const uint32_t u = __builtin_bit_cast(uint32_t, w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One more in bin d for every lane with `in`. Lanes with the first one's bin are
// counted together: weights are often alike (zeros), and atomics on one address
// take a turn each.
__device__ __forceinline__ void count(int* hist, int d, bool in) {
  const uint64_t all = __ballot(in);
  if (!all) return;
  const int lane = threadIdx.x % kWave, first = __ffsll((unsigned long long)all) - 1;
  const int common = __builtin_amdgcn_readlane(d, first);
  const uint64_t same = __ballot(in && d == common);
  if (lane == first) atomicAdd(&hist[common], __popcll(same));
  if (in && d != common) atomicAdd(&hist[d], 1);
}

struct SelectShared {
  int hist[kCopies][kBins];
  uint32_t list[kSelWaves][kListed];
  int listed[kSelWaves], above[kSelWaves], equal[kSelWaves], sums[kSelWaves];
  int digit, left;
};

__device__ __forceinline__ void clear(SelectShared& s) {
  for (int i = threadIdx.x; i < kCopies * kBins; i += kSelThreads) (&s.hist[0][0])[i] = 0;
  __syncthreads();
}

// The bin of the `take`-th largest counted, and the place in it that is wanted.
__device__ __forceinline__ void find(SelectShared& s, int take) {
  static_assert(kBins == 2 * kSelThreads, "two bins a thread");
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  __syncthreads();
  const int high = kBins - 1 - 2 * tid;  // this thread's bins: high, high - 1
  int n[2] = {0, 0};
  for (int c = 0; c < kCopies; ++c) {
    n[0] += s.hist[c][high];
    n[1] += s.hist[c][high - 1];
  }
  int up_to = n[0] + n[1];
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int x = __shfl_up(up_to, off);
    if (lane >= off) up_to += x;
  }
  if (lane == kWave - 1) s.sums[wave] = up_to;
  __syncthreads();
  for (int w = 0; w < wave; ++w) up_to += s.sums[w];
  const int before = up_to - n[0] - n[1];
  if (before < take && take <= up_to) {
    const bool second = take > before + n[0];
    s.digit = high - second;
    s.left = take - before - (second ? n[0] : 0);
  }
  __syncthreads();
}

// HELD: rows of at most kSelWaves * kHeld * kStep tokens, read once.
template <bool HELD>
__global__ __launch_bounds__(kSelThreads) void evict_select(
    CacheParams c, const int32_t* __restrict__ lens, const float* __restrict__ weights, int budget,
    int recent, int new_capacity, int32_t* __restrict__ kept, int32_t* __restrict__ new_lens,
    float* __restrict__ new_weights) {
  __shared__ SelectShared s;
  const int b = blockIdx.x / c.hkv, tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int capacity = c.capacity(), n = clamp_len(lens[b], capacity);
  const float* w = weights + (long long)blockIdx.x * capacity;
  kept += (long long)blockIdx.x * budget;
  new_weights += (long long)blockIdx.x * new_capacity;
  const int m = n < budget ? n : budget;
  if (blockIdx.x % c.hkv == 0 && tid == 0) new_lens[b] = m;
  for (int i = m + tid; i < budget; i += kSelThreads) kept[i] = -1;
  for (int i = m + tid; i < new_capacity; i += kSelThreads) new_weights[i] = 0.f;
  if (n <= budget) {
    for (int i = tid; i < n; i += kSelThreads) {
      kept[i] = i;
      new_weights[i] = w[i];
    }
    return;
  }

  const int old = n - recent, wanted = budget - recent;  // tokens that compete, and places
  const int run = HELD ? kHeld * kStep : (n + kSelWaves * kStep - 1) / (kSelWaves * kStep) * kStep;
  const int t0 = wave * run, t1 = min(t0 + run, n);
  f32x4 held[kHeld];
  // f(token, weight of it and the next three) for the lane's tokens of each step;
  // rows begin at multiples of 16 weights, so the last one's four can be read
  auto each = [&](auto f, bool first = false) {
    if (HELD) {
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int t = t0 + i * kStep + 4 * lane;
        if (first && t < t1) held[i] = *(const f32x4*)(w + t);
        if (t0 + i * kStep < t1) f(t, held[i]);
      }
      return;
    }
    constexpr int kAhead = 4;
    int t = t0 + 4 * lane;
    for (int base = t0; base < t1; base += kAhead * kStep) {
      f32x4 x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (t + i * kStep < t1) x[i] = *(const f32x4*)(w + t + i * kStep);
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (base + i * kStep < t1) f(t + i * kStep, x[i]);
      t += kAhead * kStep;
    }
  };

  int* hist = s.hist[wave % kCopies];
  uint32_t last = 0;  // the rank of the last token kept, and how many of that rank are
  int take = wanted, musts = 0, equals = 0;
  if (wanted > 0) {
    clear(s);
    each([&](int t, f32x4 x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) count(hist, rank_of(x[e]) >> 21, t + e < old);
    }, true);
    find(s, take);
    last = (uint32_t)s.digit << 21;
    take = s.left;
    // the tokens above that digit are kept; those in it are collected
    int listed = 0;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    each([&](int t, f32x4 x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t r = rank_of(x[e]);
        const bool in = t + e < old;
        musts += __popcll(__ballot(in && r >> 21 > last >> 21));
        const bool mine = in && r >> 21 == last >> 21;
        const uint64_t who = __ballot(mine);
        const int at = listed + __popcll(who & below);
        if (mine && at < kListed) s.list[wave][at] = r;
        listed += __popcll(who);
      }
    });
    if (lane == 0) s.listed[wave] = listed;
    __syncthreads();
    bool fits = true;
    for (int i = 0; i < kSelWaves; ++i) fits = fits && s.listed[i] <= kListed;
    for (int shift = 10; shift >= 0; shift -= 10) {
      const int bits = shift ? 11 : 10;
      clear(s);
      if (fits) {
        for (int i = lane; i - lane < listed; i += kWave) {
          const uint32_t r = i < listed ? s.list[wave][i] : 0;
          count(hist, r >> shift & ((1 << bits) - 1),
                i < listed && (r ^ last) >> (shift + bits) == 0);
        }
      } else {
        each([&](int t, f32x4 x) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t r = rank_of(x[e]);
            count(hist, r >> shift & ((1 << bits) - 1),
                  t + e < old && (r ^ last) >> (shift + bits) == 0);
          }
        });
      }
      find(s, take);
      last |= (uint32_t)s.digit << shift;
      take = s.left;
    }
    if (fits) {
      for (int i = lane; i - lane < listed; i += kWave) {
        const uint32_t r = i < listed ? s.list[wave][i] : 0;
        musts += __popcll(__ballot(i < listed && r > last));
        equals += __popcll(__ballot(i < listed && r == last));
      }
    } else {
      musts = 0;
      each([&](int t, f32x4 x) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t r = rank_of(x[e]);
          musts += __popcll(__ballot(t + e < old && r > last));
          equals += __popcll(__ballot(t + e < old && r == last));
        }
      });
    }
  }
  musts += max(0, t1 - max(t0, old));
  if (lane == 0) {
    s.above[wave] = musts;
    s.equal[wave] = equals;
  }
  __syncthreads();
  // places taken and equal tokens met before this wave's run; of the equal ones
  // the first `take` of the row are kept
  int base = 0, ties = 0;
  for (int i = 0; i < wave; ++i) {
    base += s.above[i];
    ties += s.equal[i];
  }
  const bool first_read = HELD && wanted == 0;
  each([&](int t, f32x4 x) {
    bool must[4], tie[4];
    uint32_t must_before = 0, tie_before = 0;  // in the lanes below
    int must_all = 0, tie_all = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t r = rank_of(x[e]);
      const bool competes = wanted > 0 && t + e < old;
      must[e] = (t + e >= old && t + e < n) || (competes && r > last);
      tie[e] = competes && r == last;
      const uint64_t a = __ballot(must[e]), q = __ballot(tie[e]);
      must_before = __builtin_amdgcn_mbcnt_hi(a >> 32,
                                              __builtin_amdgcn_mbcnt_lo((uint32_t)a, must_before));
      tie_before = __builtin_amdgcn_mbcnt_hi(q >> 32,
                                             __builtin_amdgcn_mbcnt_lo((uint32_t)q, tie_before));
      must_all += __popcll(a);
      tie_all += __popcll(q);
    }
    int at = base + (int)must_before, tied = ties + (int)tie_before;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (must[e] || (tie[e] && tied < take)) {
        const int place = at + min(tied, take);
        kept[place] = t + e;
        new_weights[place] = x[e];
      }
      at += must[e];
      tied += tie[e];
    }
    base += must_all;
    ties += tie_all;
  }, first_read);
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
  auto* select = c.capacity() <= kSelWaves * kHeld * kStep ? evict_select<true>
                                                           : evict_select<false>;
  hipLaunchKernelGGL(select, dim3(rows), dim3(kSelThreads), 0, st, c, lens, weights, budget,
                     recent, new_pages << c.shift, kept, new_lens, new_weights);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int per = kMoveThreads / (e4m3 ? 8 : 16), chunks = (budget + per - 1) / per;
  auto* kernel = e4m3 ? evict_move<true> : evict_move<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)rows * chunks)), dim3(kMoveThreads), 0, st,
                     c, lens, budget, new_table, new_pages, kept);
  return hipGetLastError();
}
