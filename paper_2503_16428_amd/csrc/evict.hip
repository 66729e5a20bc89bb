// Eviction from the paged cache by accumulated attention weight.
//
// The weight of the last token kept is found over its order-preserving integer,
// 11, 11 and 10 bits at a time, by one workgroup per 8192 tokens of a row
// (sequence, key head), in three launches:
//   evict_count    histogram of the upper 11 bits of a chunk's weights;
//   evict_collect  sums the row's histograms, finds the digit of the last place,
//                  lists the chunk's tokens that have it and counts their next
//                  11 bits;
//   evict_emit     finds that digit, and the last 10 bits from the row's lists (if
//                  not all of the digit's tokens are kept);
//                  the places of a chunk's tokens follow from the counts of the
//                  chunks before it, and it writes its kept tokens.
// Rows of at most two chunks are one workgroup's, in one launch (evict_select).
// evict_move copies the tokens' vectors to the new pages.
//
// The copies are bound by HBM: 131 MB of 4 sequences of 16,000 tokens, 8 heads, cut
// to 4096, 25 us (5.2 TB/s). The selection is a chain of loads, LDS sums and
// barriers: one workgroup a row of 16,000 tokens 16.5 us, three launches for 128K
// 5.0 + 8.5 + 11.4.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / kWave;
constexpr int kStep = 4 * kWave;                 // tokens of a wave's step, four a lane
constexpr int kSteps = 2;                        // of a wave, where a row has several workgroups
// Tokens of a workgroup.
constexpr int chunk_of(int steps) { return kSelWaves * steps * kStep; }
constexpr int kChunk = chunk_of(kSteps);
constexpr int kBins = 2048;                      // of a histogram
constexpr int kCopies = 2;                       // of it in LDS
constexpr int kMoveThreads = 256;

// What the launches leave for the next, per chunk and per row.
struct ChunkCounts {
  int above, listed;  // tokens above the first digit, tokens that have it
};
struct RowDigit {
  int digit, left;  // the first digit, and the place within it that is wanted
};
struct EvictParams {
  CacheParams c;
  const int32_t* lens;
  const float* weights;
  int budget, recent, chunks, new_capacity;
  int32_t *kept, *new_lens;
  float* new_weights;
  int* hist;            // [rows][chunks][2][kBins]
  uint32_t* list;       // [rows][chunks][kChunk]
  ChunkCounts* counts;  // [rows][chunks]
  RowDigit* digits;     // [rows]
};

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
  int above[kSelWaves], equal[kSelWaves], sums[kSelWaves];
  int digit, left, size, listed;
};

// Sum of the first n of the waves' numbers in LDS, in every lane.
__device__ __forceinline__ int sum_of_first(const int* a, int n) {
  const int lane = threadIdx.x % kSelWaves;
  int x = lane < n ? a[lane] : 0;
#pragma unroll
  for (int off = 1; off < kSelWaves; off <<= 1) x += __shfl_xor(x, off);
  return x;
}

__device__ __forceinline__ void clear(SelectShared& s) {
  for (int i = threadIdx.x; i < kCopies * kBins / 4; i += kSelThreads)
    ((int4*)&s.hist[0][0])[i] = int4{0, 0, 0, 0};
  __syncthreads();
}

// The chunk's histogram to memory.
__device__ __forceinline__ void store(const SelectShared& s, int* to) {
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kSelThreads) {
    int n = 0;
    for (int c = 0; c < kCopies; ++c) n += s.hist[c][i];
    to[i] = n;
  }
}

// The bin of the `take`-th largest of `parts` histograms that lie `stride` apart,
// how many it has, and the place in it that is wanted.
__device__ __forceinline__ void find(SelectShared& s, const int* hist, int parts, int stride,
                                     int take) {
  static_assert(kBins == 2 * kSelThreads, "two bins a thread");
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int low = kBins - 2 - 2 * tid;  // this thread's bins: low + 1, low
  int n0 = 0, n1 = 0;
#pragma unroll 16
  for (int i = 0; i < parts; ++i) {
    const int2 x = *(const int2*)(hist + (size_t)i * stride + low);
    n0 += x.y;
    n1 += x.x;
  }
  int up_to = n0 + n1;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const int x = __shfl_up(up_to, off);
    if (lane >= off) up_to += x;
  }
  if (lane == kWave - 1) s.sums[wave] = up_to;
  __syncthreads();
  up_to += sum_of_first(s.sums, wave);
  const int before = up_to - n0 - n1;
  if (before < take && take <= up_to) {
    const bool second = take > before + n0;
    s.digit = low + !second;
    s.left = take - before - (second ? n0 : 0);
    s.size = second ? n1 : n0;
  }
  __syncthreads();
}

// Whether all of the bin that was found are kept, whatever their other bits: the
// rank `last` of a bin's lowest is then made one less, of which none are (`take`).
// It is not 0: below these there are tokens that are not kept. It saves passes where
// the upper bits tell the weights apart: 2000 tokens of 8 heads 15.2 -> 13.4 us, 4 x
// 16,000 41.3 -> 40.6.
__device__ __forceinline__ bool all_kept(const SelectShared& s, uint32_t& last, int& take) {
  if (take != s.size) return false;
  --last;
  take = 0;
  return true;
}

// A workgroup's place: its row's length and tokens, and its lanes' weights.
template <int STEPS = kSteps>
struct Chunk {
  int row, index, n, old, wanted, t0;  // t0: the lane's first token
  const float* w;
  f32x4 x[STEPS];
  __device__ Chunk(const EvictParams& p) {
    row = blockIdx.x / p.chunks;
    index = blockIdx.x % p.chunks;
    n = clamp_len(p.lens[row / p.c.hkv], p.c.capacity());
    old = n - p.recent;             // tokens that compete,
    wanted = p.budget - p.recent;   // for so many places
    w = p.weights + (long long)row * p.c.capacity();
    t0 = index * kChunk + (int)threadIdx.x / kWave * (STEPS * kStep) +
         4 * ((int)threadIdx.x % kWave);
  }
  // rows begin at multiples of 16 weights and hold multiples of 16
  __device__ void load() {
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
      if (t0 + i * kStep < n) x[i] = *(const f32x4*)(w + t0 + i * kStep);
  }
  template <class F>
  __device__ void each(F f) const {
#pragma unroll
    for (int i = 0; i < STEPS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) f(t0 + i * kStep + e, x[i][e]);
  }
};

// What every chunk writes of the outputs whatever is kept: the ends behind the kept
// tokens and, where the whole row is kept, the row. Whether it is not.
template <int STEPS>
__device__ __forceinline__ bool competes(const EvictParams& p, const Chunk<STEPS>& k) {
  const int tid = threadIdx.x, m = min(k.n, p.budget);
  const int first = k.index * kSelThreads + tid, all = p.chunks * kSelThreads;
  int32_t* kept = p.kept + (long long)k.row * p.budget;
  float* new_weights = p.new_weights + (long long)k.row * p.new_capacity;
  if (k.row % p.c.hkv == 0 && first == 0) p.new_lens[k.row / p.c.hkv] = m;
  for (int i = m + first; i < p.budget; i += all) kept[i] = -1;
  for (int i = m + first; i < p.new_capacity; i += all) new_weights[i] = 0.f;
  if (k.n <= p.budget) {  // all of them
    for (int i = first; i < k.n; i += all) {
      kept[i] = i;
      new_weights[i] = k.w[i];
    }
    return false;
  }
  return true;
}

// Writes a chunk's kept tokens, wave after wave: those that do not compete, those
// above rank `last`, and of that rank the row's first `take`; `base` are kept and
// `ties` of that rank in the chunks before.
template <int STEPS>
__device__ __forceinline__ void write_kept(const EvictParams& p, const Chunk<STEPS>& k,
                                           SelectShared& s, uint32_t last, int take, int base,
                                           int ties) {
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const bool some = k.wanted > 0;
  base += max(0, k.index * kChunk - max(0, k.old));
  // this chunk's, wave after wave
  auto must = [&](int t, uint32_t r) {
    return (t >= k.old && t < k.n) || (some && t < k.old && r > last);
  };
  auto tie = [&](int t, uint32_t r) { return some && t < k.old && r == last; };
  int musts = 0, equals = 0;
  k.each([&](int t, float x) {
    const uint32_t r = rank_of(x);
    musts += __popcll(__ballot(must(t, r)));
    equals += __popcll(__ballot(tie(t, r)));
  });
  if (lane == 0) {
    s.above[wave] = musts;
    s.equal[wave] = equals;
  }
  __syncthreads();
  base += sum_of_first(s.above, wave);
  ties += sum_of_first(s.equal, wave);
  int32_t* kept = p.kept + (long long)k.row * p.budget;
  float* new_weights = p.new_weights + (long long)k.row * p.new_capacity;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    int at = base, tied = ties;  // and those of the lanes below and of this lane
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = k.t0 + i * kStep + e;
      r[e] = rank_of(k.x[i][e]);
      const uint64_t a = __ballot(must(t, r[e])), q = __ballot(tie(t, r[e]));
      at += __popcll(a & below);
      tied += __popcll(q & below);
      base += __popcll(a);
      ties += __popcll(q);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int t = k.t0 + i * kStep + e;
      const bool m = must(t, r[e]), q = tie(t, r[e]);
      if (m || (q && tied < take)) {  // of the equal ones the row's first `take`
        const int place = at + min(tied, take);
        kept[place] = t;
        new_weights[place] = k.x[i][e];
      }
      at += m;
      tied += q;
    }
  }
}

// All of it for rows of one workgroup, whose weights stay in registers.
template <int STEPS>
__global__ __launch_bounds__(kSelThreads) void evict_select(EvictParams p) {
  __shared__ SelectShared s;
  Chunk<STEPS> k(p);
  if (!competes(p, k)) return;
  k.load();
  uint32_t last = 0;
  int take = k.wanted;
  if (take > 0) {
    int* hist = s.hist[threadIdx.x / kWave % kCopies];
    for (int shift = 21; shift >= 0; shift -= shift == 21 ? 11 : 10) {
      const int bits = shift ? 11 : 10;
      clear(s);
      k.each([&](int t, float x) {
        const uint32_t r = rank_of(x);
        const bool in = shift == 21 || (r ^ last) >> (shift + bits) == 0;
        count(hist, r >> shift & ((1 << bits) - 1), in && t < k.old);
      });
      __syncthreads();
      find(s, s.hist[0], kCopies, kBins, take);
      last |= (uint32_t)s.digit << shift;
      take = s.left;
      if (all_kept(s, last, take)) break;
    }
  }
  write_kept(p, k, s, last, take, 0, 0);
}

__global__ __launch_bounds__(kSelThreads) void evict_count(EvictParams p) {
  __shared__ SelectShared s;
  Chunk<> k(p);
  if (!competes(p, k) || k.wanted == 0 || k.index * kChunk >= k.n) return;
  k.load();
  clear(s);
  int* hist = s.hist[threadIdx.x / kWave % kCopies];
  k.each([&](int t, float x) { count(hist, rank_of(x) >> 21, t < k.old); });
  store(s, p.hist + (size_t)blockIdx.x * (2 * kBins));
}

__global__ __launch_bounds__(kSelThreads) void evict_collect(EvictParams p) {
  __shared__ SelectShared s;
  Chunk<> k(p);
  if (k.n <= p.budget || k.wanted == 0 || k.index * kChunk >= k.n) return;
  const int tid = threadIdx.x, lane = tid % kWave, chunks = (k.n + kChunk - 1) / kChunk;
  k.load();
  if (tid == 0) s.listed = 0;
  clear(s);
  find(s, p.hist + (size_t)k.row * p.chunks * (2 * kBins), chunks, 2 * kBins, k.wanted);
  const uint32_t digit = s.digit;
  uint32_t* list = p.list + (size_t)blockIdx.x * kChunk;
  int* hist = s.hist[tid / kWave % kCopies];
  int above = 0;
  k.each([&](int t, float x) {
    const uint32_t r = rank_of(x);
    above += __popcll(__ballot(t < k.old && r >> 21 > digit));
    const bool in = t < k.old && r >> 21 == digit;
    const uint64_t who = __ballot(in);
    if (!who) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&s.listed, __popcll(who));
    at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & (((uint64_t)1 << lane) - 1));
    if (in) list[at] = r;
    count(hist, r >> 10 & (kBins - 1), in);
  });
  if (lane == 0) s.above[tid / kWave] = above;
  store(s, p.hist + (size_t)blockIdx.x * (2 * kBins) + kBins);
  if (tid != 0) return;
  above = 0;
  for (int i = 0; i < kSelWaves; ++i) above += s.above[i];
  p.counts[blockIdx.x] = ChunkCounts{above, s.listed};
  if (k.index == 0) p.digits[k.row] = RowDigit{(int)digit, s.left};
}

__global__ __launch_bounds__(kSelThreads) void evict_emit(EvictParams p) {
  __shared__ SelectShared s;
  Chunk<> k(p);
  if (k.n <= p.budget || k.index * kChunk >= k.n) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int chunks = (k.n + kChunk - 1) / kChunk;
  const int first = k.row * p.chunks;  // the row's chunks
  const bool some = k.wanted > 0;
  k.load();
  uint32_t last = 0;  // the rank of the last token kept, and how many of that rank are
  int take = 0, base = 0, ties = 0;  // kept, and of that rank, in the chunks before
  if (some) {
    clear(s);
    const RowDigit d = p.digits[k.row];
    find(s, p.hist + (size_t)first * (2 * kBins) + kBins, chunks, 2 * kBins, d.left);
    last = (uint32_t)d.digit << 21 | (uint32_t)s.digit << 10;
    take = s.left;
    // f(whether, rank) for the tokens listed in the first `upto` chunks, whole
    // waves at a time, a wave a chunk
    auto each_listed = [&](int upto, auto f) {
      constexpr int kAhead = 4;
      for (int i = wave; i < upto; i += kSelWaves) {
        const int listed = __builtin_amdgcn_readfirstlane(p.counts[first + i].listed);
        const uint32_t* list = p.list + (size_t)(first + i) * kChunk;
        for (int at = lane; at - lane < listed; at += kAhead * kWave) {
          uint32_t r[kAhead];
#pragma unroll
          for (int x = 0; x < kAhead; ++x)
            r[x] = at + x * kWave < listed ? list[at + x * kWave] : 0;
#pragma unroll
          for (int x = 0; x < kAhead; ++x) f(at + x * kWave < listed, r[x]);
        }
      }
    };
    if (!all_kept(s, last, take)) {
      each_listed(chunks, [&](bool in, uint32_t r) {
        count(s.hist[wave % kCopies], r & 1023, in && (r ^ last) >> 10 == 0);
      });
      __syncthreads();
      find(s, s.hist[0], kCopies, kBins, take);
      last |= s.digit;
      take = s.left;
    }
    int above = 0, equal = 0;
    each_listed(k.index, [&](bool in, uint32_t r) {
      above += __popcll(__ballot(in && r > last));
      equal += __popcll(__ballot(in && r == last));
    });
    int before = 0;
    for (int i = tid; i < k.index; i += kSelThreads) before += p.counts[first + i].above;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) before += __shfl_xor(before, off);
    if (lane == 0) {
      s.above[wave] = above + before;
      s.equal[wave] = equal;
    }
    __syncthreads();
    base = sum_of_first(s.above, kSelWaves);
    ties = sum_of_first(s.equal, kSelWaves);
    __syncthreads();
  }
  write_kept(p, k, s, last, take, base, ties);
}

// 16 lanes a token for bf16, 8 for e4m3: a 16-byte piece of its key and value
// each. Loads that are not to stay in the caches and stores that may: 10 % faster
// than both one way or the other way round (four tokens a thread: 5 % slower).
template <bool E4M3>
__global__ __launch_bounds__(kMoveThreads) void evict_move(CacheParams c,
                                                           const int32_t* __restrict__ lens,
                                                           int budget, int moves,
                                                           const int32_t* __restrict__ new_table,
                                                           int new_pages,
                                                           const int32_t* __restrict__ kept) {
  constexpr int kBytes = E4M3 ? kHeadDim : 2 * kHeadDim, kPer = kBytes / 16;
  const int row = blockIdx.x / moves, b = row / c.hkv, h = row % c.hkv;
  const int i = blockIdx.x % moves * (kMoveThreads / kPer) + threadIdx.x / kPer;
  const int piece = threadIdx.x % kPer, slot = (1 << c.shift) - 1;
  if (i >= min(budget, clamp_len(lens[b], c.capacity()))) return;
  const int t = kept[(long long)row * budget + i];
  const long long from = page_row(c.table[(long long)b * c.table_pages + (t >> c.shift)], c.pages,
                                  c.hkv, h, c.shift, t & slot);
  const long long to = page_row(new_table[(long long)b * new_pages + (i >> c.shift)], c.pages,
                                c.hkv, h, c.shift, i & slot);
  if (from < 0 || to < 0) return;
  char *k = (char*)c.k + piece * 16, *v = (char*)c.v + piece * 16;
  const u32x4 key = __builtin_nontemporal_load((const u32x4*)(k + from * kBytes));
  const u32x4 value = __builtin_nontemporal_load((const u32x4*)(v + from * kBytes));
  *(u32x4*)(k + to * kBytes) = key;
  *(u32x4*)(v + to * kBytes) = value;
  if (E4M3 && piece == 0) {
    c.k_scale[to] = c.k_scale[from];
    c.v_scale[to] = c.v_scale[from];
  }
}

int chunks_of(const CacheParams& c) { return (c.capacity() + kChunk - 1) / kChunk; }

struct Scratch {
  size_t hist, list, counts, digits, bytes;
  Scratch(const CacheParams& c, int batch) {
    const size_t rows = (size_t)batch * c.hkv, chunks = rows * chunks_of(c);
    hist = 0;
    list = hist + chunks * 2 * kBins * 4;
    counts = list + chunks * kChunk * 4;
    digits = align256(counts + chunks * sizeof(ChunkCounts));
    bytes = align256(digits + rows * sizeof(RowDigit));
  }
};

}  // namespace

// Rows that one workgroup has.
static bool single_row(const CacheParams& c) { return c.capacity() <= chunk_of(2 * kSteps); }

size_t evict_scratch_bytes(const CacheParams& c, int batch) {
  return single_row(c) ? 0 : Scratch(c, batch).bytes;
}

hipError_t launch_evict(const CacheParams& c, bool e4m3, int batch, const int32_t* lens,
                        const float* weights, int budget, int recent, const int32_t* new_table,
                        int new_pages, int32_t* kept, int32_t* new_lens, float* new_weights,
                        void* scratch, hipStream_t st) {
  const int rows = batch * c.hkv;
  const bool single = single_row(c);
  const int chunks = single ? 1 : chunks_of(c);
  const Scratch s(c, batch);
  char* at = (char*)scratch;
  const EvictParams p{c,      lens, weights,  budget,      recent,
                        chunks, new_pages << c.shift,        kept, new_lens, new_weights,
                        (int*)(at + s.hist), (uint32_t*)(at + s.list),
                        (ChunkCounts*)(at + s.counts), (RowDigit*)(at + s.digits)};
  // one launch where one workgroup has the row (before passes could be saved: 2000
  // tokens of 8 heads 22.6 -> 15.0 us, 4 x 8000 40.0 -> 30.1, 4 x 16,000 45.1 -> 41.8)
  void (*const one)(EvictParams) = c.capacity() <= kChunk ? evict_select<kSteps>
                                                          : evict_select<2 * kSteps>;
  void (*const three[])(EvictParams) = {evict_count, evict_collect, evict_emit};
  hipError_t e;
  for (int i = 0; i < (single ? 1 : 3); ++i) {
    hipLaunchKernelGGL(single ? one : three[i], dim3((unsigned)(rows * chunks)),
                       dim3(kSelThreads), 0, st, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  const int per = kMoveThreads / (e4m3 ? 8 : 16), moves = (budget + per - 1) / per;
  auto* kernel = e4m3 ? evict_move<true> : evict_move<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)rows * moves)), dim3(kMoveThreads), 0, st,
                     c, lens, budget, moves, new_table, new_pages, kept);
  return hipGetLastError();
}
