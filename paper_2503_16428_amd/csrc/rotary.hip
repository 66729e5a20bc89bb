// Rotary positions, and the append of keys (rotated on the way) and values to
// the paged cache.
//
// Eight lanes share a vector of 128: lane j holds elements 8j .. 8j+7 and
// 64+8j .. 64+8j+7 (two 16-byte loads), which are eight whole pairs in either
// pairing. A wave has eight tokens, the waves of a workgroup go over the heads in
// turn (two or one of them where there are no more heads, the others then have
// other tokens): neighbouring heads of a token, which a projection leaves side by
// side, are read together, and eight tokens of a head written together. A thread
// computes its token's eight angles once, while its first vector is on the way, and
// loads the next head's before it turns this one.
//
// Bound by HBM, every vector read and written once: 32K tokens of 32 heads 102 us
// (537 MB, 5.3 TB/s; a 1 GB copy 5.15), 115,200 of 24 heads 249 us (1.42 GB, 5.7
// TB/s). Append of 60,000 tokens of 8 heads in bf16 90 us, rotated or not (5.5 TB/s),
// in e4m3 64 (5.8); one token of 64 sequences 4 us, a chain of loads. Keys that go to
// e4m3 rotated are bound by their fp64 sines the more, the fewer heads share them: 8
// heads 79 us (4.7 TB/s), two heads 3.0 TB/s, one head of 200,000 tokens 61 us (2.5).
#include <type_traits>

#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 8;                   // lanes of a vector
constexpr int kItems = kWave / kLanes;      // tokens of a wave
constexpr int kWaves = kThreads / kWave;

// A launch: how many waves share out the heads, and how many heads a workgroup has.
struct Split {
  int waves, heads;
};
// A thread's token, and its first head and the one behind its last.
struct Place {
  long long item;
  int h, h1;
  __device__ Place(Split s, int heads) {
    const int wave = threadIdx.x / kWave;
    item = (long long)blockIdx.x * (kItems * (kWaves / s.waves)) + wave / s.waves * kItems +
           threadIdx.x % kWave / kLanes;
    h = blockIdx.y * s.heads + wave % s.waves;
    h1 = min((int)(blockIdx.y + 1) * s.heads, heads);
  }
};

__device__ __forceinline__ float bf_lo(uint32_t w) {
  return __builtin_bit_cast(float, w << 16);
}
__device__ __forceinline__ float bf_hi(uint32_t w) {
  return __builtin_bit_cast(float, w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  bf16x2 r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Sixteen values of a lane: 0 .. 7 its first chunk, 8 .. 15 its second.
struct Vec {
  float f[16];
};

__device__ __forceinline__ Vec unpack(u32x4 lo, u32x4 hi) {
  Vec v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v.f[2 * i] = bf_lo(lo[i]);
    v.f[2 * i + 1] = bf_hi(lo[i]);
    v.f[8 + 2 * i] = bf_lo(hi[i]);
    v.f[8 + 2 * i + 1] = bf_hi(hi[i]);
  }
  return v;
}

// The places in Vec of a lane's pair e, and its index among the head's 64.
template <bool IL>
__device__ __forceinline__ constexpr int first_of(int e) {
  return IL ? 2 * e : e;
}
template <bool IL>
__device__ __forceinline__ constexpr int second_of(int e) {
  return IL ? 2 * e + 1 : e + 8;
}
template <bool IL>
__device__ __forceinline__ int pair_of(int j, int e) {
  return IL ? (e < 4 ? 4 * j + e : 32 + 4 * j + e - 4) : 8 * j + e;
}

template <class T>
struct Angles {
  T c[8], s[8];
};

// Sine and cosine of a part of a turn, |t| <= 1/2: of the quarter turn next to it
// and the rest, |x| <= pi / 4, by their series to x^13 and x^12 (off by x^14 / 14!,
// at most 4e-13).
__device__ __forceinline__ void sin_cos(double t, double* s, double* c) {
  const double q = __builtin_rint(4.0 * t);
  const double x = 6.283185307179586476925 * (t - 0.25 * q), y = x * x;
  const double sine =
      x + x * y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 +
          y * (-1.0 / 39916800 + y * (1.0 / 6227020800))))));
  const double cosine =
      1.0 + y * (-1.0 / 2 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 +
          y * (-1.0 / 3628800 + y * (1.0 / 479001600))))));
  const int n = (int)q & 3;
  const double a = n & 1 ? cosine : sine, b = n & 1 ? sine : cosine;
  *s = n & 2 ? -a : a;
  *c = n == 1 || n == 2 ? -b : b;
}
// In fp32 the hardware's, which take turns: off by at most 1.26e-7 (of 2^24 turns in
// every range that was looked at). The turn's own rounding to fp32 adds up to pi 2^-25,
// 0.94e-7, so that a sine is good to 3.7 steps of 2^-24.
__device__ __forceinline__ void sin_cos(float t, float* s, float* c) {
  *s = __builtin_amdgcn_sinf(t);
  *c = __builtin_amdgcn_cosf(t);
}

// The positions of a token, and the part of a turn of its pair i: turns = pos *
// turn in fp64, exact to 2^-52 of up to 2^31 / 2 pi of them.
struct Position {
  double at[3];
  __device__ Position(const RotaryParams& p, const int32_t* pos, long long axis_stride,
                      long long item) {
#pragma unroll
    for (int x = 0; x < 3; ++x) at[x] = pos[min(x, p.axes - 1) * axis_stride + item];
  }
  __device__ double turn(const RotaryParams& p, int i) const {
    const double t = (i < p.end[0] ? at[0] : i < p.end[1] ? at[1] : at[2]) * p.turn[i];
    return t - __builtin_rint(t);
  }
};

// Angles of a lane's pairs of a token.
template <bool IL>
__device__ __forceinline__ Angles<float> angles(const RotaryParams& p, const int32_t* pos,
                                                long long axis_stride, long long item, int j,
                                                float sign) {
  const Position at(p, pos, axis_stride, item);
  Angles<float> a;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    sin_cos((float)at.turn(p, pair_of<IL>(j, e)), &a.s[e], &a.c[e]);
    a.s[e] *= sign;
  }
  return a;
}

// The same in fp64, of the workgroup's tokens, each pair by one thread.
struct SharedAngles {
  double2 sc[kItems * kWaves][64 + 1];  // sine, cosine
  __device__ void compute(const RotaryParams& p, const int32_t* pos, long long items, Split s) {
    const int per = kLanes * s.waves;  // threads of a token
    const int token = threadIdx.x / per;
    const long long item = (long long)blockIdx.x * (kThreads / per) + token;
    if (item < items) {
      const Position at(p, pos, items, item);
      for (int i = threadIdx.x % per; i < 64; i += per)
        sin_cos(at.turn(p, i), &sc[token][i].x, &sc[token][i].y);
    }
    __syncthreads();
  }
  template <bool IL>
  __device__ Angles<double> of(int token, int j) const {
    Angles<double> a;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      a.s[e] = sc[token][pair_of<IL>(j, e)].x;
      a.c[e] = sc[token][pair_of<IL>(j, e)].y;
    }
    return a;
  }
};

template <bool IL, class T>
__device__ __forceinline__ void rotate(Vec& v, const Angles<T>& a, int n, int j) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = v.f[first_of<IL>(e)], y = v.f[second_of<IL>(e)];
    const bool turned = pair_of<IL>(j, e) < n;
    v.f[first_of<IL>(e)] = turned ? (float)(x * a.c[e] - y * a.s[e]) : x;
    v.f[second_of<IL>(e)] = turned ? (float)(x * a.s[e] + y * a.c[e]) : y;
  }
}

// A lane's two pieces of a vector. Nothing here is read again before it has left
// the caches.
struct Raw {
  u32x4 lo, hi;
};
__device__ __forceinline__ Raw load(const uint16_t* p) {
  return Raw{__builtin_nontemporal_load((const u32x4*)p),
             __builtin_nontemporal_load((const u32x4*)(p + 64))};
}
__device__ __forceinline__ void store(uint16_t* p, Raw r) {
  __builtin_nontemporal_store(r.lo, (u32x4*)p);
  __builtin_nontemporal_store(r.hi, (u32x4*)(p + 64));
}
__device__ __forceinline__ Raw pack(const Vec& v) {
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = pack_bf16(v.f[2 * i], v.f[2 * i + 1]);
    hi[i] = pack_bf16(v.f[8 + 2 * i], v.f[8 + 2 * i + 1]);
  }
  return Raw{lo, hi};
}

template <bool IL>
__global__ __launch_bounds__(kThreads) void rotary_kernel(
    const uint16_t* x, Strides xs, int tokens, long long items, int heads, Split split,
    const int32_t* __restrict__ pos, RotaryParams plan, float sign, uint16_t* out, Strides os) {
  const int j = threadIdx.x % kLanes;
  const Place place(split, heads);
  const long long item = place.item;
  const int h1 = place.h1, step = split.waves;
  int h = place.h;
  if (item >= items || h >= h1) return;
  const long long b = item / tokens, t = item - b * tokens;
  x += b * xs.batch + t * xs.token + 8 * j;
  out += b * os.batch + t * os.token + 8 * j;
  Raw next = load(x + h * xs.head);
  const Angles<float> a = angles<IL>(plan, pos, items, item, j, sign);
  for (; h < h1; h += step) {
    const Raw now = next;
    if (h + step < h1) next = load(x + (h + step) * xs.head);
    Vec v = unpack(now.lo, now.hi);
    rotate<IL>(v, a, plan.n, j);
    store(out + h * os.head, pack(v));
  }
}

// ---- append

__device__ __forceinline__ float max8(float x) {
#pragma unroll
  for (int off = 1; off < kLanes; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

__device__ __forceinline__ float finite_or_0(float x) {
  return __builtin_isfinite(x) ? x : 0.f;
}

// Exponent of a vector's scale, from its values before the rotation: the least
// e >= -126 with m <= 448 * 2^e, m the largest finite magnitude, or the largest
// length of a pair where it is to be rotated. With 2^E <= the largest magnitude
// < 2^(E+1), the values times 2^-E have squares (sums of two) in [1, 8), exact
// products of 8-bit mantissas; 448 = 1.75 * 2^8 and 1.75^2 = 3.0625, so e is
// E - 8, or one more where the square is larger than that. The sum of two squares is
// rounded to fp32: a length of up to 2^-24 more than 448 * 2^e counts as that (its
// values are bounded).
template <bool IL, bool ROT>
__device__ __forceinline__ int scale_exponent(const Vec& v) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(finite_or_0(v.f[i])));
  m = max8(m);
  if (m == 0.f) return 0;
  const int E = __builtin_amdgcn_frexp_expf(m) - 1;
  float sq;
  if (ROT) {
    sq = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = ldexpf(finite_or_0(v.f[first_of<IL>(e)]), -E);
      const float y = ldexpf(finite_or_0(v.f[second_of<IL>(e)]), -E);
      sq = fmaxf(sq, __builtin_fmaf(x, x, y * y));
    }
    sq = max8(sq);
  } else {
    const float x = ldexpf(m, -E);
    sq = x * x;
  }
  const int e = E - 8 + (sq > 3.0625f);
  return e < -126 ? -126 : e;
}

__device__ __forceinline__ float bounded(float x) {
  return x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
}

__device__ __forceinline__ void store_e4m3(uint8_t* p, const Vec& v, int e) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = bounded(ldexpf(v.f[4 * i + k], -e));
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], r, true);
  }
  *(u32x2*)p = u32x2{w[0], w[1]};
  *(u32x2*)(p + 64) = u32x2{w[2], w[3]};
}

template <bool IL, bool ROT, bool E4M3>
__global__ __launch_bounds__(kThreads) void append_kernel(
    const uint16_t* __restrict__ k, Strides ks, const uint16_t* __restrict__ v, Strides vs,
    int tokens, long long items, Split split, const int32_t* __restrict__ count,
    const int32_t* __restrict__ start, const int32_t* __restrict__ pos, RotaryParams plan,
    CacheParams c) {
  // A key that goes to 8 bits is turned in fp64: a value that rounds the other way
  // is off by a sixteenth.
  __shared__ typename std::conditional<ROT && E4M3, SharedAngles, int>::type shared;
  if constexpr (ROT && E4M3) shared.compute(plan, pos, items, split);
  const int j = threadIdx.x % kLanes;
  const Place at(split, c.hkv);
  const long long item = at.item;
  const int h1 = at.h1, step = split.waves;
  int h = at.h;
  if (item >= items || h >= h1) return;
  const long long b = item / tokens, t = item - b * tokens;
  k += b * ks.batch + t * ks.token + 8 * j;
  v += b * vs.batch + t * vs.token + 8 * j;
  if (count && t >= count[b]) return;
  const long long place = start[b] + t;
  const int column = page_column(place, c.shift, c.table_pages);
  if (column < 0) return;
  Raw next_k = load(k + h * ks.head), next_v = load(v + h * vs.head);
  const int entry = c.table[b * c.table_pages + column];
  const int slot = (int)(place & ((1 << c.shift) - 1));
  if (page_row(entry, c.pages, c.hkv, 0, c.shift, slot) < 0) return;
  Angles<float> a;
  Angles<double> exact;
  if (ROT && !E4M3) a = angles<IL>(plan, pos, items, item, j, 1.f);
  if constexpr (ROT && E4M3) {
    const long long first = (long long)blockIdx.x * (kItems * (kWaves / step));  // of the workgroup
    exact = shared.template of<IL>((int)(item - first), j);
  }
  for (; h < h1; h += step) {
    const long long row = page_row(entry, c.pages, c.hkv, h, c.shift, slot);
    Raw k_now = next_k;
    const Raw v_now = next_v;
    if (h + step < h1) {
      next_k = load(k + (h + step) * ks.head);
      next_v = load(v + (h + step) * vs.head);
    }
    if (E4M3) {
      Vec key = unpack(k_now.lo, k_now.hi);
      const int ek = scale_exponent<IL, ROT>(key);
      if (ROT) rotate<IL>(key, exact, plan.n, j);
      store_e4m3((uint8_t*)c.k + row * kHeadDim + 8 * j, key, ek);
      const Vec value = unpack(v_now.lo, v_now.hi);
      const int ev = scale_exponent<IL, false>(value);
      store_e4m3((uint8_t*)c.v + row * kHeadDim + 8 * j, value, ev);
      if (j == 0) {
        c.k_scale[row] = (uint8_t)(ek + 127);
        c.v_scale[row] = (uint8_t)(ev + 127);
      }
    } else {
      if (ROT) {
        Vec key = unpack(k_now.lo, k_now.hi);
        rotate<IL>(key, a, plan.n, j);
        k_now = pack(key);
      }
      store((uint16_t*)c.k + row * kHeadDim + 8 * j, k_now);
      store((uint16_t*)c.v + row * kHeadDim + 8 * j, v_now);
    }
  }
}

// Workgroups that are to be left when their heads are made more: 32 a CU (8: 32K
// tokens of 32 heads 104.9 -> 101.0 us the other way, others alike).
constexpr long long kWant = 32 * 256;

Split split_of(long long items, int heads, dim3* grid) {
  Split s;
  s.waves = heads >= kWaves ? kWaves : heads >= 2 ? 2 : 1;
  const int tokens = kItems * (kWaves / s.waves);
  const long long groups = (items + tokens - 1) / tokens;
  const long long per = (groups * heads / kWant + s.waves - 1) / s.waves * s.waves;
  s.heads = (int)(per < s.waves ? s.waves : per > heads ? heads : per);
  *grid = dim3((unsigned)groups, (heads + s.heads - 1) / s.heads);
  return s;
}

}  // namespace

hipError_t launch_rotary(const void* x, const Strides& xs, int batch, int heads, int tokens,
                         const int32_t* pos, const RotaryParams& plan, bool interleaved,
                         bool inverse, void* out, const Strides& os, hipStream_t st) {
  const long long items = (long long)batch * tokens;
  dim3 grid;
  const Split split = split_of(items, heads, &grid);
  auto* kernel = interleaved ? rotary_kernel<true> : rotary_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, (const uint16_t*)x, xs, tokens, items,
                     heads, split, pos, plan, inverse ? -1.f : 1.f, (uint16_t*)out, os);
  return hipGetLastError();
}

hipError_t launch_append(const void* k, const Strides& ks, const void* v, const Strides& vs,
                         int batch, int tokens, const int32_t* count, const int32_t* start,
                         const int32_t* pos, const RotaryParams* plan, bool interleaved,
                         const CacheParams& c, bool e4m3, hipStream_t st) {
  const long long items = (long long)batch * tokens;
  dim3 grid;
  const Split split = split_of(items, c.hkv, &grid);
  auto* kernel = plan ? (interleaved ? (e4m3 ? append_kernel<true, true, true>
                                             : append_kernel<true, true, false>)
                                     : (e4m3 ? append_kernel<false, true, true>
                                             : append_kernel<false, true, false>))
                      : (e4m3 ? append_kernel<false, false, true>
                              : append_kernel<false, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, (const uint16_t*)k, ks,
                     (const uint16_t*)v, vs, tokens, items, split, count, start, pos,
                     plan ? *plan : RotaryParams{}, c);
  return hipGetLastError();
}
