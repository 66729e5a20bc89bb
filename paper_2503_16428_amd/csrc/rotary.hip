// Rotary positions, and the append of keys (rotated on the way) and values to
// the paged cache.
//
// Eight lanes share a vector of 128: lane j holds elements 8j .. 8j+7 and
// 64+8j .. 64+8j+7 (two 16-byte loads), which are eight whole pairs in either
// pairing. A wave has eight tokens, the waves of a workgroup go over the heads in
// turn: neighbouring heads of a token, which a projection leaves side by side, are
// read together, and eight tokens of a head written together. A thread computes
// its token's eight angles once, while its first vector is on the way, and loads
// the next head's before it turns this one.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 8;                   // lanes of a vector
constexpr int kItems = kWave / kLanes;      // tokens of a workgroup
constexpr int kWaves = kThreads / kWave;

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

struct Angles {
  float c[8], s[8];
};

// Angles of a token's pairs: turns = pos * turn in fp64 (exact to 2^-52 of up
// to 2^31 / 2 pi turns), of which the part of a turn goes to the hardware's sine
// and cosine in fp32 (inputs in turns; off by at most 1.3e-7).
template <bool IL>
__device__ __forceinline__ Angles angles(const RotaryParams& p, const int32_t* pos,
                                         long long axis_stride, long long item, int j, float sign) {
  double at[3];
#pragma unroll
  for (int x = 0; x < 3; ++x) at[x] = pos[min(x, p.axes - 1) * axis_stride + item];
  Angles a;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = pair_of<IL>(j, e);
    const double t = (i < p.end[0] ? at[0] : i < p.end[1] ? at[1] : at[2]) * p.turn[i];
    const float f = (float)(t - __builtin_rint(t));
    a.c[e] = __builtin_amdgcn_cosf(f);
    a.s[e] = sign * __builtin_amdgcn_sinf(f);
  }
  return a;
}

template <bool IL>
__device__ __forceinline__ void rotate(Vec& v, const Angles& a, int n, int j) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = v.f[first_of<IL>(e)], y = v.f[second_of<IL>(e)];
    const bool turned = pair_of<IL>(j, e) < n;
    v.f[first_of<IL>(e)] = turned ? x * a.c[e] - y * a.s[e] : x;
    v.f[second_of<IL>(e)] = turned ? x * a.s[e] + y * a.c[e] : y;
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
    const uint16_t* x, Strides xs, int tokens, long long items, int heads, int heads_per,
    const int32_t* __restrict__ pos, RotaryParams plan, float sign, uint16_t* out, Strides os) {
  const int lane = threadIdx.x % kWave, j = lane % kLanes;
  const long long item = (long long)blockIdx.x * kItems + lane / kLanes;
  int h = blockIdx.y * heads_per + threadIdx.x / kWave;
  const int h1 = min((int)(blockIdx.y + 1) * heads_per, heads);
  if (item >= items || h >= h1) return;
  const long long b = item / tokens, t = item - b * tokens;
  x += b * xs.batch + t * xs.token + 8 * j;
  out += b * os.batch + t * os.token + 8 * j;
  Raw next = load(x + h * xs.head);
  const Angles a = angles<IL>(plan, pos, items, item, j, sign);
  for (; h < h1; h += kWaves) {
    const Raw now = next;
    if (h + kWaves < h1) next = load(x + (h + kWaves) * xs.head);
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
// E - 8, or one more where the square is larger than that.
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
    int tokens, long long items, int heads_per, const int32_t* __restrict__ count,
    const int32_t* __restrict__ start, const int32_t* __restrict__ pos, RotaryParams plan,
    CacheParams c) {
  const int lane = threadIdx.x % kWave, j = lane % kLanes;
  const long long item = (long long)blockIdx.x * kItems + lane / kLanes;
  int h = blockIdx.y * heads_per + threadIdx.x / kWave;
  const int h1 = min((int)(blockIdx.y + 1) * heads_per, c.hkv);
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
  Angles a;
  if (ROT) a = angles<IL>(plan, pos, items, item, j, 1.f);
  for (; h < h1; h += kWaves) {
    const long long row = page_row(entry, c.pages, c.hkv, h, c.shift, slot);
    Raw k_now = next_k;
    const Raw v_now = next_v;
    if (h + kWaves < h1) {
      next_k = load(k + (h + kWaves) * ks.head);
      next_v = load(v + (h + kWaves) * vs.head);
    }
    if (E4M3) {
      Vec key = unpack(k_now.lo, k_now.hi);
      const int ek = scale_exponent<IL, ROT>(key);
      if (ROT) rotate<IL>(key, a, plan.n, j);
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

// Heads of a workgroup: as many as leave 32 workgroups a CU, four at least (8
// a CU: 32K tokens of 32 heads 104.9 -> 101.0 us, others alike).
constexpr long long kWant = 32 * 256;
int heads_per_group(long long groups, int heads) {
  const long long per = (groups * heads / kWant + kWaves - 1) / kWaves * kWaves;
  return (int)(per < kWaves ? kWaves : per > heads ? heads : per);
}

}  // namespace

hipError_t launch_rotary(const void* x, const Strides& xs, int batch, int heads, int tokens,
                         const int32_t* pos, const RotaryParams& plan, bool interleaved,
                         bool inverse, void* out, const Strides& os, hipStream_t st) {
  const long long items = (long long)batch * tokens, groups = (items + kItems - 1) / kItems;
  const int per = heads_per_group(groups, heads);
  const dim3 grid((unsigned)groups, (heads + per - 1) / per);
  auto* kernel = interleaved ? rotary_kernel<true> : rotary_kernel<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, (const uint16_t*)x, xs, tokens, items,
                     heads, per, pos, plan, inverse ? -1.f : 1.f, (uint16_t*)out, os);
  return hipGetLastError();
}

hipError_t launch_append(const void* k, const Strides& ks, const void* v, const Strides& vs,
                         int batch, int tokens, const int32_t* count, const int32_t* start,
                         const int32_t* pos, const RotaryParams* plan, bool interleaved,
                         const CacheParams& c, bool e4m3, hipStream_t st) {
  const long long items = (long long)batch * tokens, groups = (items + kItems - 1) / kItems;
  const int per = heads_per_group(groups, c.hkv);
  const dim3 grid((unsigned)groups, (c.hkv + per - 1) / per);
  auto* kernel = plan ? (interleaved ? (e4m3 ? append_kernel<true, true, true>
                                             : append_kernel<true, true, false>)
                                     : (e4m3 ? append_kernel<false, true, true>
                                             : append_kernel<false, true, false>))
                      : (e4m3 ? append_kernel<false, false, true>
                              : append_kernel<false, false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, st, (const uint16_t*)k, ks,
                     (const uint16_t*)v, vs, tokens, items, per, count, start, pos,
                     plan ? *plan : RotaryParams{}, c);
  return hipGetLastError();
}
