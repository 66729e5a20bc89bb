// Rotary positions, and the append of keys (rotated on the way) and values to
// the paged cache.
//
// Eight lanes share a vector of 128: lane j holds elements 8j .. 8j+7 and
// 64+8j .. 64+8j+7 (two 16-byte loads), which are eight whole pairs in either
// pairing. A thread computes its token's eight angles once and goes over heads.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kLanes = 8;                   // lanes of a vector
constexpr int kItems = kThreads / kLanes;   // tokens of a workgroup

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
// and cosine in fp32 (inputs in turns).
template <bool IL>
__device__ __forceinline__ Angles angles(const RotaryParams& p, const int32_t* pos,
                                         long long axis_stride, long long item, int j, float sign) {
  Angles a;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int i = pair_of<IL>(j, e);
    const double t = (double)pos[p.axis[i] * axis_stride + item] * p.turn[i];
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

__device__ __forceinline__ void store_bf16(uint16_t* p, const Vec& v) {
  u32x4 lo, hi;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[i] = pack_bf16(v.f[2 * i], v.f[2 * i + 1]);
    hi[i] = pack_bf16(v.f[8 + 2 * i], v.f[8 + 2 * i + 1]);
  }
  *(u32x4*)p = lo;
  *(u32x4*)(p + 64) = hi;
}

template <bool IL>
__global__ __launch_bounds__(kThreads) void rotary_kernel(
    const uint16_t* x, Strides xs, int tokens, long long items, int heads, int heads_per,
    const int32_t* __restrict__ pos, RotaryParams plan, float sign, uint16_t* out, Strides os) {
  const int j = threadIdx.x % kLanes;
  const long long item = (long long)blockIdx.x * kItems + threadIdx.x / kLanes;
  if (item >= items) return;
  const long long b = item / tokens, t = item - b * tokens;
  const Angles a = angles<IL>(plan, pos, items, item, j, sign);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, heads);
  x += b * xs.batch + t * xs.token + 8 * j;
  out += b * os.batch + t * os.token + 8 * j;
  for (int h = h0; h < h1; ++h) {
    const uint16_t* p = x + h * xs.head;
    Vec v = unpack(*(const u32x4*)p, *(const u32x4*)(p + 64));
    rotate<IL>(v, a, plan.n, j);
    store_bf16(out + h * os.head, v);
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
  const int j = threadIdx.x % kLanes;
  const long long item = (long long)blockIdx.x * kItems + threadIdx.x / kLanes;
  if (item >= items) return;
  const long long b = item / tokens, t = item - b * tokens;
  if (count && t >= count[b]) return;
  const long long place = start[b] + t;
  const int column = page_column(place, c.shift, c.table_pages);
  if (column < 0) return;
  const int entry = c.table[b * c.table_pages + column];
  const int slot = (int)(place & ((1 << c.shift) - 1));
  if (page_row(entry, c.pages, c.hkv, 0, c.shift, slot) < 0) return;
  Angles a;
  if (ROT) a = angles<IL>(plan, pos, items, item, j, 1.f);
  const int h0 = blockIdx.y * heads_per, h1 = min(h0 + heads_per, c.hkv);
  k += b * ks.batch + t * ks.token + 8 * j;
  v += b * vs.batch + t * vs.token + 8 * j;
  for (int h = h0; h < h1; ++h) {
    const long long row = page_row(entry, c.pages, c.hkv, h, c.shift, slot);
    const uint16_t *kp = k + h * ks.head, *vp = v + h * vs.head;
    const u32x4 k0 = *(const u32x4*)kp, k1 = *(const u32x4*)(kp + 64);
    const u32x4 v0 = *(const u32x4*)vp, v1 = *(const u32x4*)(vp + 64);
    if (E4M3) {
      Vec key = unpack(k0, k1);
      const int ek = scale_exponent<IL, ROT>(key);
      if (ROT) rotate<IL>(key, a, plan.n, j);
      store_e4m3((uint8_t*)c.k + row * kHeadDim + 8 * j, key, ek);
      const Vec value = unpack(v0, v1);
      const int ev = scale_exponent<IL, false>(value);
      store_e4m3((uint8_t*)c.v + row * kHeadDim + 8 * j, value, ev);
      if (j == 0) {
        c.k_scale[row] = (uint8_t)(ek + 127);
        c.v_scale[row] = (uint8_t)(ev + 127);
      }
    } else {
      uint16_t* to = (uint16_t*)c.k + row * kHeadDim + 8 * j;
      if (ROT) {
        Vec key = unpack(k0, k1);
        rotate<IL>(key, a, plan.n, j);
        store_bf16(to, key);
      } else {
        *(u32x4*)to = k0;
        *(u32x4*)(to + 64) = k1;
      }
      to = (uint16_t*)c.v + row * kHeadDim + 8 * j;
      *(u32x4*)to = v0;
      *(u32x4*)(to + 64) = v1;
    }
  }
}

// Heads that a thread goes over: as many as leave eight workgroups a CU.
int heads_per_thread(long long groups, int heads) {
  const long long want = 8 * 256;
  long long per = groups * heads / want;
  return (int)(per < 1 ? 1 : per > heads ? heads : per);
}

}  // namespace

hipError_t launch_rotary(const void* x, const Strides& xs, int batch, int heads, int tokens,
                         const int32_t* pos, const RotaryParams& plan, bool interleaved,
                         bool inverse, void* out, const Strides& os, hipStream_t st) {
  const long long items = (long long)batch * tokens, groups = (items + kItems - 1) / kItems;
  const int per = heads_per_thread(groups, heads);
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
  const int per = heads_per_thread(groups, c.hkv);
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
