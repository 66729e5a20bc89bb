// Attention of one new token per sequence over a paged cache, split over the
// length and joined.
//
// A wave takes 16 keys of a key head against up to 16 of its query heads:
//   S^T = K Q^T  by 16x16x32 bf16 MFMAs: lane (g, c) = (lane / 16, lane % 16)
//     supplies K's row c and Q's row c, and receives queries c, keys 4g .. 4g+3;
//   O^T += V^T P^T  by 16x16x4 fp32 MFMAs: step r takes the keys {4g + r}, so
//     that P stays in the registers where the softmax left it, and the lane's
//     piece of V is 8 consecutive values of row 4g + r: the i-th of them is row c
//     of the A operand of MFMA i, whose output rows are elements 8c + i.
// Neither K, V nor P passes through LDS, nothing is transposed, and P and the
// values are fp32 in the second product (v_mfma_f32_16x16x4_f32).
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 16;       // keys of a wave's step
constexpr int kRows = 16;       // query heads of a workgroup
constexpr float kScale = 0.08838834764831845f * kLog2e;  // to log2, 1 / sqrt(128)

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

struct DecodeParams {
  CacheParams c;
  const uint16_t* q;
  const int32_t* lens;
  int hq, group, row_tiles, splits;
  float* part;   // [row][split][16][128] unnormalised outputs
  float* ml;     // [row][split][16][2] (maximum in log2, sum)
  float* stat;   // [batch][hq][2] (maximum in log2, 1 / sum)
  float* z;      // [batch][hq][capacity] products in log2, or NULL
};

__device__ __forceinline__ int split_keys(int len, int splits) {
  const int per = (len + splits - 1) / splits;
  return (per + kTile * kWaves - 1) / (kTile * kWaves) * (kTile * kWaves);
}

template <bool E4M3>
__global__ __launch_bounds__(kThreads) void decode_kernel(DecodeParams p) {
  __shared__ float so[kWaves][kRows][kHeadDim + 4];
  __shared__ float sm[kWaves][kRows], sl[kWaves][kRows];
  const int tid = threadIdx.x, lane = tid % kWave, g = lane / 16, c = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int row = blockIdx.x / p.splits, split = blockIdx.x % p.splits;
  const int tile = row % p.row_tiles, bh = row / p.row_tiles;
  const int b = bh / p.c.hkv, h = bh % p.c.hkv;
  const int len = clamp_len(p.lens[b], p.c.capacity());
  const int per = split_keys(len, p.splits);
  const int t0 = split * per, t1 = min(t0 + per, len);
  float* ml = p.ml + (long long)blockIdx.x * (2 * kRows);
  if (t0 >= t1) {
    if (tid < kRows) {
      ml[2 * tid] = -__builtin_inff();
      ml[2 * tid + 1] = 0.f;
    }
    return;
  }
  const int in_group = tile * kRows + c;
  const bool real = in_group < p.group;
  const int hq = h * p.group + (real ? in_group : 0);

  bf16x8 q[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    // e4m3 keys come as 16 bytes a lane, two of these pieces
    const int d = E4M3 ? 64 * (j / 2) + 16 * g + 8 * (j % 2) : 32 * j + 8 * g;
    u32x4 u = *(const u32x4*)(p.q + ((long long)b * p.hq + hq) * kHeadDim + d);
    if (!real) u = u32x4{0, 0, 0, 0};
    q[j] = as_bf16x8(u);
  }
  f32x4 o[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -__builtin_inff(), l = 0.f;
  const int32_t* table = p.c.table + (long long)b * p.c.table_pages;

  for (int t = t0 + wave * kTile; t < t1; t += kTile * kWaves) {
    const int entry = __builtin_amdgcn_readfirstlane(table[t >> p.c.shift]);
    const int slot = t & ((1 << p.c.shift) - 1);
    const long long first = page_row(entry, p.c.pages, p.c.hkv, h, p.c.shift, slot);
    float zs[4];
    if (first < 0) {
#pragma unroll
      for (int r = 0; r < 4; ++r) zs[r] = -__builtin_inff();
    } else {
      f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
      if (E4M3) {
        const uint8_t* kp = (const uint8_t*)p.c.k + (first + c) * kHeadDim + 16 * g;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const u32x4 u = *(const u32x4*)(kp + 64 * i);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            bf16x8 a;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w = u[2 * x + e];
              const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false);
              const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
              a[4 * e] = (__bf16)lo[0];
              a[4 * e + 1] = (__bf16)lo[1];
              a[4 * e + 2] = (__bf16)hi[0];
              a[4 * e + 3] = (__bf16)hi[1];
            }
            s = mfma16(a, q[2 * i + x], s);
          }
        }
        const uint32_t sc = *(const uint32_t*)(p.c.k_scale + first + 4 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r) zs[r] = s[r] * scale_of(sc >> (8 * r) & 255) * kScale;
      } else {
        const uint16_t* kp = (const uint16_t*)p.c.k + (first + c) * kHeadDim + 8 * g;
#pragma unroll
        for (int j = 0; j < 4; ++j) s = mfma16(as_bf16x8(*(const u32x4*)(kp + 32 * j)), q[j], s);
#pragma unroll
        for (int r = 0; r < 4; ++r) zs[r] = s[r] * kScale;
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (t + 4 * g + r >= t1) zs[r] = -__builtin_inff();
    if (p.z && real) {
      float* z = p.z + ((long long)b * p.hq + hq) * p.c.capacity() + t + 4 * g;
      *(f32x4*)z = f32x4{zs[0], zs[1], zs[2], zs[3]};
    }
    if (first < 0) continue;
    float top = fmaxf(fmaxf(zs[0], zs[1]), fmaxf(zs[2], zs[3]));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (__any(top > m)) {
      const float next = fmaxf(m, top);
      // a maximum of -inf has summed nothing yet
      const float f = m == -__builtin_inff() ? 0.f : fast_exp2(m - next);
      l *= f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] *= f;
      m = next;
    }
    const float ref = m == -__builtin_inff() ? 0.f : m;
    float pr[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      pr[r] = fast_exp2(zs[r] - ref);
      l += pr[r];
    }
    uint32_t vsc = 0;
    if (E4M3) vsc = *(const uint32_t*)(p.c.v_scale + first + 4 * g);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const bool in = t + 4 * g + r < t1;
      float f[8];
      if (E4M3) {
        u32x2 u = *(const u32x2*)((const uint8_t*)p.c.v + (first + 4 * g + r) * kHeadDim + 8 * c);
        const float sc = in ? scale_of(vsc >> (8 * r) & 255) : 0.f;
        if (!in) u = u32x2{0, 0};
        pr[r] *= sc;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[e], false);
          const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[e], true);
          f[4 * e] = lo[0];
          f[4 * e + 1] = lo[1];
          f[4 * e + 2] = hi[0];
          f[4 * e + 3] = hi[1];
        }
      } else {
        u32x4 u = *(const u32x4*)((const uint16_t*)p.c.v + (first + 4 * g + r) * kHeadDim + 8 * c);
        if (!in) u = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f[2 * e] = __builtin_bit_cast(float, u[e] << 16);
          f[2 * e + 1] = __builtin_bit_cast(float, u[e] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = mfma4(f[i], pr[r], o[i]);
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // the four waves' keys, joined in their order
  if (g == 0) {
    sm[wave][c] = m;
    sl[wave][c] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < 8; ++i) so[wave][c][8 * (4 * g + r) + i] = o[i][r];
  __syncthreads();
  float* part = p.part + (long long)blockIdx.x * (kRows * kHeadDim);
  for (int i = tid; i < kRows * kHeadDim; i += kThreads) {
    const int rq = i / kHeadDim, d = i % kHeadDim;
    float top = sm[0][rq];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][rq]);
    float sum = 0.f, out = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = sm[w][rq] == -__builtin_inff() ? 0.f : fast_exp2(sm[w][rq] - top);
      sum += f * sl[w][rq];
      out += f * so[w][rq][d];
    }
    part[i] = out;
    if (d == 0) {
      ml[2 * rq] = top;
      ml[2 * rq + 1] = sum;
    }
  }
}

// One workgroup per query head, one thread per element: its splits in order.
__global__ __launch_bounds__(kHeadDim) void decode_join(DecodeParams p, uint16_t* __restrict__ o,
                                                        float* __restrict__ lse) {
  const int d = threadIdx.x, b = blockIdx.x / p.hq, hq = blockIdx.x % p.hq;
  const int h = hq / p.group, in_group = hq % p.group;
  const long long row = ((long long)b * p.c.hkv + h) * p.row_tiles + in_group / kRows;
  const int r = in_group % kRows;
  const float* ml = p.ml + (row * p.splits * kRows + r) * 2;
  const float* part = p.part + (row * p.splits * kRows + r) * kHeadDim + d;
  float top = -__builtin_inff();
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, ml[s * 2 * kRows]);
  float sum = 0.f, out = 0.f;
  for (int s = 0; s < p.splits; ++s) {
    const float ms = ml[s * 2 * kRows], ls = ml[s * 2 * kRows + 1];
    if (ls == 0.f) continue;  // no key, nothing written
    const float f = fast_exp2(ms - top);
    sum += f * ls;
    out += f * part[(long long)s * (kRows * kHeadDim)];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const __bf16 r16 = (__bf16)(out * inv);
  o[(long long)blockIdx.x * kHeadDim + d] = __builtin_bit_cast(uint16_t, r16);
  if (d == 0) {
    if (lse) lse[blockIdx.x] = sum == 0.f ? -__builtin_inff() : (top + log2f(sum)) / kLog2e;
    if (p.stat) {
      p.stat[2 * blockIdx.x] = sum == 0.f ? 0.f : top;
      p.stat[2 * blockIdx.x + 1] = inv;
    }
  }
}

// One thread per key: the weights of its group's heads, from the products.
__global__ __launch_bounds__(kThreads) void decode_weights(DecodeParams p,
                                                           float* __restrict__ weights) {
  const int capacity = p.c.capacity(), chunks = (capacity + kThreads - 1) / kThreads;
  const int row = blockIdx.x / chunks, t = blockIdx.x % chunks * kThreads + threadIdx.x;
  const int b = row / p.c.hkv, h = row % p.c.hkv;
  if (t >= clamp_len(p.lens[b], capacity)) return;
  const long long first = (long long)b * p.hq + h * p.group;
  float w = 0.f;
  for (int i = 0; i < p.group; ++i) {
    const float* st = p.stat + 2 * (first + i);
    w += fast_exp2(p.z[(first + i) * capacity + t] - st[0]) * st[1];
  }
  weights[(long long)row * capacity + t] += w;
}

constexpr int kSplitGroups = 1024;  // workgroups that the splits are to make
constexpr int kLeastKeys = 256;     // keys that a split is worth

int splits_of(const CacheParams& c, int rows) {
  const int most = (c.capacity() + kLeastKeys - 1) / kLeastKeys;
  const int want = (kSplitGroups + rows - 1) / rows;
  return want < most ? want : most;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Scratch {
  size_t part, ml, stat, z, bytes;
};

Scratch scratch_of(const CacheParams& c, int batch, int hq, bool weights) {
  const int row_tiles = (hq / c.hkv + kRows - 1) / kRows, rows = batch * c.hkv * row_tiles;
  const size_t parts = (size_t)rows * splits_of(c, rows);
  Scratch s;
  s.part = 0;
  s.ml = s.part + align256(parts * kRows * kHeadDim * 4);
  s.stat = s.ml + align256(parts * kRows * 8);
  s.z = s.stat + (weights ? align256((size_t)batch * hq * 8) : 0);
  s.bytes = s.z + (weights ? align256((size_t)batch * hq * c.capacity() * 4) : 0);
  return s;
}

}  // namespace

size_t decode_scratch_bytes(const CacheParams& c, int batch, int hq, bool weights) {
  return scratch_of(c, batch, hq, weights).bytes;
}

hipError_t launch_decode(const void* q, const CacheParams& c, bool e4m3, int batch, int hq,
                         const int32_t* lens, void* o, float* lse, float* weights, void* scratch,
                         hipStream_t st) {
  const Scratch s = scratch_of(c, batch, hq, weights != nullptr);
  DecodeParams p;
  p.c = c;
  p.q = (const uint16_t*)q;
  p.lens = lens;
  p.hq = hq;
  p.group = hq / c.hkv;
  p.row_tiles = (p.group + kRows - 1) / kRows;
  const int rows = batch * c.hkv * p.row_tiles;
  p.splits = splits_of(c, rows);
  p.part = (float*)((char*)scratch + s.part);
  p.ml = (float*)((char*)scratch + s.ml);
  p.stat = weights ? (float*)((char*)scratch + s.stat) : nullptr;
  p.z = weights ? (float*)((char*)scratch + s.z) : nullptr;
  hipLaunchKernelGGL(e4m3 ? decode_kernel<true> : decode_kernel<false>,
                     dim3((unsigned)(rows * p.splits)), dim3(kThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(decode_join, dim3(batch * hq), dim3(kHeadDim), 0, st, p, (uint16_t*)o, lse);
  if ((e = hipGetLastError()) != hipSuccess || !weights) return e;
  const int chunks = (c.capacity() + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(decode_weights, dim3((unsigned)(batch * c.hkv * chunks)), dim3(kThreads), 0,
                     st, p, weights);
  return hipGetLastError();
}
