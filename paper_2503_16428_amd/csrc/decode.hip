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
// values are fp32 in the second product.
//
// The work of a batch is its rows (sequence, key head, tile of query heads) end
// to end, in units of kWaves wave steps; every workgroup takes an equal share of
// the units, whatever the lengths, and goes through the rows in it. A row that
// one workgroup has whole is done there; of the others every share leaves a
// partial output (at most two a workgroup: its first and its last row), and
// decode_join adds them in order.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 16;  // keys of a tile
constexpr int kRows = 16;  // query heads of a tile
constexpr float kScale = 0.08838834764831845f * kLog2e;  // to log2, 1 / sqrt(128)
constexpr float kMinusInf = -__builtin_inff();

// Tiles of a wave's step: 16 KB of keys and values in either type.
template <bool E4M3>
constexpr int kTiles = E4M3 ? 2 : 2;

__host__ __device__ constexpr int unit_keys(bool e4m3) {
  return kTile * kWaves * (e4m3 ? 2 : 2);
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}
// Eight e4m3 values in bf16, which holds them exactly.
__device__ __forceinline__ bf16x8 bf16_of(uint32_t a, uint32_t b) {
  const auto p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false);
  const auto q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
  const auto r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false);
  const auto s = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
  return bf16x8{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
}
// A lane's piece of a value vector in fp32.
__device__ __forceinline__ void values(u32x4 u, float* f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[2 * e] = __builtin_bit_cast(float, u[e] << 16);
    f[2 * e + 1] = __builtin_bit_cast(float, u[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void values(u32x2 u, float* f) {
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[e], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[e], true);
    f[4 * e] = lo[0];
    f[4 * e + 1] = lo[1];
    f[4 * e + 2] = hi[0];
    f[4 * e + 3] = hi[1];
  }
}
// 2^(m - top) of a part whose maximum is m: nothing if it has summed nothing.
__device__ __forceinline__ float weight_of(float m, float top) {
  return m == kMinusInf ? 0.f : fast_exp2(m - top);
}

// A value that the compiler takes for a new one: what follows from it is not
// computed ahead and kept in registers over the main loop.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}
// A value that is the same in every lane, for the compiler to see.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x) {
  return (long long)(((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32) |
                     (uint32_t)uniform((int)x));
}

struct DecodeParams {
  CacheParams c;
  const uint16_t* q;
  const int32_t* lens;
  uint16_t* o;
  float* lse;    // or NULL
  int batch, hq, group, row_tiles, tile_rows, unit, most_workers;
  float* part;   // [2 workers][tile_rows][128] unnormalised outputs
  float* ml;     // [2 workers][tile_rows][2] (maximum in log2, sum)
  float* stat;   // [batch][hq][2] (maximum in log2, 1 / sum), or NULL
  float* z;      // [batch][hq][capacity] products in log2, or NULL
};

template <bool E4M3>
struct PieceOf {
  typedef u32x4 type;
};
template <>
struct PieceOf<true> {
  typedef u32x2 type;
};

// Units that a workgroup is to have before there are more workgroups.
constexpr int kLeastUnits = 1;

__device__ __forceinline__ int workers_of(long long units, int most) {
  const long long w = (units + kLeastUnits - 1) / kLeastUnits;
  return w < most ? (int)w : most;
}
// First unit of a worker's share.
__device__ __forceinline__ long long share(long long worker, long long units, int workers) {
  return worker * units / workers;
}

__device__ __forceinline__ int len_of(const DecodeParams& p, int b) {
  return clamp_len(p.lens[b], p.c.capacity());
}
__device__ __forceinline__ int units_of(const DecodeParams& p, int b) {
  return (len_of(p, b) + p.unit - 1) / p.unit;
}

// Sum over the workgroup's threads below this one, and over all of them.
__device__ __forceinline__ long long scan(long long x, long long* total, long long* lds) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  long long y = x;
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const long long up = __shfl_up(y, off);
    if (lane >= off) y += up;
  }
  if (lane == kWave - 1) lds[wave] = y;
  __syncthreads();
  long long before = y - x, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += lds[w];
    all += lds[w];
  }
  __syncthreads();
  *total = all;
  return before;
}

// One element of a finished row: output head `head`, element d.
__device__ __forceinline__ void write_row(const DecodeParams& p, long long head, int d, float top,
                                          float sum, float out) {
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const __bf16 r = (__bf16)(out * inv);
  p.o[head * kHeadDim + d] = __builtin_bit_cast(uint16_t, r);
  if (d != 0) return;
  if (p.lse) p.lse[head] = sum == 0.f ? kMinusInf : (top + log2f(sum)) / kLog2e;
  if (p.stat) {
    p.stat[2 * head] = sum == 0.f ? 0.f : top;
    p.stat[2 * head + 1] = inv;
  }
}

template <bool E4M3, int RT>
__global__ __launch_bounds__(kThreads, RT == 1 ? 3 : 2) void decode_kernel(DecodeParams p) {
  constexpr int TILES = kTiles<E4M3>, KP = E4M3 ? 2 : 4;  // 16-byte pieces of a lane's key
  constexpr int STEP = TILES * kTile;
  using Piece = typename PieceOf<E4M3>::type;  // 8 values
  __shared__ float so[kWaves][RT * kRows][kHeadDim + 4];
  __shared__ float sm[kWaves][RT * kRows], sl[kWaves][RT * kRows];
  __shared__ long long places[kWaves];
  __shared__ long long found[2];
  const int tid = threadIdx.x, lane = tid % kWave;
  const unsigned g = lane / 16, c = lane % 16;
  // the lane's piece of a tile's keys and values, bytes
  const uint32_t k_off = c * (E4M3 ? 128 : 256) + 16 * g;
  const uint32_t v_off = E4M3 ? 512 * g + 8 * c : 1024 * g + 16 * c;
  const int wave = uniform(tid / kWave);
  const int per_seq = p.c.hkv * p.row_tiles;

  // this workgroup's share, and the sequence that it begins in
  long long units = 0, first_before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    const int b = b0 + tid;
    long long all;
    const long long before =
        scan(b < p.batch ? (long long)units_of(p, b) * per_seq : 0, &all, places);
    if (b0 == 0) first_before = before;
    units += all;
  }
  units = uniform(units);
  const int workers = workers_of(units, p.most_workers);
  if ((int)blockIdx.x >= workers) return;
  const long long begin = share(blockIdx.x, units, workers);
  const long long end = share(blockIdx.x + 1, units, workers);
  long long running = 0;
  for (int b0 = 0; b0 < p.batch; b0 += kThreads) {
    const int b = b0 + tid;
    const long long mine = b < p.batch ? (long long)units_of(p, b) * per_seq : 0;
    long long all = 0, before = first_before;
    if (p.batch > kThreads) before = scan(mine, &all, places);
    before += running;
    if (before <= begin && begin < before + mine) {
      found[0] = b;
      found[1] = before;
    }
    running += all;
  }
  __syncthreads();
  int b = uniform((int)found[0]);
  long long at = begin - uniform(found[1]);  // units into sequence b
  long long left = end - begin;
  bool first_segment = true;

  while (left > 0) {
    const int len = uniform(len_of(p, b));
    const int row_units = (len + p.unit - 1) / p.unit;
    if (row_units == 0 || at >= (long long)row_units * per_seq) {
      at = 0;
      ++b;
      continue;
    }
    const int row = (int)(at / row_units), u0 = (int)(at - (long long)row * row_units);
    const int n = (int)min(left, (long long)(row_units - u0));
    const int h = row / p.row_tiles, tile = row % p.row_tiles;
    const int t0 = u0 * p.unit, t1 = min((u0 + n) * p.unit, len);

    bf16x8 q[RT][4];
    const int heads = p.group - tile * RT * kRows;  // of this row, if they are fewer than 16 RT
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      const unsigned ln = fresh(lane), qg = ln / 16, qc = ln % 16 + x * kRows;
      const bool real = (int)qc < heads;
      const uint16_t* from =
          p.q + ((long long)b * p.hq + h * p.group + tile * RT * kRows) * kHeadDim;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // e4m3 keys come as 16 values a lane, two of these pieces
        const unsigned d = E4M3 ? 64 * (j / 2) + 16 * qg + 8 * (j % 2) : 32 * j + 8 * qg;
        u32x4 u = *(const u32x4*)(from + (real ? qc : 0) * kHeadDim + d);
        if (!real) u = u32x4{0, 0, 0, 0};
        q[x][j] = as_bf16x8(u);
      }
    }
    f32x4 o[RT][8];
    float m[RT], l[RT];
#pragma unroll
    for (int x = 0; x < RT; ++x) {
      m[x] = kMinusInf;
      l[x] = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[x][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The table through the scalar cache: a vector load's wait would also wait
    // for every key and value in flight before it.
    typedef const __attribute__((address_space(4))) int32_t* Uniform;
    const Uniform table = (Uniform)(uintptr_t)(p.c.table + (long long)b * p.c.table_pages);
    const int last_column = (t1 - 1) >> p.c.shift;
    auto entry = [&](int t, int i) {
      const int column = (t + i * kTile) >> p.c.shift;
      return table[column < last_column ? column : last_column];
    };
    // Row of a tile's first key; where there is no page one that may be read.
    auto place = [&](int e, int t, int i) {
      const int page = (unsigned)e < (unsigned)p.c.pages ? e : 0;
      return (((long long)page * p.c.hkv + h) << p.c.shift) +
             ((t + i * kTile) & ((1 << p.c.shift) - 1));
    };
    // a wave that has no key of a short row takes one step of masked ones
    int t = t0 + wave * STEP;
    u32x4 k[TILES][KP];
    Piece v[TILES][4];
    uint32_t k_scale[TILES], v_scale[TILES];
    auto load_k = [&](const int* e, int t) {
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const long long r = place(e[i], t, i);
        const char* a = (const char*)p.c.k + r * (E4M3 ? 128 : 256);
#pragma unroll
        for (int j = 0; j < KP; ++j)
          k[i][j] = *(const u32x4*)(a + 64 * j + k_off);
        if (E4M3) k_scale[i] = *(const uint32_t*)(p.c.k_scale + r + 4u * g);
      }
    };
    auto load_v = [&](const char* a, int i, int y) {
      v[i][y] = *(const Piece*)(a + (E4M3 ? 128 : 256) * y + v_off);
    };
    auto load_scale = [&](long long r, int i) {
      if (E4M3) v_scale[i] = *(const uint32_t*)(p.c.v_scale + r + 4u * g);
    };

    // the last step's loads ahead are of its own keys, not waited for
    int t_next = t + kWaves * STEP < t1 ? t + kWaves * STEP : t;
    int now[TILES], next[TILES];
#pragma unroll
    for (int i = 0; i < TILES; ++i) now[i] = entry(t, i);
    load_k(now, t);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < TILES; ++i) {
      const long long r = place(now[i], t, i);
#pragma unroll
      for (int y = 0; y < 4; ++y) load_v((const char*)p.c.v + r * (E4M3 ? 128 : 256), i, y);
      load_scale(r, i);
    }
#pragma unroll
    for (int i = 0; i < TILES; ++i) next[i] = entry(t_next, i);
    do {
      float zs[RT][TILES][4];
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
#pragma unroll
        for (int x = 0; x < RT; ++x) {
          f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < KP; ++j) {
            if (E4M3) {
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const bf16x8 a = bf16_of(k[i][j][2 * y], k[i][j][2 * y + 1]);
                s = mfma16(a, q[x][2 * j + y], s);
              }
            } else {
              s = mfma16(as_bf16x8(k[i][j]), q[x][j], s);
            }
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            zs[x][i][r] = s[r] * kScale;
            if (E4M3) zs[x][i][r] *= scale_of(k_scale[i] >> (8 * r) & 255);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      load_k(next, t_next);
      __builtin_amdgcn_sched_barrier(0);
      // keys behind the end, and those that have no page
      bool whole = t + STEP <= t1;
#pragma unroll
      for (int i = 0; i < TILES; ++i) whole = whole && (unsigned)now[i] < (unsigned)p.c.pages;
      if (!whole) {
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
          const int valid = (unsigned)now[i] < (unsigned)p.c.pages ? t1 - t - i * kTile : 0;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if ((int)(4 * g) + r < valid) continue;
#pragma unroll
            for (int x = 0; x < RT; ++x) zs[x][i][r] = kMinusInf;
            v[i][r] = Piece{};
            if (E4M3) v_scale[i] &= ~(255u << (8 * r));
          }
        }
      }
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        if (p.z && (int)c + x * kRows < heads) {
          float* z = p.z + ((long long)b * p.hq + h * p.group + (tile * RT + x) * kRows) *
                               p.c.capacity() + t;
          const size_t at = (size_t)c * p.c.capacity() + 4 * g;
#pragma unroll
          for (int i = 0; i < TILES; ++i)
            if (t + i * kTile < t1)
              *(f32x4*)(z + i * kTile + at) =
                  f32x4{zs[x][i][0], zs[x][i][1], zs[x][i][2], zs[x][i][3]};
        }
        // The reference of the exponentials follows the maximum only where it is
        // passed by 2^8: the sums are fp32, so it needs not be the maximum.
        float top = zs[x][0][0];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, zs[x][i][r]);
        if (__any(top > m[x] + 8.f)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float to = fmaxf(m[x], top), f = weight_of(m[x], to);
          l[x] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) o[x][i] *= f;
          m[x] = to;
        }
        const float ref = m[x] == kMinusInf ? 0.f : m[x];
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            zs[x][i][r] = fast_exp2(zs[x][i][r] - ref);
            l[x] += zs[x][i][r];
          }
      }
      // the values; each of their registers takes the next step's piece as soon
      // as it has been used
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const long long row = place(next[i], t_next, i);
        float pr[RT][4];
#pragma unroll
        for (int x = 0; x < RT; ++x)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            pr[x][r] = zs[x][i][r];
            if (E4M3) pr[x][r] *= scale_of(v_scale[i] >> (8 * r) & 255);
          }
        load_scale(row, i);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float f[8];
          values(v[i][r], f);
          __builtin_amdgcn_sched_barrier(0);
          load_v((const char*)p.c.v + row * (E4M3 ? 128 : 256), i, r);
#pragma unroll
          for (int x = 0; x < RT; ++x)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[x][e] = mfma4(f[e], pr[x][r], o[x][e]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) now[i] = next[i];
      t += kWaves * STEP;
      t_next = t + kWaves * STEP < t1 ? t + kWaves * STEP : t;
#pragma unroll
      for (int i = 0; i < TILES; ++i) next[i] = entry(t_next, i);
    } while (t < t1);

    // the four waves' keys, joined in their order
    {
      const int to_lane = fresh(lane), to_g = to_lane / 16, to_c = to_lane % 16;
#pragma unroll
      for (int x = 0; x < RT; ++x) {
        l[x] += __shfl_xor(l[x], 16);
        l[x] += __shfl_xor(l[x], 32);
        if (to_g == 0) {
          sm[wave][x * kRows + to_c] = m[x];
          sl[wave][x * kRows + to_c] = l[x];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            so[wave][x * kRows + to_c][8 * (4 * to_g + r) + i] = o[x][i][r];
      }
    }
    __syncthreads();
    const bool done = u0 == 0 && n == row_units;  // the whole row
    const long long slot = 2ll * blockIdx.x + (first_segment ? 0 : 1);
    const int rows = min(RT * kRows, heads);
    for (int i = fresh(tid); i < rows * kHeadDim; i += kThreads) {
      const int rq = i / kHeadDim, d = i % kHeadDim;
      float top = sm[0][rq];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][rq]);
      float sum = 0.f, out = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = weight_of(sm[w][rq], top);
        sum += f * sl[w][rq];
        out += f * so[w][rq][d];
      }
      if (done) {
        write_row(p, (long long)b * p.hq + h * p.group + tile * RT * kRows + rq, d, top, sum, out);
      } else {
        p.part[(slot * p.tile_rows + rq) * kHeadDim + d] = out;
        if (d == 0) {
          p.ml[(slot * p.tile_rows + rq) * 2] = top;
          p.ml[(slot * p.tile_rows + rq) * 2 + 1] = sum;
        }
      }
    }
    __syncthreads();
    first_segment = false;
    at += n;
    left -= n;
  }
}

// One workgroup per query head: the parts of its row, if it has any, eight at a
// time, 32 lanes of 4 elements each, then the eight sums in order.
__global__ __launch_bounds__(kThreads) void decode_join(DecodeParams p) {
  constexpr int kLanes = kHeadDim / 4, kAtOnce = kThreads / kLanes;
  __shared__ long long places[kWaves];
  __shared__ float so[kAtOnce][kHeadDim];
  __shared__ float sl[kAtOnce], st[kAtOnce];
  const int tid = threadIdx.x, b = blockIdx.x / p.hq, hq = blockIdx.x % p.hq;
  const int h = hq / p.group, in_group = hq % p.group;
  const int tile = in_group / p.tile_rows, r = in_group % p.tile_rows;
  const int per_seq = p.c.hkv * p.row_tiles;
  long long units = 0, before = 0;
  for (int i = tid; i < p.batch; i += kThreads) {
    const long long u = (long long)units_of(p, i) * per_seq;
    units += u;
    if (i < b) before += u;
  }
  long long all, all_before;
  scan(units, &all, places);
  scan(before, &all_before, places);
  const int row_units = units_of(p, b);
  if (row_units == 0) {
    if (tid < kHeadDim) write_row(p, blockIdx.x, tid, 0.f, 0.f, 0.f);
    return;
  }
  const int workers = workers_of(all, p.most_workers);
  const long long start = all_before + (long long)(h * p.row_tiles + tile) * row_units;
  const long long stop = start + row_units;
  // the first worker whose share reaches past a unit u: share(w + 1) > u
  auto worker_at = [&](long long u) {
    long long w = u * workers / all;
    while (share(w + 1, all, workers) <= u) ++w;
    while (share(w, all, workers) > u) --w;
    return (int)w;
  };
  const int w0 = worker_at(start), w1 = worker_at(stop - 1);
  if (w0 == w1) return;  // written by decode_kernel
  // in the first worker the row is its last one, unless it is also its first
  auto slot_of = [&](int w) {
    return 2ll * w + (w == w0 && share(w, all, workers) < start ? 1 : 0);
  };
  const int part = tid / kLanes, d = tid % kLanes * 4;
  float top = kMinusInf;
  for (int w = w0 + part; w <= w1; w += kAtOnce)
    top = fmaxf(top, p.ml[(slot_of(w) * p.tile_rows + r) * 2]);
  if (d == 0) st[part] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) top = fmaxf(top, st[i]);
  f32x4 out = f32x4{0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
#pragma unroll 4
  for (int w = w0 + part; w <= w1; w += kAtOnce) {
    const long long at = slot_of(w) * p.tile_rows + r;
    const float f = weight_of(p.ml[at * 2], top);
    const f32x4 x = *(const f32x4*)(p.part + at * kHeadDim + d);
    sum += f * p.ml[at * 2 + 1];
    out += f * x;
  }
  *(f32x4*)&so[part][d] = out;
  if (d == 0) sl[part] = sum;
  __syncthreads();
  if (tid >= kHeadDim) return;
  float o = 0.f, s = 0.f;
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    o += so[i][tid];
    s += sl[i];
  }
  write_row(p, blockIdx.x, tid, top, s, o);
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

// Workgroups that share a batch's units: three a CU, as many as are resident.
constexpr int kMostWorkers = 768;

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

struct Scratch {
  size_t part, ml, stat, z, bytes;
};

// Query heads of a row: one MFMA tile, or two for wider groups, so that these
// read the keys and values half as often.
int tile_rows_of(int group) {
  return group < 2 * kRows ? group : 2 * kRows;
}

Scratch scratch_of(const CacheParams& c, int batch, int hq, bool weights) {
  const size_t rows = 2 * (size_t)kMostWorkers * tile_rows_of(hq / c.hkv);
  Scratch s;
  s.part = 0;
  s.ml = s.part + align256(rows * kHeadDim * 4);
  s.stat = s.ml + align256(rows * 8);
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
  p.o = (uint16_t*)o;
  p.lse = lse;
  p.batch = batch;
  p.hq = hq;
  p.group = hq / c.hkv;
  p.tile_rows = tile_rows_of(p.group);
  p.row_tiles = (p.group + p.tile_rows - 1) / p.tile_rows;
  p.unit = unit_keys(e4m3);
  p.part = (float*)((char*)scratch + s.part);
  p.ml = (float*)((char*)scratch + s.ml);
  p.stat = weights ? (float*)((char*)scratch + s.stat) : nullptr;
  p.z = weights ? (float*)((char*)scratch + s.z) : nullptr;
  // no more workgroups than there can be units
  const long long most = (long long)batch * c.hkv * p.row_tiles *
                         ((c.capacity() + p.unit - 1) / p.unit);
  p.most_workers = most < kMostWorkers ? (int)most : kMostWorkers;
  auto* kernel = p.tile_rows <= kRows ? (e4m3 ? decode_kernel<true, 1> : decode_kernel<false, 1>)
                                      : (e4m3 ? decode_kernel<true, 2> : decode_kernel<false, 2>);
  hipLaunchKernelGGL(kernel, dim3(p.most_workers), dim3(kThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(decode_join, dim3(batch * hq), dim3(kThreads), 0, st, p);
  if ((e = hipGetLastError()) != hipSuccess || !weights) return e;
  const int chunks = (c.capacity() + kThreads - 1) / kThreads;
  hipLaunchKernelGGL(decode_weights, dim3((unsigned)(batch * c.hkv * chunks)), dim3(kThreads), 0,
                     st, p, weights);
  return hipGetLastError();
}
