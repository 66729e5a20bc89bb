// Attention of one new token per sequence over a paged cache, split over the
// length and joined.
//
// A wave takes 16 keys of a key head against up to 16 of its query heads:
//   S^T = K Q^T  by 16x16x32 bf16 MFMAs: lane (g, c) = (lane / 16, lane % 16)
//     supplies K's row c and Q's row c, and receives queries c, keys 4g .. 4g+3;
//   O^T += V^T P^T  by 16x16x32 bf16 MFMAs over two tiles: P stays in the lane
//     where the softmax left it (keys 4g .. 4g+3 of both tiles are the lane's 8
//     values of the contraction), and of V the lane loads elements 8c .. 8c+7 of
//     those same keys, so that the i-th elements of its 8 pieces are row c of the
//     A operand of MFMA i, whose output rows are elements 8c + i: pairs of values
//     are put together within the lane, nothing moves between lanes.
// P is the sum of three bf16 values, one MFMA each (products exact), which is P in
// fp32 at three sixteenths of the time of fp32 MFMAs. (Two are off by up to 2^-15; the
// third costs nothing where loads bound: 64 sequences of up to 8000 tokens 173.8 ->
// 174.0 us, 128K 87.1 -> 86.5, rows of 2048 in 8 bits 36.7 -> 37.3; with two tiles of
// heads in 8 bits 41.4 -> 44.2.)
//
// Short rows (sequence, key head, tile of query heads) are one workgroup's each. The
// work of longer ones is the batch's rows end to end, in units of kWaves wave steps;
// every workgroup takes an equal share of the units, whatever the lengths, and goes
// through the rows in it. A row that one workgroup has whole is done there; of the
// others every share leaves a partial output (at most two a workgroup: its first and
// its last row), and decode_join adds them in order.
//
// Bound by HBM: with tiles filled up to 16 heads and P in three parts 32 flops a byte
// of bf16 keys and values, which keeps the matrix cores busy for 8 to 9 % of the time
// that the loads take. 64 sequences of up to 8000 tokens, 32 / 8 heads, 1.08 GB:
// 171 us in decode_kernel (6.3 TB/s; a kernel that only loads does 6.2 to 7.0), 5.8
// in decode_join; one of 128K 82 + 5; e4m3, 16 of up to 20,011, 28 / 4 heads, with
// weights 38 + 9. About 6 us of each are the chain of first loads and the end.
#include "serve.h"

using namespace xattn;

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kTile = 16;  // keys of a tile
constexpr int kRows = 16;  // query heads of a tile
constexpr float kScale = 0.08838834764831845f * kLog2e;  // to log2, 1 / sqrt(128)
constexpr float kMinusInf = -__builtin_inff();

constexpr int kTiles = 2;  // of a wave's step: the 32 keys of a PV MFMA
constexpr int kUnit = kTile * kTiles * kWaves;

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
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
// p and q as sums of three bf16 values each: the upper halves of their bits, those of
// what is left, and what is left then, at most the last eight bits of a mantissa. No
// part of a positive weight is 0, so that an infinite value times it is infinite: the
// lower two are at least 2^-30 p each, and their sum is off by no more than that makes.
struct Split {
  uint32_t upper, middle, lower;
};
__device__ __forceinline__ Split split(float p, float q) {
  const auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
  const auto upper = [](float x) {
    return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffff0000u);
  };
  const auto pack = [&](float x, float y) {
    return __builtin_amdgcn_perm(bits(y), bits(x), 0x07060302u);
  };
  const float least_p = p * 0x1p-30f, least_q = q * 0x1p-30f;
  const float a = fmaxf(p - upper(p), least_p), b = fmaxf(q - upper(q), least_q);
  return Split{pack(p, q), pack(a, b),
               pack(fmaxf(a - upper(a), least_p), fmaxf(b - upper(b), least_q))};
}
// Elements 2n and 2n + 1 (n = 0 .. 3) of a lane's four rows of a tile, in bf16:
// rows 0, 1 and rows 2, 3 of the one, then of the other.
__device__ __forceinline__ void columns(const u32x4* v, int n, uint32_t* even, uint32_t* odd) {
  even[0] = __builtin_amdgcn_perm(v[1][n], v[0][n], 0x05040100u);
  even[1] = __builtin_amdgcn_perm(v[3][n], v[2][n], 0x05040100u);
  odd[0] = __builtin_amdgcn_perm(v[1][n], v[0][n], 0x07060302u);
  odd[1] = __builtin_amdgcn_perm(v[3][n], v[2][n], 0x07060302u);
}
__device__ __forceinline__ void columns(const u32x2* v, int n, uint32_t* even, uint32_t* odd) {
  // bytes 2n, 2n + 1 of rows 0, 1 and of rows 2, 3: of the one, then of the other
  const uint32_t pick = n % 2 ? 0x07030602u : 0x05010400u;
  const uint32_t a = __builtin_amdgcn_perm(v[1][n / 2], v[0][n / 2], pick);
  const uint32_t b = __builtin_amdgcn_perm(v[3][n / 2], v[2][n / 2], pick);
  const auto bits = [](auto x) { return __builtin_bit_cast(uint32_t, x); };
  even[0] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false));
  even[1] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false));
  odd[0] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true));
  odd[1] = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true));
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

struct DecodeParams {
  CacheParams c;
  const uint16_t* q;
  const int32_t* lens;
  uint16_t* o;
  float* lse;    // or NULL
  int batch, hq, group, row_tiles, tile_rows;
  int most_workers;  // or 0: every row is one workgroup's
  // 1 / (2^8 times the table's tokens), a factor of the weights in the values' product:
  // no sum of it then passes the largest value
  float least;
  float* part;   // [2 workers][tile_rows][128] unnormalised outputs
  float* ml;     // [2 workers][tile_rows][2] (maximum in log2, sum)
  float* stat;   // [batch][hq][2] (maximum in log2, sum) of whole rows, or NULL
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

// How `units` are shared out: the first `more` workgroups have per + 1 of them,
// the others per; no more workgroups than half the units (one key head, 64K: 20.4
// -> 16.8 us for the fewer parts to join).
struct Shares {
  int workers, per, more;
  __device__ Shares(int units, int most) {
    workers = min((units + 1) / 2, most);
    per = workers ? (unsigned)units / (unsigned)workers : 0;
    more = units - workers * per;
  }
  __device__ int first(int worker) const { return worker * per + min(worker, more); }
  __device__ int worker_of(int unit) const {
    const int early = more * (per + 1);
    const bool is_early = unit < early;
    const unsigned from = is_early ? unit : unit - early;
    return (int)(from / (unsigned)(is_early ? per + 1 : per)) + (is_early ? 0 : more);
  }
};

__device__ __forceinline__ int len_of(const DecodeParams& p, int b) {
  return clamp_len(p.lens[b], p.c.capacity());
}
// Units of a sequence's rows (all of its key heads and tiles of heads).
__device__ __forceinline__ int units_of(const DecodeParams& p, int b) {
  return (len_of(p, b) + kUnit - 1) / kUnit * (p.c.hkv * p.row_tiles);
}

// Sums over the wave's lanes up to this one, by moves within rows of 16 lanes and
// from row to row: short code, which every launch fetches anew.
__device__ __forceinline__ int scan_of_wave(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // 1, 2, 4, 8 lanes up
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 of rows 0, 2 up
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2, 3
  return x;
}
__device__ __forceinline__ int sum_of_wave(int x) {
  return __builtin_amdgcn_readlane(scan_of_wave(x), kWave - 1);
}

// Four elements of a finished row: output head `head`, elements d .. d + 3.
__device__ __forceinline__ void write_row(const DecodeParams& p, long long head, int d, float top,
                                          float sum, f32x4 out) {
  const float inv = sum == 0.f ? 0.f : 1.f / (sum * p.least);
  typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
  const bf16x4 r = {(__bf16)(out[0] * inv), (__bf16)(out[1] * inv), (__bf16)(out[2] * inv),
                    (__bf16)(out[3] * inv)};
  *(bf16x4*)(p.o + head * kHeadDim + d) = r;
  if (d != 0) return;
  if (p.lse) p.lse[head] = sum == 0.f ? kMinusInf : (top + log2f(sum)) / kLog2e;
  if (p.stat) {
    p.stat[2 * head] = top;
    p.stat[2 * head + 1] = sum;
  }
}

// WHOLE: a workgroup has a row, and nothing is left to join.
template <bool E4M3, int RT, bool WHOLE>
__global__ __launch_bounds__(kThreads, RT == 1 ? 3 : 2) void decode_kernel(DecodeParams p) {
  constexpr int TILES = kTiles, KP = E4M3 ? 2 : 4;  // 16-byte pieces of a lane's key
  constexpr int STEP = TILES * kTile;
  using Piece = typename PieceOf<E4M3>::type;  // 8 values
  __shared__ __attribute__((aligned(16))) float so[kWaves][RT * kRows][kHeadDim + 4];
  __shared__ float sm[kWaves][RT * kRows], sl[kWaves][RT * kRows];
  const int tid = threadIdx.x, lane = tid % kWave;
  const unsigned g = lane / 16, c = lane % 16;
  // the lane's piece of a tile's keys and values, bytes
  const uint32_t k_off = c * (E4M3 ? 128 : 256) + 16 * g;
  const uint32_t v_off = E4M3 ? 512 * g + 8 * c : 1024 * g + 16 * c;
  const int wave = uniform(tid / kWave);
  const int per_row = p.c.hkv * p.row_tiles;
  int b, at, left, len;  // the sequence, units into it, units to do, its length
  if constexpr (WHOLE) {
    b = (unsigned)blockIdx.x / (unsigned)per_row;
    const int row = blockIdx.x - b * per_row;
    len = uniform(len_of(p, b));
    left = (len + kUnit - 1) / kUnit;
    at = row * left;
    if (left == 0) {  // no key
      const int h = RT == 1 ? row : (unsigned)row / (unsigned)p.row_tiles;
      const int first = RT == 1 ? 0 : (row - h * p.row_tiles) * RT * kRows;
      const int rows = min(RT * kRows, p.group - first);
      for (int i = tid; i < rows * (kHeadDim / 4); i += kThreads)
        write_row(p, (long long)b * p.hq + h * p.group + first + i / (kHeadDim / 4),
                  i % (kHeadDim / 4) * 4, 0.f, 0.f, f32x4{0.f, 0.f, 0.f, 0.f});
    }
  } else {
    // This workgroup's share, and the sequence that it begins in. Every wave finds
    // out for itself, without a barrier: its lanes have equal runs of the batch.
    const int run = (p.batch + kWave - 1) / kWave;
    const int b0 = min(lane * run, p.batch), b1 = min(b0 + run, p.batch);
    int mine = 0, my_len = 0;
    for (int i = b0; i < b1; ++i) {
      my_len = len_of(p, i);
      mine += (my_len + kUnit - 1) / kUnit * per_row;
    }
    const int before = scan_of_wave(mine);
    const Shares shares(__builtin_amdgcn_readlane(before, kWave - 1), p.most_workers);
    if ((int)blockIdx.x >= shares.workers) return;
    const int begin = shares.first(blockIdx.x);
    left = shares.first(blockIdx.x + 1) - begin;
    const int holder = __ffsll((unsigned long long)__ballot(begin < before)) - 1;
    int my_b = b0, my_at = begin - (before - mine);
    if (lane == holder && run > 1)
      for (;; ++my_b) {
        my_len = len_of(p, my_b);
        const int u = (my_len + kUnit - 1) / kUnit * per_row;
        if (my_at < u) break;
        my_at -= u;
      }
    b = __builtin_amdgcn_readlane(my_b, holder);
    at = __builtin_amdgcn_readlane(my_at, holder);
    len = __builtin_amdgcn_readlane(my_len, holder);
  }
  bool first_segment = true;

  while (left > 0) {
    const int row_units = (len + kUnit - 1) / kUnit;
    if (at >= row_units * per_row) {
      at = 0;
      len = uniform(len_of(p, ++b));
      continue;
    }
    const int row = (unsigned)at / (unsigned)row_units, u0 = at - row * row_units;
    const int n = min(left, row_units - u0);
    // groups of one tile of MFMA columns are one tile
    const int h = RT == 1 ? row : (unsigned)row / (unsigned)p.row_tiles;
    const int tile = RT == 1 ? 0 : row - h * p.row_tiles;
    const int t0 = u0 * kUnit, t1 = min((u0 + n) * kUnit, len);

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
    // Values pass the caches by: 7 % faster. (Keys, of which a load has halves of
    // lines, are slower that way; brought to LDS in whole lines they are as fast on
    // long rows and 12 % slower on short ones.)
    auto load_v = [&](const char* a, int i, int y) {
      v[i][y] = __builtin_nontemporal_load((const Piece*)(a + (E4M3 ? 128 : 256) * y + v_off));
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
      u32x4 upper[RT], middle[RT], lower[RT];
#pragma unroll
      for (int x = 0; x < RT; ++x)
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            zs[x][i][r] *= E4M3 ? p.least * scale_of(v_scale[i] >> (8 * r) & 255) : p.least;
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const Split w = split(zs[x][i][2 * r], zs[x][i][2 * r + 1]);
            upper[x][2 * i + r] = w.upper;
            middle[x][2 * i + r] = w.middle;
            lower[x][2 * i + r] = w.lower;
          }
        }
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        uint32_t e[4], f[4];
        columns(v[0], n, e, f);
        columns(v[1], n, e + 2, f + 2);
        const bf16x8 even = as_bf16x8(u32x4{e[0], e[1], e[2], e[3]});
        const bf16x8 odd = as_bf16x8(u32x4{f[0], f[1], f[2], f[3]});
#pragma unroll
        for (int x = 0; x < RT; ++x) {
#pragma unroll
          for (const u32x4& part : {upper[x], middle[x], lower[x]}) {
            o[x][2 * n] = mfma16(even, as_bf16x8(part), o[x][2 * n]);
            o[x][2 * n + 1] = mfma16(odd, as_bf16x8(part), o[x][2 * n + 1]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const long long row = place(next[i], t_next, i);
#pragma unroll
        for (int y = 0; y < 4; ++y) load_v((const char*)p.c.v + row * (E4M3 ? 128 : 256), i, y);
        load_scale(row, i);
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
    const bool done = WHOLE || (u0 == 0 && n == row_units);  // the whole row
    const long long slot = 2ll * blockIdx.x + (first_segment ? 0 : 1);
    const int rows = min(RT * kRows, heads);
    constexpr int kLanes = kHeadDim / 4;  // threads of a head, four elements each
    for (int i = fresh(tid); i < rows * kLanes; i += kThreads) {
      const int rq = i / kLanes, d = i % kLanes * 4;
      float top = sm[0][rq];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm[w][rq]);
      float sum = 0.f;
      f32x4 out = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = weight_of(sm[w][rq], top);
        sum += f * sl[w][rq];
        out += f * *(const f32x4*)&so[w][rq][d];
      }
      if (done) {
        write_row(p, (long long)b * p.hq + h * p.group + tile * RT * kRows + rq, d, top, sum, out);
      } else {
        *(f32x4*)(p.part + (slot * p.tile_rows + rq) * kHeadDim + d) = out;
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

// Where a row's parts lie: of workgroup `first` in its slot 0 or 1, of the
// others up to `last` in slot 0; none where one workgroup had the whole row.
struct Parts {
  int first, last, slot;
  __device__ long long at(int worker) const {
    return 2ll * worker + (worker == first ? slot : 0);
  }
};

// The parts of sequence b's row (key head and tile of heads). Every wave for itself.
__device__ __forceinline__ Parts parts_of(const DecodeParams& p, int b, int row) {
  if (p.most_workers == 0) return Parts{0, 0, 0};
  int all = 0, before = 0;
  for (int i = threadIdx.x % kWave; i < p.batch; i += kWave) {
    const int u = units_of(p, i);
    all += u;
    if (i < b) before += u;
  }
  const Shares shares(sum_of_wave(all), p.most_workers);
  const int row_units = (len_of(p, b) + kUnit - 1) / kUnit;
  const int start = sum_of_wave(before) + row * row_units;
  Parts r;
  r.first = shares.worker_of(start);
  r.last = shares.worker_of(start + row_units - 1);
  r.slot = shares.first(r.first) < start;
  return r;
}

// Threads of decode_join: half as many are 2 us faster for 2048 heads, others alike.
constexpr int kJoin = 128, kJoinWaves = kJoin / kWave;
// One workgroup per query head: the parts of its row, if it has any, four at a
// time, 32 lanes of 4 elements each, then the four sums in order.
__device__ __forceinline__ void join(const DecodeParams& p, int head) {
  constexpr int kLanes = kHeadDim / 4, kAtOnce = kJoin / kLanes;
  __shared__ __attribute__((aligned(16))) float so[kAtOnce][kHeadDim];
  __shared__ float sf[kMostWorkers], sl[kMostWorkers], st[kJoinWaves];
  const int tid = threadIdx.x, b = head / p.hq, hq = head % p.hq;
  const int h = hq / p.group, in_group = hq % p.group;
  const int tile = in_group / p.tile_rows, r = in_group % p.tile_rows;
  if (len_of(p, b) == 0) {
    if (tid < kLanes) write_row(p, head, 4 * tid, 0.f, 0.f, f32x4{0.f, 0.f, 0.f, 0.f});
    return;
  }
  const Parts parts = parts_of(p, b, h * p.row_tiles + tile);
  const int n = parts.last - parts.first + 1;
  if (n == 1) return;  // written by decode_kernel
  const int lane = tid % kWave, wave = tid / kWave;
  float top = kMinusInf;
  for (int i = tid; i < n; i += kJoin) {
    const float* ml = p.ml + (parts.at(parts.first + i) * p.tile_rows + r) * 2;
    sf[i] = ml[0];
    sl[i] = ml[1];
    top = fmaxf(top, ml[0]);
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) top = fmaxf(top, __shfl_xor(top, off));
  if (lane == 0) st[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kJoinWaves; ++i) top = fmaxf(top, st[i]);
  float sum = 0.f;
  for (int i = tid; i < n; i += kJoin) {
    sf[i] = weight_of(sf[i], top);
    sum += sf[i] * sl[i];
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) sum += __shfl_xor(sum, off);
  __syncthreads();
  if (lane == 0) st[wave] = sum;
  const int part = tid / kLanes, d = tid % kLanes * 4;
  f32x4 out = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int i = part; i < n; i += kAtOnce) {
    const long long at = parts.at(parts.first + i) * p.tile_rows + r;
    out += sf[i] * *(const f32x4*)(p.part + at * kHeadDim + d);
  }
  *(f32x4*)&so[part][d] = out;
  __syncthreads();
  if (tid >= kLanes) return;
  out = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) out += *(const f32x4*)&so[i][d];
  sum = 0.f;
#pragma unroll
  for (int i = 0; i < kJoinWaves; ++i) sum += st[i];
  write_row(p, head, d, top, sum, out);
}

constexpr int kWeightKeys = 4 * kJoin;  // keys of a workgroup's weights

// The weights of 512 keys of a key head, from the products, a tile of its heads
// after the other. First the heads' maxima and sums, four lanes a head.
__device__ __forceinline__ void add_weights(const DecodeParams& p, int chunk, int seq_head,
                                            float* __restrict__ weights) {
  __shared__ float stat[2 * kRows][2];
  const int r = threadIdx.x / 4, sub = threadIdx.x % 4;
  const int b = seq_head / p.c.hkv, h = seq_head % p.c.hkv, capacity = p.c.capacity();
  const int len = len_of(p, b), t = chunk * kWeightKeys + 4 * (int)threadIdx.x;
  if (chunk * kWeightKeys >= len) return;
  // rows are multiples of 16 keys, so that four can be read at the end too
  float* to = weights + (long long)seq_head * capacity + t;
  f32x4 w = f32x4{0.f, 0.f, 0.f, 0.f};
  if (t < len) w = *(const f32x4*)to;
  for (int tile = 0; tile < p.row_tiles; ++tile) {
    const int heads = min(p.tile_rows, p.group - tile * p.tile_rows);
    const long long first = (long long)b * p.hq + h * p.group + tile * p.tile_rows;
    // the first heads' products are on the way while the sums are found
    constexpr int kAhead = 8;
    const float* z = p.z + first * capacity + t;
    f32x4 u[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i < heads && t < len) u[i] = *(const f32x4*)(z + (size_t)i * capacity);
    const Parts parts = parts_of(p, b, h * p.row_tiles + tile);
    float top = kMinusInf, sum = 0.f;
    if (r < heads) {
      if (parts.first == parts.last) {
        top = p.stat[2 * (first + r)];
        sum = sub == 0 ? p.stat[2 * (first + r) + 1] : 0.f;
      } else {
#pragma unroll 4
        for (int x = parts.first + sub; x <= parts.last; x += 4) {
          const float* ml = p.ml + (parts.at(x) * p.tile_rows + r) * 2;
          const float m = ml[0], l = ml[1], to = fmaxf(top, m);
          sum = sum * weight_of(top, to) + l * weight_of(m, to);
          top = to;
        }
      }
    }
#pragma unroll
    for (int off = 1; off < 4; off <<= 1) {
      const float m = __shfl_xor(top, off), l = __shfl_xor(sum, off), to = fmaxf(top, m);
      sum = sum * weight_of(top, to) + l * weight_of(m, to);
      top = to;
    }
    __syncthreads();
    if (sub == 0 && r < heads) {
      stat[r][0] = sum == 0.f ? 0.f : top;
      stat[r][1] = sum == 0.f ? 0.f : 1.f / sum;
    }
    __syncthreads();
    if (t >= len) continue;
    f32x4 sums = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](f32x4 x, int i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[e] += fast_exp2(x[e] - stat[i][0]) * stat[i][1];
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (i < heads) add(u[i], i);
#pragma unroll 4
    for (int i = kAhead; i < heads; ++i) add(*(const f32x4*)(z + (size_t)i * capacity), i);
    w += sums;
  }
  if (t >= len) return;
  if (t + 4 <= len) {
    *(f32x4*)to = w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (t + e < len) to[e] = w[e];
}

// The first batch * hq workgroups join a head each; the others add the weights.
__global__ __launch_bounds__(kJoin) void decode_join(DecodeParams p, int chunks,
                                                        float* __restrict__ weights) {
  const int heads = p.most_workers ? p.batch * p.hq : 0, i = blockIdx.x;
  if (i < heads)
    join(p, i);
  else
    add_weights(p, (i - heads) % chunks, (i - heads) / chunks, weights);
}

struct Scratch {
  size_t part, ml, stat, z, bytes;
};

// Query heads of a row: one MFMA tile, or two for wider groups, so that these
// read the keys and values half as often.
int tile_rows_of(int group) {
  return group < 2 * kRows ? group : 2 * kRows;
}

// Whether every row is one workgroup's: where rows are short, or not long and either
// many or e4m3 (half the bytes a key). Then there are no parts and no join, and a
// workspace only for weights. In us a call among others, the launch of the join among
// them, shares and join / whole rows, 32 / 8 heads unless noted, of up to as many keys as
// the table holds:
//    512 keys  1 sequence 11.1 / 9.0, e4m3 10.6 / 8.0; 64 25.0 / 18.0, 19.3 / 12.2;
//              256 69.0 / 51.2, 47.5 / 32.3
//    640 keys  1 sequence 11.5 / 9.7, 8 12.7 / 10.8, 1 of 4 / 1 heads 10.9 / 10.1
//    768 keys  1 sequence 11.1 / 11.1, 8 12.7 / 11.7, 1 of 4 / 1 heads 11.1 / 11.2
//    896 keys  1 sequence 12.1 / 12.9, e4m3 11.6 / 10.5; 8 13.1 / 13.1, 12.1 / 11.2; 1
//              of 4 / 1 heads 11.3 / 12.1, 10.6 / 10.0
//   1024 keys  1 sequence 11.4 / 13.9, e4m3 10.6 / 10.7; 8 13.4 / 14.4, 12.5 / 11.8;
//              64 33.6 / 30.3, 23.1 / 17.6; 256 112.5 / 98.2, 73.7 / 55.4; 64 of 40 / 2
//              heads 23.9 / 16.2, 21.2 / 17.0; 32 of 24 / 24 heads 44.0 / 44.5, 28.4 / 25.8
//   2048 keys  1 sequence 11.3 / 23.8, e4m3 10.5 / 18.6; 64 58.4 / 57.1, 37.0 / 30.5;
//              32 of 24 / 24 heads 73.5 / 85.4, 46.4 / 48.0
// The kernels alone, one sequence of 4 / 1 heads, shares + join / whole rows: 512 keys
// 5.9 + 3.7 / 7.6, 640 5.9 + 3.6 / 8.6, 768 6.0 + 3.6 / 9.7, 896 5.9 + 3.4 / 10.7: the
// second launch's host time makes up for the longer kernel up to 768.
bool whole_rows(const CacheParams& c, bool e4m3, int rows) {
  return c.capacity() <= 768 || (c.capacity() <= 1024 && (e4m3 || rows >= 128));
}

Scratch scratch_of(const CacheParams& c, bool e4m3, int batch, int hq, bool weights) {
  const int group = hq / c.hkv, tile_rows = tile_rows_of(group);
  const int rows = batch * c.hkv * ((group + tile_rows - 1) / tile_rows);
  const size_t parts = whole_rows(c, e4m3, rows) ? 0 : 2 * (size_t)kMostWorkers * tile_rows;
  Scratch s;
  s.part = 0;
  s.ml = s.part + align256(parts * kHeadDim * 4);
  s.stat = s.ml + align256(parts * 8);
  s.z = s.stat + (weights ? align256((size_t)batch * hq * 8) : 0);
  s.bytes = s.z + (weights ? align256((size_t)batch * hq * c.capacity() * 4) : 0);
  return s;
}

}  // namespace

size_t decode_scratch_bytes(const CacheParams& c, bool e4m3, int batch, int hq, bool weights) {
  return scratch_of(c, e4m3, batch, hq, weights).bytes;
}

hipError_t launch_decode(const void* q, const CacheParams& c, bool e4m3, int batch, int hq,
                         const int32_t* lens, void* o, float* lse, float* weights, void* scratch,
                         hipStream_t st) {
  const Scratch s = scratch_of(c, e4m3, batch, hq, weights != nullptr);
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
  p.least = 0x1p-8f;  // the largest weight is up to 2^8
  for (int n = c.capacity(); n > 1; n = (n + 1) / 2) p.least *= 0.5f;
  p.part = (float*)((char*)scratch + s.part);
  p.ml = (float*)((char*)scratch + s.ml);
  p.stat = weights ? (float*)((char*)scratch + s.stat) : nullptr;
  p.z = weights ? (float*)((char*)scratch + s.z) : nullptr;
  const int rows = batch * c.hkv * p.row_tiles;
  const bool whole = whole_rows(c, e4m3, rows);
  // no more workgroups than there can be shares
  const long long units = (long long)rows * ((c.capacity() + kUnit - 1) / kUnit);
  p.most_workers = whole ? 0 : decode_workers(rows, p.tile_rows > kRows);
  if ((units + 1) / 2 < p.most_workers) p.most_workers = (int)((units + 1) / 2);
  void (*const kernels[2][2][2])(DecodeParams) = {
      {{decode_kernel<false, 1, false>, decode_kernel<false, 1, true>},
       {decode_kernel<false, 2, false>, decode_kernel<false, 2, true>}},
      {{decode_kernel<true, 1, false>, decode_kernel<true, 1, true>},
       {decode_kernel<true, 2, false>, decode_kernel<true, 2, true>}}};
  hipLaunchKernelGGL(kernels[e4m3][p.tile_rows > kRows][whole],
                     dim3((unsigned)(whole ? rows : p.most_workers)), dim3(kThreads), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || (whole && !weights)) return e;
  const int chunks = weights ? (c.capacity() + kWeightKeys - 1) / kWeightKeys : 0;
  const int heads = whole ? 0 : batch * hq;
  hipLaunchKernelGGL(decode_join, dim3((unsigned)(heads + batch * c.hkv * chunks)), dim3(kJoin), 0,
                     st, p, chunks, weights);
  return hipGetLastError();
}
