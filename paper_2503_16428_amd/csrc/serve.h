// Internal declarations of the calls for serving after the prefill: rotary
// positions, the paged cache, one new token's attention, eviction.
#pragma once

#include "common.h"

namespace xattn {

// Tokens that a row of the page table can hold, and of a length read from
// device memory the part that it does hold.
__host__ __device__ inline int clamp_len(int len, int capacity) {
  return len < 0 ? 0 : len > capacity ? capacity : len;
}

// Row of a page's token in a [pages][hkv][page] array (page = 1 << shift), or
// -1 where the table's entry is no page. 64 bits: a pool of 2^24 rows of 256
// bytes already passes 32.
__host__ __device__ inline long long page_row(int entry, int pages, int hkv, int head, int shift,
                                              int slot) {
  if ((unsigned)entry >= (unsigned)pages) return -1;
  return (((long long)entry * hkv + head) << shift) + slot;
}

// Page-table column of token t of a sequence, or -1 where the row has none.
__host__ __device__ inline int page_column(long long t, int shift, int table_pages) {
  return t < 0 || (t >> shift) >= table_pages ? -1 : (int)(t >> shift);
}

// Parts of a workspace begin at multiples of 256 bytes.
inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// One array of vectors, [batch][heads][tokens] with strides in elements.
struct Strides {
  long long batch, head, token;
};

// Whether two arrays of vectors with the same sizes and strides have an element in
// common, the second one's first element `apart` elements behind the first one's. From
// the smallest stride on each is at least what the smaller ones span, so that at most
// two multiples of the largest can come as near as the rest reaches, and so on down.
inline bool vectors_meet(long long apart, const Strides& s, int batch, int heads, int tokens) {
  long long stride[3] = {s.batch, s.head, s.token}, size[3] = {batch, heads, tokens};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] > stride[i]) {
        const long long a = stride[i], b = size[i];
        stride[i] = stride[j], size[i] = size[j];
        stride[j] = a, size[j] = b;
      }
  for (int pick = 0; pick < 8; ++pick) {
    long long rest = apart;
    bool inside = true;
    for (int i = 0; i < 3 && inside; ++i) {
      if (size[i] == 1) continue;
      long long n = rest / stride[i] - (rest % stride[i] < 0) + (pick >> i & 1);
      inside = n > -size[i] && n < size[i];
      rest -= n * stride[i];
    }
    if (inside && rest > -kHeadDim && rest < kHeadDim) return true;
  }
  return false;
}

// A plan as the kernels take it (by value): turns per position of each pair, the
// first pairs behind axes 0 and 1, and how many pairs are rotated.
struct RotaryParams {
  double turn[64];
  int axes, end[2], n;
};

// The cache and one batch's page table (by value).
struct CacheParams {
  void *k, *v;
  uint8_t *k_scale, *v_scale;
  const int32_t* table;
  int pages, shift, hkv, table_pages;
  __host__ __device__ int capacity() const { return table_pages << shift; }
};

// Workgroups that share a decode's work: two a CU, or three where rows are many and a
// workgroup often begins a new one, which the others of its CU then make up for. All
// of them have to be resident, or the equal shares take a second turn: of the kernel
// for two tiles of heads (groups of more than 16) a CU holds two. In us, two / three a
// CU, 8 key heads, groups of 4: one sequence of 128K 88 / 92, 4 of 32K 87 / 91, 48 of
// up to 8000 132 / 137, in 8 bits 77 / 82; 64 of up to 8000 178 / 175, 103 / 99, of up
// to 2000 60 / 59, 40 / 36; 64 of 2048, a row each, 86 / 93. Two tiles: 512 sequences
// of up to 4000, 32 / 1 heads, 131 / 144, in 8 bits 94 / 108, all of 4000 184 / 214;
// 1024 of up to 2000 168 / 190; 600 of up to 2500, 20 / 1 heads, 101 / 115. (Any number
// that is no multiple of the CUs gives some of them more work: 384, 103 us at 128K.)
constexpr int kMostWorkers = 768;
inline int decode_workers(int rows, bool two_tiles) {
  return rows >= 512 && !two_tiles ? kMostWorkers : 512;
}

}  // namespace xattn

hipError_t launch_rotary(const void* x, const xattn::Strides& xs, int batch, int heads, int tokens,
                         const int32_t* pos, const xattn::RotaryParams& plan, bool interleaved,
                         bool inverse, void* out, const xattn::Strides& os, hipStream_t st);
hipError_t launch_append(const void* k, const xattn::Strides& ks, const void* v,
                         const xattn::Strides& vs, int batch, int tokens, const int32_t* count,
                         const int32_t* start, const int32_t* pos,
                         const xattn::RotaryParams* plan, bool interleaved,
                         const xattn::CacheParams& c, bool e4m3, hipStream_t st);
size_t decode_scratch_bytes(const xattn::CacheParams& c, bool e4m3, int batch, int hq,
                            bool weights);
hipError_t launch_decode(const void* q, const xattn::CacheParams& c, bool e4m3, int batch, int hq,
                         const int32_t* lens, void* o, float* lse, float* weights, void* scratch,
                         hipStream_t st);
size_t evict_scratch_bytes(const xattn::CacheParams& c, int batch);
hipError_t launch_evict(const xattn::CacheParams& c, bool e4m3, int batch, const int32_t* lens,
                        const float* weights, int budget, int recent, const int32_t* new_table,
                        int new_pages, int32_t* kept, int32_t* new_lens, float* new_weights,
                        void* scratch, hipStream_t st);
