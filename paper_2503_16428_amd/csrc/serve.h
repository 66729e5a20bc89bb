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

// One array of vectors, [batch][heads][tokens] with strides in elements.
struct Strides {
  long long batch, head, token;
};

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
