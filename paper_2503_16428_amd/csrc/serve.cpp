// C ABI of the calls for serving after the prefill: argument validation and
// workspace sizing. Declarations and contracts are in include/xattn.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>

#include "serve.h"
#include "xattn.h"

namespace xattn_host {
extern thread_local char g_err[512];
int fail(int code, const char* fmt, ...);
}  // namespace xattn_host

namespace {

using xattn_host::fail;
using xattn::CacheParams;
using xattn::RotaryParams;
using xattn::Strides;

int ok() {
  xattn_host::g_err[0] = '\0';
  return XATTN_OK;
}

int launched(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(XATTN_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  return ok();
}

int check_aligned(const void* p, const char* name, size_t align) {
  if ((uintptr_t)p % align != 0)
    return fail(XATTN_ERR_ARG, "%s must be aligned to %zu bytes", name, align);
  return XATTN_OK;
}

int check_pointer(const void* p, const char* name, size_t align) {
  if (!p) return fail(XATTN_ERR_ARG, "%s must be non-NULL", name);
  return check_aligned(p, name, align);
}

// Strides of [batch][heads][tokens] vectors; of a dimension of size 1 unused. Those
// of an output keep its vectors apart: from the smallest on, each passes all that
// the ones before it span.
int check_strides(const int64_t* s, const char* name, int batch, int heads, int tokens,
                  bool written, Strides* out) {
  if (!s) return fail(XATTN_ERR_ARG, "the strides of %s are NULL", name);
  const int size[3] = {batch, heads, tokens};
  long long v[3];
  for (int i = 0; i < 3; ++i) {
    v[i] = size[i] == 1 ? 0 : s[i];
    if (v[i] < 0 || v[i] % 8 != 0 || v[i] > (1ll << 40))
      return fail(XATTN_ERR_ARG, "stride %d of %s must be a multiple of 8 from 0 to 2^40 (got %lld)",
                  i, name, (long long)s[i]);
  }
  if (written) {
    int by_stride[3] = {0, 1, 2};
    std::sort(by_stride, by_stride + 3, [&](int a, int b) { return v[a] < v[b]; });
    double span = xattn::kHeadDim;  // elements; a sum may pass 64 bits
    for (int i : by_stride) {
      if (size[i] == 1) continue;
      if ((double)v[i] < span)
        return fail(XATTN_ERR_ARG, "stride %d of the output %s lets its vectors overlap (%lld)", i,
                    name, (long long)s[i]);
      span += (double)v[i] * (size[i] - 1);
    }
  }
  *out = Strides{v[0], v[1], v[2]};
  return XATTN_OK;
}

// The rotation's output: x itself, or no memory of x. It is decided where both have the
// same strides (two slices of one projection, say); others are the caller's to keep apart.
int check_out(const void* x, const Strides& xs, const void* out, const Strides& os, int batch,
              int heads, int tokens) {
  if (xs.batch != os.batch || xs.head != os.head || xs.token != os.token || x == out)
    return XATTN_OK;
  const long long apart = ((long long)(uintptr_t)out - (long long)(uintptr_t)x) / 2;
  if (!xattn::vectors_meet(apart, xs, batch, heads, tokens)) return XATTN_OK;
  return fail(XATTN_ERR_ARG, "out must be x itself or lie apart from it");
}

constexpr double kTurn = 0.15915494309189533576888;  // 1 / 2 pi

int check_plan(const xattn_rotary_plan* plan, RotaryParams* out) {
  if (!plan) return fail(XATTN_ERR_ARG, "plan is NULL");
  if (plan->axes < 1 || plan->axes > 3)
    return fail(XATTN_ERR_ARG, "axes must be 1, 2 or 3 (got %d)", plan->axes);
  if (plan->interleaved != 0 && plan->interleaved != 1)
    return fail(XATTN_ERR_ARG, "interleaved must be 0 or 1 (got %d)", plan->interleaved);
  if (!plan->freq) return fail(XATTN_ERR_ARG, "freq is NULL");
  *out = RotaryParams{};
  int n = 0;
  for (int a = 0; a < 3; ++a) {
    const int pairs = plan->pairs[a];
    if (a < plan->axes ? pairs < 1 || pairs > 64 : pairs != 0)
      return fail(XATTN_ERR_ARG, "pairs[%d] = %d with %d axes", a, pairs, plan->axes);
    if (n + pairs > 64) return fail(XATTN_ERR_ARG, "more than 64 pairs");
    n += pairs;
    if (a < 2) out->end[a] = n;
  }
  // 0 * x is 0 unless x is infinite or NaN
  double finite = 0.0;
  for (int i = 0; i < n; ++i) {
    out->turn[i] = plan->freq[i] * kTurn;
    finite += 0.0 * plan->freq[i];
  }
  if (!(finite == 0.0)) return fail(XATTN_ERR_ARG, "a frequency is not finite");
  out->axes = plan->axes;
  out->n = n;
  return XATTN_OK;
}

int check_tokens(int batch, int heads, int tokens) {
  if (batch < 1 || heads < 1 || tokens < 1)
    return fail(XATTN_ERR_ARG, "sizes must be positive (batch=%d heads=%d tokens=%d)", batch, heads,
                tokens);
  if ((long long)batch * tokens > (1ll << 26) || heads > 65535)
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^26 tokens or 65535 heads");
  return XATTN_OK;
}

int check_cache(const xattn_cache* cache, const int32_t* table, int table_pages, int batch,
                CacheParams* out) {
  if (!cache) return fail(XATTN_ERR_ARG, "cache is NULL");
  int shift = 4;
  while (shift < 8 && cache->page != 1 << shift) ++shift;
  if (cache->page != 1 << shift)
    return fail(XATTN_ERR_ARG, "page must be 16, 32, 64, 128 or 256 (got %d)", cache->page);
  if (cache->pages < 1 || cache->hkv < 1 || cache->head_dim < 1)
    return fail(XATTN_ERR_ARG, "pages, hkv and head_dim must be positive (%d, %d, %d)",
                cache->pages, cache->hkv, cache->head_dim);
  if (cache->head_dim != xattn::kHeadDim)
    return fail(XATTN_ERR_UNSUPPORTED, "head_dim %d not supported (only %d)", cache->head_dim,
                xattn::kHeadDim);
  if (cache->type != XATTN_CACHE_BF16 && cache->type != XATTN_CACHE_E4M3)
    return fail(XATTN_ERR_ARG, "unknown cache type %d", cache->type);
  if (batch < 1) return fail(XATTN_ERR_ARG, "batch must be positive (got %d)", batch);
  if (table_pages < 1)
    return fail(XATTN_ERR_ARG, "the page table must have columns (got %d)", table_pages);
  if ((long long)table_pages << shift > (1ll << 30))
    return fail(XATTN_ERR_UNSUPPORTED, "a page table row of more than 2^30 tokens");
  if ((long long)batch * cache->hkv > 65535 * 16ll)
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^20 sequences times key heads");
  *out = CacheParams{cache->k, cache->v, cache->k_scale, cache->v_scale, table, cache->pages,
                     shift, cache->hkv, table_pages};
  return XATTN_OK;
}

int check_cache_arrays(const xattn_cache* c, const int32_t* table) {
  int rc;
  if ((rc = check_pointer(c->k, "the cache's k", 16)) ||
      (rc = check_pointer(c->v, "the cache's v", 16)) ||
      (rc = check_pointer(table, "table", 4)))
    return rc;
  if (c->type == XATTN_CACHE_E4M3)
    if ((rc = check_pointer(c->k_scale, "the cache's k_scale", 4)) ||
        (rc = check_pointer(c->v_scale, "the cache's v_scale", 4)))
      return rc;
  return XATTN_OK;
}

int check_workspace(const void* workspace, size_t bytes, size_t need) {
  if (need && (!workspace || bytes < need || (uintptr_t)workspace % 16 != 0))
    return fail(XATTN_ERR_WORKSPACE, "a 16-byte aligned workspace of %zu bytes needed, %zu given",
                need, workspace ? bytes : (size_t)0);
  return XATTN_OK;
}

// Arrays that are to lie apart, as far as one of two is written: bytes [at, at + bytes).
struct Extent {
  const char* name;
  const void* at;  // NULL: not given
  size_t bytes;
  bool written;
};
int check_apart(std::initializer_list<Extent> all) {
  for (auto a = all.begin(); a != all.end(); ++a)
    for (auto b = all.begin(); b != a; ++b) {
      if (!a->at || !b->at || !(a->written || b->written)) continue;
      const uintptr_t x = (uintptr_t)a->at, y = (uintptr_t)b->at;
      if (x < y + b->bytes && y < x + a->bytes)
        return fail(XATTN_ERR_ARG, "%s and %s share memory", b->name, a->name);
    }
  return XATTN_OK;
}

int check_decode(const xattn_cache* cache, int batch, int hq, const int32_t* table,
                 int table_pages, CacheParams* c) {
  int rc;
  if ((rc = check_cache(cache, table, table_pages, batch, c))) return rc;
  if (hq < 1 || hq % cache->hkv != 0)
    return fail(XATTN_ERR_ARG, "hq (%d) must be a positive multiple of hkv (%d)", hq, cache->hkv);
  // grids of one workgroup a head, and of one a head and 256 tokens
  if ((long long)batch * hq > (1 << 20) ||
      (long long)batch * cache->hkv * ((c->capacity() + 255) / 256) > (1 << 23))
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^20 query heads or 2^31 cached vectors a batch");
  // units of 128 keys of every row of up to 32 heads, in 32 bits
  const long long tiles = (hq / cache->hkv + 31) / 32;
  if (batch * cache->hkv * tiles * ((c->capacity() + 127) / 128) > (1 << 30))
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^30 units of 128 keys and 32 heads a batch");
  return XATTN_OK;
}

// Bytes of a cache's keys (or values), and of their scales.
size_t vector_bytes(const CacheParams& c, bool e4m3) {
  return ((size_t)c.pages * c.hkv << c.shift) * xattn::kHeadDim * (e4m3 ? 1 : 2);
}
size_t scale_bytes(const CacheParams& c) { return (size_t)c.pages * c.hkv << c.shift; }

int check_evict(const xattn_cache* cache, const int32_t* table, int table_pages, int batch,
                CacheParams* c) {
  if (int rc = check_cache(cache, table, table_pages, batch, c)) return rc;
  if ((long long)batch * cache->hkv * c->capacity() > (1ll << 31))
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^31 cached vectors a batch");
  return XATTN_OK;
}

}  // namespace

extern "C" {

int xattn_rotary(const void* x, const int64_t* x_strides, int batch, int heads, int tokens,
                 int head_dim, const int32_t* pos, const xattn_rotary_plan* plan, int inverse,
                 void* out, const int64_t* out_strides, void* stream) {
  int rc;
  Strides xs, os;
  RotaryParams p;
  if ((rc = check_tokens(batch, heads, tokens))) return rc;
  if (head_dim != xattn::kHeadDim)
    return fail(head_dim < 1 ? XATTN_ERR_ARG : XATTN_ERR_UNSUPPORTED,
                "head_dim %d not supported (only %d)", head_dim, xattn::kHeadDim);
  if (inverse != 0 && inverse != 1)
    return fail(XATTN_ERR_ARG, "inverse must be 0 or 1 (got %d)", inverse);
  if ((rc = check_plan(plan, &p)) ||
      (rc = check_strides(x_strides, "x", batch, heads, tokens, false, &xs)) ||
      (rc = check_strides(out_strides, "out", batch, heads, tokens, true, &os)) ||
      (rc = check_pointer(x, "x", 16)) || (rc = check_pointer(out, "out", 16)) ||
      (rc = check_pointer(pos, "pos", 4)) ||
      (rc = check_out(x, xs, out, os, batch, heads, tokens)))
    return rc;
  return launched(launch_rotary(x, xs, batch, heads, tokens, pos, p, plan->interleaved != 0,
                                inverse != 0, out, os, (hipStream_t)stream),
                  "xattn_rotary");
}

int xattn_cache_append(const void* k, const int64_t* k_strides, const void* v,
                       const int64_t* v_strides, int batch, int tokens, const int32_t* count,
                       const int32_t* start, const int32_t* table, int table_pages,
                       const int32_t* pos, const xattn_rotary_plan* plan,
                       const xattn_cache* cache, void* stream) {
  int rc;
  CacheParams c;
  Strides ks, vs;
  RotaryParams p;
  if ((rc = check_cache(cache, table, table_pages, batch, &c)) ||
      (rc = check_tokens(batch, cache->hkv, tokens)))
    return rc;
  if (!pos != !plan) return fail(XATTN_ERR_ARG, "pos and plan go together");
  if ((plan && (rc = check_plan(plan, &p))) ||
      (rc = check_strides(k_strides, "k", batch, cache->hkv, tokens, false, &ks)) ||
      (rc = check_strides(v_strides, "v", batch, cache->hkv, tokens, false, &vs)) ||
      (rc = check_pointer(k, "k", 16)) || (rc = check_pointer(v, "v", 16)) ||
      (rc = check_pointer(start, "start", 4)) || (rc = check_aligned(count, "count", 4)) ||
      (rc = check_aligned(pos, "pos", 4)) || (rc = check_cache_arrays(cache, table)))
    return rc;
  return launched(launch_append(k, ks, v, vs, batch, tokens, count, start, pos,
                                plan ? &p : nullptr, plan && plan->interleaved, c,
                                cache->type == XATTN_CACHE_E4M3, (hipStream_t)stream),
                  "xattn_cache_append");
}

int xattn_decode_workspace_size(const xattn_cache* cache, int batch, int hq, int table_pages,
                                int weights, size_t* bytes) {
  int rc;
  CacheParams c;
  if ((rc = check_decode(cache, batch, hq, nullptr, table_pages, &c))) return rc;
  if (!bytes) return fail(XATTN_ERR_ARG, "bytes is NULL");
  *bytes = decode_scratch_bytes(c, cache->type == XATTN_CACHE_E4M3, batch, hq, weights != 0);
  return ok();
}

int xattn_decode(const void* q, const xattn_cache* cache, int batch, int hq,
                 const int32_t* table, int table_pages, const int32_t* lens, void* o, float* lse,
                 float* weights, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  CacheParams c;
  if ((rc = check_decode(cache, batch, hq, table, table_pages, &c)) ||
      (rc = check_pointer(q, "q", 16)) || (rc = check_pointer(o, "o", 16)) ||
      (rc = check_pointer(lens, "lens", 4)) || (rc = check_cache_arrays(cache, table)) ||
      (rc = check_aligned(lse, "lse", 4)) || (rc = check_aligned(weights, "weights", 16)))
    return rc;
  const bool e4m3 = cache->type == XATTN_CACHE_E4M3;
  const size_t need = decode_scratch_bytes(c, e4m3, batch, hq, weights != nullptr);
  if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
  const size_t rows = (size_t)batch * hq, vectors = vector_bytes(c, e4m3);
  const size_t q_bytes = rows * xattn::kHeadDim * 2;
  if ((rc = check_apart(
           {{"q", o == q ? nullptr : q, q_bytes, false},  // a head's q is read before its o is written
            {"table", table, (size_t)batch * table_pages * 4, false},
            {"lens", lens, (size_t)batch * 4, false},
            {"the cache's k", c.k, vectors, false},
            {"the cache's v", c.v, vectors, false},
            {"the cache's k_scale", c.k_scale, scale_bytes(c), false},
            {"the cache's v_scale", c.v_scale, scale_bytes(c), false},
            {"o", o, q_bytes, true},
            {"lse", lse, rows * 4, true},
            {"weights", weights, (size_t)batch * c.hkv * c.capacity() * 4, true},
            {"workspace", need ? workspace : nullptr, need, true}})))
    return rc;
  return launched(launch_decode(q, c, e4m3, batch, hq, lens, o, lse, weights, workspace,
                                (hipStream_t)stream),
                  "xattn_decode");
}

int xattn_evict_workspace_size(const xattn_cache* cache, int batch, int table_pages,
                               size_t* bytes) {
  int rc;
  CacheParams c;
  if ((rc = check_evict(cache, nullptr, table_pages, batch, &c))) return rc;
  if (!bytes) return fail(XATTN_ERR_ARG, "bytes is NULL");
  *bytes = evict_scratch_bytes(c, batch);
  return ok();
}

int xattn_cache_evict(const xattn_cache* cache, int batch, const int32_t* table, int table_pages,
                      const int32_t* lens, const float* weights, int budget, int recent,
                      const int32_t* new_table, int new_pages, int32_t* kept, int32_t* new_lens,
                      float* new_weights, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  CacheParams c;
  if ((rc = check_evict(cache, table, table_pages, batch, &c))) return rc;
  if (budget < 1 || recent < 0 || recent > budget)
    return fail(XATTN_ERR_ARG, "1 <= budget and 0 <= recent <= budget (got %d, %d)", budget,
                recent);
  if (new_pages < 1 || ((long long)new_pages << c.shift) < budget)
    return fail(XATTN_ERR_ARG, "%d new pages do not hold a budget of %d", new_pages, budget);
  if ((long long)new_pages << c.shift > (1ll << 30) ||
      (long long)batch * c.hkv * ((budget + 15) / 16) > (1 << 23))
    return fail(XATTN_ERR_UNSUPPORTED, "more than 2^27 kept vectors a batch");
  if ((rc = check_cache_arrays(cache, table)) || (rc = check_pointer(lens, "lens", 4)) ||
      (rc = check_pointer(weights, "weights", 16)) ||
      (rc = check_pointer(new_table, "new_table", 4)) || (rc = check_pointer(kept, "kept", 4)) ||
      (rc = check_pointer(new_lens, "new_lens", 4)) ||
      (rc = check_pointer(new_weights, "new_weights", 4)))
    return rc;
  if (new_table == table) return fail(XATTN_ERR_ARG, "new_table is table");
  const size_t rows = (size_t)batch * c.hkv;
  const size_t need = evict_scratch_bytes(c, batch);
  const bool e4m3 = cache->type == XATTN_CACHE_E4M3;
  if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
  if ((rc = check_apart(
           {{"table", table, (size_t)batch * table_pages * 4, false},
            {"lens", lens, (size_t)batch * 4, false},
            {"weights", weights, rows * c.capacity() * 4, false},
            {"new_table", new_table, (size_t)batch * new_pages * 4, false},
            {"the cache's k", c.k, vector_bytes(c, e4m3), false},
            {"the cache's v", c.v, vector_bytes(c, e4m3), false},
            {"the cache's k_scale", c.k_scale, scale_bytes(c), false},
            {"the cache's v_scale", c.v_scale, scale_bytes(c), false},
            {"kept", kept, rows * budget * 4, true},
            {"new_lens", new_lens, (size_t)batch * 4, true},
            {"new_weights", new_weights, (rows * new_pages << c.shift) * 4, true},
            {"workspace", need ? workspace : nullptr, need, true}})))
    return rc;
  return launched(launch_evict(c, e4m3, batch, lens, weights, budget,
                               recent, new_table, new_pages, kept, new_lens, new_weights,
                               workspace, (hipStream_t)stream),
                  "xattn_cache_evict");
}

}  // extern "C"
