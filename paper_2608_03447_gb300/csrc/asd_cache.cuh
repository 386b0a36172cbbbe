// libasd: what the cache entry points share: the checked view of one layer of a
// paged cache, 16-bit and 32-bit storage types, and division by the page size.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "asd.h"

namespace asd_detail {

// ---------------------------------------------------------------- storage types

template <typename T> struct Store;
template <> struct Store<float> {
  static __device__ __forceinline__ float widen(float v) { return v; }
  static __device__ __forceinline__ float narrow(float v) { return v; }
};
template <> struct Store<__nv_bfloat16> {
  static __device__ __forceinline__ float widen(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
};
template <> struct Store<__half> {
  static __device__ __forceinline__ float widen(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
};

inline size_t store_bytes(int dtype) { return dtype == ASD_F32 ? 4 : 2; }

// ---------------------------------------------------------------- pages

// Division of a slot number (0 <= s < 2^31) by the page size: a shift where it
// is a power of two, a 64-bit product with ceil(2^(31 + w) / d) otherwise, which
// is exact for 31-bit numerators (w: the bits of d - 1).
struct PageDiv {
  uint64_t mul;
  int shift;
  int size;
  __host__ __device__ __forceinline__ int quot(int s) const {
    return mul ? static_cast<int>((static_cast<uint64_t>(static_cast<uint32_t>(s)) * mul) >> shift) : s >> shift;
  }
};

inline PageDiv page_div(int size) {
  PageDiv d = {0, 0, size};
  int w = 0;
  while ((1ll << w) < size) ++w;
  d.shift = w;
  if ((1ll << w) != size) {
    d.shift = 31 + w;
    d.mul = ((1ull << d.shift) + static_cast<uint64_t>(size) - 1) / static_cast<uint64_t>(size);
  }
  return d;
}

// One layer of a cache, as the kernels see it.
struct CacheView {
  char* k;
  char* v;
  long long page_stride, token_stride, head_stride;  // elements
  const int32_t* table;
  int table_width;
  int pages;
  int slots;  // that a request's row of the table covers (clamped to 2^31 - 1)
  PageDiv div;
};

// The element offset of a slot of request b (head 0), or -1 where its page id
// is out of range. slot < slots. The page table is read by ordinary loads: a
// page's entry serves its slots.
__device__ __forceinline__ long long slot_offset(const CacheView& c, int b, int slot) {
  const int at = c.div.quot(slot);
  const int page = c.table[static_cast<long long>(b) * c.table_width + at];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(c.pages)) return -1;
  return page * c.page_stride + static_cast<long long>(slot - at * c.div.size) * c.token_stride;
}

// ---------------------------------------------------------------- argument checks (host)

inline int check_cache(const asd_kv_cache* c) {
  if (!c) return ASD_ERR_NULL;
  if (c->dtype != ASD_F32 && c->dtype != ASD_BF16 && c->dtype != ASD_F16) return ASD_ERR_DTYPE;
  if (c->layers < 1 || c->pages < 0 || c->page_size < 1 || c->heads < 1 || c->head_dim < 1 ||
      c->head_dim > ASD_MAX_HEAD_DIM || c->B < 0 || c->table_width < 0)
    return ASD_ERR_SHAPE;
  if (c->layer_stride < 0 || c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0) return ASD_ERR_SHAPE;
  if (c->pages > 0 && (!c->k || !c->v)) return ASD_ERR_NULL;
  if (c->B > 0 && c->table_width > 0 && !c->page_table) return ASD_ERR_NULL;
  const size_t es = store_bytes(c->dtype);
  if (reinterpret_cast<uintptr_t>(c->k) % es != 0 || reinterpret_cast<uintptr_t>(c->v) % es != 0 ||
      reinterpret_cast<uintptr_t>(c->page_table) % 4 != 0)
    return ASD_ERR_ALIGN;
  return ASD_OK;
}

inline CacheView cache_view(const asd_kv_cache* c, int layer) {
  CacheView w = {};
  const long long at = layer * c->layer_stride * static_cast<long long>(store_bytes(c->dtype));
  w.k = static_cast<char*>(c->k) + at;
  w.v = static_cast<char*>(c->v) + at;
  w.page_stride = c->page_stride;
  w.token_stride = c->token_stride;
  w.head_stride = c->head_stride;
  w.table = c->page_table;
  w.table_width = c->table_width;
  w.pages = c->pages;
  const long long slots = static_cast<long long>(c->table_width) * c->page_size;
  w.slots = slots > 0x7fffffffll ? 0x7fffffff : static_cast<int>(slots);
  w.div = page_div(c->page_size);
  return w;
}

// Whether rows that start at p with these strides (elements of es bytes) can be
// read in words of `bytes`.
inline bool rows_aligned(const void* p, size_t es, size_t bytes, long long s0, long long s1, long long s2) {
  const long long n = static_cast<long long>(bytes / es);
  return reinterpret_cast<uintptr_t>(p) % bytes == 0 && s0 % n == 0 && s1 % n == 0 && s2 % n == 0;
}

}  // namespace asd_detail
