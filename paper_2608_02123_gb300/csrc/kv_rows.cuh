// What the entry points over rows of several requests share: the description
// of rows and cache (include/pctree.h, "Rows of several requests") on the
// device, and conversions of the two 16-bit types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pctree_common.cuh"

namespace pct {

struct KvRows {
  const int32_t* row_start;
  const int32_t* n_rows;
  const int32_t* prefix_len;
  const int32_t* page_table;   // NULL: request r's only page is page r
  int batch, total_rows, page_size, n_pages, max_pages;
};

// Whether request r's rows and slots lie inside the row tensors and its page
// table.
__device__ __forceinline__ bool kv_request_ok(const KvRows& k, int start, int n, int prefix) {
  return n >= 0 && prefix >= 0 && start >= 0 &&
         static_cast<long long>(start) + n <= k.total_rows &&
         static_cast<long long>(prefix) + n <=
             static_cast<long long>(k.max_pages) * k.page_size;
}

// The page of a request's page-table entry, or -1 if it is no page.
__device__ __forceinline__ int kv_page(const KvRows& k, int r, int entry) {
  const int p = k.page_table == nullptr
                    ? r
                    : k.page_table[static_cast<size_t>(r) * k.max_pages + entry];
  return p >= 0 && p < k.n_pages ? p : -1;
}

// Checks of the sizes the configurations share.
inline pctree_status kv_check(int batch, int total_rows, int Hkv, int page_size, int n_pages,
                              int max_pages, int dtype) {
  if (batch < 1 || total_rows < 1 || Hkv < 1 || page_size < 1 || n_pages < 1 || max_pages < 1)
    return PCTREE_ERR_INVALID_ARG;
  if (dtype != PCTREE_BF16 && dtype != PCTREE_F16) return PCTREE_ERR_INVALID_ARG;
  if (batch > PCTREE_KV_MAX_BATCH || Hkv > 65535 || total_rows > (1 << 30) ||
      page_size > (1 << 30) ||
      static_cast<long long>(max_pages) * page_size > (1ll << 30))
    return PCTREE_ERR_UNSUPPORTED;
  return PCTREE_OK;
}

// A contiguous cache has one page a request.
inline bool kv_table_ok(const int32_t* page_table, int batch, int n_pages, int max_pages) {
  return page_table != nullptr || (n_pages >= batch && max_pages == 1);
}

inline bool kv_al16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <bool F16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
  if constexpr (F16) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  } else {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
}

// Two floats rounded to nearest even, the lower half holding the first.
template <bool F16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if constexpr (F16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
}

}  // namespace pct
