// Shared declarations of the serving entry points: packed prompts and the paged 4-bit cache.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "../../include/hyperattn.h"
#include "common.cuh"

namespace hyperattn {

// the device status word of the bounded waits (api.cu); 0 or a hyperattn_status
int device_status_word(cudaStream_t st, int** status);

namespace {

constexpr int kGroup = 32;              // numbers that share a scale and a minimum
constexpr int kBlockTokens = 16;        // tokens of a cache block

template <int D>
struct Block {                          // bytes of a cache block (see the header for the order inside)
  static constexpr int kGroups = D / kGroup;
  static constexpr int kBytes = 20 * D;
  static constexpr int kV = 8 * D, kScaleK = 16 * D, kScaleV = 18 * D;
};

struct CacheView {
  uint8_t* pages;
  int num_pages, page, heads;           // page: tokens
};
template <int D>
__device__ __forceinline__ uint8_t* block_at(const CacheView& c, int page, int head, int sub) {
  return c.pages + (((size_t)page * c.heads + head) * (c.page / kBlockTokens) + sub) * Block<D>::kBytes;
}

inline bool bad_cache(const hyperattn_cache& c, int* rc) {
  *rc = HYPERATTN_OK;
  if (!c.pages || c.num_pages <= 0 || c.kv_heads <= 0) *rc = HYPERATTN_INVALID_ARGUMENT;
  else if ((c.d != 64 && c.d != 128) || c.page_tokens <= 0 || c.page_tokens % kBlockTokens || c.page_tokens > 1024) *rc = HYPERATTN_UNSUPPORTED_SHAPE;
  else if ((long long)c.num_pages * c.page_tokens > 0x7fffffffLL) *rc = HYPERATTN_UNSUPPORTED_SHAPE;
  else if (reinterpret_cast<uintptr_t>(c.pages) & 15) *rc = HYPERATTN_MISALIGNED;
  return *rc != HYPERATTN_OK;
}
inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
inline bool bad_stride(long long s) { return s < 0 || s % 8 != 0; }

// two numbers of a 16-bit type as fp32, and back
template <class T> __device__ __forceinline__ float2 to_float2(uint32_t v);
template <> __device__ __forceinline__ float2 to_float2<__nv_bfloat16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
template <> __device__ __forceinline__ float2 to_float2<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
template <class T> __device__ __forceinline__ uint32_t from_float2(float a, float b);
template <> __device__ __forceinline__ uint32_t from_float2<__nv_bfloat16>(float a, float b) {
  __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&t);
}
template <> __device__ __forceinline__ uint32_t from_float2<__half>(float a, float b) {
  __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&t);
}
// first index of an ascending array whose value exceeds x (n: none)
__device__ __forceinline__ int upper_bound(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

}  // namespace
}  // namespace hyperattn
