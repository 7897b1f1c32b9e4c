// Declarations shared by the decoder operators' translation units (4-bit cache, its attention,
// 8-bit linear layers).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "../../include/fgq_decoder.h"
#include "fgq_device.cuh"

namespace fgq {
namespace dec {

// Tokens, features and channels beyond this are refused: kernels round up to tiles, and step past the end, in 32 bits.
constexpr int MAX_SIZE = INT32_MAX - 65535;
inline bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline bool valid_float(int t) { return t == FGQ_F32 || t == FGQ_BF16 || t == FGQ_F16; }
inline bool nonfinite_host(float v) { return !(v - v == 0.0f); }
inline int float_bytes(int t) { return t == FGQ_F32 ? 4 : 2; }
inline bool stride16(int64_t elems, int t) { return (elems * float_bytes(t)) % 16 == 0; }

// FGQ_OK, or what is wrong with a cache.
inline fgq_status check_cache(const fgq_kv_cache* c) {
  if (!c || !c->k_codes || !c->k_params || !c->v_codes || !c->v_params) return FGQ_ERR_ARG;
  if (c->pages <= 0 || c->page_size <= 0 || c->page_size % 16 != 0 || c->kv_heads <= 0) return FGQ_ERR_ARG;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return FGQ_ERR_ARG;
  if ((c->group != 32 && c->group != 64 && c->group != 128) || c->head_dim % c->group != 0) return FGQ_ERR_ARG;
  if (!aligned(c->k_codes, 16) || !aligned(c->k_params, 16) || !aligned(c->v_codes, 16) || !aligned(c->v_params, 16))
    return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

// The cache as kernels take it.
struct CacheView {
  uint8_t* k_codes;
  uint32_t* k_params;
  uint8_t* v_codes;
  uint32_t* v_params;
  const int32_t* table;  // [B][max_pages]
  int pages, page_size, kv_heads, max_pages;
  int page_shift;  // log2(page_size), or -1
};

inline CacheView view(const fgq_kv_cache* c, const int32_t* table, int max_pages) {
  CacheView v;
  v.k_codes = static_cast<uint8_t*>(c->k_codes);
  v.k_params = static_cast<uint32_t*>(c->k_params);
  v.v_codes = static_cast<uint8_t*>(c->v_codes);
  v.v_params = static_cast<uint32_t*>(c->v_params);
  v.table = table;
  v.pages = c->pages;
  v.page_size = c->page_size;
  v.kv_heads = c->kv_heads;
  v.max_pages = max_pages;
  v.page_shift = -1;
  for (int s = 4; s < 31; ++s)
    if (c->page_size == 1 << s) v.page_shift = s;
  return v;
}

__device__ __forceinline__ uint32_t page_of(const CacheView& c, uint32_t pos) {
  return c.page_shift >= 0 ? pos >> c.page_shift : pos / (uint32_t)c.page_size;
}

// Row (page, head, slot) of position pos of sequence b in the cache's rows, or -1 where the
// position is outside the table or its entry is no page.
__device__ __forceinline__ int64_t cache_row(const CacheView& c, int b, int head, int64_t pos) {
  if (pos < 0 || pos >= (int64_t)c.max_pages * c.page_size) return -1;
  const uint32_t pi = page_of(c, (uint32_t)pos);  // the sum of two int32 values
  const int page = __ldg(c.table + (int64_t)b * c.max_pages + pi);
  if (page < 0 || page >= c.pages) return -1;
  const int slot = (int)(pos - (int64_t)pi * c.page_size);
  return ((int64_t)page * c.kv_heads + head) * c.page_size + slot;
}

// Eight consecutive elements, 16-byte aligned, as fp32, and back.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8], __nv_bfloat16) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(uint4 u, float (&x)[8], __half) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  unpack8(__ldg(reinterpret_cast<const uint4*>(p)), x, T());
}
// The smaller and the larger, NaN where either is.
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t r;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b, __nv_bfloat16) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b, __half) {
  uint32_t r;
  asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b, __half) {
  uint32_t r;
  asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack2(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// Eight elements as loaded, for loads issued ahead of their use; their extremes (NaN where one is).
template <typename T>
struct Raw8 {
  uint4 v;
  __device__ __forceinline__ void extremes(float& lo, float& hi) const {
    const float2 a = unpack2(min2_nan(min2_nan(v.x, v.y, T()), min2_nan(v.z, v.w, T()), T()), T());
    const float2 b = unpack2(max2_nan(max2_nan(v.x, v.y, T()), max2_nan(v.z, v.w, T()), T()), T());
    lo = min_nan(a.x, a.y);
    hi = max_nan(b.x, b.y);
  }
  __device__ __forceinline__ void load(const T* p) { v = __ldg(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void unpack(float (&x)[8]) const { unpack8(v, x, T()); }
};
template <>
struct Raw8<float> {
  float x[8];
  __device__ __forceinline__ void extremes(float& lo, float& hi) const {
    lo = min_nan(min_nan(min_nan(x[0], x[1]), min_nan(x[2], x[3])), min_nan(min_nan(x[4], x[5]), min_nan(x[6], x[7])));
    hi = max_nan(max_nan(max_nan(x[0], x[1]), max_nan(x[2], x[3])), max_nan(max_nan(x[4], x[5]), max_nan(x[6], x[7])));
  }
  __device__ __forceinline__ void load(const float* p) { load8(p, x); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  }
  __device__ __forceinline__ void unpack(float (&y)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
  }
};
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()),
                                            pack2(x[6], x[7], T()));
}
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_float(float v, float& o) { o = v; }
__device__ __forceinline__ void from_float(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_float(float v, __half& o) { o = __float2half_rn(v); }

__device__ __forceinline__ bool nonfinite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }

// rint(fp32(a / b)) for |a / b| < 256, given inv = fp32(1 / b): the product a inv is within 2^-22 of
// the quotient, relatively, so it rounds to the same integer unless it lies within 1e-4 of a half;
// only there (and where inv overflowed) is the division made.
__device__ __forceinline__ float rint_quotient(float a, float b, float inv) {
  const float q = a * inv;
  float r = rintf(q);
  if (!(fabsf(fabsf(q - r) - 0.5f) >= 1e-4f)) r = rintf(__fdiv_rn(a, b));
  return r;
}

// Every thread of the cluster's blocks; shared memory written before is seen after.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}

}  // namespace dec
}  // namespace fgq
