// The 4-bit cache of keys and values: quantization as it is written, and its read-back.
//
// Per group of G values of one token and head: lo = min rounded down to bf16, s = (max - lo) / 15
// rounded up to bf16, codes round((x - lo) / s).  Eight consecutive values, a 16-byte load of 16-bit
// elements, make one 32-bit word of a key row, or two 16-bit units of a value row; the G / 8 threads of
// a group find its extremes by shuffles.  Both kernels move each byte once and are bound by HBM;
// consecutive threads take consecutive values of the dense side, and the 32 to 128 bytes of a cache
// row are written by neighbouring threads, so that L2 merges them into whole sectors.
#include <type_traits>

#include "decoder_internal.cuh"

namespace fgq {
namespace {

using namespace dec;

constexpr int KV_THREADS = 256;

struct KvArgs {
  CacheView c;
  const void* k;
  const void* v;
  void* k_out;
  void* v_out;
  int64_t bs[2], ts[2];  // batch and token strides of k and v, in elements
  const int32_t* starts;
  const int32_t* lens;  // or nullptr
  int B, T;
  unsigned int* err;
};

// bf16 values next to x, as fp32: at or below it, and (x >= 0) at or above it.
__device__ __forceinline__ float bf16_down(float x) {
  const uint32_t u = __float_as_uint(x);
  return __uint_as_float(((u & 0x80000000u) ? u + 0xffffu : u) & 0xffff0000u);
}
__device__ __forceinline__ float bf16_up_pos(float x) {
  return __uint_as_float((__float_as_uint(x) + 0xffffu) & 0xffff0000u);
}

// blockIdx.x: rows (token, head) of a sequence, KV_THREADS / (D / 8) a block; blockIdx.y: sequences
// (strided); blockIdx.z: keys, values.
template <typename T, int D, int G>
__global__ void __launch_bounds__(KV_THREADS) kv_append_kernel(const __grid_constant__ KvArgs a) {
  constexpr int LR = D / 8, GL = G / 8, NB = D / 32, NG = D / G, RPB = KV_THREADS / LR;
  const int of_v = blockIdx.z;
  const int tid = threadIdx.x, u = tid % LR;  // values 8 u .. 8 u + 7 of the row
  const uint32_t r = blockIdx.x * RPB + tid / LR;  // below 2^32: the host checks
  const int t = (int)(r / (uint32_t)a.c.kv_heads), head = (int)(r - (uint32_t)t * (uint32_t)a.c.kv_heads);
  const T* src = static_cast<const T*>(of_v ? a.v : a.k);
  const int64_t bs = of_v ? a.bs[1] : a.bs[0], ts = of_v ? a.ts[1] : a.ts[0];
  uint8_t* codes = of_v ? a.c.v_codes : a.c.k_codes;
  uint32_t* params = of_v ? a.c.v_params : a.c.k_params;
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int n = a.lens ? min(__ldg(a.lens + b), a.T) : a.T;
    const bool live = t < n;  // rows of a warp may differ: every lane takes part in the shuffles
    if (!__any_sync(FULL_MASK, live)) continue;
    float x[8];
    int64_t row = -1;
    if (live) {
      load8(src + b * bs + t * ts + (int64_t)head * D + 8 * u, x);
      row = cache_row(a.c, b, head, (int64_t)__ldg(a.starts + b) + t);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.0f;
    }
    float lo = x[0], hi = x[0];
    bool bad = nonfinite(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      lo = fminf(lo, x[i]);
      hi = fmaxf(hi, x[i]);
      bad |= nonfinite(x[i]);
    }
#pragma unroll
    for (int o = 1; o < GL; o <<= 1) {
      lo = fminf(lo, __shfl_xor_sync(FULL_MASK, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(FULL_MASK, hi, o));
    }
    const uint32_t bads = __ballot_sync(FULL_MASK, bad);
    bad = (bads >> ((tid & 31) & ~(GL - 1)) & (uint32_t)((1ull << GL) - 1)) != 0;
    // differences of values beyond 2^126 may overflow: halves of them do not
    const bool huge = std::is_same<T, __half>::value ? false : fmaxf(fabsf(lo), fabsf(hi)) > 8.507059e37f;
    const float f = huge ? 0.5f : 1.0f;
    const float l = fmaxf(bf16_down(lo * f), huge ? -1.6947657e38f : -3.3895314e38f);
    const float s = bf16_up_pos(fmaxf(__fdiv_rn(hi * f - l, 15.0f), 0.0f));
    const float inv = __frcp_rn(s);
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = s > 0.0f ? rint_quotient(x[i] * f - l, s, inv) : 0.0f;
      c[i] = bad ? 0u : (uint32_t)min(max((int)q, 0), 15);
    }
    if (live && row < 0) record_error(a.err, FGQ_ERR_ARG);
    if (live && bad) record_error(a.err, FGQ_ERR_NONFINITE);
    if (row < 0) continue;  // no shuffle follows before the next any_sync of this warp
    const int j = u >> 2, v = u & 3;  // block of 32, quarter of it
    if (!of_v) {
      const uint32_t w = c[0] | c[2] << 4 | c[4] << 8 | c[6] << 12 | c[1] << 16 | c[3] << 20 | c[5] << 24 | c[7] << 28;
      reinterpret_cast<uint32_t*>(codes)[row * (D / 8) + v * NB + j] = w;
    } else {
      uint16_t* dst = reinterpret_cast<uint16_t*>(codes) + row * (D / 4) + 2 * v * NB + j;
      dst[0] = (uint16_t)(c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12);
      dst[NB] = (uint16_t)(c[4] | c[5] << 4 | c[6] << 8 | c[7] << 12);
    }
    if (u % GL == 0) {
      const float g = huge ? 2.0f : 1.0f;
      params[row * NG + u / GL] =
          bad ? 0u : (__float_as_uint(l * g) & 0xffff0000u) | (__float_as_uint(s * g) >> 16);
    }
  }
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(const __grid_constant__ KvArgs a) {
  constexpr int LR = D / 8, GL = G / 8, NB = D / 32, NG = D / G, RPB = KV_THREADS / LR;
  const int of_v = blockIdx.z;
  const int tid = threadIdx.x, u = tid % LR;
  const uint32_t r = blockIdx.x * RPB + tid / LR;  // below 2^32: the host checks
  const int t = (int)(r / (uint32_t)a.c.kv_heads), head = (int)(r - (uint32_t)t * (uint32_t)a.c.kv_heads);
  if (t >= a.T) return;
  T* dst = static_cast<T*>(of_v ? a.v_out : a.k_out);
  const uint8_t* codes = of_v ? a.c.v_codes : a.c.k_codes;
  const uint32_t* params = of_v ? a.c.v_params : a.c.k_params;
  const int j = u >> 2, v = u & 3;
  for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
    const int n = a.lens ? min(__ldg(a.lens + b), a.T) : a.T;
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
    if (t < n) {
      const int64_t row = cache_row(a.c, b, head, (int64_t)__ldg(a.starts + b) + t);
      if (row < 0) {
        record_error(a.err, FGQ_ERR_ARG);
      } else {
        const uint32_t p = params[row * NG + u / GL];
        const float lo = __uint_as_float(p & 0xffff0000u), s = __uint_as_float(p << 16);
        uint32_t c[8];
        if (!of_v) {
          const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[row * (D / 8) + v * NB + j];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            c[2 * i] = w >> (4 * i) & 15u;
            c[2 * i + 1] = w >> (16 + 4 * i) & 15u;
          }
        } else {
          const uint16_t* cs = reinterpret_cast<const uint16_t*>(codes) + row * (D / 4) + 2 * v * NB + j;
          const uint32_t w = (uint32_t)cs[0] | (uint32_t)cs[NB] << 16;
#pragma unroll
          for (int i = 0; i < 8; ++i) c[i] = w >> (4 * i) & 15u;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(s, (float)c[i], lo);  // s c is exact in fp32
      }
    }
    store8(dst + (((int64_t)b * a.T + t) * a.c.kv_heads + head) * D + 8 * u, x);
  }
}

template <typename T, int D, int G>
fgq_status launch_kv(const KvArgs& a, bool append, cudaStream_t s) {
  constexpr int RPB = KV_THREADS / (D / 8);
  const int64_t rows = (int64_t)a.T * a.c.kv_heads, blocks = (rows + RPB - 1) / RPB;
  if (rows > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)blocks, (unsigned)(a.B < 65535 ? a.B : 65535), 2);
  if (append)
    kv_append_kernel<T, D, G><<<grid, KV_THREADS, 0, s>>>(a);
  else
    kv_read_kernel<T, D, G><<<grid, KV_THREADS, 0, s>>>(a);
  return after_launch();
}

template <typename T>
fgq_status launch_kv_t(const KvArgs& a, int D, int G, bool append, cudaStream_t s) {
  if (D == 64) return G == 32 ? launch_kv<T, 64, 32>(a, append, s) : launch_kv<T, 64, 64>(a, append, s);
  if (D == 128)
    return G == 32   ? launch_kv<T, 128, 32>(a, append, s)
           : G == 64 ? launch_kv<T, 128, 64>(a, append, s)
                     : launch_kv<T, 128, 128>(a, append, s);
  return G == 32   ? launch_kv<T, 256, 32>(a, append, s)
         : G == 64 ? launch_kv<T, 256, 64>(a, append, s)
                   : launch_kv<T, 256, 128>(a, append, s);
}

fgq_status run_kv(const KvArgs& a, int type, int D, int G, bool append, cudaStream_t s) {
  if (type == FGQ_F32) return launch_kv_t<float>(a, D, G, append, s);
  return type == FGQ_BF16 ? launch_kv_t<__nv_bfloat16>(a, D, G, append, s) : launch_kv_t<__half>(a, D, G, append, s);
}

// What both calls ask of their common arguments.
fgq_status check_kv(const fgq_kv_cache* cache, const void* k, const void* v, int type, int B, int T,
                    const int32_t* table, int max_pages, const int32_t* starts, const int32_t* lens) {
  if (B < 0 || T < 0 || max_pages < 0 || !valid_float(type)) return FGQ_ERR_ARG;
  const fgq_status st = check_cache(cache);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  if (!k || !v || !table || !starts) return FGQ_ERR_ARG;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(table, 4) || !aligned(starts, 4) || !aligned(lens, 4))
    return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

}  // namespace
}  // namespace fgq

using namespace fgq;

extern "C" {

fgq_status fgq_kv_append(const fgq_kv_cache* cache, const void* k, const void* v, fgq_float_type type, int B, int T,
                         int64_t k_batch_stride, int64_t k_token_stride, int64_t v_batch_stride,
                         int64_t v_token_stride, const int32_t* page_table, int max_pages, const int32_t* starts,
                         const int32_t* lens, cudaStream_t stream) {
  const fgq_status st = check_kv(cache, k, v, type, B, T, page_table, max_pages, starts, lens);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  if (!dec::stride16(k_batch_stride, type) || !dec::stride16(k_token_stride, type) ||
      !dec::stride16(v_batch_stride, type) || !dec::stride16(v_token_stride, type))
    return FGQ_ERR_ALIGN;
  KvArgs a = {};
  a.c = dec::view(cache, page_table, max_pages);
  a.k = k;
  a.v = v;
  a.bs[0] = k_batch_stride;
  a.bs[1] = v_batch_stride;
  a.ts[0] = k_token_stride;
  a.ts[1] = v_token_stride;
  a.starts = starts;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.err = device_error_word();
  return run_kv(a, type, cache->head_dim, cache->group, true, stream);
}

fgq_status fgq_kv_read(const fgq_kv_cache* cache, void* k, void* v, fgq_float_type type, int B, int T,
                       const int32_t* page_table, int max_pages, const int32_t* starts, const int32_t* lens,
                       cudaStream_t stream) {
  const fgq_status st = check_kv(cache, k, v, type, B, T, page_table, max_pages, starts, lens);
  if (st != FGQ_OK || B == 0 || T == 0) return st;
  KvArgs a = {};
  a.c = dec::view(cache, page_table, max_pages);
  a.k_out = k;
  a.v_out = v;
  a.starts = starts;
  a.lens = lens;
  a.B = B;
  a.T = T;
  a.err = device_error_word();
  return run_kv(a, type, cache->head_dim, cache->group, false, stream);
}

}  // extern "C"
