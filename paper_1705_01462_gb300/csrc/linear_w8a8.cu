// Linear layers on 8-bit integers: per-token quantization, the product for few tokens, and the C entries.
//
// y[p][m] = scale_p wscale_m sum_k q[p][k] wq[m][k] + bias_m.  int8 values are exact in fp16 and their
// products and sums exact in fp32 below 2^24, so both products run on fp16 matrix instructions (sm_103a's
// integer tensor rate is far below): few tokens here, bound by the weights' bytes, and more in
// gemm_w8a8.cu on tcgen05.
#include <type_traits>

#include "decoder_internal.cuh"
#include "linear_internal.cuh"
#include "kv_attention.cuh"  // mma16816

namespace fgq {
namespace {

using namespace dec;

// ------------------------------------------------------------------ per-token quantization
// One block per token: the row's largest magnitude, then its codes; a row of up to QT_THREADS * 8 * QT_HELD
// elements is read once and held in registers.  OUT16: codes as fp16 in rows of `pitch` elements, zero past K
// (the operand of gemm_w8a8.cu); else int8 [P][K].
constexpr int QT_THREADS = 256;
constexpr int QT_HELD = 4;

__device__ __forceinline__ float block_max(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(FULL_MASK, v, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < QT_THREADS / 32; ++i) v = fmaxf(v, red[i]);
  return v;
}

// What turns x into its code: rint(fp32(127 x / amax)).
struct TokenScale {
  float pre, amax, inv;  // 127 x can overflow for amax above 2^120: both are scaled down first
};
__device__ __forceinline__ TokenScale token_scale(float amax) {
  TokenScale t;
  t.pre = amax > 1.329228e36f ? 1.52587890625e-5f : 1.0f;
  t.amax = amax * t.pre;
  t.inv = __frcp_rn(t.amax);
  return t;
}
__device__ __forceinline__ float token_code(float x, const TokenScale& t) {
  return fminf(fmaxf(rint_quotient(x * t.pre * 127.0f, t.amax, t.inv), -127.0f), 127.0f);
}

template <typename T, bool VEC, bool OUT16>
__global__ void __launch_bounds__(QT_THREADS) quantize_tokens_kernel(const T* __restrict__ x, int K, int64_t ldx,
                                                                     void* __restrict__ out, int64_t pitch,
                                                                     float* __restrict__ scale, unsigned int* err) {
  __shared__ float red[QT_THREADS / 32];
  const int64_t p = blockIdx.x;
  const T* row = x + p * ldx;
  const int tid = threadIdx.x;
  float mx = 0.0f;
  bool bad = false;
  float held[VEC ? QT_HELD : 1][8];
  if (VEC) {
#pragma unroll
    for (int c = 0; c < QT_HELD; ++c) {
      const int k = 8 * (tid + c * QT_THREADS);
#pragma unroll
      for (int i = 0; i < 8; ++i) held[c][i] = 0.0f;
      if (k < K) load8(row + k, held[c]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mx = fmaxf(mx, fabsf(held[c][i]));
        bad |= nonfinite(held[c][i]);
      }
    }
    for (int k = 8 * (tid + QT_HELD * QT_THREADS); k < K; k += 8 * QT_THREADS) {
      float v[8];
      load8(row + k, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        mx = fmaxf(mx, fabsf(v[i]));
        bad |= nonfinite(v[i]);
      }
    }
  } else {
    for (int k = tid; k < K; k += QT_THREADS) {
      const float v = to_float(row[k]);
      mx = fmaxf(mx, fabsf(v));
      bad |= nonfinite(v);
    }
  }
  bad = __syncthreads_or(bad);
  const float amax = bad ? 0.0f : block_max(mx, red);
  if (tid == 0) {
    scale[p] = __fdiv_rn(amax, 127.0f);
    if (bad) record_error(err, FGQ_ERR_NONFINITE);
  }
  const TokenScale ts = token_scale(amax);
  auto put8 = [&](int k, const float (&v)[8]) {
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = amax > 0.0f ? token_code(v[i], ts) : 0.0f;
    if (OUT16) {
      store8(static_cast<__half*>(out) + p * pitch + k, c);
    } else {
      uint32_t w[2] = {0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)((int)c[i] & 255) << (8 * (i & 3));
      *reinterpret_cast<uint2*>(static_cast<int8_t*>(out) + p * pitch + k) = make_uint2(w[0], w[1]);
    }
  };
  if (VEC) {
#pragma unroll
    for (int c = 0; c < QT_HELD; ++c) {
      const int k = 8 * (tid + c * QT_THREADS);
      if (k < K) put8(k, held[c]);
    }
    for (int k = 8 * (tid + QT_HELD * QT_THREADS); k < K; k += 8 * QT_THREADS) {
      float v[8];
      load8(row + k, v);
      put8(k, v);
    }
    if (OUT16)
      for (int k = K + tid; k < pitch; k += QT_THREADS) static_cast<__half*>(out)[p * pitch + k] = __float2half_rn(0.0f);
  } else {
    const int to = OUT16 ? (int)pitch : K;
    for (int k = tid; k < to; k += QT_THREADS) {
      const float v = k < K ? to_float(row[k]) : 0.0f;
      const float c = amax > 0.0f && k < K ? token_code(v, ts) : 0.0f;
      if (OUT16)
        static_cast<__half*>(out)[p * pitch + k] = __float2half_rn(c);
      else
        static_cast<int8_t*>(out)[p * pitch + k] = (int8_t)(int)c;
    }
  }
}

template <typename T>
fgq_status launch_quantize_tokens_t(const T* x, int P, int K, int64_t ldx, void* out, int64_t pitch, bool out16,
                                    float* scale, cudaStream_t s) {
  // eight elements at a time: 16-byte aligned input rows, 8-byte aligned int8 rows
  const bool vec = K % 8 == 0 && aligned(x, 16) && stride16(ldx, sizeof(T) == 4 ? FGQ_F32 : FGQ_BF16) &&
                   (out16 || (pitch % 8 == 0 && aligned(out, 8)));
  unsigned int* err = device_error_word();
  if (vec && out16)
    quantize_tokens_kernel<T, true, true><<<P, QT_THREADS, 0, s>>>(x, K, ldx, out, pitch, scale, err);
  else if (vec)
    quantize_tokens_kernel<T, true, false><<<P, QT_THREADS, 0, s>>>(x, K, ldx, out, pitch, scale, err);
  else if (out16)
    quantize_tokens_kernel<T, false, true><<<P, QT_THREADS, 0, s>>>(x, K, ldx, out, pitch, scale, err);
  else
    quantize_tokens_kernel<T, false, false><<<P, QT_THREADS, 0, s>>>(x, K, ldx, out, pitch, scale, err);
  return after_launch();
}

fgq_status launch_quantize_tokens(const void* x, int type, int P, int K, int64_t ldx, void* out, int64_t pitch,
                                  bool out16, float* scale, cudaStream_t s) {
  if (type == FGQ_F32)
    return launch_quantize_tokens_t(static_cast<const float*>(x), P, K, ldx, out, pitch, out16, scale, s);
  if (type == FGQ_BF16)
    return launch_quantize_tokens_t(static_cast<const __nv_bfloat16*>(x), P, K, ldx, out, pitch, out16, scale, s);
  return launch_quantize_tokens_t(static_cast<const __half*>(x), P, K, ldx, out, pitch, out16, scale, s);
}

// ------------------------------------------------------------------ few tokens
// A block takes 16 output channels and 8 NT tokens; its 8 warps take every eighth piece of 64 reduction
// elements, weights as the 16 rows of mma.m16n8k16 and tokens as its columns, and join their sums in
// shared memory.  Thread (g, t) of a warp loads 16 consecutive bytes of rows g and g + 8 (and of token g):
// they are its operands of four k-steps, the order of k being free as long as both sides agree.
constexpr int FEW_WARPS = 8;

struct FewArgs {
  const void* x;  // float tokens, ldx elements apart, or nullptr:
  int64_t ldx;
  const int8_t* q;  // int8 tokens and their scales
  const float* scale;
  const int8_t* wq;
  const float* wscale;
  const float* bias;
  void* y;
  int P, K, M, ytype;
  unsigned int* err;
};

// Four int8 of w as two fp16 pairs.
__device__ __forceinline__ void s8_to_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);  // 1024 + 128 + v
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

// 16 bytes from row + k, zero from byte K on; ALIGNED: row + k is 16-byte aligned and K a multiple of 16.
template <bool ALIGNED>
__device__ __forceinline__ uint4 load16(const int8_t* row, int k, int K) {
  if (ALIGNED) return k < K ? __ldg(reinterpret_cast<const uint4*>(row + k)) : make_uint4(0u, 0u, 0u, 0u);
  uint32_t w[4] = {0u, 0u, 0u, 0u};
  if (k + 19 <= K) {  // whole words around the 16 bytes, all inside the row from k - 3 on
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + k);
    const uint32_t sh = 8u * (uint32_t)(at & 3);
    if (sh == 0) {
      const uint32_t* a = reinterpret_cast<const uint32_t*>(at);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __ldg(a + i);
    } else if (k >= 3) {
      const uint32_t* a = reinterpret_cast<const uint32_t*>(at & ~uintptr_t(3));
      uint32_t v[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) v[i] = __ldg(a + i);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(v[i], v[i + 1], sh);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i >> 2] |= (uint32_t)(uint8_t)__ldg(row + k + i) << (8 * (i & 3));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (k + i < K) w[i >> 2] |= (uint32_t)(uint8_t)__ldg(row + k + i) << (8 * (i & 3));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// The tokens' int8 codes in shared memory where the block quantizes them itself: rows a multiple of 16
// bytes long and 64 off a multiple of 128, so that eight rows' pieces meet all banks.
__host__ __device__ constexpr int few_row_bytes(int K) { return (K + 63) / 128 * 128 + 64; }

// X: the type of float tokens that the block quantizes itself (a launch and a round trip less), or int8_t for
// tokens quantized before.
template <int NT, bool ALIGNED, typename X>
__global__ void __launch_bounds__(32 * FEW_WARPS) few_tokens_kernel(const __grid_constant__ FewArgs a) {
  constexpr bool FLOAT = !std::is_same<X, int8_t>::value;
  constexpr int AHEAD = 2;  // pieces of 64 whose weights are loaded ahead
  __shared__ float sums[FEW_WARPS][8 * NT][17];
  __shared__ float red[8 * NT][FEW_WARPS], tscale[8 * NT];
  extern __shared__ __align__(16) uint8_t codes[];  // [8 NT][few_row_bytes(K)], FLOAT only
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int m0 = blockIdx.x * 16, p0 = blockIdx.y * 8 * NT;
  const int np = min(8 * NT, a.P - p0);
  const int8_t* wa = a.wq + (int64_t)min(m0 + g, a.M - 1) * a.K;
  const int8_t* wb = a.wq + (int64_t)min(m0 + g + 8, a.M - 1) * a.K;
  uint4 na[AHEAD], nb[AHEAD];
  int kn = 64 * warp + 16 * t;  // the next piece to load
#pragma unroll
  for (int i = 0; i < AHEAD; ++i, kn += 64 * FEW_WARPS) {
    na[i] = load16<ALIGNED>(wa, kn, a.K);
    nb[i] = load16<ALIGNED>(wb, kn, a.K);
  }
  const int row_bytes = few_row_bytes(a.K);
  if constexpr (FLOAT) {
    const X* x = static_cast<const X*>(a.x) + (int64_t)p0 * a.ldx;
    bool bad = false;
    for (int p = 0; p < np; ++p) {
      float mx = 0.0f;
      for (int k = 8 * threadIdx.x; k < a.K; k += 8 * 32 * FEW_WARPS) {
        float v[8];
        load8(x + p * a.ldx + k, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          mx = fmaxf(mx, fabsf(v[i]));
          if (nonfinite(v[i])) mx = INFINITY;  // the whole row, as the quantizer has it
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(FULL_MASK, mx, o));
      if (lane == 0) red[p][warp] = mx;
    }
    __syncthreads();
    for (int p = 0; p < 8 * NT; ++p) {
      float amax = 0.0f;
      if (p < np) {
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) amax = fmaxf(amax, red[p][w]);
      }
      if (nonfinite(amax)) {
        bad = true;
        amax = 0.0f;
      }
      if (threadIdx.x == 0) tscale[p] = __fdiv_rn(amax, 127.0f);
      const TokenScale ts = token_scale(amax);
      for (int k = 8 * threadIdx.x; k < row_bytes; k += 8 * 32 * FEW_WARPS) {
        uint32_t w[2] = {0u, 0u};
        if (amax > 0.0f && k < a.K) {
          float v[8];
          load8(x + p * a.ldx + k, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i >> 2] |= (uint32_t)((int)token_code(v[i], ts) & 255) << (8 * (i & 3));
        }
        *reinterpret_cast<uint2*>(codes + p * row_bytes + k) = make_uint2(w[0], w[1]);
      }
    }
    if (bad && threadIdx.x == 0) record_error(a.err, FGQ_ERR_NONFINITE);
    __syncthreads();
  }
  float acc[NT][4];
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0.0f;
  auto piece = [&](int k, uint4 va, uint4 vb) {  // 16 bytes of this thread's rows from element k
    uint32_t ha[8], hb[8];
    s8_to_h2(va.x, ha[0], ha[1]), s8_to_h2(va.y, ha[2], ha[3]), s8_to_h2(va.z, ha[4], ha[5]), s8_to_h2(va.w, ha[6], ha[7]);
    s8_to_h2(vb.x, hb[0], hb[1]), s8_to_h2(vb.y, hb[2], hb[3]), s8_to_h2(vb.z, hb[4], hb[5]), s8_to_h2(vb.w, hb[6], hb[7]);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int p = 8 * nt + g;
      uint4 vx;
      if constexpr (FLOAT)
        vx = k < row_bytes ? *reinterpret_cast<const uint4*>(codes + p * row_bytes + k) : make_uint4(0u, 0u, 0u, 0u);
      else
        vx = p < np ? load16<ALIGNED>(a.q + (int64_t)(p0 + p) * a.K, k, a.K) : make_uint4(0u, 0u, 0u, 0u);
      uint32_t hx[8];
      s8_to_h2(vx.x, hx[0], hx[1]), s8_to_h2(vx.y, hx[2], hx[3]), s8_to_h2(vx.z, hx[4], hx[5]), s8_to_h2(vx.w, hx[6], hx[7]);
#pragma unroll
      for (int s = 0; s < 4; ++s)
        mma16816(acc[nt], ha[2 * s], hb[2 * s], ha[2 * s + 1], hb[2 * s + 1], hx[2 * s], hx[2 * s + 1]);
    }
  };
  for (int k0 = 64 * warp; k0 < a.K; k0 += 64 * FEW_WARPS * AHEAD) {
    uint4 ca[AHEAD], cb[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i, kn += 64 * FEW_WARPS) {
      ca[i] = na[i];
      cb[i] = nb[i];
      na[i] = load16<ALIGNED>(wa, kn, a.K);  // zeros past the end
      nb[i] = load16<ALIGNED>(wb, kn, a.K);
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int k = k0 + 64 * FEW_WARPS * i;
      if (k < a.K) piece(k + 16 * t, ca[i], cb[i]);  // the same for the whole warp
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) sums[warp][8 * nt + 2 * t + (i & 1)][g + 8 * (i >> 1)] = acc[nt][i];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * 8 * NT; i += 32 * FEW_WARPS) {
    const int m = m0 + (i & 15), p = p0 + (i >> 4);
    if (m >= a.M || p >= a.P) continue;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < FEW_WARPS; ++w) v += sums[w][i >> 4][i & 15];
    v = v * ((FLOAT ? tscale[i >> 4] : __ldg(a.scale + p)) * __ldg(a.wscale + m));
    if (a.bias) v += __ldg(a.bias + m);
    store_typed(a.y, a.ytype, (int64_t)p * a.M + m, v);
  }
}

template <int NT, typename X>
fgq_status launch_few_nt(const FewArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)((a.M + 15) / 16), (unsigned)((a.P + 8 * NT - 1) / (8 * NT)));
  const int smem = std::is_same<X, int8_t>::value ? 0 : 8 * NT * few_row_bytes(a.K);
  if (a.K % 16 == 0 && (a.x || aligned(a.q, 16)) && aligned(a.wq, 16))
    few_tokens_kernel<NT, true, X><<<grid, 32 * FEW_WARPS, smem, s>>>(a);
  else
    few_tokens_kernel<NT, false, X><<<grid, 32 * FEW_WARPS, smem, s>>>(a);
  return after_launch();
}

fgq_status launch_few(const FewArgs& a, cudaStream_t s) {
  if (a.P <= 8) return launch_few_nt<1, int8_t>(a, s);
  if (a.P <= 16) return launch_few_nt<2, int8_t>(a, s);
  return launch_few_nt<4, int8_t>(a, s);
}

// Float tokens that each block quantizes for itself: up to 8 of them while a block's share (every block has
// all of it to do) stays small, 32 KB of codes, with rows that can be loaded eight elements at a time.
constexpr int FUSED_MAX_P = 8, FUSED_MAX_CODES = 32768;
bool fused_fits(const void* x, int type, int P, int K, int64_t ldx) {
  return P <= FUSED_MAX_P && 8 * few_row_bytes(K) <= FUSED_MAX_CODES && K % 8 == 0 && aligned(x, 16) &&
         (P == 1 || stride16(ldx, type));
}
fgq_status launch_few_float(const FewArgs& a, int type, cudaStream_t s) {
  if (type == FGQ_F32) return launch_few_nt<1, float>(a, s);
  return type == FGQ_BF16 ? launch_few_nt<1, __nv_bfloat16>(a, s) : launch_few_nt<1, __half>(a, s);
}

constexpr int FEW_MAX_P = 32;  // tokens up to which the few-token kernel runs

fgq_status check_product(const void* x, int P, int K, const int8_t* wq, const float* wscale, int M, const float* bias,
                         const void* y, int ytype) {
  if (P < 0 || K < 0 || M < 0 || !valid_float(ytype)) return FGQ_ERR_ARG;
  if (P == 0 || M == 0) return FGQ_OK;
  if (!wscale || !y || (K > 0 && (!x || !wq))) return FGQ_ERR_ARG;
  if (!aligned(wscale, 4) || !aligned(bias, 4) || !aligned(y, float_bytes(ytype))) return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

}  // namespace
}  // namespace fgq

using namespace fgq;

extern "C" {

fgq_status fgq_quantize_tokens(const void* x, fgq_float_type type, int P, int K, int64_t ldx, int8_t* q, float* scale,
                               cudaStream_t stream) {
  if (P < 0 || K < 0 || !dec::valid_float(type) || (P > 1 && ldx < K)) return FGQ_ERR_ARG;
  if (P == 0) return FGQ_OK;
  if (!scale || (K > 0 && (!x || !q))) return FGQ_ERR_ARG;
  if (!dec::aligned(x, dec::float_bytes(type)) || !dec::aligned(scale, 4)) return FGQ_ERR_ALIGN;
  return launch_quantize_tokens(x, type, P, K, ldx, q, K, false, scale, stream);
}

fgq_status fgq_gemm_w8a8(const int8_t* q, const float* scale, int P, int K, const int8_t* wq, const float* wscale,
                         int M, const float* bias, void* y, fgq_float_type ytype, cudaStream_t stream) {
  const fgq_status st = check_product(q, P, K, wq, wscale, M, bias, y, ytype);
  if (st != FGQ_OK || P == 0 || M == 0) return st;
  if (!scale) return FGQ_ERR_ARG;
  if (!dec::aligned(scale, 4)) return FGQ_ERR_ALIGN;
  if (P > FEW_MAX_P && K > 0) return launch_gemm_w8a8(q, nullptr, 0, scale, P, K, wq, wscale, M, bias, y, ytype, stream);
  const FewArgs a = {nullptr, 0, q, scale, wq, wscale, bias, y, P, K, M, ytype, nullptr};
  return launch_few(a, stream);
}

fgq_status fgq_linear_w8a8(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const int8_t* wq,
                           const float* wscale, int M, const float* bias, void* y, cudaStream_t stream) {
  fgq_status st = check_product(x, P, K, wq, wscale, M, bias, y, type);
  if (st == FGQ_OK && P > 1 && ldx < K) st = FGQ_ERR_ARG;
  if (st != FGQ_OK || P == 0 || M == 0) return st;
  if (!dec::aligned(x, dec::float_bytes(type))) return FGQ_ERR_ALIGN;
  if (fused_fits(x, type, P, K, ldx)) {
    const FewArgs a = {x, ldx, nullptr, nullptr, wq, wscale, bias, y, P, K, M, type, device_error_word()};
    return launch_few_float(a, type, stream);
  }
  const bool few = P <= FEW_MAX_P || K == 0;
  const int64_t pitch = few ? K : gemm_w8a8_pitch(K);
  const size_t q_bytes = ((size_t)P * pitch * (few ? 1 : 2) + 255) / 256 * 256;
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(q_bytes + (size_t)P * 4, stream));
  if (!tmp) return FGQ_ERR_CUDA;
  float* scale = reinterpret_cast<float*>(tmp + q_bytes);
  st = launch_quantize_tokens(x, type, P, K, ldx, tmp, pitch, !few, scale, stream);
  if (st == FGQ_OK && few) {
    const FewArgs a = {nullptr, 0, reinterpret_cast<const int8_t*>(tmp), scale, wq, wscale, bias, y, P, K, M, type, nullptr};
    st = launch_few(a, stream);
  } else if (st == FGQ_OK) {
    st = launch_gemm_w8a8(nullptr, tmp, pitch, scale, P, K, wq, wscale, M, bias, y, type, stream);
  }
  if (cudaFreeAsync(tmp, stream) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

}  // extern "C"
