// Linear layers on 8-bit integers: per-token quantization, the product for few tokens, and the C entries.
//
// y[p][m] = scale_p wscale_m sum_k q[p][k] wq[m][k] + bias_m.  int8 values are exact in fp16 and their
// products and sums exact in fp32 below 2^24, so both products run on fp16 matrix instructions (sm_103a's
// integer tensor rate is far below): few tokens here, bound by the weights' bytes, and more in
// gemm_w8a8.cu on tcgen05.
#include <type_traits>

#include "decoder_internal.cuh"
#include "linear_internal.cuh"
#include "kv_attention.cuh"  // matrix instruction, cluster helpers
#include "tc_common.cuh"

namespace fgq {
namespace {

using namespace dec;

// ------------------------------------------------------------------ per-token quantization
// What turns x into its code: rint(fp32(127 x / amax)).
struct TokenScale {
  float pre, amax, inv;  // 127 x overflows for amax above 2^120, 1 / amax for tiny ones: both scaled, exactly
};
__device__ __forceinline__ TokenScale token_scale(float amax) {
  TokenScale t;
  t.pre = amax > 1.329228e36f ? 1.52587890625e-5f : (amax < 8.271806e-25f ? 1.8446744e19f : 1.0f);  // 2^-16, 2^64
  t.amax = amax * t.pre;
  t.inv = __frcp_rn(t.amax);
  return t;
}
__device__ __forceinline__ float token_code(float x, const TokenScale& t) {
  return fminf(fmaxf(rint_quotient(x * t.pre * 127.0f, t.amax, t.inv), -127.0f), 127.0f);
}

// Codes of eight values as fp32 integers plus kMagicF (whose low bits are the integers).  16-bit types: the
// correctly rounded quotients, by the reciprocal RN(1 / amax) and the quotients' exact remainders (Markstein):
// of 127 x by an amax of at most 11 bits, no quotient lies within 2^-12 ulp of a rounding boundary.
template <typename T>
__device__ __forceinline__ void token_codes8(const float (&x)[8], const TokenScale& t, uint32_t (&c)[8]) {
  if constexpr (std::is_same<T, float>::value) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = __float_as_uint(token_code(x[i], t) + kMagicF);
  } else {
    const uint64_t s2 = pack_f2(127.0f * t.pre, 127.0f * t.pre), y2 = pack_f2(t.inv, t.inv);
    const uint64_t b2 = pack_f2(-t.amax, -t.amax), m2 = pack_f2(kMagicF, kMagicF);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t a = mul_f2(pack_f2(x[2 * i], x[2 * i + 1]), s2), q = mul_f2(a, y2);
      float c0, c1;
      unpack_f2(add_f2(fma_f2(fma_f2(q, b2, a), y2, q), m2), c0, c1);
      c[2 * i] = __float_as_uint(c0);
      c[2 * i + 1] = __float_as_uint(c1);
    }
  }
}
__device__ __forceinline__ uint2 pack_codes8(const uint32_t (&c)[8]) {
  return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}

// int8 weights to expand to fp16 rows of `pitch` elements (zero past K) beside the tokens' quantization.
struct Expand {
  const int8_t* src;
  __half* dst;
  int rows, aligned;
};

// Four int8 of w as two fp16 pairs.
__device__ __forceinline__ void s8_to_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  const uint32_t u = w ^ 0x80808080u;
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);  // 1024 + 128 + v
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}
__device__ __forceinline__ void s8_to_h2(uint4 v, uint32_t (&h)[8]) {
  s8_to_h2(v.x, h[0], h[1]), s8_to_h2(v.y, h[2], h[3]), s8_to_h2(v.z, h[4], h[5]), s8_to_h2(v.w, h[6], h[7]);
}

// 16 bytes from row + k of a matrix [base, end), zero from byte K of the row on.  ALIGNED: row + k is 16-byte
// aligned and K a multiple of 16.  Otherwise two aligned loads around them, put right; where those would leave
// the matrix, byte by byte.  READONLY: the data is older than the kernel.
template <bool ALIGNED, bool READONLY>
__device__ __forceinline__ uint4 load16(const int8_t* row, int k, int K, const int8_t* base, const int8_t* end) {
  if (k >= K) return make_uint4(0u, 0u, 0u, 0u);
  if (ALIGNED) {
    const uint4* p = reinterpret_cast<const uint4*>(row + k);
    return READONLY ? __ldg(p) : __ldcg(p);
  }
  const uintptr_t at = reinterpret_cast<uintptr_t>(row + k), lo = at & ~uintptr_t(15);
  uint32_t r[4] = {0u, 0u, 0u, 0u};
  if (lo < reinterpret_cast<uintptr_t>(base) || lo + 32 > reinterpret_cast<uintptr_t>(end)) {
#pragma unroll 1
    for (int i = 0; i < 16 && k + i < K; ++i) {
      const uint32_t v = (uint32_t)(uint8_t)row[k + i] << (8 * (i & 3));
      r[0] |= i < 4 ? v : 0u;
      r[1] |= i >= 4 && i < 8 ? v : 0u;
      r[2] |= i >= 8 && i < 12 ? v : 0u;
      r[3] |= i >= 12 ? v : 0u;
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
  }
  const uint4* p = reinterpret_cast<const uint4*>(lo);
  const uint4 a = READONLY ? __ldg(p) : __ldcg(p), b = READONLY ? __ldg(p + 1) : __ldcg(p + 1);
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  const uint32_t off = (uint32_t)(at & 15);
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = off & 8 ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = off & 4 ? w[i + 1] : w[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = __funnelshift_r(w[i], w[i + 1], 8 * (off & 3));
    const int left = K - k - 4 * i;  // bytes of this word that the row still has
    if (left < 4) r[i] &= left <= 0 ? 0u : (1u << (8 * left)) - 1u;
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}

// One row of int8 as fp16, by one warp.
template <bool ALIGNED>
__device__ __forceinline__ void expand_row(const Expand& e, int row, int K, int64_t pitch, int lane) {
  const int8_t* src = e.src + (int64_t)row * K;
  __half* dst = e.dst + (int64_t)row * pitch;
  const int8_t* end = e.src + (int64_t)e.rows * K;
#pragma unroll 2
  for (int k = 16 * lane; k < pitch; k += 512) {
    uint32_t h[8];
    s8_to_h2(load16<ALIGNED, true>(src, k, K, e.src, end), h);
    *reinterpret_cast<uint4*>(dst + k) = make_uint4(h[0], h[1], h[2], h[3]);
    *reinterpret_cast<uint4*>(dst + k + 8) = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

// WPR warps a token (one where there are many short rows, so that no barrier stands between load and store; eight
// otherwise), 8 / WPR tokens a block: the row's largest magnitude, then its codes.  Rows of up to 256 WPR HELD
// elements are read once and held in registers.  OUT16: codes as fp16 in rows of `pitch` elements, zero past K
// (the operand of gemm_w8a8.cu); else int8 [P][K].  Blocks past the tokens' expand weights, a warp a row.
constexpr int QT_THREADS = 256, QT_WARPS = QT_THREADS / 32;

template <typename T, bool VEC, bool OUT16, int WPR>
__global__ void __launch_bounds__(QT_THREADS) quantize_tokens_kernel(const T* __restrict__ x, int P, int K, int64_t ldx,
                                                                     void* __restrict__ out, int64_t pitch,
                                                                     float* __restrict__ scale, unsigned int* err,
                                                                     const __grid_constant__ Expand e) {
  constexpr int RPB = QT_WARPS / WPR, HELD = WPR == 1 ? 8 : 4, LANES = 32 * WPR;
  __shared__ float red[QT_WARPS];
  pdl_trigger();  // the product may be brought up; it waits for this kernel's end
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int qblocks = (P + RPB - 1) / RPB;
  if ((int)blockIdx.x >= qblocks) {
    for (int row = ((int)blockIdx.x - qblocks) * QT_WARPS + warp; row < e.rows; row += ((int)gridDim.x - qblocks) * QT_WARPS) {
      if (e.aligned)
        expand_row<true>(e, row, K, pitch, lane);
      else
        expand_row<false>(e, row, K, pitch, lane);
    }
    return;
  }
  const int p = blockIdx.x * RPB + warp / WPR;
  const int tid = threadIdx.x % LANES;
  if (p >= P) return;  // with WPR = 8 there is no such block
  const T* row = x + (int64_t)p * ldx;
  float mx = 0.0f;
  Raw8<T> held[VEC ? HELD : 1];
  if constexpr (VEC) {
#pragma unroll
    for (int c = 0; c < HELD; ++c) {
      const int k = 8 * (tid + c * LANES);
      held[c].zero();
      if (k < K) held[c].load(row + k);
    }
    float lo, hi;
#pragma unroll
    for (int c = 0; c < HELD; ++c) {
      held[c].extremes(lo, hi);
      mx = max_nan(mx, max_nan(-lo, hi));
    }
    for (int k = 8 * (tid + HELD * LANES); k < K; k += 8 * LANES) {
      Raw8<T> v;
      v.load(row + k);
      v.extremes(lo, hi);
      mx = max_nan(mx, max_nan(-lo, hi));
    }
  } else {
    for (int k = tid; k < K; k += LANES) mx = max_nan(mx, fabsf(to_float(row[k])));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(FULL_MASK, mx, o));
  if constexpr (WPR > 1) {
    if (lane == 0) red[warp] = mx;
    __syncthreads();
    mx = red[0];
#pragma unroll
    for (int i = 1; i < WPR; ++i) mx = max_nan(mx, red[i]);
  }
  const bool bad = nonfinite(mx);
  const float amax = bad ? 0.0f : mx;
  if (tid == 0) {
    scale[p] = __fdiv_rn(amax, 127.0f);
    if (bad) record_error(err, FGQ_ERR_NONFINITE);
  }
  const TokenScale ts = token_scale(amax);
  auto put8 = [&](int k, const Raw8<T>& raw) {
    float v[8];
    raw.unpack(v);
    uint32_t c[8];
    if (amax > 0.0f) {
      token_codes8<T>(v, ts, c);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = (uint32_t)kMagicI;
    }
    if (OUT16) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(c[i]) - kMagicF;
      store8(static_cast<__half*>(out) + p * pitch + k, f);
    } else {
      *reinterpret_cast<uint2*>(static_cast<int8_t*>(out) + p * pitch + k) = pack_codes8(c);
    }
  };
  if constexpr (VEC) {
#pragma unroll
    for (int c = 0; c < HELD; ++c) {
      const int k = 8 * (tid + c * LANES);
      if (k < K) put8(k, held[c]);
    }
    for (int k = 8 * (tid + HELD * LANES); k < K; k += 8 * LANES) {
      Raw8<T> v;
      v.load(row + k);
      put8(k, v);
    }
    if (OUT16)
      for (int k = K + tid; k < pitch; k += LANES) static_cast<__half*>(out)[p * pitch + k] = __float2half_rn(0.0f);
  } else {
    const int to = OUT16 ? (int)pitch : K;
    for (int k = tid; k < to; k += LANES) {
      const float v = k < K ? to_float(row[k]) : 0.0f;
      const float c = amax > 0.0f && k < K ? token_code(v, ts) : 0.0f;
      if (OUT16)
        static_cast<__half*>(out)[p * pitch + k] = __float2half_rn(c);
      else
        static_cast<int8_t*>(out)[p * pitch + k] = (int8_t)(int)c;
    }
  }
}

template <typename T, bool VEC, bool OUT16>
fgq_status launch_quantize_tokens_w(const T* x, int P, int K, int64_t ldx, void* out, int64_t pitch, float* scale,
                                    const Expand& e, cudaStream_t s) {
  unsigned int* err = device_error_word();
  // blocks for the weights, a warp a row, up to eight of them an SM
  const int64_t most = 8ll * device_sms(), want = ((int64_t)e.rows + QT_WARPS - 1) / QT_WARPS;
  const unsigned eb = (unsigned)(want < most ? want : most);
  if (VEC && P >= 8 * device_sms() && K <= 2048)
    quantize_tokens_kernel<T, VEC, OUT16, 1><<<(P + 7) / 8 + eb, QT_THREADS, 0, s>>>(x, P, K, ldx, out, pitch, scale, err, e);
  else
    quantize_tokens_kernel<T, VEC, OUT16, 8><<<P + eb, QT_THREADS, 0, s>>>(x, P, K, ldx, out, pitch, scale, err, e);
  return after_launch();
}

template <typename T>
fgq_status launch_quantize_tokens_t(const T* x, int P, int K, int64_t ldx, void* out, int64_t pitch, bool out16,
                                    float* scale, const Expand& e, cudaStream_t s) {
  // eight elements at a time: 16-byte aligned input rows, 8-byte aligned int8 rows
  const bool vec = K % 8 == 0 && aligned(x, 16) && (P == 1 || stride16(ldx, sizeof(T) == 4 ? FGQ_F32 : FGQ_BF16)) &&
                   (out16 || (pitch % 8 == 0 && aligned(out, 8)));
  if (vec)
    return out16 ? launch_quantize_tokens_w<T, true, true>(x, P, K, ldx, out, pitch, scale, e, s)
                 : launch_quantize_tokens_w<T, true, false>(x, P, K, ldx, out, pitch, scale, e, s);
  return out16 ? launch_quantize_tokens_w<T, false, true>(x, P, K, ldx, out, pitch, scale, e, s)
               : launch_quantize_tokens_w<T, false, false>(x, P, K, ldx, out, pitch, scale, e, s);
}

fgq_status launch_quantize_tokens(const void* x, int type, int P, int K, int64_t ldx, void* out, int64_t pitch,
                                  bool out16, float* scale, const Expand& e, cudaStream_t s) {
  if (type == FGQ_F32)
    return launch_quantize_tokens_t(static_cast<const float*>(x), P, K, ldx, out, pitch, out16, scale, e, s);
  if (type == FGQ_BF16)
    return launch_quantize_tokens_t(static_cast<const __nv_bfloat16*>(x), P, K, ldx, out, pitch, out16, scale, e, s);
  return launch_quantize_tokens_t(static_cast<const __half*>(x), P, K, ldx, out, pitch, out16, scale, e, s);
}

// int8 tokens and weights as fp16 rows, a warp a row.
__global__ void __launch_bounds__(256) expand_kernel(const __grid_constant__ Expand w, const __grid_constant__ Expand q, int K,
                                                     int64_t pitch) {
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  for (int row = blockIdx.x * 8 + (threadIdx.x >> 5); row < w.rows + q.rows; row += gridDim.x * 8) {
    const Expand& e = row < w.rows ? w : q;
    const int r = row < w.rows ? row : row - w.rows;
    if (e.aligned)
      expand_row<true>(e, r, K, pitch, lane);
    else
      expand_row<false>(e, r, K, pitch, lane);
  }
}

// ------------------------------------------------------------------ few tokens
// A block takes 32 output channels, 8 NT tokens and its share of K; its 8 warps take every eighth piece of 64
// reduction elements, weights as the rows of mma.m16n8k16 (two tiles of 16) and tokens as its columns.  Thread
// (g, t) of a warp loads 16 consecutive bytes of rows g, g + 8, g + 16 and g + 24 (and of token g): they are its
// operands of four k-steps, the order of k being free as long as both sides agree.  Four pieces' weights
// (16 loads a thread; two with 32 tokens, whose sums need the registers) are under way at any time, the first ones
// before the tokens are there.  The warps' sums
// are joined in shared memory; K is split over a cluster of up to 8 blocks where channels alone leave SMs idle,
// and the cluster joins through shared memory too, always in the same order.
constexpr int FEW_WARPS = 8, FEW_M = 32;

struct FewArgs {
  const void* x;  // float tokens, ldx elements apart, or nullptr:
  int64_t ldx;
  const int8_t* q;  // int8 tokens and their scales
  const float* scale;
  const int8_t* wq;
  const float* wscale;
  const float* bias;
  void* y;
  int P, K, M, ytype, splits;
  unsigned int* err;
  int early;  // the kernel before is this library's quantizer: weights may be loaded while it runs
};

// The tokens' int8 codes in shared memory where the block quantizes them itself: rows a multiple of 16
// bytes long and 64 off a multiple of 128, so that eight rows' pieces meet all banks.
__host__ __device__ constexpr int few_row_bytes(int pieces) { return (64 * pieces + 63) / 128 * 128 + 64; }
// Most pieces of a split block.
__host__ __device__ constexpr int few_pieces(int K, int splits) { return ((K + 63) / 64 + splits - 1) / splits; }

// X: the type of float tokens that the block quantizes itself (a launch and a round trip less), or int8_t for
// tokens that a kernel before has quantized.
template <int NT, bool ALIGNED, typename X>
__global__ void __launch_bounds__(32 * FEW_WARPS, 2) few_tokens_kernel(const __grid_constant__ FewArgs a) {
  constexpr bool FLOAT = !std::is_same<X, int8_t>::value;
  constexpr int NP = 8 * NT, AHEAD = NT >= 4 ? 2 : 4;
  extern __shared__ __align__(16) uint8_t few_smem[];
  float* sums = reinterpret_cast<float*>(few_smem);                        // [warp][token][33]
  uint8_t* codes = few_smem + FEW_WARPS * NP * (FEW_M + 1) * sizeof(float);  // [token][few_row_bytes], FLOAT only
  __shared__ float red[NP][FEW_WARPS], tscale[NP];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int sp = blockIdx.x % a.splits, m0 = blockIdx.x / a.splits * FEW_M, p0 = blockIdx.y * NP;
  const int np = min(NP, a.P - p0);
  const int pieces = (a.K + 63) / 64;
  const int c0 = (int)((int64_t)pieces * sp / a.splits), c1 = (int)((int64_t)pieces * (sp + 1) / a.splits);
  const int8_t* wend = a.wq + (int64_t)a.M * a.K;
  const int8_t* wrow[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) wrow[i] = a.wq + (int64_t)min(m0 + g + 8 * i, a.M - 1) * a.K;
  uint4 w[AHEAD][4];
  auto fetch = [&](int c, uint4 (&v)[4]) {
    const int k = c < c1 ? 64 * c + 16 * t : a.K;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load16<ALIGNED, true>(wrow[i], k, a.K, a.wq, wend);
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) fetch(c0 + warp + i * FEW_WARPS, w[i]);

  const int row_bytes = few_row_bytes(few_pieces(a.K, a.splits));
  if constexpr (FLOAT) {
    const X* x = static_cast<const X*>(a.x) + (int64_t)p0 * a.ldx;
    float mx[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) mx[p] = 0.0f;
    for (int k = 8 * threadIdx.x; k < a.K; k += 8 * 32 * FEW_WARPS) {
      Raw8<X> raw[NP];  // all rows' loads at once
#pragma unroll
      for (int p = 0; p < NP; ++p)
        if (p < np) raw[p].load(x + p * a.ldx + k);
#pragma unroll
      for (int p = 0; p < NP; ++p)
        if (p < np) {
          float lo, hi;
          raw[p].extremes(lo, hi);
          mx[p] = max_nan(mx[p], max_nan(-lo, hi));
        }
    }
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p < np) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mx[p] = max_nan(mx[p], __shfl_xor_sync(FULL_MASK, mx[p], o));
        if (lane == 0) red[p][warp] = mx[p];
      }
    __syncthreads();
    bool bad = false;
    TokenScale ts[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (p < np) {
        float amax = red[p][0];
#pragma unroll
        for (int i = 1; i < FEW_WARPS; ++i) amax = max_nan(amax, red[p][i]);
        if (nonfinite(amax)) {  // the whole row is 0, as the quantizer has it
          bad = true;
          amax = 0.0f;
        }
        if (threadIdx.x == 0) tscale[p] = __fdiv_rn(amax, 127.0f);
        ts[p] = token_scale(amax);
      }
    for (int i = 8 * threadIdx.x; i < 64 * (c1 - c0); i += 8 * 32 * FEW_WARPS) {
      const int k = 64 * c0 + i;
      Raw8<X> raw[NP];
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        raw[p].zero();
        if (p < np && k < a.K) raw[p].load(x + p * a.ldx + k);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p)
        if (p < np) {
          uint2 q = make_uint2(0u, 0u);
          if (ts[p].amax > 0.0f) {
            float v[8];
            raw[p].unpack(v);
            uint32_t c[8];
            token_codes8<X>(v, ts[p], c);
            q = pack_codes8(c);
          }
          *reinterpret_cast<uint2*>(codes + p * row_bytes + i) = q;
        }
    }
    if (bad && threadIdx.x == 0 && blockIdx.x == 0) record_error(a.err, FGQ_ERR_NONFINITE);
    __syncthreads();
  } else {
    pdl_wait();
  }

  float acc[2][NT][4];
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[mt][i][e] = 0.0f;
  const int8_t* qend = a.q + (int64_t)a.P * a.K;
  for (int c = c0 + warp; c < c1; c += FEW_WARPS * AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int ci = c + i * FEW_WARPS;
      if (ci >= c1) break;  // the same for the whole warp
      uint32_t h[4][8];
#pragma unroll
      for (int r = 0; r < 4; ++r) s8_to_h2(w[i][r], h[r]);
      fetch(ci + AHEAD * FEW_WARPS, w[i]);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int p = 8 * nt + g;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (p < np) {
          if constexpr (FLOAT)
            v = *reinterpret_cast<const uint4*>(codes + p * row_bytes + 64 * (ci - c0) + 16 * t);
          else
            v = load16<ALIGNED, false>(a.q + (int64_t)(p0 + p) * a.K, 64 * ci + 16 * t, a.K, a.q, qend);
        }
        uint32_t hx[8];
        s8_to_h2(v, hx);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
          for (int mt = 0; mt < 2; ++mt)
            mma16816(acc[mt][nt], h[2 * mt][2 * s], h[2 * mt + 1][2 * s], h[2 * mt][2 * s + 1], h[2 * mt + 1][2 * s + 1],
                     hx[2 * s], hx[2 * s + 1]);
      }
    }
  }
#pragma unroll
  for (int mt = 0; mt < 2; ++mt)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[(warp * NP + 8 * nt + 2 * t + (e & 1)) * (FEW_M + 1) + 16 * mt + g + 8 * (e >> 1)] = acc[mt][nt][e];
  __syncthreads();
  auto put = [&](int i, float v) {  // sum i = token * 32 + channel
    const int tok = i / FEW_M, m = m0 + i % FEW_M, p = p0 + tok;
    if (m >= a.M || p >= a.P) return;
    // as gemm_w8a8.cu has it: the two kernels give the same bits wherever the sums are exact
    v = fmaf(v, (FLOAT ? tscale[tok] : __ldcg(a.scale + p)) * __ldg(a.wscale + m), a.bias ? __ldg(a.bias + m) : 0.0f);
    store_typed(a.y, a.ytype, (int64_t)p * a.M + m, v);
  };
#pragma unroll
  for (int n = 0; n < NP * FEW_M / (32 * FEW_WARPS); ++n) {
    const int i = threadIdx.x + n * 32 * FEW_WARPS;
    float* at = sums + i / FEW_M * (FEW_M + 1) + i % FEW_M;
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < FEW_WARPS; ++k) v += at[k * NP * (FEW_M + 1)];
    if (a.splits == 1)
      put(i, v);
    else
      *at = v;  // the first warp's place: no other thread reads it in this loop
  }
  if (a.splits > 1) {
    cluster_sync();
    for (int i = threadIdx.x + 32 * FEW_WARPS * sp; i < np * FEW_M; i += 32 * FEW_WARPS * a.splits) {
      float v = 0.0f;
      for (int k = 0; k < a.splits; ++k) v += ld_cluster(sums + i / FEW_M * (FEW_M + 1) + i % FEW_M, k);
      put(i, v);
    }
    cluster_sync();  // no block leaves while another may read its sums
  }
}

constexpr int FEW_MAX_CODES = 65536;  // bytes of codes that a block quantizes itself, at most

template <int NT, bool ALIGNED, typename X>
fgq_status launch_few_kernel(const FewArgs& a, cudaStream_t s) {
  constexpr bool FLOAT = !std::is_same<X, int8_t>::value;
  constexpr int SUMS = FEW_WARPS * 8 * NT * (FEW_M + 1) * 4;
  const int smem = SUMS + (FLOAT ? 8 * NT * few_row_bytes(few_pieces(a.K, a.splits)) : 0);
  if (!tc::smem_attr_once<few_tokens_kernel<NT, ALIGNED, X>>(SUMS + (FLOAT ? FEW_MAX_CODES : 0))) return FGQ_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((a.M + FEW_M - 1) / FEW_M * a.splits), (unsigned)((a.P + 8 * NT - 1) / (8 * NT)));
  cfg.blockDim = dim3(32 * FEW_WARPS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  unsigned n = 0;
  if (a.early) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (a.splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)a.splits;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return after_launch(cudaLaunchKernelEx(&cfg, few_tokens_kernel<NT, ALIGNED, X>, a));
}

template <int NT, typename X>
fgq_status launch_few_nt(const FewArgs& a, cudaStream_t s) {
  return a.K % 16 == 0 && (a.x || aligned(a.q, 16)) && aligned(a.wq, 16) ? launch_few_kernel<NT, true, X>(a, s)
                                                                         : launch_few_kernel<NT, false, X>(a, s);
}

// Blocks that share a K: about two blocks an SM, each with 16 pieces at least (two a warp).
int few_splits(int P, int K, int M, int nt) {
  const int64_t blocks = (int64_t)((M + FEW_M - 1) / FEW_M) * ((P + 8 * nt - 1) / (8 * nt));
  int splits = 1;
  while (splits < 8 && blocks * splits * 2 <= 2 * device_sms() && (K + 63) / 64 >= 32 * splits) splits *= 2;
  return splits;
}
int few_nt(int P) { return P <= 8 ? 1 : (P <= 16 ? 2 : 4); }

fgq_status launch_few(FewArgs a, cudaStream_t s) {
  const int nt = few_nt(a.P);
  a.splits = few_splits(a.P, a.K, a.M, nt);
  // more tokens than a grid has rows of blocks for (only without features, whose bias any number of tokens takes here)
  const int most = 65535 * 8 * nt;
  for (; a.P > most; a.P -= most) {
    FewArgs part = a;
    part.P = most;
    const fgq_status st = launch_few_nt<4, int8_t>(part, s);
    if (st != FGQ_OK) return st;
    a.scale += most;
    a.y = static_cast<uint8_t*>(a.y) + (int64_t)most * a.M * float_bytes(a.ytype);
  }
  return nt == 1 ? launch_few_nt<1, int8_t>(a, s) : nt == 2 ? launch_few_nt<2, int8_t>(a, s) : launch_few_nt<4, int8_t>(a, s);
}

// 16-bit tokens that each block quantizes for itself: rows that can be loaded eight elements at a time, codes that fit
// beside the sums, and few elements, as every block has all of the rows' maxima to find.  It saves the caller a launch and a
// temporary and costs the device time.  Calls from Python one after another, so and with a quantizing launch of their own: one and
// two tokens, 4096 -> 4096, 12.5 us both, four, 2048 -> 2000, 9.5 and 10.8, eight, 1024 -> 1024, 8.4 and 10.3 (up to 4 us
// saved where the host is slower); the same calls from a graph, weights from HBM: 9.9 and 8.8, 10.2 and 9.0, 7.0 and 5.6, 6.6
// and 4.0.  With 16384 elements, or fp32 ones, both are slower so: four tokens, 4096 -> 4096, 14.4 and 12.6 (11.4 and 9.0),
// four fp32 ones, 2048 -> 2000, 12.4 and 10.5 (10.4 and 5.9).
constexpr int FUSED_MAX_P = 8, FUSED_MAX_ELEMS = 8192;
bool fused_fits(const void* x, int type, int P, int K, int M, int64_t ldx) {
  return type != FGQ_F32 && P <= FUSED_MAX_P && (int64_t)P * K <= FUSED_MAX_ELEMS && K % 8 == 0 && aligned(x, 16) &&
         (P == 1 || stride16(ldx, type)) && 8 * few_row_bytes(few_pieces(K, few_splits(P, K, M, 1))) <= FEW_MAX_CODES;
}
// Whether outputs take the place of tokens: blocks that quantize for themselves would read what others have written.
bool outputs_over_tokens(const void* x, const void* y, int type, int P, int K, int M, int64_t ldx) {
  const uintptr_t xb = reinterpret_cast<uintptr_t>(x), yb = reinterpret_cast<uintptr_t>(y);
  const uint64_t xn = ((uint64_t)(P - 1) * (P > 1 ? ldx : 0) + K) * float_bytes(type), yn = (uint64_t)P * M * float_bytes(type);
  return xb < yb + yn && yb < xb + xn;
}
fgq_status launch_few_float(FewArgs a, int type, cudaStream_t s) {
  a.splits = few_splits(a.P, a.K, a.M, 1);
  return type == FGQ_BF16 ? launch_few_nt<1, __nv_bfloat16>(a, s) : launch_few_nt<1, __half>(a, s);
}

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// Tokens up to which the few-token kernel runs, in us here and on tcgen05: 64 tokens, 4096 -> 4096 19.8 and 25.0, 1024 ->
// 8192 17.1 and 18.3, 8192 -> 1024 15.0 and 25.0; 80 tokens 29.0 and 25.1, 22.1 and 18.6, 20.6 and 25.0.
constexpr int FEW_MAX_P = 64;

fgq_status check_product(const void* x, int P, int K, const int8_t* wq, const float* wscale, int M, const float* bias,
                         const void* y, int ytype) {
  if (P < 0 || K < 0 || M < 0 || !valid_float(ytype)) return FGQ_ERR_ARG;
  if (P == 0 || M == 0) return FGQ_OK;
  if (P > MAX_SIZE || K > MAX_SIZE || M > MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
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
  if (P > dec::MAX_SIZE || K > dec::MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
  if (!scale || (K > 0 && (!x || !q))) return FGQ_ERR_ARG;
  if (!dec::aligned(x, dec::float_bytes(type)) || !dec::aligned(scale, 4)) return FGQ_ERR_ALIGN;
  return launch_quantize_tokens(x, type, P, K, ldx, q, K, false, scale, Expand{}, stream);
}

fgq_status fgq_gemm_w8a8(const int8_t* q, const float* scale, int P, int K, const int8_t* wq, const float* wscale,
                         int M, const float* bias, void* y, fgq_float_type ytype, cudaStream_t stream) {
  const fgq_status st = check_product(q, P, K, wq, wscale, M, bias, y, ytype);
  if (st != FGQ_OK || P == 0 || M == 0) return st;
  if (!scale) return FGQ_ERR_ARG;
  if (!dec::aligned(scale, 4)) return FGQ_ERR_ALIGN;
  if (P > FEW_MAX_P && K > 0) {
    const GemmPlan plan = plan_gemm_w8a8(P, K, M);
    const size_t w_bytes = up256((size_t)M * plan.pitch * 2), q_bytes = up256((size_t)P * plan.pitch * 2);
    uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(w_bytes + q_bytes + plan.part_bytes, stream));
    if (!tmp) return FGQ_ERR_CUDA;
    const bool k16 = K % 16 == 0;
    const Expand we = {wq, reinterpret_cast<__half*>(tmp), M, k16 && dec::aligned(wq, 16)};
    const Expand qe = {q, reinterpret_cast<__half*>(tmp + w_bytes), P, k16 && dec::aligned(q, 16)};
    const int64_t blocks = ((int64_t)P + M + 7) / 8, most = 8ll * device_sms();
    expand_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, stream>>>(we, qe, K, plan.pitch);
    fgq_status r = after_launch();
    if (r == FGQ_OK)
      r = launch_gemm_w8a8(plan, qe.dst, we.dst, reinterpret_cast<float*>(tmp + w_bytes + q_bytes), scale, P, wscale, M, bias,
                           y, ytype, stream);
    if (cudaFreeAsync(tmp, stream) != cudaSuccess && r == FGQ_OK) r = FGQ_ERR_CUDA;
    return r;
  }
  const FewArgs a = {nullptr, 0, q, scale, wq, wscale, bias, y, P, K, M, ytype, 1, nullptr, 0};
  return launch_few(a, stream);
}

fgq_status fgq_linear_w8a8(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const int8_t* wq,
                           const float* wscale, int M, const float* bias, void* y, cudaStream_t stream) {
  fgq_status st = check_product(x, P, K, wq, wscale, M, bias, y, type);
  if (st == FGQ_OK && P > 1 && ldx < K) st = FGQ_ERR_ARG;
  if (st != FGQ_OK || P == 0 || M == 0) return st;
  if (!dec::aligned(x, dec::float_bytes(type))) return FGQ_ERR_ALIGN;
  if (K > 0 && fused_fits(x, type, P, K, M, ldx) && !outputs_over_tokens(x, y, type, P, K, M, ldx)) {
    const FewArgs a = {x, ldx, nullptr, nullptr, wq, wscale, bias, y, P, K, M, type, 1, device_error_word(), 0};
    return launch_few_float(a, type, stream);
  }
  const bool few = P <= FEW_MAX_P || K == 0;
  const GemmPlan plan = few ? GemmPlan{} : plan_gemm_w8a8(P, K, M);
  const size_t q_bytes = up256((size_t)P * (few ? (int64_t)K : 2 * plan.pitch)), s_bytes = up256((size_t)P * 4);
  const size_t w_bytes = few ? 0 : up256((size_t)M * plan.pitch * 2);
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(q_bytes + s_bytes + w_bytes + plan.part_bytes, stream));
  if (!tmp) return FGQ_ERR_CUDA;
  float* scale = reinterpret_cast<float*>(tmp + q_bytes);
  if (few) {
    st = launch_quantize_tokens(x, type, P, K, ldx, tmp, K, false, scale, Expand{}, stream);
    if (st == FGQ_OK) {
      const FewArgs a = {nullptr, 0, reinterpret_cast<const int8_t*>(tmp), scale, wq, wscale, bias, y, P, K, M, type, 1, nullptr, 1};
      st = launch_few(a, stream);
    }
  } else {
    // tokens to fp16 codes and weights to fp16 in one launch
    __half* w16 = reinterpret_cast<__half*>(tmp + q_bytes + s_bytes);
    const Expand we = {wq, w16, M, K % 16 == 0 && dec::aligned(wq, 16)};
    st = launch_quantize_tokens(x, type, P, K, ldx, tmp, plan.pitch, true, scale, we, stream);
    if (st == FGQ_OK)
      st = launch_gemm_w8a8(plan, tmp, w16, reinterpret_cast<float*>(tmp + q_bytes + s_bytes + w_bytes), scale, P, wscale, M,
                            bias, y, type, stream);
  }
  if (cudaFreeAsync(tmp, stream) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

}  // extern "C"
