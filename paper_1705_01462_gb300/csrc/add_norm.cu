// Between two blocks of a decoder: the norm of a block's output, its gate and scale, the residual sum, and the norm that the
// next block reads, in one pass over the data.
//
//   u = post(x),  s = r + scale gate u,  y = pre(s);   norm(z) = z' / sqrt(mean z'^2 + eps) weight + bias
//
// A row is held in registers (fp32) from its load to its last store, so each input is read and each output written once:
// the kernel is bound by those bytes, or by instructions where bf16 rows pass both norms and a gate.  The threads of a row each hold up to
// CH pieces of 8 elements, two in a packed register pair; a layer norm takes its mean first and then the squares of what is
// left, so that a large mean costs no bits.  Sums of a row meet in the same order always: in registers, by shuffles, over the
// warps through shared memory.  Rows past 16384 elements are read again for each sum instead (long_kernel).
// 8192 x 4096, device time (floor): fp32 78.7 us (79), bf16 layer norms 42.3 (39.5), bf16 with both norms and a gate for each 2048
// 48.5 (39.5; 57 with unpacked arithmetic, then 49.5).  What did not help there, beside 49.5: a persistent block with the next row's loads under way to
// registers (56) or to a ring in shared memory, which takes the place of the weights in L1 (80); 128 threads a row (57).
#include <cmath>

#include "decoder_internal.cuh"

namespace fgq {
namespace {

using namespace dec;

struct NormArgs {
  const void* x;
  const void* gate;
  const void* r;
  void* s;
  void* y;
  int64_t ldx, ldg, ldr, lds;
  fgq_norm post, pre;
  float scale;
  float part, rest;  // 1 / K: a power of two, which costs no bits, times the rest
  int P, K, tokens_per_gate, has_post, has_pre;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_MASK, v, o);
  return v;
}

// Sum over the NT threads of a row, in all of them.  (What they bring has been divided by about the row's length, so that squares of values up
// to 1e18 stay in fp32's range in rows of any length.)  `red` is the block's; two sums in turn take its two halves, so that
// one barrier a sum is enough.
template <int NT>
__device__ __forceinline__ float row_sum(float v, float (*red)[32], int& turn) {
  v = warp_sum(v);
  if constexpr (NT > 32) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) red[turn][warp] = v;
    __syncthreads();
    v = red[turn][lane & (NT / 32 - 1)];
#pragma unroll
    for (int o = NT / 64; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_MASK, v, o);
    turn ^= 1;
  }
  return v;
}

using f2 = unsigned long long;  // two fp32 values, as the packed instructions take them

// Eight consecutive elements as four pairs.  CONST: of memory that the kernel does not write (weights, gates; x and r may be outputs' places, and go
// past L1, which is left to the weights, unless two pieces share its sectors: 8192 x 4096 fp32 85.7 us so and 90.5 past it, 8192 x 8192
// bf16 93.3 and 88.8).
template <bool CONST>
__device__ __forceinline__ void load_pairs(const float* p, f2 (&v)[4]) {
  ulonglong2 a, b;
  if constexpr (CONST)
    a = __ldg(reinterpret_cast<const ulonglong2*>(p)), b = __ldg(reinterpret_cast<const ulonglong2*>(p) + 1);
  else
    a = reinterpret_cast<const ulonglong2*>(p)[0], b = reinterpret_cast<const ulonglong2*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y;
}
template <bool CONST, typename T>
__device__ __forceinline__ void load_pairs(const T* p, f2 (&v)[4]) {
  const uint4* q = reinterpret_cast<const uint4*>(p);
  const uint4 u = CONST ? __ldg(q) : __ldcg(q);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = unpack2(w[i], T());
    v[i] = pack_f2(f.x, f.y);
  }
}

// Piece c of a row, eight elements of thread tid (VEC: consecutive ones); zeros past the row.
template <typename T, bool VEC, bool CONST>
__device__ __forceinline__ void load_piece(const T* row, int c, int tid, int NT, int K, f2 (&v)[4]) {
  if constexpr (VEC) {
    const int k = 8 * (tid + c * NT);
    if (k < K) {
      load_pairs<CONST>(row + k, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = 0ull;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = tid + (8 * c + 2 * i) * NT;
      v[i] = pack_f2(k < K ? to_float(row[k]) : 0.0f, k + NT < K ? to_float(row[k + NT]) : 0.0f);
    }
  }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_piece(T* row, int c, int tid, int NT, int K, const f2 (&v)[4]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack_f2(v[i], f[2 * i], f[2 * i + 1]);
  if constexpr (VEC) {
    const int k = 8 * (tid + c * NT);
    if (k < K) store8(row + k, f);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = tid + (8 * c + i) * NT;
      if (k < K) from_float(f[i], row[k]);
    }
  }
}

// v to its norm, in registers.  Elements past the row are 0 before and after.
template <int NT, int CH, bool VEC>
__device__ __forceinline__ void normalise(f2 (&v)[CH][4], const NormArgs& args, const fgq_norm& n, int tid, float (*red)[32], int& turn) {
  const int K = args.K;
  float a, b;
  if (n.kind == FGQ_NORM_LAYER) {
    f2 sum = 0ull;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum = add_f2(sum, v[c][i]);
    unpack_f2(sum, a, b);
    const float mean = row_sum<NT>((a + b) * args.part, red, turn) * args.rest;
    const f2 off = pack_f2(-mean, -mean);
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = VEC ? 8 * (tid + c * NT) : tid + (8 * c + 2 * i) * NT;
        v[c][i] = k < K ? add_f2(v[c][i], off) : 0ull;
        if (!VEC && k < K && k + NT >= K) v[c][i] &= 0xffffffffull;  // the second of a pair
      }
  }
  f2 sq = 0ull;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) sq = fma_f2(v[c][i], v[c][i], sq);
  unpack_f2(sq, a, b);
  const float inv = rsqrtf(row_sum<NT>((a + b) * args.part, red, turn) * args.rest + n.eps);
  const f2 inv2 = pack_f2(inv, inv);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[c][i] = mul_f2(v[c][i], inv2);
    f2 w[4];
    if (n.weight) {
      load_piece<float, VEC, true>(n.weight, c, tid, NT, K, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = mul_f2(v[c][i], w[i]);
    }
    if (n.bias) {
      load_piece<float, VEC, true>(n.bias, c, tid, NT, K, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = add_f2(v[c][i], w[i]);
    }
  }
}

// NT threads a row; blocks of at least 128 threads.
// 512 threads with two pieces: three blocks an SM (8192 x 8192 bf16 86 us, 95 with two), of rows that are not 16-byte pieces two (8192 x 8001 155 us, 199
// with three, whose registers spill).
template <typename T, typename R, int NT, int CH, bool VEC>
__global__ void __launch_bounds__(NT < 128 ? 128 : NT, NT == 512 && CH == 2 ? (VEC ? 3 : 2) : 1)
    add_norm_kernel(const __grid_constant__ NormArgs a) {
  constexpr int RPB = NT < 128 ? 128 / NT : 1;
  __shared__ float red[2][32];
  const int tid = threadIdx.x % NT, p = (int)blockIdx.x * RPB + (int)threadIdx.x / NT;
  if (p >= a.P) return;  // whole warps; with one row a block there is no such block
  int turn = 0;
  f2 v[CH][4];
  Raw8<R> raw[VEC ? CH : 1];  // the residual as loaded
  f2 rs[VEC ? 1 : CH][4];
  const T* x = static_cast<const T*>(a.x) + p * a.ldx;
  const R* res = static_cast<const R*>(a.r) + p * a.ldr;
#pragma unroll
  for (int c = 0; c < CH; ++c) load_piece<T, VEC, false>(x, c, tid, NT, a.K, v[c]);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if constexpr (VEC) {
      raw[c].zero();
      if (a.r && 8 * (tid + c * NT) < a.K) raw[c].template load_written<sizeof(T) == 4>(res + 8 * (tid + c * NT));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) rs[c][i] = 0ull;
      if (a.r) load_piece<R, false, false>(res, c, tid, NT, a.K, rs[c]);
    }
  }
  if (a.has_post) normalise<NT, CH, VEC>(v, a, a.post, tid, red, turn);
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + (int64_t)(p / a.tokens_per_gate) * a.ldg : nullptr;
  const f2 scale = pack_f2(a.scale, a.scale);
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    if (gate) {
      f2 g[4];
      load_piece<T, VEC, true>(gate, c, tid, NT, a.K, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = mul_f2(v[c][i], g[i]);
    }
    if constexpr (VEC) {
      float r[8];
      raw[c].unpack(r);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = fma_f2(scale, v[c][i], pack_f2(r[2 * i], r[2 * i + 1]));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[c][i] = fma_f2(scale, v[c][i], rs[c][i]);
    }
    if (a.s) store_piece<R, VEC>(static_cast<R*>(a.s) + p * a.lds, c, tid, NT, a.K, v[c]);
  }
  if (a.has_pre) {
    normalise<NT, CH, VEC>(v, a, a.pre, tid, red, turn);
    T* y = static_cast<T*>(a.y) + (int64_t)p * a.K;
#pragma unroll
    for (int c = 0; c < CH; ++c) store_piece<T, VEC>(y, c, tid, NT, a.K, v[c]);
  }
}

// Rows that registers do not hold, a block each: every sum reads the row again.  Elements are written in the last loop only,
// each by the thread that reads it, so outputs may take the place of inputs.
constexpr int LONG_THREADS = 1024;
template <typename T, typename R>
__global__ void __launch_bounds__(LONG_THREADS) long_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[2][32];
  int turn = 0;
  const int p = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + p * a.ldx;
  const R* r = a.r ? static_cast<const R*>(a.r) + p * a.ldr : nullptr;
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + (int64_t)(p / a.tokens_per_gate) * a.ldg : nullptr;
  // means of f(k) over the row, in pieces that keep fp32's bits
  auto mean_of = [&](auto f) {
    float total = 0.0f;
    for (int k = threadIdx.x; k < a.K; k += LONG_THREADS * 64) {
      float part = 0.0f;
      for (int i = 0; i < 64; ++i) {
        const int64_t at = (int64_t)k + (int64_t)i * LONG_THREADS;
        if (at < a.K) part += f((int)at);
      }
      total += part * a.part;
    }
    return row_sum<LONG_THREADS>(total, red, turn) * a.rest;
  };
  auto stats = [&](auto value, const fgq_norm& n, float& mean, float& inv) {
    mean = 0.0f;
    if (n.kind == FGQ_NORM_LAYER) mean = mean_of(value);
    const float m = mean;
    inv = rsqrtf(mean_of([&](int k) {
                   const float z = value(k) - m;
                   return z * z;
                 }) + n.eps);
  };
  auto apply = [&](float z, const fgq_norm& n, float mean, float inv, int k) {
    z = (z - mean) * inv;
    if (n.weight) z *= __ldg(n.weight + k);
    return n.bias ? z + __ldg(n.bias + k) : z;
  };
  float m0 = 0.0f, i0 = 0.0f, m1 = 0.0f, i1 = 0.0f;
  if (a.has_post) stats([&](int k) { return to_float(x[k]); }, a.post, m0, i0);
  auto stream = [&](int k) {
    float u = to_float(x[k]);
    if (a.has_post) u = apply(u, a.post, m0, i0, k);
    if (gate) u *= to_float(gate[k]);
    return fmaf(a.scale, u, r ? to_float(r[k]) : 0.0f);
  };
  if (a.has_pre) stats(stream, a.pre, m1, i1);
  for (int64_t at = threadIdx.x; at < a.K; at += LONG_THREADS) {
    const int k = (int)at;
    const float s = stream(k);
    if (a.s) from_float(s, static_cast<R*>(a.s)[p * a.lds + k]);
    if (a.has_pre) from_float(apply(s, a.pre, m1, i1, k), static_cast<T*>(a.y)[(int64_t)p * a.K + k]);
  }
}

template <typename T, typename R, bool VEC>
fgq_status launch_add_norm(const NormArgs& a, cudaStream_t s) {
  const unsigned P = (unsigned)a.P;
  // few rows: one piece a thread, for shorter chains of a single row; many: two, for fewer barriers a byte.  4096 bf16 values, both norms, us so
  // and so: 1 row 2.83 and 2.99, 304 rows 3.61 and 3.74, 2432 rows 16.8 and 14.9; of 2048 values 2.36 and 2.64, 2.93 and 3.22, 8.1 and 7.2
  const bool few = a.P <= 2 * device_sms();
  if (a.K <= 512)
    add_norm_kernel<T, R, 32, 2, VEC><<<(P + 3) / 4, 128, 0, s>>>(a);
  else if (a.K <= 1024)
    add_norm_kernel<T, R, 128, 1, VEC><<<P, 128, 0, s>>>(a);
  else if (a.K <= 2048)
    few ? add_norm_kernel<T, R, 256, 1, VEC><<<P, 256, 0, s>>>(a) : add_norm_kernel<T, R, 128, 2, VEC><<<P, 128, 0, s>>>(a);
  else if (a.K <= 4096)
    few ? add_norm_kernel<T, R, 512, 1, VEC><<<P, 512, 0, s>>>(a) : add_norm_kernel<T, R, 256, 2, VEC><<<P, 256, 0, s>>>(a);
  else if (a.K <= 8192)
    add_norm_kernel<T, R, 512, 2, VEC><<<P, 512, 0, s>>>(a);
  else if (a.K <= 16384)
    add_norm_kernel<T, R, 1024, 2, VEC><<<P, 1024, 0, s>>>(a);
  else
    long_kernel<T, R><<<P, LONG_THREADS, 0, s>>>(a);
  return after_launch();
}

template <typename T, typename R>
fgq_status launch_add_norm(const NormArgs& a, int type, int rtype, cudaStream_t s) {
  auto rows16 = [&](const void* p, int64_t ld, int t) { return !p || (aligned(p, 16) && stride16(ld, t)); };
  const bool vec = a.K % 8 == 0 && rows16(a.x, a.ldx, type) && rows16(a.gate, a.ldg, type) && rows16(a.r, a.ldr, rtype) &&
                   rows16(a.s, a.lds, rtype) && rows16(a.y, a.K, type) && aligned(a.post.weight, 16) && aligned(a.post.bias, 16) &&
                   aligned(a.pre.weight, 16) && aligned(a.pre.bias, 16);
  return vec ? launch_add_norm<T, R, true>(a, s) : launch_add_norm<T, R, false>(a, s);
}

// FGQ_OK, or what is wrong with a norm.
fgq_status check_norm(const fgq_norm* n) {
  if (!n) return FGQ_OK;
  if (n->kind != FGQ_NORM_RMS && n->kind != FGQ_NORM_LAYER) return FGQ_ERR_ARG;
  if (!(n->eps > 0.0f) || nonfinite_host(n->eps)) return FGQ_ERR_ARG;
  return FGQ_OK;
}

}  // namespace
}  // namespace fgq

using namespace fgq;

extern "C" fgq_status fgq_add_norm(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const fgq_norm* post,
                                   const void* gate, int64_t ldg, int tokens_per_gate, float scale, const void* r,
                                   fgq_float_type rtype, int64_t ldr, void* s, int64_t lds, const fgq_norm* pre, void* y,
                                   cudaStream_t stream) {
  if (P < 0 || K < 1 || !dec::valid_float(type) || !dec::valid_float(rtype) || (rtype != type && rtype != FGQ_F32)) return FGQ_ERR_ARG;
  if (check_norm(post) != FGQ_OK || check_norm(pre) != FGQ_OK || dec::nonfinite_host(scale)) return FGQ_ERR_ARG;
  if (P == 0) return FGQ_OK;
  if ((pre != nullptr) != (y != nullptr) || (!y && !s) || (gate && tokens_per_gate < 1) || !x) return FGQ_ERR_ARG;
  if (P > 1 && (ldx < K || (r && ldr < K) || (s && lds < K))) return FGQ_ERR_ARG;
  if (gate && P > tokens_per_gate && ldg < K) return FGQ_ERR_ARG;
  if (P > 1 && ((y == x && ldx != K) || (s && s == r && lds != ldr))) return FGQ_ERR_ARG;  // another row's inputs would be overwritten
  if (P > dec::MAX_SIZE || K > dec::MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
  const uintptr_t e = dec::float_bytes(type), re = dec::float_bytes(rtype);
  if (!dec::aligned(x, e) || !dec::aligned(gate, e) || !dec::aligned(r, re) || !dec::aligned(s, re) || !dec::aligned(y, e))
    return FGQ_ERR_ALIGN;
  for (const fgq_norm* n : {post, pre})
    if (n && (!dec::aligned(n->weight, 4) || !dec::aligned(n->bias, 4))) return FGQ_ERR_ALIGN;
  NormArgs a = {};
  a.x = x, a.gate = gate, a.r = r, a.s = s, a.y = y;
  // a single row may have any stride
  a.ldx = P > 1 ? ldx : 0, a.ldr = P > 1 ? ldr : 0, a.lds = P > 1 ? lds : 0, a.ldg = gate && P > tokens_per_gate ? ldg : 0;
  if (post) a.post = *post, a.has_post = 1;
  if (pre) a.pre = *pre, a.has_pre = 1;
  int log2k = 0;
  frexp((double)K, &log2k);
  a.part = (float)ldexp(1.0, -log2k), a.rest = (float)(1.0 / ldexp((double)K, -log2k));
  a.scale = scale, a.P = P, a.K = K, a.tokens_per_gate = gate ? tokens_per_gate : 1;
  if (type == FGQ_F32) return launch_add_norm<float, float>(a, type, rtype, stream);
  if (type == FGQ_BF16)
    return rtype == FGQ_F32 ? launch_add_norm<__nv_bfloat16, float>(a, type, rtype, stream)
                            : launch_add_norm<__nv_bfloat16, __nv_bfloat16>(a, type, rtype, stream);
  return rtype == FGQ_F32 ? launch_add_norm<__half, float>(a, type, rtype, stream)
                          : launch_add_norm<__half, __half>(a, type, rtype, stream);
}
