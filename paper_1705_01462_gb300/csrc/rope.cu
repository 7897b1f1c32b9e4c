// Rotary positions: heads' pairs turned by angles that grow with their token's position.
//
// (a, b) -> m (a cos - b sin, b cos + a sin), angle = 2 pi frac(position turns_j).  turns_j is held as a 64-bit fraction
// of a turn, so the fraction at a position is the low half of an integer product, exact at any distance, where an
// fp32 angle at position 100000 would be off by 0.004 radians; its top 32 bits, as half turns in [-1, 1), go to sincospi.
//
// A thread takes one unit of a token's heads: V consecutive values and their partners (half: V pairs; interleaved: V / 2
// pairs; past rot: V values to copy), 16 bytes each, turns them by angles found once, and does so for every HG-th head, the loads of
// four heads ahead of their stores.  Bound by bytes: heads read and written once.  4 x 8192 tokens, 40 heads of 128, bf16: 109 us,
// 91% of the copy rate (154 with each head's loads behind the stores of the one before).
#include <cmath>
#include <type_traits>

#include "decoder_internal.cuh"

namespace fgq {
namespace {

using namespace dec;

constexpr int RP_THREADS = 256;

struct RopeArgs {
  const void* x;
  void* y;
  int64_t xbs, xts, ybs, yts;
  const uint64_t* table;
  const int32_t* starts;
  const int32_t* lens;
  float magnitude;
  int inverse;
  int tokens, T, heads, D, rot;
  int units, turning, hg, per_block;  // units of a head, those that turn, groups of heads, tokens of a block
};

// V elements as loaded, and as fp32: 16 bytes, or one element.
template <typename T, int V>
struct Piece {
  using Raw = typename std::conditional<V == 1, T, uint4>::type;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void unpack(float (&v)[V]) const {
    if constexpr (V == 1) {
      v[0] = to_float(raw);
    } else if constexpr (std::is_same<T, float>::value) {
      v[0] = __uint_as_float(raw.x), v[1] = __uint_as_float(raw.y), v[2] = __uint_as_float(raw.z), v[3] = __uint_as_float(raw.w);
    } else {
      unpack8(raw, v, T());
    }
  }
  static __device__ __forceinline__ void store(T* p, const float (&v)[V]) {
    if constexpr (V == 1)
      from_float(v[0], *p);
    else if constexpr (std::is_same<T, float>::value)
      *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
      store8(p, v);
  }
};

// V = 16 bytes of elements, or 1.  A unit that turns is two pieces of V (half) or one (interleaved; V = 1: two elements).
template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(RP_THREADS) rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int PAIRS = HALF || V == 1 ? V : V / 2, HB = 4;
  constexpr bool TWO = HALF || V == 1;  // pieces of a unit that turns
  const int first = (int)blockIdx.x * a.per_block, per_token = a.units * a.hg;
  const int n = min(a.per_block, a.tokens - first) * per_token;
  const bool copy = a.x != a.y;
  for (int li = threadIdx.x; li < n; li += RP_THREADS) {
    const int tk = li / per_token, in = li - tk * per_token;
    const int h0 = in / a.units, u = in - h0 * a.units;
    const int token = first + tk, b = token / a.T, i = token - b * a.T;
    const bool live = !a.lens || i < __ldg(a.lens + b);
    const bool turn = u < a.turning && live;
    if (!turn && !copy) continue;
    const T* x = static_cast<const T*>(a.x) + b * a.xbs + i * a.xts;
    T* y = static_cast<T*>(a.y) + b * a.ybs + i * a.yts;
    // where the unit's pieces are in a head
    int at0, at1;
    if (u < a.turning) {
      at0 = HALF || V > 1 ? u * V : 2 * u;
      at1 = HALF ? at0 + a.rot / 2 : (V > 1 ? -1 : at0 + 1);
    } else {
      at0 = a.rot + (u - a.turning) * V;
      at1 = -1;
    }
    float c[PAIRS], s[PAIRS];
    if (turn) {
      const int64_t pos = (int64_t)__ldg(a.starts + b) + i;
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) {
        const uint64_t phase = (uint64_t)pos * __ldg(reinterpret_cast<const unsigned long long*>(a.table) + u * PAIRS + j);
        const float half_turns = (float)(int)(phase >> 32) * 4.656612873077393e-10f;  // 2^-31
        sincospif(half_turns, &s[j], &c[j]);
        c[j] *= a.magnitude;
        s[j] *= a.inverse ? -a.magnitude : a.magnitude;
      }
    }
    // HB heads' loads at once: the stores between would hold them back, as y may be x
    for (int h = h0; h < a.heads; h += HB * a.hg) {
      Piece<T, V> p[HB], q[HB];
#pragma unroll
      for (int n = 0; n < HB; ++n) {
        const T* head = x + (int64_t)(h + n * a.hg) * a.D;
        if (h + n * a.hg < a.heads) {
          p[n].load(head + at0);
          if (TWO && at1 >= 0) q[n].load(head + at1);
        }
      }
#pragma unroll
      for (int n = 0; n < HB; ++n) {
        if (h + n * a.hg >= a.heads) break;
        T* head = y + (int64_t)(h + n * a.hg) * a.D;
        float f[V], e[V];
        p[n].unpack(f);
        if constexpr (TWO) {
          if (at1 >= 0) {
            q[n].unpack(e);
            if (turn) {
#pragma unroll
              for (int j = 0; j < V; ++j) {
                const float u = f[j], v = e[j];
                f[j] = fmaf(u, c[j], -v * s[j]);
                e[j] = fmaf(v, c[j], u * s[j]);
              }
            }
            Piece<T, V>::store(head + at1, e);
          }
        } else if (turn) {
#pragma unroll
          for (int j = 0; j < PAIRS; ++j) {
            const float u = f[2 * j], v = f[2 * j + 1];
            f[2 * j] = fmaf(u, c[j], -v * s[j]);
            f[2 * j + 1] = fmaf(v, c[j], u * s[j]);
          }
        }
        Piece<T, V>::store(head + at0, f);
      }
    }
  }
}

template <typename T>
fgq_status launch_rope(RopeArgs a, int layout, cudaStream_t s) {
  constexpr int V = 16 / (int)sizeof(T);
  const bool half = layout == FGQ_ROPE_HALF;
  const int type = sizeof(T) == 4 ? FGQ_F32 : FGQ_BF16;
  const bool vec = a.D % V == 0 && a.rot % (half ? 2 * V : V) == 0 && aligned(a.x, 16) && aligned(a.y, 16) &&
                   stride16(a.xbs, type) && stride16(a.xts, type) && stride16(a.ybs, type) && stride16(a.yts, type);
  const int v = vec ? V : 1;
  a.turning = half ? a.rot / 2 / v : (vec ? a.rot / V : a.rot / 2);
  a.units = a.turning + (a.x != a.y ? (a.D - a.rot) / v : 0);
  // heads that share a thread's angles: as many as leave two blocks an SM
  const int64_t most = 2ll * RP_THREADS * device_sms(), all = (int64_t)a.tokens * a.units;
  int64_t hg = (most + all - 1) / all;
  const int64_t fewest = (a.heads + 15) / 16;
  a.hg = (int)(hg > a.heads ? a.heads : (hg < fewest ? fewest : hg));
  const int per_token = a.units * a.hg;
  a.per_block = per_token >= RP_THREADS ? 1 : RP_THREADS / per_token;
  const unsigned grid = (unsigned)(((int64_t)a.tokens + a.per_block - 1) / a.per_block);
  if (half)
    vec ? rope_kernel<T, V, true><<<grid, RP_THREADS, 0, s>>>(a) : rope_kernel<T, 1, true><<<grid, RP_THREADS, 0, s>>>(a);
  else
    vec ? rope_kernel<T, V, false><<<grid, RP_THREADS, 0, s>>>(a) : rope_kernel<T, 1, false><<<grid, RP_THREADS, 0, s>>>(a);
  return after_launch();
}

// Whether no two of the outputs' tokens, n elements each, share memory: one axis steps past all of the other.
bool apart(int B, int64_t batch_stride, int T, int64_t token_stride, double n) {
  const double b = fabs((double)batch_stride), t = fabs((double)token_stride);
  return (T == 1 || t >= n) && (B == 1 || b >= n) && (T == 1 || B == 1 || b >= (T - 1) * t + n || t >= (B - 1) * b + n);
}

}  // namespace
}  // namespace fgq

using namespace fgq;

extern "C" {

fgq_status fgq_rope_table(int rot, double base, fgq_rope_scaling scaling, double factor, double length, double low,
                          double high, uint64_t* table) {
  if (!table || rot < 2 || rot % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return FGQ_ERR_ARG;
  if (scaling != FGQ_ROPE_PLAIN && scaling != FGQ_ROPE_LINEAR && scaling != FGQ_ROPE_BASE && scaling != FGQ_ROPE_RAMP)
    return FGQ_ERR_ARG;
  if (scaling != FGQ_ROPE_PLAIN && (!(factor >= 1.0) || !std::isfinite(factor))) return FGQ_ERR_ARG;
  if (scaling == FGQ_ROPE_RAMP && (!(length > 0.0) || !std::isfinite(length) || !std::isfinite(low) || !std::isfinite(high) ||
                                   !(high > low)))
    return FGQ_ERR_ARG;
  const double two_pi = 6.283185307179586476925;
  if (scaling == FGQ_ROPE_BASE && rot > 2) base *= pow(factor, (double)rot / (rot - 2));
  for (int j = 0; j < rot / 2; ++j) {
    double f = pow(base, -2.0 * j / rot) / two_pi;  // turns a position, below 1 / 6
    if (scaling == FGQ_ROPE_LINEAR) f /= factor;
    if (scaling == FGQ_ROPE_RAMP) {
      double k = (length * f - low) / (high - low);
      k = k < 0.0 ? 0.0 : (k > 1.0 ? 1.0 : k);
      f = k * f + (1.0 - k) * f / factor;
    }
    table[j] = (uint64_t)nearbyint(ldexp(f, 64));
  }
  return FGQ_OK;
}

fgq_status fgq_rope(const void* x, void* y, fgq_float_type type, int B, int T, int heads, int head_dim,
                    int64_t x_batch_stride, int64_t x_token_stride, int64_t y_batch_stride, int64_t y_token_stride, int rot,
                    fgq_rope_layout layout, const uint64_t* table, float magnitude, int inverse, const int32_t* starts,
                    const int32_t* lens, cudaStream_t stream) {
  if (B < 0 || T < 0 || heads < 0 || head_dim < 0 || !dec::valid_float(type)) return FGQ_ERR_ARG;
  if (rot < 2 || rot % 2 != 0 || rot > head_dim || (inverse != 0 && inverse != 1) || dec::nonfinite_host(magnitude)) return FGQ_ERR_ARG;
  if (layout != FGQ_ROPE_HALF && layout != FGQ_ROPE_INTERLEAVED) return FGQ_ERR_ARG;
  if (B == 0 || T == 0 || heads == 0) return FGQ_OK;
  if (!x || !y || !table || !starts) return FGQ_ERR_ARG;
  if (x == y && ((B > 1 && x_batch_stride != y_batch_stride) || (T > 1 && x_token_stride != y_token_stride))) return FGQ_ERR_ARG;
  const uintptr_t e = dec::float_bytes(type);
  if (!dec::aligned(x, e) || !dec::aligned(y, e) || !dec::aligned(table, 8) || !dec::aligned(starts, 4) || !dec::aligned(lens, 4))
    return FGQ_ERR_ALIGN;
  if (head_dim > 65536 || heads > INT32_MAX / head_dim || (int64_t)B * T > INT32_MAX || (int64_t)B * T * heads > INT32_MAX)
    return FGQ_ERR_UNSUPPORTED;
  if (!apart(B, y_batch_stride, T, y_token_stride, (double)heads * head_dim)) return FGQ_ERR_ARG;
  // an axis of one element may have any stride
  RopeArgs a = {};
  a.x = x, a.y = y;
  a.xbs = B > 1 ? x_batch_stride : 0, a.xts = T > 1 ? x_token_stride : 0;
  a.ybs = B > 1 ? y_batch_stride : 0, a.yts = T > 1 ? y_token_stride : 0;
  a.table = table, a.starts = starts, a.lens = lens;
  a.magnitude = magnitude, a.inverse = inverse;
  a.tokens = B * T, a.T = T, a.heads = heads, a.D = head_dim, a.rot = rot;
  if (type == FGQ_F32) return launch_rope<float>(a, layout, stream);
  if (type == FGQ_BF16) return launch_rope<__nv_bfloat16>(a, layout, stream);
  return launch_rope<__half>(a, layout, stream);
}

}  // extern "C"
