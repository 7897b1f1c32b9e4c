// Mixture of experts on 4-bit weights, for few tokens.
//
//   l = router x;  the `top` largest, their weights g;  y = sum_j g_j down_e (silu(gate_e x) * (up_e x)),  e = the j-th choice
//
// Kernels of a layer, each brought up while the one before it runs:
//   route_kernel    a cluster four tokens: products of 8 elements in fp32, their sums as pairs of fp32 (two-sum), so that a
//                   logit is off by 8 roundings of its terms' magnitudes at most (with terms of random signs by about one of itself,
//                   so that the choice is that of 64-bit sums but for near ties; pairs throughout took 64 tokens of 64 experts from
//                   11.2 to 18.3 us); the largest one by one, and their weights;
//   group_kernel    (more than four tokens, or choices that are given) one block: choices sorted by expert, and cut into units of
//                   tokens that share an expert;
//   resident_kernel (w4_resident.cuh) 16 rows of gate and of up for a unit of up to 8 tokens: silu(gate) up in fp32; then of down;
//   or, with more choices an expert, the kernels of gemm_w4_experts.cu for units of 32 to 256;
//   combine_kernel  each token's choices by their weights, in their order.
// Bound by the bytes of the experts' weights, each read once (again from L2 for each further unit of an expert), and before them by the way
// from logits to units: of 165 us for 64 tokens of 6 of 64 experts, 4096 -> 1536, routing takes 11 and the grouping 7 more, combining 4; of 22 us for one
// token of 8 of 64 experts, 2048 -> 1024, routing takes 5 (3 with one expert to choose), each layer about 7, combining 2.
#include <type_traits>

#include "w4_launch.h"
#include "w4_many.h"

namespace fgq {
namespace w4 {
namespace {

constexpr int MAX_EXPERTS = 1024, MAX_TOP = 32;
constexpr int MAX_CHOICES = 4096;  // of a pass: what group_kernel holds
static_assert(MAX_CHOICES < 1 << 16 && MAX_CHOICES >= MAX_TOP, "group_kernel's sums");

// ------------------------------------------------------------------ routing
struct RouteArgs {
  const void* x;
  const void* router;
  int64_t ldx;
  int32_t* ids;
  float* weights;
  // what group_kernel would find, where the tokens are one cluster's
  Unit* units;
  Choice* choices;
  int32_t* places;
  unsigned* tops;
  int* nunits;  // units, choices
  int P, K, E, top, score, renormalize;
  float scale;
};

// hi + lo += h + l, hi the rounded sum of all and lo what it leaves out (two-sum).
__device__ __forceinline__ void add_pair(float& hi, float& lo, float h, float l) {
  const float t = hi + h, b = t - hi;
  lo += ((hi - (t - b)) + (h - b)) + l;
  hi = t;
}

// fp32 numbers as whole ones of the same order (no NaN); 0 has one sign.
__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }

// A cluster of eight blocks takes four tokens: its 128 warps share the experts, `ks` of them each expert's row, and leave
// the logits, as ordered pairs of fp32, in the first block's shared memory; there a warp a token takes the largest one by one.
constexpr int RT_WARPS = 16, RT_CLUSTER = 8, RT_TOKENS = 4;

// Eight elements as loaded, where the source has the load: the compiler may not move it to its use.
template <typename T>
struct Ahead8 {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i)
      asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                   : "l"(reinterpret_cast<const uint4*>(p) + i));
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[4 * i] = __uint_as_float(v[i].x), x[4 * i + 1] = __uint_as_float(v[i].y);
        x[4 * i + 2] = __uint_as_float(v[i].z), x[4 * i + 3] = __uint_as_float(v[i].w);
      }
    } else {
      unpack8(v[0], x, T());
    }
  }
};

// TOKENS of a cluster; VEC: 16-byte pieces of aligned rows.
template <typename T, typename R, int TOKENS, bool VEC>
__global__ void __cluster_dims__(RT_CLUSTER, 1, 1) __launch_bounds__(32 * RT_WARPS)
    route_kernel(const __grid_constant__ RouteArgs a, int ks) {
  __shared__ float2 part[RT_WARPS][TOKENS];
  __shared__ unsigned long long keys[TOKENS][MAX_EXPERTS];  // of the first block
  __shared__ int chosen[TOKENS * MAX_TOP];
  __shared__ float chosen_w[TOKENS * MAX_TOP];
  __shared__ int ahead[TOKENS * MAX_TOP];
  pdl_trigger();
  // another block's shared memory may be written once that block runs: they meet before the first keys, after the first products
  asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)blockIdx.x % RT_CLUSTER, p0 = (int)blockIdx.x / RT_CLUSTER * TOKENS;
  const int np = min(TOKENS, a.P - p0), kpart = warp % ks, per_pass = RT_CLUSTER * RT_WARPS / ks;
  const T* x = static_cast<const T*>(a.x) + p0 * a.ldx;
  for (int e0 = 0; e0 < a.E; e0 += per_pass) {
    const int e = e0 + (rank * RT_WARPS + warp) / ks;
    float hi[TOKENS], lo[TOKENS];
#pragma unroll
    for (int i = 0; i < TOKENS; ++i) hi[i] = lo[i] = 0.0f;
    if (e < a.E) {
      const R* wr = static_cast<const R*>(a.router) + (int64_t)e * a.K;
      const T* row[TOKENS];  // tokens past the last are read as the last
#pragma unroll
      for (int i = 0; i < TOKENS; ++i) row[i] = x + min(i, np - 1) * a.ldx;
      auto add = [&](int i, const float (&v)[8], const float (&w)[8]) {
        float s = v[0] * w[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) s = fmaf(v[j], w[j], s);
        add_pair(hi[i], lo[i], s, 0.0f);
      };
      if constexpr (VEC) {  // BATCH steps' loads at once
        constexpr int BATCH = sizeof(T) == 4 || sizeof(R) == 4 ? 2 : 4;
        const int step = 256 * ks;
        for (int k0 = 8 * (lane + 32 * kpart); k0 < a.K; k0 += BATCH * step) {
          Ahead8<R> wc[BATCH];
          Ahead8<T> xc[BATCH][TOKENS];
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            const int k = min(k0 + b * step, a.K - 8);  // past the row: its last again, left out below
            wc[b].load(wr + k);
#pragma unroll
            for (int i = 0; i < TOKENS; ++i) xc[b][i].load(row[i] + k);
          }
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            if (k0 + b * step >= a.K) break;
            float w[8];
            wc[b].unpack(w);
#pragma unroll
            for (int i = 0; i < TOKENS; ++i) {
              float v[8];
              xc[b][i].unpack(v);
              add(i, v, w);
            }
          }
        }
      } else {
        for (int k = 8 * (lane + 32 * kpart); k < a.K; k += 256 * ks) {
          float w[8], v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = k + j < a.K ? to_float(wr[k + j]) : 0.0f;
#pragma unroll
          for (int i = 0; i < TOKENS; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = k + j < a.K ? to_float(row[i][k + j]) : 0.0f;
            add(i, v, w);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TOKENS; ++i)
      if (i < np) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const float h = __shfl_xor_sync(FULL_MASK, hi[i], o), l = __shfl_xor_sync(FULL_MASK, lo[i], o);
          // the same operands in the same order in both lanes
          float a0 = lane & o ? h : hi[i], a1 = lane & o ? l : lo[i];
          add_pair(a0, a1, lane & o ? hi[i] : h, lane & o ? lo[i] : l);
          hi[i] = a0, lo[i] = a1;
        }
        if (lane == 0) part[warp][i] = make_float2(hi[i], lo[i]);
      }
    __syncthreads();
    if (e0 == 0) asm volatile("barrier.cluster.wait;" ::: "memory");
    const int el = (int)threadIdx.x / TOKENS, i = (int)threadIdx.x % TOKENS;  // an expert of this block, a token
    const int ee = e0 + rank * (RT_WARPS / ks) + el;
    if (el < RT_WARPS / ks && i < np && ee < a.E) {
      float h = part[el * ks][i].x, l = part[el * ks][i].y;
      for (int s = 1; s < ks; ++s) add_pair(h, l, part[el * ks + s][i].x, part[el * ks + s][i].y);
      // infinite sums have no rest, and what their two-sums left is NaN; NaN counts as the smallest
      const float r = nonfinite(h) ? h : h + l, rest = l - (r - h);
      unsigned long long key = 1ull;
      if (r == r) key = (unsigned long long)order_of(r) << 32 | (nonfinite(r) ? 0x80000000u : order_of(rest));
      uint32_t at;
      asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(&keys[i][ee])));
      asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at), "l"(key) : "memory");
    }
    __syncthreads();
  }
  cluster_sync();
  if (rank != 0) return;
  if (warp < np) {
    const unsigned long long* key = keys[warp];
    const int p = p0 + warp, count = (a.E + 31) / 32;
    bool bad = false;
    for (int i = 0; i < count; ++i) bad |= lane + 32 * i < a.E && key[lane + 32 * i] == 1ull;
    bad = __any_sync(FULL_MASK, bad);
    unsigned taken = 0;  // of this lane's, a bit each
    float best_h = 0.0f, best_l = 0.0f, mine = 0.0f, total = 0.0f;  // the largest; lane j: the j-th choice's value; their sum
    int mine_id = 0;
    auto value = [&](unsigned long long k) {  // less the largest, rounded
      return (of_order((uint32_t)(k >> 32)) - best_h) + (of_order((uint32_t)k) - best_l);
    };
    for (int j = 0; j < a.top; ++j) {
      unsigned long long k = 0;
      int id = 0x7fffffff;
      for (int i = 0; i < count; ++i) {
        const int e = lane + 32 * i;
        if (e < a.E && !(taken >> i & 1u) && key[e] > k) {
          k = key[e];
          id = e;
        }
      }
      // the largest upper half, of those lanes the largest lower half, of those the lowest index
      const unsigned h = __reduce_max_sync(FULL_MASK, (unsigned)(k >> 32));
      const bool in = (unsigned)(k >> 32) == h;
      const unsigned l = __reduce_max_sync(FULL_MASK, in ? (unsigned)k : 0u);
      id = (int)__reduce_min_sync(FULL_MASK, in && (unsigned)k == l ? (unsigned)id : 0x7fffffffu);
      k = (unsigned long long)h << 32 | l;
      if ((id & 31) == lane) taken |= 1u << (id >> 5);
      if (j == 0) best_h = of_order((uint32_t)(k >> 32)), best_l = of_order((uint32_t)k);
      // sigmoid scores through exponentials of numbers below 0, which do not overflow; where all are to be divided by their sum, without the
      // largest's exponential, a factor of each: scores far below fp32's smallest have a ratio all the same
      const float logit = of_order((uint32_t)(k >> 32));
      float f;
      if (a.score == FGQ_SCORE_SOFTMAX)
        f = expf(value(k));
      else if (logit < 0.0f)
        f = expf(a.renormalize && best_h < 0.0f ? value(k) : logit) / (1.0f + expf(logit));
      else
        f = 1.0f / (1.0f + expf(-logit));
      if (lane == j) {
        mine = f;
        mine_id = id;
      }
      total += f;
    }
    if (a.score == FGQ_SCORE_SOFTMAX && !a.renormalize) {
      total = 0.0f;
      for (int i = 0; i < count; ++i)
        if (lane + 32 * i < a.E) total += expf(value(key[lane + 32 * i]));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(FULL_MASK, total, o);
    }
    float w = mine;
    if (a.score == FGQ_SCORE_SOFTMAX || a.renormalize) w /= total;
    w *= a.scale;
    if (bad) w = __uint_as_float(0x7fc00000u);
    if (lane < a.top) {
      a.ids[(int64_t)p * a.top + lane] = mine_id;
      a.weights[(int64_t)p * a.top + lane] = w;
      chosen[warp * a.top + lane] = mine_id;
      chosen_w[warp * a.top + lane] = w;
    }
  }
  if (!a.units) return;
  // the choices by expert, each counting for itself; a unit an expert, as four tokens fit every unit
  __syncthreads();
  const int n = np * a.top, c = (int)threadIdx.x;
  int e = 0, place = 0, same = 0, lead = 0;
  if (c < n) {
    e = chosen[c];
    lead = 1;
    for (int j = 0; j < n; ++j) {
      const int f = chosen[j];
      place += f < e || (f == e && j < c);
      same += f == e;
      if (f == e && j < c) lead = 0;
    }
    ahead[c] = lead;
  }
  __syncthreads();
  if (c < n) {
    a.choices[place] = {c / a.top, chosen_w[c]};
    a.places[c] = place;
    a.tops[c] = 0u;
    if (lead) {
      int u = 0;
      for (int j = 0; j < n; ++j) u += ahead[j] && chosen[j] < e;
      a.units[u] = {e, place, same, 0};
    }
  }
  if (warp == 0) {
    int u = 0;
    for (int j = lane; j < n; j += 32) u += ahead[j];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(FULL_MASK, u, o);
    if (lane == 0) a.nunits[0] = u, a.nunits[1] = n;
  }
}

// ------------------------------------------------------------------ tokens as operand rows
// A block a token: fp32 in three bf16 parts, 16-bit types copied to aligned rows; zeros up to a multiple of 8.  (Brought into form by the
// products themselves, 64 tokens of 6 of 64 experts 4096 -> 1536 took 16 us more, for all types: registers spilled.)
template <typename T>
__global__ void __launch_bounds__(256) operand_rows_kernel(const T* __restrict__ x, int K, int64_t ldx, uint16_t* dst, int64_t pitch) {
  pdl_trigger();
  const T* row = x + blockIdx.x * ldx;
  for (int64_t k = threadIdx.x; k < pitch; k += 256) {
    if constexpr (std::is_same<T, float>::value) {
      uint16_t p[3];
      three_parts(k < K ? row[k] : 0.0f, p);
      uint16_t* to = dst + 3 * pitch * blockIdx.x + k;
      to[0] = p[0], to[pitch] = p[1], to[2 * pitch] = p[2];
    } else {
      dst[pitch * blockIdx.x + k] = k < K ? row[k] : (uint16_t)0;
    }
  }
}

// ------------------------------------------------------------------ choices by expert
constexpr int GR_THREADS = 1024;

__global__ void __launch_bounds__(GR_THREADS) group_kernel(const int32_t* ids, const float* weights, int A, int top, int E, int cap,
                                                           Unit* units, Choice* choices, int32_t* places, unsigned* tops, int* nunits) {
  __shared__ int count[MAX_EXPERTS], start[MAX_EXPERTS], id[MAX_CHOICES], warp_sums[GR_THREADS / 32];
  __shared__ float weight[MAX_CHOICES];
  pdl_trigger();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  count[t] = 0;
  __syncthreads();
  pdl_wait();
  for (int i = t; i < A; i += GR_THREADS) {
    const int e = __ldcg(ids + i);
    id[i] = e;
    weight[i] = __ldcg(weights + i);
    tops[i] = 0u;
    if (e >= 0 && e < E)
      atomicAdd(&count[e], 1);
    else
      places[i] = -1;
  }
  __syncthreads();
  // choices and units before expert t, both in one word
  const int n = count[t], mine = n | (n + cap - 1) / cap << 16;  // 0 from E on
  int s = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(FULL_MASK, s, o);
    if (lane >= o) s += u;
  }
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  int before = lane < warp ? warp_sums[lane] : 0, total = warp_sums[lane];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    before += __shfl_xor_sync(FULL_MASK, before, o);
    total += __shfl_xor_sync(FULL_MASK, total, o);
  }
  before += s - mine;
  const int first = before & 0xffff, u0 = before >> 16;
  start[t] = first;
  for (int u = 0; u * cap < n; ++u) units[u0 + u] = {t, first + u * cap, min(cap, n - u * cap), 0};
  if (t == 0) nunits[0] = total >> 16, nunits[1] = total & 0xffff;
  __syncthreads();
  for (int e = warp; e < E; e += GR_THREADS / 32) {  // each expert's choices in the order they came
    const int want = count[e];
    int at = start[e], found = 0;
    for (int i = 0; found < want; i += 32) {
      const bool hit = i + lane < A && id[i + lane] == e;
      const unsigned m = __ballot_sync(FULL_MASK, hit);
      if (hit) {
        const int place = at + __popc(m & ((1u << lane) - 1u));
        choices[place] = {(i + lane) / top, weight[i + lane]};
        places[i + lane] = place;
      }
      at += __popc(m);
      found += __popc(m);
    }
  }
}

// ------------------------------------------------------------------ the choices' outputs together
// y[p] = sum_j weights[p][j] z[places[p][j]], V values a thread.  (Done by whichever unit of a row tile is the last in the kernel before,
// which saves a launch, one token took 25.1 us on the device in place of 21.5, four 50 in place of 32: a fence for each row tile.)
template <int V>
__global__ void __launch_bounds__(256) combine_kernel(const float* z, const int32_t* places, const float* weights, int top, int K, void* y,
                                                      int ytype) {
  __shared__ int at[MAX_TOP];
  __shared__ float by[MAX_TOP];
  const int p = blockIdx.y, m = ((int)blockIdx.x * 256 + (int)threadIdx.x) * V;
  // these are of kernels before the one that this one waits for
  if ((int)threadIdx.x < top) {
    at[threadIdx.x] = __ldcg(places + p * top + threadIdx.x);
    by[threadIdx.x] = __ldcg(weights + p * top + threadIdx.x);
  }
  __syncthreads();
  pdl_wait();
  if (m >= K) return;
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.0f;
#pragma unroll 8
  for (int j = 0; j < top; ++j) {
    if (at[j] < 0) continue;  // the same for the whole block
    const float* row = z + (int64_t)at[j] * K + m;
    if constexpr (V == 4) {
      const float4 f = __ldcg(reinterpret_cast<const float4*>(row));
      v[0] = fmaf(by[j], f.x, v[0]), v[1] = fmaf(by[j], f.y, v[1]), v[2] = fmaf(by[j], f.z, v[2]), v[3] = fmaf(by[j], f.w, v[3]);
    } else {
      v[0] = fmaf(by[j], __ldcg(row), v[0]);
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) store_typed(y, ytype, (int64_t)p * K + m + i, v[i]);
}

// ------------------------------------------------------------------ host side
template <typename T, typename R, int TOKENS>
fgq_status launch_route_tokens(const RouteArgs& a, bool vec, cudaStream_t s) {
  int ks = 1;  // warps that share an expert's row
  while (ks < RT_WARPS && RT_CLUSTER * RT_WARPS / (2 * ks) >= a.E) ks *= 2;
  const unsigned grid = (unsigned)(((int64_t)a.P + TOKENS - 1) / TOKENS * RT_CLUSTER);
  if (vec)
    route_kernel<T, R, TOKENS, true><<<grid, 32 * RT_WARPS, 0, s>>>(a, ks);
  else
    route_kernel<T, R, TOKENS, false><<<grid, 32 * RT_WARPS, 0, s>>>(a, ks);
  return after_launch();
}
template <typename T, typename R>
fgq_status launch_route_t(const RouteArgs& a, bool vec, cudaStream_t s) {
  return a.P == 1 ? launch_route_tokens<T, R, 1>(a, vec, s) : launch_route_tokens<T, R, RT_TOKENS>(a, vec, s);
}
fgq_status launch_route(const RouteArgs& a, int type, int rtype, cudaStream_t s) {
  const bool vec = a.K % 8 == 0 && aligned(a.x, 16) && aligned(a.router, 16) && (a.P == 1 || stride16(a.ldx, type));
  if (type == FGQ_F32) return launch_route_t<float, float>(a, vec, s);
  if (type == FGQ_BF16)
    return rtype == FGQ_F32 ? launch_route_t<__nv_bfloat16, float>(a, vec, s) : launch_route_t<__nv_bfloat16, __nv_bfloat16>(a, vec, s);
  return rtype == FGQ_F32 ? launch_route_t<__half, float>(a, vec, s) : launch_route_t<__half, __half>(a, vec, s);
}

struct Route {
  const void* router;
  int rtype, E, score, renormalize;
  float scale;
};

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// How tokens are held in shared memory: as many as a unit may have (0: not even one fits), a unit's, and the plans of both layers.
struct HeldPlan {
  int most, cap;
  ResidentPlan hidden, down;
};
HeldPlan plan_units(int type, int pass, int ctk, int per, int ctf, int down_per) {
  HeldPlan p = {};
  const int parts = type == FGQ_F32 ? 3 : 2;  // of a hidden value
  for (int cap = type == FGQ_F32 ? 4 : 8; cap > 0; cap /= 2) {
    const int c = pass < cap ? pass : cap;
    p.hidden = type == FGQ_F32 ? plan_resident<2, 2, GATED_AHEAD>(ctk, per, c * columns_per_token(3)) : plan_resident<2, 1, GATED_AHEAD>(ctk, per, c);
    p.down = plan_held(2, ctf, down_per, c * columns_per_token(parts));
    p.most = cap;
    p.cap = c;
    if (p.hidden.warps > 0 && p.down.warps > 0) return p;
  }
  p.most = p.cap = 0;
  return p;
}

// Units of an expert on average up to which tokens are held.  bf16, us so and on the products of many tokens: 8 experts 2048 -> 1024, 2 a
// token, 64 tokens 33 and 39, 128 tokens 45 and 42; 128 experts 2048 -> 768, 8 a token, 256 tokens 238 and 271, 512 tokens 425 and 402;
// units of 2 (8 experts 4096 -> 14336) 16 tokens 327 and 413, 24 tokens 512 and 415; fp32, 32 experts 4096 -> 1024, 4 a token, 40 tokens
// 127 and 150, 128 tokens 260 and 151.
constexpr int HELD_UNITS = 2;
// Up to so many choices an expert on average units have 32 tokens in place of 64 (us, 8 experts 4096 -> 14336, 2 a token: bf16, 64 tokens 404 and 436,
// 128 tokens 555 and 439; fp32, 64 tokens 416 and 555, 128 tokens 569 and 557), 64 in place of 128 (bf16, 128 tokens 439 and 561; 8 experts
// 2048 -> 1024, 256 tokens 71 and 54), and 128 in place of 256, of fp32 always, where two rows a token fill a product's columns (bf16, 32 experts
// 4096 -> 1024, 4 a token, 1024 tokens 399 and 433; 8 experts 4096 -> 14336, 1024 tokens 1506 and 1402).
constexpr int UNIT_32_MAX = 16, UNIT_64_MAX = 32, UNIT_128_MAX = 128;

// route == nullptr: ids and weights are given.
fgq_status run_experts(const void* x, int type, int P, int64_t ldx, const Route* route, const int32_t* ids, const float* weights,
                       int top, const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down, void* y, cudaStream_t s) {
  const int K = gate->cols, F = gate->rows, E = gate->experts;
  const int most = MAX_CHOICES / top, pass = P < most ? P : most, A = pass * top;  // tokens and choices of a pass
  const int parts = type == FGQ_F32 ? 3 : 1;
  const int64_t hpitch = (int64_t)row_tiles(F) * TILE_ROWS, xpitch = parts * copied_pitch(K);
  const HeldPlan plan = plan_units(type, pass, col_tiles(K), TILE_COLS / gate->group, col_tiles(F), TILE_COLS / down->group);
  const bool held = A <= (int64_t)HELD_UNITS * plan.most * E;
  const bool small = A <= (int64_t)UNIT_32_MAX * E, large = type != FGQ_F32 && A > (int64_t)UNIT_128_MAX * E;
  const int cap = held ? plan.cap : (small ? 32 : (A <= (int64_t)UNIT_64_MAX * E ? 64 : (large ? 256 : 128)));
  const bool direct = !held || (type != FGQ_F32 && pieces16(x, type, P, K, ldx));
  const int most_units = (A < E || pass == 1 ? A : E) + A / cap;
  const size_t b_x = direct ? 0 : up256((size_t)pass * xpitch * 2);
  const size_t b_h = held ? up256((size_t)A * hpitch * 4) : up256(experts_many_bytes(type, A, K, F));
  const size_t b_units = up256(sizeof(Unit) * most_units), b_choices = up256(sizeof(Choice) * (size_t)A), b_n = 256;
  const size_t b_places = up256(4 * (size_t)A), b_z = up256(4 * (size_t)A * K), b_ids = route ? b_places : 0;
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(b_x + b_h + b_units + b_choices + b_n + 2 * b_places + b_z + 2 * b_ids, s));
  if (!tmp) return FGQ_ERR_CUDA;
  uint8_t* at = tmp;
  auto take = [&](size_t n) {
    uint8_t* p = at;
    at += n;
    return p;
  };
  uint16_t* xc = reinterpret_cast<uint16_t*>(take(b_x));
  void* h = take(b_h);
  Unit* units = reinterpret_cast<Unit*>(take(b_units));
  Choice* choices = reinterpret_cast<Choice*>(take(b_choices));
  int* nunits = reinterpret_cast<int*>(take(b_n));
  int32_t* places = reinterpret_cast<int32_t*>(take(b_places));
  unsigned* tops = reinterpret_cast<unsigned*>(take(b_places));
  float* z = reinterpret_cast<float*>(take(b_z));
  int32_t* own_ids = reinterpret_cast<int32_t*>(take(b_ids));
  float* own_weights = reinterpret_cast<float*>(take(b_ids));
  const Matrix mg = matrix(gate), mu = matrix(up), md = matrix(down);
  fgq_status st = FGQ_OK;
  for (int p0 = 0; p0 < P && st == FGQ_OK; p0 += pass) {
    const int np = P - p0 < pass ? P - p0 : pass, na = np * top;
    const uint8_t* xp = static_cast<const uint8_t*>(x) + p0 * ldx * float_bytes(type);
    TokenRows rows = {xp, ldx, K, ROWS_COPIED};
    if (!direct) {
      if (type == FGQ_F32)
        operand_rows_kernel<<<np, 256, 0, s>>>(reinterpret_cast<const float*>(xp), K, ldx, xc, copied_pitch(K));
      else
        operand_rows_kernel<<<np, 256, 0, s>>>(reinterpret_cast<const uint16_t*>(xp), K, ldx, xc, copied_pitch(K));
      st = after_launch();
      if (st != FGQ_OK) break;
      rows = {xc, xpitch, (int)copied_pitch(K), ROWS_COPIED};
    }
    const int32_t* pid = ids ? ids + (int64_t)p0 * top : own_ids;
    const float* pw = weights ? weights + (int64_t)p0 * top : own_weights;
    const bool one = route && np <= RT_TOKENS && cap >= np;  // a cluster's tokens: it leaves units and choices itself
    if (route) {
      const RouteArgs ra = {xp, route->router, ldx, own_ids, own_weights, one ? units : nullptr, choices, places, tops, nunits, np, K, E, top,
                            route->score, route->renormalize, route->scale};
      st = launch_route(ra, type, route->rtype, s);
      if (st != FGQ_OK) break;
    }
    if (!one) {
      if (route) {
        st = after_launch(launch_pdl(group_kernel, dim3(1), dim3(GR_THREADS), 0, s, pid, pw, na, top, E, cap, units, choices, places, tops, nunits));
      } else {  // the kernel before is the caller's, or the copy
        group_kernel<<<1, GR_THREADS, 0, s>>>(pid, pw, na, top, E, cap, units, choices, places, tops, nunits);
        st = after_launch();
      }
      if (st != FGQ_OK) break;
    }
    const int nu = one ? (na < E ? na : E) : (na < E || np == 1 ? na : E + na / cap);  // units at most
    if (held) {
      const int64_t hi = (int64_t)nu * mg.rt, di = (int64_t)nu * md.rt;
      if (hi > INT32_MAX || di > INT32_MAX) {
        st = FGQ_ERR_UNSUPPORTED;
        break;
      }
      ResidentArgs ra = {};
      ra.w = mg, ra.up = mu, ra.x = rows, ra.M = F, ra.units = units, ra.choices = choices, ra.nunits = nunits;
      ra.h = static_cast<float*>(h), ra.hpitch = hpitch, ra.top = tops, ra.one = np == 1;
      ra.items = one && np == 1 ? (int)hi : 0;  // one token picks distinct experts
      st = type == FGQ_F32 ? launch_held_gated_f32(ra, plan.hidden, hi, s)
                           : (type == FGQ_BF16 ? launch_held_gated_bf16(ra, plan.hidden, hi, s) : launch_held_gated_f16(ra, plan.hidden, hi, s));
      if (st != FGQ_OK) break;
      ra.w = md, ra.M = K, ra.z = z, ra.items = ra.items ? (int)di : 0;
      st = type == FGQ_F32 ? launch_held_down_f32(ra, plan.down, di, s) : launch_held_down_16(ra, plan.down, di, s);
    } else {
      st = launch_experts_many({mg, mu, md, units, choices, nunits, K, F, na, cap, nu, h, z}, xp, type, ldx, s);
    }
    if (st != FGQ_OK) break;
    const bool four = K % 4 == 0;
    const dim3 cg((unsigned)((K + (four ? 1023 : 255)) / (four ? 1024 : 256)), (unsigned)np);
    void* yp = static_cast<uint8_t*>(y) + (int64_t)p0 * K * float_bytes(type);
    st = after_launch(launch_pdl(four ? combine_kernel<4> : combine_kernel<1>, cg, dim3(256), 0, s, static_cast<const float*>(z),
                                 static_cast<const int32_t*>(places), pw, top, K, yp, type));
  }
  if (cudaFreeAsync(tmp, s) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

fgq_status check_experts(const void* x, int type, int P, int64_t ldx, int top, const fgq_w4* gate, const fgq_w4* up,
                         const fgq_w4* down, const void* y) {
  if (P < 0 || !valid_float(type)) return FGQ_ERR_ARG;
  for (const fgq_w4* w : {gate, up, down}) {
    const fgq_status st = check_weights(w);
    if (st != FGQ_OK) return st;
  }
  const int K = gate->cols, F = gate->rows, E = gate->experts;
  if (up->cols != K || up->rows != F || up->experts != E || up->group != gate->group || down->rows != K || down->cols != F ||
      down->experts != E)
    return FGQ_ERR_ARG;
  if (top < 1 || top > MAX_TOP || (P > 1 && ldx < K)) return FGQ_ERR_ARG;
  if (P == 0 || K == 0) return FGQ_OK;
  if (E > MAX_EXPERTS || P > MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
  if (!x || !y || E < 1 || F < 1) return FGQ_ERR_ARG;
  const uintptr_t e = float_bytes(type);
  if (!aligned(x, e) || !aligned(y, e)) return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

fgq_status check_route(const void* x, int type, int P, int K, int64_t ldx, const void* router, int rtype, int E, int top, int score,
                       int renormalize, float scale) {
  if (P < 0 || K < 1 || E < 1 || !valid_float(type) || !valid_float(rtype) || (rtype != type && rtype != FGQ_F32)) return FGQ_ERR_ARG;
  if ((score != FGQ_SCORE_SOFTMAX && score != FGQ_SCORE_SIGMOID) || (renormalize != 0 && renormalize != 1) || nonfinite_host(scale))
    return FGQ_ERR_ARG;
  if (top < 1 || top > E || (P > 1 && ldx < K)) return FGQ_ERR_ARG;
  if (P == 0) return FGQ_OK;
  if (E > MAX_EXPERTS || top > MAX_TOP || P > 1 << 29 || K > MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
  if (!x || !router) return FGQ_ERR_ARG;
  if (!aligned(x, float_bytes(type)) || !aligned(router, float_bytes(rtype))) return FGQ_ERR_ALIGN;
  return FGQ_OK;
}

}  // namespace
}  // namespace w4
}  // namespace fgq

using namespace fgq;

extern "C" {

fgq_status fgq_route_tokens(const void* x, fgq_float_type type, int P, int K, int64_t ldx, const void* router,
                            fgq_float_type rtype, int E, int top, fgq_score score, int renormalize, float scale, int32_t* ids,
                            float* weights, cudaStream_t stream) {
  using namespace w4;
  fgq_status st = check_route(x, type, P, K, ldx, router, rtype, E, top, score, renormalize, scale);
  if (st != FGQ_OK || P == 0) return st;
  if (!ids || !weights) return FGQ_ERR_ARG;
  if (!aligned(ids, 4) || !aligned(weights, 4)) return FGQ_ERR_ALIGN;
  return launch_route({x, router, P > 1 ? ldx : 0, ids, weights, nullptr, nullptr, nullptr, nullptr, nullptr, P, K, E, top, score, renormalize, scale},
                      type, rtype, stream);
}

fgq_status fgq_experts_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const int32_t* ids, const float* weights, int top,
                          const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down, void* y, cudaStream_t stream) {
  using namespace w4;
  const fgq_status st = check_experts(x, type, P, ldx, top, gate, up, down, y);
  if (st != FGQ_OK || P == 0 || gate->cols == 0) return st;
  if (!ids || !weights) return FGQ_ERR_ARG;
  if (!aligned(ids, 4) || !aligned(weights, 4)) return FGQ_ERR_ALIGN;
  return run_experts(x, type, P, P > 1 ? ldx : 0, nullptr, ids, weights, top, gate, up, down, y, stream);
}

fgq_status fgq_moe_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const void* router, fgq_float_type rtype, int top,
                      fgq_score score, int renormalize, float scale, const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down,
                      void* y, cudaStream_t stream) {
  using namespace w4;
  fgq_status st = check_experts(x, type, P, ldx, top, gate, up, down, y);
  if (st != FGQ_OK) return st;
  st = check_route(x, type, P, gate->cols, ldx, router, rtype, gate->experts, top, score, renormalize, scale);
  if (st != FGQ_OK || P == 0) return st;
  const Route route = {router, rtype, gate->experts, score, renormalize, scale};
  return run_experts(x, type, P, P > 1 ? ldx : 0, &route, nullptr, nullptr, top, gate, up, down, y, stream);
}

}  // extern "C"
