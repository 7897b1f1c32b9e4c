// Mixture of experts on 4-bit weights, for few tokens.
//
//   l = router x;  the `top` largest, their weights g;  y = sum_j g_j down_e (silu(gate_e x) * (up_e x)),  e = the j-th choice
//
// Kernels of a layer, each brought up while the one before it runs:
//   logits_kernel   four warps an expert, four tokens: products of 8 elements in fp32, their sums as pairs of fp32 (two-sum), so that a
//                   logit is off by about one fp32 rounding and the choice is that of 64-bit sums but for near ties;
//   select_kernel   a warp a token: the largest one by one, then the weights;
//   group_kernel    one block: choices sorted by expert, and cut into units of up to CAP tokens that share an expert;
//   hidden_kernel   a block 16 rows of gate and the same 16 of up, for one unit: silu(gate) up, left as bf16 parts;
//   down_kernel     a block 16 rows of down, for all units: sums stay with the block, so nothing is added up across blocks
//                   and no order depends on which comes first.
// Bound by the bytes of the experts' weights, each read once (again from L2 where more than CAP tokens share an expert).
#include <type_traits>

#include "linear_internal.cuh"
#include "w4.cuh"

namespace fgq {
namespace w4 {
namespace {

constexpr int MAX_EXPERTS = 1024, MAX_TOP = 32;
constexpr int CHUNK = 128;  // tokens of a pass

// ------------------------------------------------------------------ routing
struct RouteArgs {
  const void* x;
  const void* router;
  double* logits;  // [P][E]
  int64_t ldx;
  int P, K, E;
};

template <typename T>
__device__ __forceinline__ void load_row8(const T* row, int k, int K, bool vec, float (&v)[8]) {
  if (vec) {
    load8(row + k, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < K ? to_float(row[k + i]) : 0.0f;
  }
}

constexpr int LG_WARPS = 8, LG_SPLIT = 4, LG_TOKENS = 4;
template <typename T, typename R>
__global__ void __launch_bounds__(32 * LG_WARPS) logits_kernel(const __grid_constant__ RouteArgs a, int vec) {
  __shared__ double part[LG_WARPS][LG_TOKENS];
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int e = (int)blockIdx.x * (LG_WARPS / LG_SPLIT) + warp / LG_SPLIT, p0 = (int)blockIdx.y * LG_TOKENS;
  const int np = min(LG_TOKENS, a.P - p0);
  float hi[LG_TOKENS], lo[LG_TOKENS];
#pragma unroll
  for (int i = 0; i < LG_TOKENS; ++i) hi[i] = lo[i] = 0.0f;
  if (e < a.E) {
    const R* wr = static_cast<const R*>(a.router) + (int64_t)e * a.K;
    const T* x = static_cast<const T*>(a.x) + p0 * a.ldx;
#pragma unroll 2
    for (int k = 8 * (lane + 32 * (warp % LG_SPLIT)); k < a.K; k += 256 * LG_SPLIT) {
      float w[8];
      load_row8(wr, k, a.K, vec, w);
#pragma unroll
      for (int i = 0; i < LG_TOKENS; ++i)
        if (i < np) {
          float v[8];
          load_row8(x + i * a.ldx, k, a.K, vec, v);
          float s = v[0] * w[0];
#pragma unroll
          for (int j = 1; j < 8; ++j) s = fmaf(v[j], w[j], s);
          const float t = hi[i] + s, b = t - hi[i];  // t + the second line's sum = hi + s exactly
          lo[i] += (hi[i] - (t - b)) + (s - b);
          hi[i] = t;
        }
    }
  }
#pragma unroll
  for (int i = 0; i < LG_TOKENS; ++i) {
    double v = (double)hi[i] + (double)lo[i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_MASK, v, o);
    // an overflow leaves NaN in the second sum: the first says what it was
    const float h = hi[i];
    const unsigned inf = __ballot_sync(FULL_MASK, nonfinite(h));
    if (inf) {
      float f = h;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) f += __shfl_xor_sync(FULL_MASK, f, o);
      v = (double)f;
    }
    if (lane == 0) part[warp][i] = v;
  }
  __syncthreads();
  if (threadIdx.x < (LG_WARPS / LG_SPLIT) * LG_TOKENS) {
    const int el = threadIdx.x / LG_TOKENS, i = threadIdx.x % LG_TOKENS, ee = (int)blockIdx.x * (LG_WARPS / LG_SPLIT) + el;
    if (ee < a.E && i < np) {
      double v = 0.0;
#pragma unroll
      for (int s = 0; s < LG_SPLIT; ++s) v += part[el * LG_SPLIT + s][i];
      a.logits[(int64_t)(p0 + i) * a.E + ee] = v;
    }
  }
}

// A unit of work: up to CAP choices of one expert, `count` of them from `start` on in the sorted order.
struct Unit {
  int expert, start, count, pad;
};

struct SelectArgs {
  const double* logits;
  int32_t* ids;
  float* weights;
  // P == 1: what group_kernel would find
  Unit* units;
  int32_t* order;
  int* nunits;
  int P, E, top, score, renormalize;
  float scale;
};

// 64-bit floats as whole numbers of the same order; NaN below all.
__device__ __forceinline__ long long order_key(double v) {
  const long long b = __double_as_longlong(v);
  return v == v ? (b < 0 ? b ^ 0x7fffffffffffffffll : b) : (long long)0x8000000000000000ull;
}
__device__ __forceinline__ double key_value(long long k) { return __longlong_as_double(k < 0 ? k ^ 0x7fffffffffffffffll : k); }

template <int EL>
__global__ void __launch_bounds__(128) select_kernel(const __grid_constant__ SelectArgs a) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, p = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 5);
  if (p >= a.P) return;
  constexpr long long NONE = (long long)0x8000000000000000ull;
  long long key[EL];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < EL; ++i) {
    const int e = lane + 32 * i;
    double v = 0.0;
    if (e < a.E) {
      v = __ldcg(a.logits + (int64_t)p * a.E + e);
      bad |= !(v == v);
    }
    key[i] = e < a.E ? order_key(v) : NONE;
  }
  bad = __any_sync(FULL_MASK, bad);
  unsigned taken = 0;  // of this lane's, a bit each
  double best = 0.0;   // the largest
  float mine = 0.0f, total = 0.0f;  // lane j: the j-th choice's value; their sum
  int mine_id = 0;
  for (int j = 0; j < a.top; ++j) {
    long long k = NONE;
    int id = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const bool open = !(taken >> i & 1u) && lane + 32 * i < a.E;
      if (open && (id == 0x7fffffff || key[i] > k)) {
        k = key[i];
        id = lane + 32 * i;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const long long k2 = __shfl_xor_sync(FULL_MASK, k, o);
      const int id2 = __shfl_xor_sync(FULL_MASK, id, o);
      if (k2 > k || (k2 == k && id2 < id)) {
        k = k2;
        id = id2;
      }
    }
    if ((id & 31) == lane) taken |= 1u << (id >> 5);
    const double v = key_value(k);
    if (j == 0) best = v;
    const float f = a.score == FGQ_SCORE_SOFTMAX ? expf((float)(v - best)) : 1.0f / (1.0f + expf(-(float)v));
    if (lane == j) {
      mine = f;
      mine_id = id;
    }
    total += f;
  }
  if (a.score == FGQ_SCORE_SOFTMAX && !a.renormalize) {
    total = 0.0f;
#pragma unroll
    for (int i = 0; i < EL; ++i)
      if (lane + 32 * i < a.E) total += expf((float)(key_value(key[i]) - best));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(FULL_MASK, total, o);
  }
  float w = mine;
  if (a.score == FGQ_SCORE_SOFTMAX || a.renormalize) w /= total;
  w *= a.scale;
  if (bad) w = __uint_as_float(0x7fc00000u);
  int rank = 0;  // by expert
  if (a.units)
    for (int j = 0; j < a.top; ++j) rank += __shfl_sync(FULL_MASK, mine_id, j) < mine_id;
  if (lane < a.top) {
    a.ids[(int64_t)p * a.top + lane] = mine_id;
    a.weights[(int64_t)p * a.top + lane] = w;
    if (a.units) {
      a.units[rank] = {mine_id, rank, 1, 0};
      a.order[rank] = lane;
    }
  }
  if (a.units && lane == 0) *a.nunits = a.top;
}

// ------------------------------------------------------------------ choices by expert
constexpr int GR_THREADS = 1024;

// Sum of the values of the threads before this one; `total`: of all.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(FULL_MASK, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();  // the sums of the scan before have been read
  if (lane == 31) warp_sums[warp] = s;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < GR_THREADS / 32; ++i) {
    const int u = warp_sums[i];
    before += i < warp ? u : 0;
    total += u;
  }
  return before + s - v;
}

__global__ void __launch_bounds__(GR_THREADS) group_kernel(const int32_t* ids, int A, int E, int cap, Unit* units, int32_t* order,
                                                           int* nunits) {
  __shared__ int count[MAX_EXPERTS], start[MAX_EXPERTS], id[CHUNK * MAX_TOP], warp_sums[GR_THREADS / 32];
  pdl_trigger();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  count[t] = 0;
  __syncthreads();
  pdl_wait();
  for (int i = t; i < A; i += GR_THREADS) {
    const int e = __ldcg(ids + i);
    id[i] = e;
    if (e >= 0 && e < E) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  const int n = count[t];  // 0 from E on
  int total;
  const int first = block_scan(n, warp_sums, total);
  const int u0 = block_scan((n + cap - 1) / cap, warp_sums, total);
  start[t] = first;
  for (int u = 0; u * cap < n; ++u) units[u0 + u] = {t, first + u * cap, min(cap, n - u * cap), 0};
  if (t == 0) *nunits = total;
  __syncthreads();
  for (int e = warp; e < E; e += GR_THREADS / 32) {  // each expert's choices in the order they came
    const int want = count[e];
    int at = start[e], found = 0;
    for (int i = 0; found < want; i += 32) {
      const bool hit = i + lane < A && id[i + lane] == e;
      const unsigned m = __ballot_sync(FULL_MASK, hit);
      if (hit) order[at + __popc(m & ((1u << lane) - 1u))] = i + lane;
      at += __popc(m);
      found += __popc(m);
    }
  }
}

// ------------------------------------------------------------------ silu(gate x) * (up x)
constexpr int WARPS = 8, AHEAD = 2;

struct HiddenArgs {
  Matrix gate, up;
  TokenRows x;
  const Unit* units;
  const int32_t* order;
  const int* nunits;
  uint16_t* h;  // [choice][parts][hpitch], in sorted order
  int64_t hpitch;
  int F, top, splits;
};

// v as PARTS bf16 values that add up to it: all of it in three, within 2^-17 in two.
template <int PARTS>
__device__ __forceinline__ void hidden_parts(float v, uint16_t (&p)[3]) {
  if constexpr (PARTS == 3) {
    three_parts(v, p);
  } else {
    const float a = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
    const __nv_bfloat16 b = __float2bfloat16_rn(v - a);
    p[0] = (uint16_t)(__float_as_uint(a) >> 16);
    p[1] = *reinterpret_cast<const uint16_t*>(&b);
  }
}

template <typename T, int NT, int PER, int PARTS, int HPARTS>
__global__ void __launch_bounds__(32 * WARPS) hidden_kernel(const __grid_constant__ HiddenArgs a) {
  constexpr int STAGE = 8 * NT * 256, CPT = columns_per_token(PARTS);
  extern __shared__ __align__(16) uint8_t w4_smem[];
  __shared__ int64_t rows[8 * NT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int sp = blockIdx.x % a.splits, item = blockIdx.x / a.splits;
  const int unit = item / a.gate.rt, mt = item - unit * a.gate.rt;
  pdl_wait();
  pdl_trigger();  // from here on the kernel after may read the units
  if (unit >= __ldcg(a.nunits)) return;
  const int4 u = __ldcg(reinterpret_cast<const int4*>(a.units) + unit);  // expert, start, count
  const int c0 = (int)((int64_t)a.gate.ct * sp / a.splits), c1 = (int)((int64_t)a.gate.ct * (sp + 1) / a.splits);
  const int64_t first = ((int64_t)u.x * a.gate.rt + mt) * a.gate.ct;
  Tile<PER> tile[AHEAD][2];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int kt = c0 + warp + i * WARPS;
    if (kt < c1) {
      tile[i][0].load(a.gate.codes, a.gate.scales, first + kt, lane);
      tile[i][1].load(a.up.codes, a.up.scales, first + kt, lane);
    }
  }
  if (threadIdx.x < 8 * NT) {
    const int tok = threadIdx.x / CPT, part = threadIdx.x % CPT;
    rows[threadIdx.x] = tok < u.z && part < PARTS
                            ? 2 * ((int64_t)(__ldcg(a.order + u.y + tok) / a.top) * a.x.pitch + part * (a.x.pitch / PARTS)) : -1;
  }
  __syncthreads();
  const uint8_t* xb = static_cast<const uint8_t*>(a.x.data);
  uint8_t* ring = w4_smem + warp * AHEAD * STAGE;
  const uint32_t ring_at = smem_u32(ring);
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    const int kt = c0 + warp + i * WARPS;
    if (kt < c1) fetch_tokens<NT>(ring_at + i * STAGE, xb, rows, kt, a.x.kvalid, lane);
    cp_async_commit();
  }
  float sum[2][NT][4];
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[m][nt][e] = 0.0f;
  for (int kt = c0 + warp; kt < c1; kt += AHEAD * WARPS) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int at = kt + i * WARPS, next = at + AHEAD * WARPS;
      if (at >= c1) break;  // the same for the whole warp
      cp_async_wait<AHEAD - 1>();
      __syncwarp();
      multiply<T, 2, NT, PER>(tile[i], ring + i * STAGE, sum, lane);
      __syncwarp();
      if (next < c1) {
        tile[i][0].load(a.gate.codes, a.gate.scales, first + next, lane);
        tile[i][1].load(a.up.codes, a.up.scales, first + next, lane);
        fetch_tokens<NT>(ring_at + i * STAGE, xb, rows, next, a.x.kvalid, lane);
      }
      cp_async_commit();
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  constexpr int LD = 33;
  float* sums = reinterpret_cast<float*>(w4_smem);  // [warp][column][gate rows, up rows]
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[(warp * 8 * NT + 8 * nt + 2 * t + (e & 1)) * LD + 16 * m + g + 8 * (e >> 1)] = sum[m][nt][e];
  __syncthreads();
  // each value's sum over warps and parts, to the first warp's place
  for (int i = threadIdx.x; i < u.z * 32; i += 32 * WARPS) {
    float* at = sums + i / 32 * CPT * LD + i % 32;
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k)
#pragma unroll
      for (int part = 0; part < PARTS; ++part) v += at[(k * 8 * NT + part) * LD];
    *at = v;
  }
  if (a.splits > 1)
    cluster_sync();
  else
    __syncthreads();
  for (int i = threadIdx.x + 32 * WARPS * sp; i < u.z * 16; i += 32 * WARPS * a.splits) {
    const int tok = i / 16, f = i % 16;
    const float* at = sums + tok * CPT * LD + f;
    float gv = 0.0f, uv = 0.0f;
    if (a.splits == 1) {
      gv = at[0], uv = at[16];
    } else {
      for (int k = 0; k < a.splits; ++k) {
        gv += ld_cluster(at, k);
        uv += ld_cluster(at + 16, k);
      }
    }
    gv *= Operand<T>::BACK;
    uv *= Operand<T>::BACK;
    const int col = mt * TILE_ROWS + f;
    const float v = col < a.F ? gv / (1.0f + expf(-gv)) * uv : 0.0f;
    uint16_t p[3];
    hidden_parts<HPARTS>(v, p);
    uint16_t* to = a.h + (int64_t)(u.y + tok) * HPARTS * a.hpitch + col;
#pragma unroll
    for (int part = 0; part < HPARTS; ++part) to[part * a.hpitch] = p[part];
  }
  if (a.splits > 1) cluster_sync();  // no block leaves while another may read its sums
}

// ------------------------------------------------------------------ down
struct DownArgs {
  Matrix down;
  const uint16_t* h;
  int64_t hpitch;
  const Unit* units;
  const int32_t* order;
  const int* nunits;
  const float* weights;
  void* y;
  int P, K, ytype, top, splits;
};

// The block's warps share the pairs (unit, tile column) in runs of equal length; at a unit's end (or its share of it) a warp adds
// what it has, by the router's weights, to sums of its own for each token and row.
template <int NT, int PER, int HPARTS>
__global__ void __launch_bounds__(32 * WARPS) down_kernel(const __grid_constant__ DownArgs a) {
  using T = __nv_bfloat16;
  constexpr int STAGE = 8 * NT * 256, CPT = columns_per_token(HPARTS);
  extern __shared__ __align__(16) uint8_t w4_smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int sp = blockIdx.x % a.splits, mt = blockIdx.x / a.splits;
  constexpr int LD = TILE_ROWS + 1;
  float* part = reinterpret_cast<float*>(w4_smem + WARPS * AHEAD * STAGE);  // [warp][token][LD]
  float* own = part + warp * a.P * LD;
  uint8_t* ring = w4_smem + warp * AHEAD * STAGE;
  const uint32_t ring_at = smem_u32(ring);
  for (int i = lane; i < a.P * LD; i += 32) own[i] = 0.0f;
  __syncwarp();
  // units, the choices' order and their weights are those of kernels before the one that this one waits for
  const int ct = a.down.ct;
  const int64_t n = (int64_t)__ldcg(a.nunits) * ct;
  const int share = sp * WARPS + warp, shares = a.splits * WARPS;
  const int64_t q0 = n * share / shares, q1 = n * (share + 1) / shares;
  struct Place {
    int unit, kt;
    int4 u;
  };
  auto place = [&](int64_t q) {
    Place c;
    c.unit = (int)(q / ct);
    c.kt = (int)(q - (int64_t)c.unit * ct);
    c.u = q < q1 ? __ldcg(reinterpret_cast<const int4*>(a.units) + c.unit) : make_int4(0, 0, 0, 0);
    return c;
  };
  auto advance = [&](Place& c, bool more) {
    if (++c.kt == ct) {
      c.kt = 0;
      ++c.unit;
      if (more) c.u = __ldcg(reinterpret_cast<const int4*>(a.units) + c.unit);
    }
  };
  Tile<PER> tile[AHEAD][1];
  auto weights = [&](int i, const Place& c) {
    tile[i][0].load(a.down.codes, a.down.scales, ((int64_t)c.u.x * a.down.rt + mt) * ct + c.kt, lane);
  };
  auto hidden = [&](int i, const Place& c) {
    const int chunk = lane & 15, k = c.kt * TILE_COLS + 8 * chunk;
#pragma unroll
    for (int j = 0; j < 4 * NT; ++j) {
      const int col = 2 * j + (lane >> 4), tok = col / CPT, p = col % CPT;
      const bool live = tok < c.u.z && p < HPARTS && k < a.hpitch;
      cp_async16(ring_at + i * STAGE + chunk_at(col, chunk), live ? a.h + ((int64_t)(c.u.y + tok) * HPARTS + p) * a.hpitch + k : a.h, live);
    }
  };
  Place ahead = place(q0);
  {
    Place c = ahead;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (q0 + i < q1) {
        weights(i, c);
        advance(c, q0 + i + 1 < q1);
      }
  }
  pdl_wait();
  Place now = ahead;
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    if (q0 + i < q1) {
      hidden(i, ahead);
      advance(ahead, q0 + i + 1 < q1);
    }
    cp_async_commit();
  }
  float sum[1][NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[0][nt][e] = 0.0f;
  for (int64_t q = q0; q < q1; q += AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      if (q + i >= q1) break;
      cp_async_wait<AHEAD - 1>();
      __syncwarp();
      multiply<T, 1, NT, PER>(tile[i], ring + i * STAGE, sum, lane);
      __syncwarp();
      if (q + i + AHEAD < q1) {
        weights(i, ahead);
        hidden(i, ahead);
        advance(ahead, q + i + AHEAD + 1 < q1);
      }
      cp_async_commit();
      if (now.kt == ct - 1 || q + i + 1 == q1) {  // the unit's last tile here
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float v0, v1;  // rows g and g + 8 of this lane's token
          int tok;
          bool mine = true;
          if constexpr (HPARTS == 2) {
            v0 = sum[0][nt][0] + sum[0][nt][1];
            v1 = sum[0][nt][2] + sum[0][nt][3];
            tok = 4 * nt + t;
          } else {
            v0 = sum[0][nt][0] + sum[0][nt][1];
            v1 = sum[0][nt][2] + sum[0][nt][3];
            v0 += __shfl_xor_sync(FULL_MASK, v0, 1);
            v1 += __shfl_xor_sync(FULL_MASK, v1, 1);
            tok = 2 * nt + (t >> 1);
            mine = (t & 1) == 0;
          }
          mine &= tok < now.u.z;
          int token = -1;
          float w = 0.0f;
          if (mine) {
            const int choice = __ldcg(a.order + now.u.y + tok);
            token = choice / a.top;
            w = __ldcg(a.weights + choice) * Operand<T>::BACK;
          }
          float* at = own + token * LD;
          auto add = [&]() {
            at[g] = fmaf(w, v0, at[g]);
            at[g + 8] = fmaf(w, v1, at[g + 8]);
          };
          // a token that has the expert twice has both places beside one another
          constexpr int STEP = HPARTS == 2 ? 1 : 2;
          const int before = __shfl_up_sync(FULL_MASK, token, STEP);
          if (__any_sync(FULL_MASK, mine && t >= STEP && before == token)) {
            for (int i = 0; i < 4; ++i) {
              if (mine && t == i) add();
              __syncwarp();
            }
          } else if (mine) {
            add();
          }
          __syncwarp();
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[0][nt][e] = 0.0f;
        }
      }
      advance(now, q + i + 1 < q1);
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  for (int i = threadIdx.x; i < a.P * TILE_ROWS; i += 32 * WARPS) {
    float* at = part + i / TILE_ROWS * LD + i % TILE_ROWS;
    float v = 0.0f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) v += at[k * a.P * LD];
    *at = v;  // the first warp's place
  }
  if (a.splits > 1)
    cluster_sync();
  else
    __syncthreads();
  for (int i = threadIdx.x + 32 * WARPS * sp; i < a.P * TILE_ROWS; i += 32 * WARPS * a.splits) {
    const float* at = part + i / TILE_ROWS * LD + i % TILE_ROWS;
    float v = 0.0f;
    if (a.splits == 1)
      v = at[0];
    else
      for (int k = 0; k < a.splits; ++k) v += ld_cluster(at, k);
    const int m = mt * TILE_ROWS + i % TILE_ROWS;
    if (m < a.K) store_typed(a.y, a.ytype, (int64_t)(i / TILE_ROWS) * a.K + m, v);
  }
  if (a.splits > 1) cluster_sync();  // no block leaves while another may read its sums
}

// ------------------------------------------------------------------ host side
template <typename... KArgs>
fgq_status launch_chained(void (*kernel)(KArgs...), dim3 grid, unsigned threads, size_t smem, int splits, cudaStream_t s, KArgs... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  unsigned n = 0;
  attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[n++].val.programmaticStreamSerializationAllowed = 1;
  if (splits > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = (unsigned)splits;
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return after_launch(cudaLaunchKernelEx(&cfg, kernel, args...));
}

template <typename T, typename R>
fgq_status launch_logits_t(const RouteArgs& a, bool vec, cudaStream_t s) {
  for (int p = 0; p < a.P; p += 65535 * LG_TOKENS) {
    RouteArgs part = a;
    part.P = a.P - p < 65535 * LG_TOKENS ? a.P - p : 65535 * LG_TOKENS;
    part.x = static_cast<const T*>(a.x) + p * a.ldx;
    part.logits = a.logits + (int64_t)p * a.E;
    constexpr int EPB = LG_WARPS / LG_SPLIT;
    logits_kernel<T, R><<<dim3((a.E + EPB - 1) / EPB, (part.P + LG_TOKENS - 1) / LG_TOKENS), 32 * LG_WARPS, 0, s>>>(part, vec);
    const fgq_status st = after_launch();
    if (st != FGQ_OK) return st;
  }
  return FGQ_OK;
}
fgq_status launch_logits(const RouteArgs& a, int type, int rtype, cudaStream_t s) {
  const bool vec = a.K % 8 == 0 && aligned(a.x, 16) && aligned(a.router, 16) && (a.P == 1 || stride16(a.ldx, type));
  if (type == FGQ_F32) return launch_logits_t<float, float>(a, vec, s);
  if (type == FGQ_BF16)
    return rtype == FGQ_F32 ? launch_logits_t<__nv_bfloat16, float>(a, vec, s) : launch_logits_t<__nv_bfloat16, __nv_bfloat16>(a, vec, s);
  return rtype == FGQ_F32 ? launch_logits_t<__half, float>(a, vec, s) : launch_logits_t<__half, __half>(a, vec, s);
}
fgq_status launch_select(const SelectArgs& a, cudaStream_t s) {
  const dim3 grid(((unsigned)a.P + 3) / 4);
  if (a.E <= 64) return launch_chained(select_kernel<2>, grid, 128, 0, 1, s, a);
  if (a.E <= 256) return launch_chained(select_kernel<8>, grid, 128, 0, 1, s, a);
  return launch_chained(select_kernel<32>, grid, 128, 0, 1, s, a);
}

struct Route {
  const void* router;
  int rtype, E, score, renormalize;
  float scale;
};

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

template <int NT, int PARTS, int HPARTS, typename T, int PER>
fgq_status launch_hidden_k(const HiddenArgs& a, int blocks, cudaStream_t s) {
  constexpr int RING = WARPS * AHEAD * 8 * NT * 256, SUMS = WARPS * 8 * NT * 33 * 4, BYTES = RING > SUMS ? RING : SUMS;
  if (!tc::smem_attr_once<hidden_kernel<T, NT, PER, PARTS, HPARTS>>(BYTES)) return FGQ_ERR_CUDA;
  return launch_chained(hidden_kernel<T, NT, PER, PARTS, HPARTS>, dim3((unsigned)blocks), 32 * WARPS, BYTES, a.splits, s, a);
}
template <int NT, int PARTS, int HPARTS, typename T>
fgq_status launch_hidden_per(const HiddenArgs& a, int blocks, cudaStream_t s) {
  if (a.gate.per == 4) return launch_hidden_k<NT, PARTS, HPARTS, T, 4>(a, blocks, s);
  if (a.gate.per == 2) return launch_hidden_k<NT, PARTS, HPARTS, T, 2>(a, blocks, s);
  return launch_hidden_k<NT, PARTS, HPARTS, T, 1>(a, blocks, s);
}
template <int NT, int HPARTS, int PER>
fgq_status launch_down_k(const DownArgs& a, cudaStream_t s) {
  constexpr int RING = WARPS * AHEAD * 8 * NT * 256, MOST = RING + WARPS * CHUNK * (TILE_ROWS + 1) * 4;
  static_assert(MOST <= 232448, "shared memory budget");
  if (!tc::smem_attr_once<down_kernel<NT, PER, HPARTS>>(MOST)) return FGQ_ERR_CUDA;
  return launch_chained(down_kernel<NT, PER, HPARTS>, dim3((unsigned)(a.down.rt * a.splits)), 32 * WARPS,
                        RING + WARPS * a.P * (TILE_ROWS + 1) * 4, a.splits, s, a);
}
template <int NT, int HPARTS>
fgq_status launch_down_per(const DownArgs& a, cudaStream_t s) {
  if (a.down.per == 4) return launch_down_k<NT, HPARTS, 4>(a, s);
  if (a.down.per == 2) return launch_down_k<NT, HPARTS, 2>(a, s);
  return launch_down_k<NT, HPARTS, 1>(a, s);
}

// Tokens of a unit: 8, which the columns of one product hold, or 16 where experts have more on average.  fp32 tokens take
// four columns each.
fgq_status launch_hidden(const HiddenArgs& a, int type, int cap, int blocks, cudaStream_t s) {
  if (type == FGQ_F32) return launch_hidden_per<4, 3, 3, __nv_bfloat16>(a, blocks, s);
  if (type == FGQ_BF16)
    return cap == 8 ? launch_hidden_per<1, 1, 2, __nv_bfloat16>(a, blocks, s) : launch_hidden_per<2, 1, 2, __nv_bfloat16>(a, blocks, s);
  return cap == 8 ? launch_hidden_per<1, 1, 2, __half>(a, blocks, s) : launch_hidden_per<2, 1, 2, __half>(a, blocks, s);
}
fgq_status launch_down(const DownArgs& a, int type, int cap, cudaStream_t s) {
  if (type == FGQ_F32) return launch_down_per<4, 3>(a, s);
  return cap == 8 ? launch_down_per<2, 2>(a, s) : launch_down_per<4, 2>(a, s);
}

// route == nullptr: ids and weights are given.
fgq_status run_experts(const void* x, int type, int P, int64_t ldx, const Route* route, const int32_t* ids, const float* weights,
                       int top, const fgq_w4* gate, const fgq_w4* up, const fgq_w4* down, void* y, cudaStream_t s) {
  const int K = gate->cols, F = gate->rows, E = gate->experts;
  const int pass = P < CHUNK ? P : CHUNK, A = pass * top;  // of the largest pass
  const int parts = type == FGQ_F32 ? 3 : 1, hparts = type == FGQ_F32 ? 3 : 2;
  const bool direct = direct_tokens(x, type, P, K, ldx);
  const int64_t hpitch = (int64_t)row_tiles(F) * TILE_ROWS;
  const int cap = type != FGQ_F32 && (int64_t)A > 8ll * E ? 16 : 8;
  const int most_units = (A < E || P == 1 ? A : E) + A / cap;
  const size_t b_x = direct ? 0 : up256(copied_bytes(type, pass, K)), b_h = up256((size_t)A * hparts * hpitch * 2);
  const size_t b_units = up256(sizeof(Unit) * most_units), b_order = up256(4 * (size_t)A), b_n = 256;
  const size_t b_logits = route ? up256(8 * (size_t)pass * E) : 0, b_ids = route ? up256(4 * (size_t)A) : 0;
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(b_x + b_h + b_units + b_order + b_n + b_logits + 2 * b_ids, s));
  if (!tmp) return FGQ_ERR_CUDA;
  uint8_t* at = tmp;
  auto take = [&](size_t n) {
    uint8_t* p = at;
    at += n;
    return p;
  };
  void* xc = take(b_x);
  uint16_t* h = reinterpret_cast<uint16_t*>(take(b_h));
  Unit* units = reinterpret_cast<Unit*>(take(b_units));
  int32_t* order = reinterpret_cast<int32_t*>(take(b_order));
  int* nunits = reinterpret_cast<int*>(take(b_n));
  double* logits = reinterpret_cast<double*>(take(b_logits));
  int32_t* own_ids = reinterpret_cast<int32_t*>(take(b_ids));
  float* own_weights = reinterpret_cast<float*>(take(b_ids));
  const Matrix mg = matrix(gate), mu = matrix(up), md = matrix(down);
  fgq_status st = FGQ_OK;
  for (int p0 = 0; p0 < P && st == FGQ_OK; p0 += CHUNK) {
    const int np = P - p0 < CHUNK ? P - p0 : CHUNK, na = np * top;
    const uint8_t* xp = static_cast<const uint8_t*>(x) + p0 * ldx * float_bytes(type);
    TokenRows rows = {xp, ldx, K};
    if (!direct) {
      st = launch_copy_tokens(xp, type, np, K, ldx, xc, s);
      if (st != FGQ_OK) break;
      const int64_t pitch = copied_pitch(K);
      rows = {xc, parts * pitch, (int)pitch};
    }
    const int32_t* pid = ids ? ids + (int64_t)p0 * top : own_ids;
    const float* pw = weights ? weights + (int64_t)p0 * top : own_weights;
    if (route) {
      const RouteArgs ra = {xp, route->router, logits, ldx, np, K, E};
      st = launch_logits(ra, type, route->rtype, s);
      if (st != FGQ_OK) break;
      const SelectArgs sa = {logits, own_ids, own_weights, np == 1 ? units : nullptr, order, nunits, np, E, top, route->score,
                             route->renormalize, route->scale};
      st = launch_select(sa, s);
      if (st != FGQ_OK) break;
    }
    if (!route || np > 1) {
      // without a router the kernel before is the caller's, or the copy
      if (route)
        st = launch_chained(group_kernel, dim3(1), GR_THREADS, 0, 1, s, pid, na, E, cap, units, order, nunits);
      else {
        group_kernel<<<1, GR_THREADS, 0, s>>>(pid, na, E, cap, units, order, nunits);
        st = after_launch();
      }
      if (st != FGQ_OK) break;
    }
    HiddenArgs ha = {mg, mu, rows, units, order, nunits, h, hpitch, F, top, 1};
    const int nu = (na < E || np == 1 ? na : E) + (np == 1 ? 0 : na / cap);
    // blocks that share K or the units: up to two an SM, a tile for each warp
    const int64_t hb = (int64_t)nu * mg.rt;
    while (ha.splits < 8 && hb * ha.splits * 2 <= 2 * device_sms() && mg.ct >= 2 * WARPS * ha.splits) ha.splits *= 2;
    if (hb * ha.splits > INT32_MAX) st = FGQ_ERR_UNSUPPORTED;
    if (st == FGQ_OK) st = launch_hidden(ha, type, cap, (int)(hb * ha.splits), s);
    if (st != FGQ_OK) break;
    DownArgs da = {md, h, hpitch, units, order, nunits, pw, static_cast<uint8_t*>(y) + (int64_t)p0 * K * float_bytes(type), np, K,
                   type, top, 1};
    while (da.splits < 8 && (int64_t)md.rt * da.splits * 2 <= 2 * device_sms() && (int64_t)nu * md.ct >= 2 * WARPS * da.splits)
      da.splits *= 2;
    st = launch_down(da, type, cap, s);
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
  if (E > MAX_EXPERTS || top > MAX_TOP || P > MAX_SIZE || K > MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
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
  double* logits = static_cast<double*>(scratch_alloc(8 * (size_t)P * E, stream));
  if (!logits) return FGQ_ERR_CUDA;
  st = launch_logits({x, router, logits, P > 1 ? ldx : 0, P, K, E}, type, rtype, stream);
  if (st == FGQ_OK) st = launch_select({logits, ids, weights, nullptr, nullptr, nullptr, P, E, top, score, renormalize, scale}, stream);
  if (cudaFreeAsync(logits, stream) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
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
