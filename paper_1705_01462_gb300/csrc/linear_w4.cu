// Linear layers on 4-bit weights with a scale for each group: quantization, the product for few tokens, and operands
// of the product for many.
//
// y[p][m] = sum_g s_mg sum_{k in g} c_mk x_pk + bias_m.  For few tokens codes c are exact matrix operands and 16-bit tokens are as they
// are (fp32 ones in three bf16 parts), so a group's sum is that of exact products in fp32, and takes its scale in fp32.
#include <type_traits>

#include "linear_internal.cuh"
#include "w4_launch.h"
#include "w4_many.h"

namespace fgq {
namespace w4 {
namespace {

// ------------------------------------------------------------------ weights to 4 bits and back
// A warp a tile of 16 rows and 128 columns, lane (g, t) as in the products: words j of rows g and g + 8.
__global__ void __launch_bounds__(256) quantize_kernel(const float* __restrict__ w, uint8_t* codes, uint16_t* scales, int rows,
                                                       int cols, int rt, int ct, int per, int64_t tiles, unsigned int* err) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < tiles; at += (int64_t)gridDim.x * 8) {
    const int64_t e = at / ((int64_t)rt * ct);
    const int in = (int)(at - e * rt * ct), mt = in / ct, kt = in - mt * ct;
    bool bad = false;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int m = mt * TILE_ROWS + g + 8 * r;
      const float* row = w + (e * rows + m) * cols;
      float v[4][8], amax[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        amax[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int64_t k = (int64_t)kt * TILE_COLS + 32 * j + 8 * t + i;
          v[j][i] = m < rows && k < cols ? row[k] : 0.0f;
          amax[j] = max_nan(amax[j], fabsf(v[j][i]));
        }
        amax[j] = max_nan(amax[j], __shfl_xor_sync(FULL_MASK, amax[j], 1));
        amax[j] = max_nan(amax[j], __shfl_xor_sync(FULL_MASK, amax[j], 2));
      }
      uint32_t word[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float top = amax[j];  // of the whole group
        if (per == 2) top = max_nan(amax[j & ~1], amax[j | 1]);
        if (per == 1) top = max_nan(max_nan(amax[0], amax[1]), max_nan(amax[2], amax[3]));
        if (nonfinite(top)) {
          bad = true;
          top = 0.0f;
        }
        const float q = __fdiv_rn(top, 7.0f);
        const uint32_t up = (__float_as_uint(q) + 0xffffu) & 0xffff0000u;  // a value above bf16's largest is none: top / 7 is
        const float s = __uint_as_float(up);                               // below it
        if (t == 0 && j % (4 / per) == 0) scales[at * (TILE_ROWS * per) + (g + 8 * r) * per + j / (4 / per)] = (uint16_t)(up >> 16);
        word[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int c = s > 0.0f ? __float2int_rn(fminf(fmaxf(__fdiv_rn(v[j][i], s), -7.0f), 7.0f)) : 0;
          word[j] |= (uint32_t)(c + 8) << (4 * ((i >> 1) + 4 * (i & 1)));
        }
      }
      reinterpret_cast<uint4*>(codes + at * TILE_BYTES)[32 * r + lane] = make_uint4(word[0], word[1], word[2], word[3]);
    }
    if (bad) record_error(err, FGQ_ERR_NONFINITE);
  }
}

__global__ void __launch_bounds__(256) read_kernel(const uint8_t* codes, const uint16_t* scales, float* __restrict__ w, int rows,
                                                   int cols, int rt, int ct, int per, int64_t tiles) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < tiles; at += (int64_t)gridDim.x * 8) {
    const int64_t e = at / ((int64_t)rt * ct);
    const int in = (int)(at - e * rt * ct), mt = in / ct, kt = in - mt * ct;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int m = mt * TILE_ROWS + g + 8 * r;
      const uint4 v = reinterpret_cast<const uint4*>(codes + at * TILE_BYTES)[32 * r + lane];
      const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float s = __uint_as_float((uint32_t)scales[at * (TILE_ROWS * per) + (g + 8 * r) * per + j / (4 / per)] << 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int64_t k = (int64_t)kt * TILE_COLS + 32 * j + 8 * t + i;
          const int n = (int)(word[j] >> (4 * ((i >> 1) + 4 * (i & 1))) & 15u);
          if (m < rows && k < cols) w[(e * rows + m) * cols + k] = (float)(n - 8) * s;
        }
      }
    }
  }
}

// ------------------------------------------------------------------ tokens that outputs would overwrite
// A block a token: its row, zeros up to `pitch` elements.
template <typename E>
__global__ void __launch_bounds__(256) copy_tokens_kernel(const E* __restrict__ x, int K, int64_t ldx, E* dst, int64_t pitch) {
  pdl_trigger();
  for (int64_t k = threadIdx.x; k < pitch; k += 256) dst[pitch * blockIdx.x + k] = k < K ? x[blockIdx.x * ldx + k] : E(0);
}

// ------------------------------------------------------------------ few tokens
fgq_status launch_few(RowsArgs a, bool early, cudaStream_t s) {
  const int cpt = a.ytype == FGQ_F32 ? columns_per_token(3) : 1;
  const int64_t columns = (int64_t)a.P * cpt;
  const int nt = columns <= 8 ? 1 : (columns <= 16 ? 2 : 4);
  const int tokens = 8 * nt / cpt;
  const int64_t tiles = ((int64_t)a.P + tokens - 1) / tokens;
  // One tile of tokens is held in shared memory where it fits, but a small matrix takes no longer to stream than the tokens to arrive.  bf16, us
  // held and not: 8 tokens, 4096 -> 4096 7.5 and 6.0, 4096 -> 6144 8.2 and 8.5, 4096 -> 14336 11.2 and 14.2; one token 4096 -> 4096 5.6 and
  // 5.6, 1024 -> 2048 3.5 and 3.7; 16 tokens, 4096 -> 8192 12.4 and 10.6, 4096 -> 14336 14.5 and 16.9.
  const int64_t weights = (int64_t)a.w.rt * a.w.ct * (TILE_ROWS * TILE_COLS);
  if (nt == 1 ? columns < 4 || weights > 1 << 24 : nt == 2 && weights > 1 << 25) {
    const ResidentPlan plan = plan_held(nt, a.w.ct, a.w.per, (int)columns);
    if (plan.warps > 0) {
      ResidentArgs r = {};
      r.w = a.w, r.x = a.x, r.bias = a.bias, r.y = a.y, r.P = a.P, r.M = a.M, r.ytype = a.ytype, r.early = early;
      r.items = a.w.rt;
      if (a.ytype == FGQ_F32) return launch_held_f32(r, nt, plan, early, s);
      return a.ytype == FGQ_BF16 ? launch_held_bf16(r, nt, plan, early, s) : launch_held_f16(r, nt, plan, early, s);
    }
  }
  const int64_t items = (int64_t)((a.w.rt + WARPS - 1) / WARPS) * tiles;
  if (items > INT32_MAX / 8) return FGQ_ERR_UNSUPPORTED;
  const RowsPlan plan = plan_rows(items, a.w.ct);
  a.items = (int)items;
  a.token_tiles = (int)tiles;
  a.splits = plan.splits;
  a.early = early;
  if (a.ytype == FGQ_F32) return launch_rows_f32(a, nt, plan.grid, early, s);
  return a.ytype == FGQ_BF16 ? launch_rows_bf16(a, nt, plan.grid, early, s) : launch_rows_f16(a, nt, plan.grid, early, s);
}

// ------------------------------------------------------------------ operands of the product for many tokens
// What the blocks past the tokens do: find the exponent of each weight row's largest scale (subnormal ones: of the smallest normal), and
// where w16 is given, write its rows as fp16, c s 2^(12 - e), `parts` blocks a row tile.  Groups past the matrix count as 0.
struct Weights {
  Matrix w;
  int* wexp;      // all rows of the tiles; or nullptr:
  __half* w16;    // [M][pitch]
  float* wscale;  // [M]: 2^(e - 12)
  int64_t pitch;
  int M, parts;
};
__device__ __forceinline__ void prepare_weights(const Weights& a, int block) {
  __shared__ uint32_t top[TILE_ROWS];
  const Matrix& w = a.w;
  const int mt = block / a.parts, part = block - mt * a.parts;
  if (threadIdx.x < TILE_ROWS) top[threadIdx.x] = 0u;
  __syncthreads();
  const uint16_t* sc = w.scales + (int64_t)mt * w.ct * TILE_ROWS * w.per;
  // magnitudes compare as whole numbers; the order of maxima does not matter.  Eight scales a load
  const int n = w.ct * TILE_ROWS * w.per / 8;
  for (int i = threadIdx.x; i < n; i += 256) {
    const uint4 v = __ldg(reinterpret_cast<const uint4*>(sc) + i);
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = 8 * i + 2 * k + h;
        if (at % w.per < w.live || at < (w.ct - 1) * TILE_ROWS * w.per) atomicMax(&top[at / w.per % TILE_ROWS], u[k] >> 16 * h & 0x7fffu);
      }
    }
  }
  __syncthreads();
  auto exponent = [&](int r) { return max((int)(top[r] >> 7) - 127, -126); };
  if (!a.w16) {
    if (threadIdx.x < TILE_ROWS) a.wexp[mt * TILE_ROWS + threadIdx.x] = exponent(threadIdx.x);
    return;
  }
  if (part == 0 && threadIdx.x < TILE_ROWS && mt * TILE_ROWS + (int)threadIdx.x < a.M)
    a.wscale[mt * TILE_ROWS + threadIdx.x] = pow2f(exponent(threadIdx.x) - 12);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int e0 = 12 - exponent(g), e1 = 12 - exponent(g + 8);
  for (int kt = part * 8 + warp; kt < w.ct; kt += a.parts * 8) {
    const int64_t at = (int64_t)mt * w.ct + kt;
    uint4 v[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) v[r] = __ldg(reinterpret_cast<const uint4*>(w.codes + at * TILE_BYTES) + 32 * r + lane);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int m = mt * TILE_ROWS + g + 8 * r, e = r ? e1 : e0;
      if (m >= a.M) continue;
      const uint32_t word[4] = {v[r].x, v[r].y, v[r].z, v[r].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t k = (int64_t)kt * TILE_COLS + 32 * j + 8 * t;
        if (k >= a.pitch) continue;
        float s = __uint_as_float((uint32_t)__ldg(w.scales + at * (TILE_ROWS * w.per) + (g + 8 * r) * w.per + j * w.per / 4) << 16);
        s = s * pow2f(e / 2) * pow2f(e - e / 2);  // in two factors: 2^e passes fp32's largest for subnormal rows
        if (kt == w.ct - 1 && j * w.per / 4 >= w.live) s = 0.0f;
        *reinterpret_cast<uint4*>(a.w16 + m * a.pitch + k) = scaled_codes(word[j], pack2(s, s, __half()));
      }
    }
  }
}

// A block a token, the blocks past them for the weights.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) prepare_kernel(const T* __restrict__ x, int P, int K, int64_t ldx, __half* dst, int64_t pitch,
                                                      float* scale, const __grid_constant__ Weights w) {
  pdl_trigger();
  const int p = blockIdx.x;
  if (p < P)
    token_row<T, VEC>(x + p * ldx, K, dst + p * pitch * (std::is_same<T, float>::value ? 2 : 1), pitch, scale + p);
  else
    prepare_weights(w, p - P);
}

__global__ void __launch_bounds__(256) ones_kernel(float* p, int n) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n) p[i] = 1.0f;
}

inline size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

bool overlap(const void* x, const void* y, int type, int P, int K, int M, int64_t ldx) {
  const uintptr_t xb = reinterpret_cast<uintptr_t>(x), yb = reinterpret_cast<uintptr_t>(y);
  const uint64_t xn = ((uint64_t)(P - 1) * (P > 1 ? ldx : 0) + K) * float_bytes(type), yn = (uint64_t)P * M * float_bytes(type);
  return xb < yb + yn && yb < xb + xn;
}

// From here on weights are expanded in memory for the product on pairs of SMs, which saves shared-memory traffic for the bytes.
// bf16, us so and in gemm_w4.cu: 1024 tokens, 4096 -> 14336 108.8 and 102.0, 4096 -> 4096 36.9 and 36.1; 1280 tokens 130.9 and 134.0, 54.5 and
// 65.2; 2048 tokens 184.8 and 206.4, 59.0 and 70.1, but 1024 -> 2048 20.2 and 18.4.
constexpr int EXPAND_MIN_P = 1025;
constexpr int64_t EXPAND_MIN_WEIGHTS = 1 << 23;

fgq_status run_many(const void* x, int type, int P, int K, int64_t ldx, const fgq_w4* w, const float* bias, void* y, cudaStream_t s) {
  const int M = w->rows;
  const bool expand = type != FGQ_F32 && P >= EXPAND_MIN_P && (int64_t)K * M >= EXPAND_MIN_WEIGHTS;
  Weights wt = {matrix(w), nullptr, nullptr, nullptr, 0, M, 1};
  const int parts = type == FGQ_F32 ? 2 : 1;
  const ManyPlan plan = plan_many(P, parts, wt.w.ct, M);
  const GemmPlan pairs = expand ? plan_gemm_w8a8(P, K, M) : GemmPlan{};
  // fp16 tokens are operands as they are (expanded: where their rows are whole K-tiles beside one another)
  const bool vec = K % 8 == 0 && pieces16(x, type, P, K, ldx);
  const bool direct = type == FGQ_F16 && vec && !overlap(x, y, type, P, K, M, ldx) && (!expand || (K == pairs.pitch && (P == 1 || ldx == K)));
  const int64_t pitch = expand ? pairs.pitch : (direct && P > 1 ? ldx : copied_pitch(K));
  const size_t e_bytes = up256((size_t)wt.w.rt * TILE_ROWS * 4), x_bytes = direct ? 0 : up256((size_t)P * parts * pitch * 2);
  const size_t s_bytes = direct && !expand ? 0 : up256((size_t)P * 4), w_bytes = expand ? up256((size_t)M * pitch * 2) : 0;
  const size_t p_bytes = expand ? pairs.part_bytes : plan.part_bytes;
  uint8_t* tmp = static_cast<uint8_t*>(scratch_alloc(e_bytes + x_bytes + s_bytes + w_bytes + p_bytes, s));
  if (!tmp) return FGQ_ERR_CUDA;
  __half* x16 = reinterpret_cast<__half*>(tmp + e_bytes);
  float* xscale = s_bytes ? reinterpret_cast<float*>(tmp + e_bytes + x_bytes) : nullptr;
  float* part = reinterpret_cast<float*>(tmp + e_bytes + x_bytes + s_bytes + w_bytes);
  if (expand) {
    wt.w16 = reinterpret_cast<__half*>(tmp + e_bytes + x_bytes + s_bytes);
    wt.wscale = reinterpret_cast<float*>(tmp);
    wt.pitch = pitch;
    wt.parts = (wt.w.ct + 7) / 8;
    while (wt.parts > 1 && (int64_t)wt.parts * wt.w.rt > 8ll * device_sms()) wt.parts = (wt.parts + 1) / 2;
  } else {
    wt.wexp = reinterpret_cast<int*>(tmp);
  }
  const int tokens = direct ? 0 : P;
  const int64_t blocks = tokens + (int64_t)wt.w.rt * wt.parts;
  fgq_status st = FGQ_ERR_UNSUPPORTED;
  if (blocks <= INT32_MAX) {
    const unsigned grid = (unsigned)blocks;
    if (type == FGQ_BF16) {
      const __nv_bfloat16* xb = static_cast<const __nv_bfloat16*>(x);
      vec ? prepare_kernel<__nv_bfloat16, true><<<grid, 256, 0, s>>>(xb, tokens, K, ldx, x16, pitch, xscale, wt)
          : prepare_kernel<__nv_bfloat16, false><<<grid, 256, 0, s>>>(xb, tokens, K, ldx, x16, pitch, xscale, wt);
    } else if (type == FGQ_F32) {
      const float* xf = static_cast<const float*>(x);
      vec ? prepare_kernel<float, true><<<grid, 256, 0, s>>>(xf, tokens, K, ldx, x16, pitch, xscale, wt)
          : prepare_kernel<float, false><<<grid, 256, 0, s>>>(xf, tokens, K, ldx, x16, pitch, xscale, wt);
    } else {
      const __half* xh = static_cast<const __half*>(x);
      vec ? prepare_kernel<__half, true><<<grid, 256, 0, s>>>(xh, tokens, K, ldx, x16, pitch, xscale, wt)
          : prepare_kernel<__half, false><<<grid, 256, 0, s>>>(xh, tokens, K, ldx, x16, pitch, xscale, wt);
    }
    st = after_launch();
  }
  if (st == FGQ_OK && expand && direct) {
    ones_kernel<<<(P + 255) / 256, 256, 0, s>>>(xscale, P);
    st = after_launch();
  }
  const void* rows = direct ? x : x16;
  if (st == FGQ_OK)
    st = expand ? launch_gemm_w8a8(pairs, rows, wt.w16, part, xscale, P, wt.wscale, M, bias, y, type, s)
                : launch_many(plan, wt.w, wt.wexp, rows, pitch, direct ? K : (int)pitch, xscale, P, M, part, bias, y, type, s);
  if (cudaFreeAsync(tmp, s) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

// Outputs without features: the bias.
__global__ void __launch_bounds__(256) bias_kernel(const float* bias, void* y, int ytype, int P, int M) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)P * M; i += (int64_t)gridDim.x * 256)
    store_typed(y, ytype, i, bias ? __ldg(bias + i % M) : 0.0f);
}

// Whether the kernels of few tokens run: up to 16 tokens (fp32: 8), or a product of tokens and weights up to which reading the weights again
// for every 32 (8) tokens costs less than what the other way starts with.  bf16, us there and in gemm_w4.cu: 16 tokens, 4096 -> 14336 14.5 and 22.5;
// 32 tokens, 4096 -> 8192 16.8 and 18.4, 4096 -> 14336 28.6 and 22.8; 64 tokens, 2048 -> 2048 6.9 and 11.1, 4096 -> 4096 14.2 and 14.7; 128 tokens
// 24.0 and 17.7, 2048 -> 4096 14.7 and 15.2; 256 tokens 20.6 and 19.3, 1024 -> 2048 10.6 and 13.9.  fp32: 8 tokens, 4096 -> 14336 24.0 and 26.9; 16 tokens,
// 4096 -> 4096 13.1 and 13.3; 64 tokens, 1024 -> 2048 9.0 and 11.1, 2048 -> 2048 14.0 and 11.8; 128 tokens, 512 -> 512 5.7 and 8.5.
bool few_tokens(int type, int P, int K, int M) {
  if (const int which = debug_linear_w4_kernel()) return which == 1;
  const int few = type == FGQ_F32 ? 8 : 16, tile = type == FGQ_F32 ? 8 : 32;
  const int64_t most = type == FGQ_F32 ? 1ll << 27 : 1ll << 30, tokens = ((int64_t)P + tile - 1) / tile * tile;
  return P <= few || (tokens <= most && (int64_t)K * M <= most / tokens);
}

}  // namespace

}  // namespace w4
}  // namespace fgq

using namespace fgq;

extern "C" {

size_t fgq_w4_code_bytes(int rows, int cols) {
  if (rows < 0 || cols < 0) return 0;
  return (size_t)w4::row_tiles(rows) * w4::col_tiles(cols) * w4::TILE_BYTES;
}
size_t fgq_w4_scale_bytes(int rows, int cols, int group) {
  if (rows < 0 || cols < 0 || !w4::valid_group(group)) return 0;
  return (size_t)w4::row_tiles(rows) * w4::col_tiles(cols) * w4::TILE_ROWS * (w4::TILE_COLS / group) * 2;
}

fgq_status fgq_quantize_weights_w4(const float* w, const fgq_w4* out, cudaStream_t stream) {
  const fgq_status st = w4::check_weights(out);
  if (st != FGQ_OK) return st;
  const int64_t tiles = (int64_t)w4::row_tiles(out->rows) * w4::col_tiles(out->cols) * out->experts;
  if (tiles == 0) return FGQ_OK;
  if (!w) return FGQ_ERR_ARG;
  if (!dec::aligned(w, 4)) return FGQ_ERR_ALIGN;
  const int64_t blocks = (tiles + 7) / 8, most = 16ll * device_sms();
  const w4::Matrix m = w4::matrix(out);
  w4::quantize_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, stream>>>(
      w, static_cast<uint8_t*>(const_cast<void*>(out->codes)), static_cast<uint16_t*>(const_cast<void*>(out->scales)), out->rows,
      out->cols, m.rt, m.ct, m.per, tiles, device_error_word());
  return after_launch();
}

fgq_status fgq_read_weights_w4(const fgq_w4* w, float* out, cudaStream_t stream) {
  const fgq_status st = w4::check_weights(w);
  if (st != FGQ_OK) return st;
  const int64_t tiles = (int64_t)w4::row_tiles(w->rows) * w4::col_tiles(w->cols) * w->experts;
  if (tiles == 0) return FGQ_OK;
  if (!out) return FGQ_ERR_ARG;
  if (!dec::aligned(out, 4)) return FGQ_ERR_ALIGN;
  const int64_t blocks = (tiles + 7) / 8, most = 16ll * device_sms();
  const w4::Matrix m = w4::matrix(w);
  w4::read_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, stream>>>(m.codes, m.scales, out, w->rows, w->cols, m.rt,
                                                                                m.ct, m.per, tiles);
  return after_launch();
}

fgq_status fgq_linear_w4(const void* x, fgq_float_type type, int P, int64_t ldx, const fgq_w4* w, const float* bias, void* y,
                         cudaStream_t stream) {
  using namespace w4;
  if (P < 0 || !valid_float(type)) return FGQ_ERR_ARG;
  const fgq_status ok = check_weights(w);
  if (ok != FGQ_OK) return ok;
  if (w->experts != 1) return FGQ_ERR_ARG;
  const int K = w->cols, M = w->rows;
  if (P > 1 && ldx < K) return FGQ_ERR_ARG;
  if (P == 0 || M == 0) return FGQ_OK;
  if (P > (type == FGQ_F32 ? MAX_SIZE / 2 : MAX_SIZE)) return FGQ_ERR_UNSUPPORTED;  // many fp32 tokens are two rows each, counted in 32 bits
  if (!y || (K > 0 && !x)) return FGQ_ERR_ARG;
  const uintptr_t e = float_bytes(type);
  if (!aligned(x, e) || !aligned(y, e) || !aligned(bias, 4)) return FGQ_ERR_ALIGN;
  if (K == 0) {
    const int64_t blocks = ((int64_t)P * M + 255) / 256, most = 8ll * device_sms();
    bias_kernel<<<(unsigned)(blocks < most ? blocks : most), 256, 0, stream>>>(bias, y, type, P, M);
    return after_launch();
  }
  if (!few_tokens(type, P, K, M)) return run_many(x, type, P, K, P > 1 ? ldx : 0, w, bias, y, stream);
  RowsArgs a = {};
  a.w = matrix(w), a.x = token_rows(x, type, P, K, P > 1 ? ldx : 0), a.bias = bias, a.y = y, a.P = P, a.M = M, a.ytype = type;
  // tokens that outputs would overwrite are copied first, and those of a large matrix that are not in pieces of 16 bytes (us, 8 tokens of bf16,
  // 4095 -> 14336 11.9 in place of 21.0; 4095 -> 4096 takes 8.1 as it is)
  if (!overlap(x, y, type, P, K, M, ldx) && (a.x.load != ROWS_SINGLE || P == 1 || (int64_t)K * M <= 1 << 24)) return launch_few(a, false, stream);
  const int64_t pitch = copied_pitch(K);
  void* tmp = scratch_alloc((size_t)P * pitch * float_bytes(type), stream);
  if (!tmp) return FGQ_ERR_CUDA;
  if (type == FGQ_F32)
    copy_tokens_kernel<<<P, 256, 0, stream>>>(static_cast<const float*>(x), K, ldx, static_cast<float*>(tmp), pitch);
  else
    copy_tokens_kernel<<<P, 256, 0, stream>>>(static_cast<const uint16_t*>(x), K, ldx, static_cast<uint16_t*>(tmp), pitch);
  fgq_status st = after_launch();
  a.x = {tmp, pitch, (int)pitch, type == FGQ_F32 ? ROWS_PIECES : ROWS_COPIED};
  if (st == FGQ_OK) st = launch_few(a, true, stream);
  if (cudaFreeAsync(tmp, stream) != cudaSuccess && st == FGQ_OK) st = FGQ_ERR_CUDA;
  return st;
}

}  // extern "C"
