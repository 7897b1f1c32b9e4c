// What the products on 4-bit weights share: the tile layout, codes as matrix operands, and the loop of one warp.
#pragma once

#include "decoder_internal.cuh"
#include "kv_attention.cuh"  // cluster helpers
#include "tc_common.cuh"

namespace fgq {
namespace w4 {

using namespace dec;

constexpr int TILE_ROWS = 16, TILE_COLS = 128, TILE_BYTES = TILE_ROWS * TILE_COLS / 2;

inline int row_tiles(int rows) { return (int)(((int64_t)rows + TILE_ROWS - 1) / TILE_ROWS); }
inline int col_tiles(int cols) { return (int)(((int64_t)cols + TILE_COLS - 1) / TILE_COLS); }
inline bool valid_group(int g) { return g == 32 || g == 64 || g == 128; }

// FGQ_OK, or what is wrong with weights.
inline fgq_status check_weights(const fgq_w4* w) {
  if (!w || w->experts < 0 || w->rows < 0 || w->cols < 0 || !valid_group(w->group)) return FGQ_ERR_ARG;
  if (w->rows > MAX_SIZE || w->cols > MAX_SIZE) return FGQ_ERR_UNSUPPORTED;
  const int64_t tiles = (int64_t)row_tiles(w->rows) * col_tiles(w->cols);
  if (tiles > INT32_MAX || tiles * w->experts > INT32_MAX) return FGQ_ERR_UNSUPPORTED;
  if (tiles * w->experts > 0) {
    if (!w->codes || !w->scales) return FGQ_ERR_ARG;
    if (!aligned(w->codes, 16) || !aligned(w->scales, 16)) return FGQ_ERR_ALIGN;
  }
  return FGQ_OK;
}

// One matrix as kernels take it; `per` groups a tile's row.
struct Matrix {
  const uint8_t* codes;
  const uint16_t* scales;  // bf16
  int rt, ct, per;
  int live;  // groups of the last column tile that hold columns of the matrix: what stands for the others is no scale of its rows
};
inline Matrix matrix(const fgq_w4* w) {
  return {static_cast<const uint8_t*>(w->codes), static_cast<const uint16_t*>(w->scales), row_tiles(w->rows), col_tiles(w->cols),
          TILE_COLS / w->group, ((w->cols - 1) % TILE_COLS) / w->group + 1};
}

// Eight codes n of a word as four pairs of matrix operands (n - 8) UNIT: pair i holds values 2 i and 2 i + 1.  In the low
// byte of a 16-bit float, n and 16 n are subnormals (or, in bf16, carry on past them in the same steps): one AND and one packed
// multiply-add a pair make the centred code, exactly.
template <typename T>
struct Operand;
template <>
struct Operand<__half> {  // n 2^-24 2^15 - 8 2^-9
  static constexpr uint32_t MUL_LO = 0x78007800u, MUL_HI = 0x68006800u, OFF = 0xa400a400u;
  static constexpr float BACK = 512.0f;  // 1 / UNIT
  static __device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
  }
  // d = a b: no registers to clear
  static __device__ __forceinline__ void mma_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Operand<__nv_bfloat16> {  // n 2^-133 2^127 - 8 2^-6
  static constexpr uint32_t MUL_LO = 0x7f007f00u, MUL_HI = 0x7d007d00u, OFF = 0xbe00be00u;
  static constexpr float BACK = 64.0f;
  static __device__ __forceinline__ uint32_t fma2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
  }
  // d = a b: no registers to clear
  static __device__ __forceinline__ void mma_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <typename T>
__device__ __forceinline__ void code_pairs(uint32_t w, uint32_t (&h)[4]) {
  using O = Operand<T>;
  const uint32_t v = w >> 8;
  h[0] = O::fma2(w & 0x000f000fu, O::MUL_LO, O::OFF);
  h[1] = O::fma2(w & 0x00f000f0u, O::MUL_HI, O::OFF);
  h[2] = O::fma2(v & 0x000f000fu, O::MUL_LO, O::OFF);
  h[3] = O::fma2(v & 0x00f000f0u, O::MUL_HI, O::OFF);
}

// Scales of one row of a tile, PER of them, as loaded.
template <int PER>
struct Scales;
template <>
struct Scales<4> {
  uint2 v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = __ldg(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void read(const uint16_t* p) { v = *reinterpret_cast<const uint2*>(p); }  // shared memory
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? v.x : v.y;
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
};
template <>
struct Scales<2> {
  uint32_t v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = __ldg(reinterpret_cast<const uint32_t*>(p)); }
  __device__ __forceinline__ void read(const uint16_t* p) { v = *reinterpret_cast<const uint32_t*>(p); }  // shared memory
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i ? v & 0xffff0000u : v << 16); }
};
template <>
struct Scales<1> {
  uint16_t v;
  __device__ __forceinline__ void load(const uint16_t* p) { v = __ldg(p); }
  __device__ __forceinline__ void read(const uint16_t* p) { v = *p; }  // shared memory
  __device__ __forceinline__ float get(int) const { return __uint_as_float((uint32_t)v << 16); }
};

// What one thread holds of a tile: 16 bytes of rows g and g + 8, and their scales.
template <int PER>
struct Tile {
  uint4 w[2];
  Scales<PER> s[2];
  // tile number `at` of the matrix; lane = 4 g + t
  __device__ __forceinline__ void load(const uint8_t* codes, const uint16_t* scales, int64_t at, int lane) {
    const uint4* p = reinterpret_cast<const uint4*>(codes + at * TILE_BYTES) + lane;
    w[0] = __ldg(p);
    w[1] = __ldg(p + 32);
    const uint16_t* q = scales + at * (TILE_ROWS * PER) + (lane >> 2) * PER;
    s[0].load(q);
    s[1].load(q + 8 * PER);
  }
  __device__ __forceinline__ uint32_t word(int r, int j) const {
    return j == 0 ? w[r].x : (j == 1 ? w[r].y : (j == 2 ? w[r].z : w[r].w));
  }
};

// Tiles in shared memory: codes, then scales, as in memory.
template <int PER>
constexpr int tile_bytes() {
  return TILE_BYTES + TILE_ROWS * PER * 2;
}
// A tile to shared address `to`, by a warp; codes and scales: the tile's, 16 bytes on a lane.
template <int PER>
__device__ __forceinline__ void copy_tile(uint32_t to, const uint8_t* codes, const uint8_t* scales, int lane) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\ncp.async.cg.shared.global [%0 + 512], [%1 + 512], 16;" ::"r"(to), "l"(codes) : "memory");
  if (lane < 2 * PER) asm volatile("cp.async.cg.shared.global [%0 + 1024], [%1], 16;" ::"r"(to), "l"(scales) : "memory");
}
template <int PER>
__device__ __forceinline__ void read_tile(Tile<PER>& tile, const uint8_t* from, int lane) {
  tile.w[0] = *reinterpret_cast<const uint4*>(from + 16 * lane);
  tile.w[1] = *reinterpret_cast<const uint4*>(from + 512 + 16 * lane);
  const uint16_t* s = reinterpret_cast<const uint16_t*>(from + TILE_BYTES) + (lane >> 2) * PER;
  tile.s[0].read(s);
  tile.s[1].read(s + 8 * PER);
}

// A stage of tokens in shared memory: 8 NT columns of 128 values, 256 bytes each, 16-byte chunks of odd columns
// moved by 64 bytes, so that eight lanes that read two columns meet all banks.
__device__ __forceinline__ uint32_t chunk_at(int col, int chunk) { return (uint32_t)(col * 256 + ((chunk ^ ((col & 1) << 2)) << 4)); }

// sum[mt][nt] += tile mt times the stage's columns; sums are in units of 1 / BACK.  Sums of two columns are a packed pair: [0] of
// row g, [1] of row g + 8.
using pair_t = unsigned long long;
// Where a thread's pieces of a stage of `cols` columns are: chunk 4 j + t of column 8 nt + g, for even and odd j.  Columns that the
// stage does not have are read as its last: nothing takes their sums.
template <int NT>
struct Pieces {
  uint32_t even[NT], odd[NT];
  __device__ __forceinline__ Pieces(int cols, int lane) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = min(8 * nt + (lane >> 2), cols - 1);
      even[nt] = chunk_at(c, lane & 3);
      odd[nt] = chunk_at(c, 4 + (lane & 3));
    }
  }
};
template <typename T, int MT, int NT, int PER>
__device__ __forceinline__ void multiply(const Tile<PER> (&tile)[MT], const uint8_t* stage, const Pieces<NT>& at, pair_t (&sum)[MT][NT][2]) {
#pragma unroll
  for (int gi = 0; gi < PER; ++gi) {
    float acc[MT][NT][4];
#pragma unroll
    for (int j = gi * (4 / PER); j < (gi + 1) * (4 / PER); ++j) {
      uint4 b[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) b[nt] = *reinterpret_cast<const uint4*>(stage + (j & 1 ? at.odd[nt] : at.even[nt]) + (j >> 1) * 128);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t u[4], v[4];
        code_pairs<T>(tile[mt].word(0, j), u);
        code_pairs<T>(tile[mt].word(1, j), v);
        const uint32_t a0[4] = {u[0], v[0], u[1], v[1]}, a1[4] = {u[2], v[2], u[3], v[3]};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (j == gi * (4 / PER))
            Operand<T>::mma_new(acc[mt][nt], a0, b[nt].x, b[nt].y);
          else
            Operand<T>::mma(acc[mt][nt], a0, b[nt].x, b[nt].y);
          Operand<T>::mma(acc[mt][nt], a1, b[nt].z, b[nt].w);
        }
      }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const float s0 = tile[mt].s[0].get(gi), s1 = tile[mt].s[1].get(gi);
      const pair_t p0 = pack_f2(s0, s0), p1 = pack_f2(s1, s1);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        sum[mt][nt][0] = fma_f2(pack_f2(acc[mt][nt][0], acc[mt][nt][1]), p0, sum[mt][nt][0]);
        sum[mt][nt][1] = fma_f2(pack_f2(acc[mt][nt][2], acc[mt][nt][3]), p1, sum[mt][nt][1]);
      }
    }
  }
}

// How a block shares its work.  Eight warps take 16 rows of weights each (MT tiles of them), all on the same 8 NT columns of
// tokens: a stage is one tile column, its tokens copied once into shared memory, STAGES of them in a ring that one barrier a
// stage keeps in order, and its weights loaded by each warp for itself, AHEAD stages before they are multiplied.  Sums stay in
// registers over all stages.
constexpr int WARPS = 8, THREADS = 32 * WARPS;

template <int NT>
struct Ring {
  static constexpr int STAGES = NT >= 8 ? 4 : 5, BYTES = 8 * NT * 256, COPIES = (8 * NT + 15) / 16;
  static constexpr int TOTAL = STAGES * BYTES;
};

// The 16-byte pieces of a stage of 16-bit tokens that one thread copies: piece tid % 16 of columns tid / 16 + 16 i.
template <int NT>
struct Columns {
  int64_t off[Ring<NT>::COPIES];  // bytes from the tokens' start, or -1: zeros
  // columns [128 kt, + 128); those from kvalid (a multiple of 8) on are zeros
  __device__ __forceinline__ void copy(uint32_t stage, const uint8_t* base, int kt, int kvalid) const {
    const int chunk = threadIdx.x & 15, k = kt * TILE_COLS + 8 * chunk;
#pragma unroll
    for (int i = 0; i < Ring<NT>::COPIES; ++i) {
      const int col = (int)(threadIdx.x >> 4) + 16 * i;
      if (NT == 1 && col >= 8) break;
      const bool live = off[i] >= 0 && k < kvalid;
      cp_async16(stage + chunk_at(col, chunk), live ? base + off[i] + 2 * (int64_t)k : base, live ? 16u : 0u);
    }
  }
};

// A unit of work of the experts: up to `cap` choices of one expert, `count` of them from `start` on in the order sorted by expert.
struct Unit {
  int expert, start, count, pad;
};
// A choice in that order: its token and the router's weight.
struct Choice {
  int token;
  float weight;
};

// Tokens as they are given, rows of elements of their type (the experts': 16-bit elements in pieces, fp32 in three rows of bf16 parts).
enum { ROWS_COPIED = 0, ROWS_SINGLE = 1, ROWS_PIECES = 2 };
struct TokenRows {
  const void* data;
  int64_t pitch;  // elements between tokens
  int kvalid;     // elements of a row
  // ROWS_COPIED: 16-bit elements in 16-byte pieces that are operands as they are; or elements to be loaded one by one, or (fp32) in pieces
  int load;
};
__host__ __device__ constexpr int columns_per_token(int parts) { return parts == 3 ? 4 : parts; }

// fp32 in parts of 8 significant bits, each cut off and the last exact.
__device__ __forceinline__ void three_parts(float v, uint16_t (&p)[3]) {
  const float a = __uint_as_float(__float_as_uint(v) & 0xffff0000u), r = v - a;
  const float b = __uint_as_float(__float_as_uint(r) & 0xffff0000u), c = r - b;
  p[0] = (uint16_t)(__float_as_uint(a) >> 16);
  p[1] = (uint16_t)(__float_as_uint(b) >> 16);
  p[2] = (uint16_t)(__float_as_uint(c) >> 16);
}

// Eight elements of a token on their way through registers: fp32 to three bf16 parts, 16-bit ones as they are.
template <int PARTS>
struct Eight {
  uint32_t v[PARTS == 3 ? 8 : 4];
  // elements [k, + 8) of a row; zeros past its end, and where row < 0
  __device__ __forceinline__ void load(const TokenRows& x, int64_t row, int k) {
    const int n = row < 0 ? 0 : x.kvalid - k;
    if constexpr (PARTS == 3) {
      const uint32_t* p = static_cast<const uint32_t*>(x.data) + row * x.pitch + k;
      if (x.load == ROWS_PIECES && n >= 8) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p)), b = __ldcg(reinterpret_cast<const uint4*>(p) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        return;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < n ? __ldcg(p + i) : 0u;
    } else {
      const unsigned short* p = static_cast<const unsigned short*>(x.data) + row * x.pitch + k;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < n ? __ldcg(p + 2 * i) : 0u, hi = 2 * i + 1 < n ? __ldcg(p + 2 * i + 1) : 0u;
        v[i] = lo | hi << 16;
      }
    }
  }
  // as columns of token `tok` in a stage, piece `chunk`; fp32: three of them, and one of zeros
  __device__ __forceinline__ void store(uint8_t* stage, int tok, int chunk) const {
    if constexpr (PARTS == 3) {
      uint32_t w[3][4];
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint16_t p[3], q[3];
        three_parts(__uint_as_float(v[2 * h]), p);
        three_parts(__uint_as_float(v[2 * h + 1]), q);
#pragma unroll
        for (int c = 0; c < 3; ++c) w[c][h] = p[c] | (uint32_t)q[c] << 16;
      }
#pragma unroll
      for (int c = 0; c < 3; ++c)
        *reinterpret_cast<uint4*>(stage + chunk_at(4 * tok + c, chunk)) = make_uint4(w[c][0], w[c][1], w[c][2], w[c][3]);
      *reinterpret_cast<uint4*>(stage + chunk_at(4 * tok + 3, chunk)) = make_uint4(0u, 0u, 0u, 0u);
    } else {
      *reinterpret_cast<uint4*>(stage + chunk_at(tok, chunk)) = make_uint4(v[0], v[1], v[2], v[3]);
    }
  }
};

// How tokens are loaded: pieces of 16 bytes where they end with the row.
inline bool pieces16(const void* x, int type, int P, int K, int64_t ldx) {
  return K % (type == FGQ_F32 ? 4 : 8) == 0 && aligned(x, 16) && (P == 1 || stride16(ldx, type));
}
inline TokenRows token_rows(const void* x, int type, int P, int K, int64_t ldx) {
  const bool pieces = pieces16(x, type, P, K, ldx);
  return {x, ldx, K, pieces ? (type == FGQ_F32 ? ROWS_PIECES : ROWS_COPIED) : ROWS_SINGLE};
}
inline int64_t copied_pitch(int K) { return ((int64_t)K + 7) / 8 * 8; }

}  // namespace w4
}  // namespace fgq
