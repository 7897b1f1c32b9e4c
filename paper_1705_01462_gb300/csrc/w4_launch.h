// Launches of the few-token products, one translation unit for each type of tokens.
#pragma once

#include "w4_resident.cuh"

namespace fgq {
namespace w4 {

// A linear layer; columns of tokens that a block takes: 8 nt, nt 1, 2 or 4.
fgq_status launch_rows_bf16(const RowsArgs& a, int nt, unsigned grid, bool chained, cudaStream_t s);
fgq_status launch_rows_f16(const RowsArgs& a, int nt, unsigned grid, bool chained, cudaStream_t s);
fgq_status launch_rows_f32(const RowsArgs& a, int nt, unsigned grid, bool chained, cudaStream_t s);
// The same with tokens held in shared memory: up to 8 nt columns (nt 1 or 2), where plan_resident finds room for them.
fgq_status launch_held_bf16(const ResidentArgs& a, int nt, const ResidentPlan& plan, bool chained, cudaStream_t s);
fgq_status launch_held_f16(const ResidentArgs& a, int nt, const ResidentPlan& plan, bool chained, cudaStream_t s);
fgq_status launch_held_f32(const ResidentArgs& a, int nt, const ResidentPlan& plan, bool chained, cudaStream_t s);
// Gate and up, and down (of 16-bit tokens, of fp32), `items` at most: 8 tokens a unit (fp32: 4).
fgq_status launch_held_gated_bf16(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s);
fgq_status launch_held_gated_f16(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s);
fgq_status launch_held_gated_f32(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s);
fgq_status launch_held_down_16(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s);
fgq_status launch_held_down_f32(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s);

template <typename T, int MT, int NT, int PARTS, int MODE, int AHEAD>
fgq_status launch_held_per(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, bool chained, cudaStream_t s) {
  if (a.w.per == 4) return launch_resident<T, MT, NT, 4, PARTS, MODE, AHEAD>(a, plan, items, chained, s);
  if (a.w.per == 2) return launch_resident<T, MT, NT, 2, PARTS, MODE, AHEAD>(a, plan, items, chained, s);
  return launch_resident<T, MT, NT, 1, PARTS, MODE, AHEAD>(a, plan, items, chained, s);
}
// Tiles under way of a warp: four, or two pairs.
constexpr int HELD_AHEAD = 4, GATED_AHEAD = 2, ROWS_AHEAD = 4;
inline ResidentPlan plan_held(int nt, int ct, int per, int cols) {
  return nt == 1 ? plan_resident<1, 1, HELD_AHEAD>(ct, per, cols) : plan_resident<1, 2, HELD_AHEAD>(ct, per, cols);
}
template <typename T, int PARTS>
fgq_status launch_held_type(const ResidentArgs& a, int nt, const ResidentPlan& plan, bool chained, cudaStream_t s) {
  if (nt == 1) return launch_held_per<T, 1, 1, PARTS, MODE_LINEAR, HELD_AHEAD>(a, plan, a.items, chained, s);
  return launch_held_per<T, 1, 2, PARTS, MODE_LINEAR, HELD_AHEAD>(a, plan, a.items, chained, s);
}

template <typename T, int NT, int PER, int PARTS>
fgq_status launch_rows_load(const RowsArgs& a, unsigned grid, bool chained, cudaStream_t s) {
  if constexpr (PARTS == 1)
    if (a.x.load == ROWS_COPIED) return launch_rows<T, NT, PER, PARTS, ROWS_AHEAD, false>(a, grid, chained, s);
  return launch_rows<T, NT, PER, PARTS, ROWS_AHEAD, true>(a, grid, chained, s);
}
template <typename T, int NT, int PARTS>
fgq_status launch_rows_per(const RowsArgs& a, unsigned grid, bool chained, cudaStream_t s) {
  if (a.w.per == 4) return launch_rows_load<T, NT, 4, PARTS>(a, grid, chained, s);
  return a.w.per == 2 ? launch_rows_load<T, NT, 2, PARTS>(a, grid, chained, s) : launch_rows_load<T, NT, 1, PARTS>(a, grid, chained, s);
}
template <typename T, int PARTS>
fgq_status launch_rows_type(const RowsArgs& a, int nt, unsigned grid, bool chained, cudaStream_t s) {
  if (nt == 1) return launch_rows_per<T, 1, PARTS>(a, grid, chained, s);
  return nt == 2 ? launch_rows_per<T, 2, PARTS>(a, grid, chained, s) : launch_rows_per<T, 4, PARTS>(a, grid, chained, s);
}

}  // namespace w4
}  // namespace fgq
