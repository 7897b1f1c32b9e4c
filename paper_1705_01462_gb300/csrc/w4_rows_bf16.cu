// Few bf16 tokens with 4-bit weights.
#include "w4_launch.h"

namespace fgq {
namespace w4 {

fgq_status launch_rows_bf16(const RowsArgs& a, int nt, unsigned grid, bool chained, cudaStream_t s) {
  return launch_rows_type<__nv_bfloat16, 1>(a, nt, grid, chained, s);
}
fgq_status launch_held_bf16(const ResidentArgs& a, int nt, const ResidentPlan& plan, bool chained, cudaStream_t s) {
  return launch_held_type<__nv_bfloat16, 1>(a, nt, plan, chained, s);
}
fgq_status launch_held_gated_bf16(const ResidentArgs& a, const ResidentPlan& plan, int64_t items, cudaStream_t s) {
  return launch_held_per<__nv_bfloat16, 2, 1, 1, MODE_GATED, GATED_AHEAD>(a, plan, items, true, s);
}

}  // namespace w4
}  // namespace fgq
