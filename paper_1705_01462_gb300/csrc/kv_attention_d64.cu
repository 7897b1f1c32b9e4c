// The few-row attention kernel for heads of 64 values.
#include "kv_attention_launch.cuh"

namespace fgq {
namespace dec {

AttnKernel attention_kernel_2(int gb, bool split, int rows) {
  if (gb == 1) return pick<2, 1>(split, rows);
  return pick<2, 2>(split, rows);
}

}  // namespace dec
}  // namespace fgq
