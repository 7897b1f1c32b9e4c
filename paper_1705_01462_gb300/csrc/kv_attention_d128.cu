// The few-row attention kernel for heads of 128 values.
#include "kv_attention_launch.cuh"

namespace fgq {
namespace dec {

AttnKernel attention_kernel_4(int gb, bool split, int rows) {
  if (gb == 1) return pick<4, 1>(split, rows);
  if (gb == 2) return pick<4, 2>(split, rows);
  return pick<4, 4>(split, rows);
}

}  // namespace dec
}  // namespace fgq
