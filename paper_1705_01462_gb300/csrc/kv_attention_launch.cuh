// Launches of the few-row attention kernel, shared by the files that instantiate it per head size.
#pragma once

#include "kv_attention.cuh"
#include "tc_common.cuh"

namespace fgq {
namespace dec {

template <int NB, int GB, bool SPLIT, int NT>
fgq_status launch_attention(const AttnArgs& a, unsigned blocks, cudaStream_t s) {
  constexpr int bytes = AttnSmem<NB, GB>::template bytes<NT>();
  if (!tc::smem_attr_once<kv_attention_kernel<NB, GB, SPLIT, NT>>(bytes)) return FGQ_ERR_CUDA;
  if (!a.cluster) {
    kv_attention_kernel<NB, GB, SPLIT, NT><<<blocks, 32 * AT_WARPS, bytes, s>>>(a);
    return after_launch();
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(32 * AT_WARPS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)a.chunks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return after_launch(cudaLaunchKernelEx(&cfg, kv_attention_kernel<NB, GB, SPLIT, NT>, a));
}

// fp32 inputs double the queries' and probabilities' operands, and 256-value heads the sums: both keep to 8 rows.
template <int NB, int GB>
AttnKernel pick(bool split, int rows) {
  constexpr int per_sm = attention_blocks_per_sm<NB, 1>();
  constexpr float rate = NB == 2 ? 130.0f : (NB == 4 ? 83.0f : 60.0f);
  if (split) return {launch_attention<NB, GB, true, 1>, 8, per_sm, true, 8.0f, 3.5f, 0.7f * rate};
  if constexpr (NB <= 4) {
    if (rows > 8) return {launch_attention<NB, GB, false, 2>, 16, attention_blocks_per_sm<NB, 2>(), true, 8.0f, 3.5f, (NB == 2 ? 0.9f : 0.85f) * rate};
  }
  return {launch_attention<NB, GB, false, 1>, 8, per_sm, true, 8.0f, 3.5f, rate};
}

}  // namespace dec
}  // namespace fgq
