// The attention kernel for long suffixes (attn_pipeline.h): workgroup = 4 query heads of one KV group x 64 tokens (256 rows in
// any case), four waves of 64 rows, one workgroup per CU, K and V rings of eight 8 KiB slots.
#include "attn_merge.h"
#include "attn_pipeline.h"

namespace calvo {
namespace pipe {

using namespace attn;
using Cfg = PipeCfg<4, 8, 2>;

// 480 of the 512 registers that a wave alone on its SIMD may have (the attribute counts half of
// the unified VGPR+AGPR file on this target): the remaining 32 per SIMD lane let a wave of the
// ingest scatter kernel become resident next to the attention waves, so the loading stage keeps
// moving while attention occupies every CU.
__global__ void __launch_bounds__(256, 1) __attribute__((amdgpu_num_vgpr(240))) attn_pipe_kernel(AttnParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  clock_begin(p.clock);
  if (append_wg(p)) return;
  attn_pipeline<Cfg>(p, smem);
}

}  // namespace pipe

int attn_pipe_tile_tokens(int heads_per_wg) { return 32 * pipe::Cfg::HB * pipe::Cfg::NW / heads_per_wg; }

hipError_t attn_pipe_prepare() {
  return hipFuncSetAttribute((const void*)pipe::attn_pipe_kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                             pipe::Cfg::LDS_BYTES);
}

hipError_t launch_attn_pipe(const AttnParams& p, hipStream_t stream) {
  if (p.n_items <= 0) return hipSuccess;
  const unsigned grid = (unsigned)p.n_items * (unsigned)(p.n_q_heads / p.heads_per_wg);
  hipLaunchKernelGGL(pipe::attn_pipe_kernel, dim3(grid + attn::append_wgs(p)), dim3(64 * pipe::Cfg::NW), pipe::Cfg::LDS_BYTES, stream, p);
  return hipGetLastError();
}

hipError_t launch_merge_splits(const AttnParams& p, const int32_t* split_tiles, int n_split_tiles, hipStream_t stream) {
  if (n_split_tiles <= 0) return hipSuccess;
  const unsigned slots = (unsigned)n_split_tiles * (unsigned)(p.n_q_heads / p.heads_per_wg) * (unsigned)p.row_blocks_per_wg;
  if (slots * 32u <= pipe::kMergeSingleRows / 2)
    hipLaunchKernelGGL((pipe::merge_splits_kernel<1, 32>), dim3(slots * 8u), dim3(256), 0, stream, p, split_tiles);
  else if (slots * 32u <= pipe::kMergeSingleRows)
    hipLaunchKernelGGL((pipe::merge_splits_kernel<1, 16>), dim3(slots * 8u), dim3(256), 0, stream, p, split_tiles);
  else
    hipLaunchKernelGGL((pipe::merge_splits_kernel<4, 16>), dim3(slots * 2u), dim3(256), 0, stream, p, split_tiles);
  return hipGetLastError();
}

}  // namespace calvo
