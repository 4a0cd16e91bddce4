// Attention with a window and first tokens on the pipelined bodies (attn_pipeline.h): bf16, 128-wide heads.  A tile's list of sub-tiles has
// those in front that all its rows see, which the steady loop runs without a mask; the others (where windows begin, the diagonal, first tokens that end
// inside a sub-tile) are met behind it one by one (WinPipeCfg).
// Power bounds long launches, as it does the causal ones, and what is outside the steady loop: 14 us of a workgroup's start, masked sub-tiles and end.
// 32Q/8KV: 0+32768 tokens behind 4096 1666 us, 1270 TFLOP/s of the pairs that are seen; 16384+2048 behind 4096 (one workgroup per CU) 122 us, 1130;
// 28096+28, 28304+61 and 38304+209 behind 8192 (60 pieces of 128 rows) 49.5 us and 8 of merging.
#include "attn_merge.h"
#include "attn_pipeline.h"

namespace calvo {
namespace window {

using namespace attn;
using Large = WinPipeCfg<4, 8, 2>;
using Small = WinPipeCfg<4, 5, 1>;

// register limits as those of the causal kernels (attn_pipe.hip, attn_duo.hip)
__global__ void __launch_bounds__(256, 1) __attribute__((amdgpu_num_vgpr(240))) window_pipe_kernel(WinParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  attn_pipeline<Large>(p, smem);
}
__global__ void __launch_bounds__(256, 2) __attribute__((amdgpu_num_vgpr(120))) window_duo_kernel(WinParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  attn_pipeline<Small>(p, smem);
}

}  // namespace window

hipError_t attn_window_pipe_prepare() {
  const hipError_t e = hipFuncSetAttribute((const void*)window::window_pipe_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, window::Large::LDS_BYTES);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)window::window_duo_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, window::Small::LDS_BYTES);
}

hipError_t launch_attn_window_pipe(const WinParams& p, int variant, int n_items, const int32_t* split_tiles, int n_split_tiles, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const unsigned groups = (unsigned)(p.n_q_heads / p.heads_per_wg), grid = (unsigned)n_items * groups;
  if (variant == kAttnPipe) hipLaunchKernelGGL(window::window_pipe_kernel, dim3(grid), dim3(256), window::Large::LDS_BYTES, stream, p);
  else hipLaunchKernelGGL(window::window_duo_kernel, dim3(grid), dim3(256), window::Small::LDS_BYTES, stream, p);
  if (n_split_tiles > 0) {
    const unsigned slots = (unsigned)n_split_tiles * groups * (unsigned)p.row_blocks_per_wg;
    if (slots * 32u <= pipe::kMergeSingleRows / 2)
      hipLaunchKernelGGL((pipe::merge_splits_kernel<1, 32, WinParams>), dim3(slots * 8u), dim3(256), 0, stream, p, split_tiles);
    else if (slots * 32u <= pipe::kMergeSingleRows)
      hipLaunchKernelGGL((pipe::merge_splits_kernel<1, 16, WinParams>), dim3(slots * 8u), dim3(256), 0, stream, p, split_tiles);
    else
      hipLaunchKernelGGL((pipe::merge_splits_kernel<4, 16, WinParams>), dim3(slots * 2u), dim3(256), 0, stream, p, split_tiles);
  }
  return hipGetLastError();
}

}  // namespace calvo
