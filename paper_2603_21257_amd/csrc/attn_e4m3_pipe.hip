// Attention over a pool of 8-bit floats on the pipelined bodies (attn_pipeline.h, WinPipe8Cfg): 128-wide heads, tiles of many rows.  K and V are widened once
// for a workgroup, on their way into LDS, and from there on all is as over a bf16 pool.  32Q/8KV, calls queued back to back: 16384+2048 tokens 433 us, 1350
// TFLOP/s for one caller whose clock has come up, 431 to 441 for several in turn, 0+16384 1620 us (1360) and 1654 to 1718 (1280 to 1330; a large library
// product 1400): power, as over bf16 pools, which take the same time and twice the memory.  Short queries (28096+28, 28304+61, 38304+209) 170 us, 1015: rows of
// tiles that tokens do not fill, starts and ends of pieces, and 8 us of merging.  256 registers and 133 accumulation registers: with 240 the compiler moved
// results of products between the two.
#include "attn_merge.h"
#include "attn_pipeline.h"

namespace calvo {
namespace e4m3 {

using namespace attn;
using Large = WinPipe8Cfg<4, 8, 2>;
using Small = WinPipe8Cfg<4, 4, 1>;

__global__ void __launch_bounds__(256, 1) __attribute__((amdgpu_num_vgpr(256))) e4m3_pipe_kernel(WinParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  attn_pipeline<Large>(p, smem);
}
__global__ void __launch_bounds__(256, 2) __attribute__((amdgpu_num_vgpr(120))) e4m3_duo_kernel(WinParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  attn_pipeline<Small>(p, smem);
}

}  // namespace e4m3

hipError_t attn_e4m3_pipe_prepare() {
  const hipError_t e = hipFuncSetAttribute((const void*)e4m3::e4m3_pipe_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, e4m3::Large::LDS_BYTES);
  if (e != hipSuccess) return e;
  return hipFuncSetAttribute((const void*)e4m3::e4m3_duo_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, e4m3::Small::LDS_BYTES);
}

hipError_t launch_attn_e4m3_pipe(const WinParams& p, int variant, int n_items, const int32_t* split_tiles, int n_split_tiles, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const unsigned grid = (unsigned)n_items * (unsigned)(p.n_q_heads / p.heads_per_wg);
  if (variant == kAttnPipe) hipLaunchKernelGGL(e4m3::e4m3_pipe_kernel, dim3(grid), dim3(256), e4m3::Large::LDS_BYTES, stream, p);
  else hipLaunchKernelGGL(e4m3::e4m3_duo_kernel, dim3(grid), dim3(256), e4m3::Small::LDS_BYTES, stream, p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_merge_window(p, split_tiles, n_split_tiles, stream);
}

}  // namespace calvo
