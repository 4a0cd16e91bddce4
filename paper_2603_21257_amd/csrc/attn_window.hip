// Launches of the attention with a sliding window and first tokens that stay visible (calvo_window_attn), on packed rows
// (attn_rows_body.h): every element type, head width and group size.
// 32 requests of 300 to 33000 tokens, one new one each, 32Q/8KV behind 4096: 75 us, 4.6 TB/s of K and V, bound by those reads.  One such request
// behind 1024: 9 us, bound by the chain start, lookup, K, V, combination, merge of nine pieces.  bf16 D = 64, 16Q/4KV, 4111+300 behind 2048: 17.3 us, one
// workgroup on each of 152 CUs; fp32 D = 64, 8Q/2KV, 1000+128 behind 300: 9.9 us.
#include "attn_rows_body.h"

namespace calvo {
namespace rows {

template <class C>
hipError_t launch_window(const WinParams& p, unsigned grid, const int32_t* split_tiles, int n_split_tiles, hipStream_t stream) {
  hipLaunchKernelGGL(attn_rows_kernel<C>, dim3(grid), dim3(64 * C::NW), C::LDS_BYTES, stream, p);
  if (n_split_tiles > 0) {
    const unsigned slots = (unsigned)n_split_tiles * (unsigned)p.n_kv_heads;
    hipLaunchKernelGGL((merge_rows_kernel<typename C::T, C::DP, C::ROWS, WinParams>), dim3(slots * (C::ROWS / 4)), dim3(256), 0, stream, p,
                       split_tiles);
  }
  return hipGetLastError();
}

// f(configuration) for an element type, head width and tiling: those of the causal launches (attn_rows_shape), and up to 128-wide heads one
// block of 16 rows for single tokens (window_plan.cpp)
template <typename F>
auto with_window_cfg(int dtype, int head_dim, int tile_rows, F&& f) {
  typedef uint16_t B16;
  if (dtype == CALVO_F32) {
    if (head_dim == 64) return tile_rows == 16 ? f(WinRowsCfg<float, 64, 1, 2, 8, true>{}) : f(WinRowsCfg<float, 64, 2, 2, 8, true>{});
    if (head_dim < 64) return tile_rows == 16 ? f(WinRowsCfg<float, 64, 1, 2, 8, false>{}) : f(WinRowsCfg<float, 64, 2, 2, 8, false>{});
    if (head_dim == 128) return tile_rows == 16 ? f(WinRowsCfg<float, 128, 1, 1, 8, true>{}) : f(WinRowsCfg<float, 128, 2, 1, 4, true>{});
    if (head_dim < 128) return tile_rows == 16 ? f(WinRowsCfg<float, 128, 1, 1, 8, false>{}) : f(WinRowsCfg<float, 128, 2, 1, 4, false>{});
    if (head_dim == 256) return tile_rows == 32 ? f(WinRowsCfg<float, 256, 2, 1, 4, true>{}) : f(WinRowsCfg<float, 256, 1, 1, 4, true>{});
    return tile_rows == 32 ? f(WinRowsCfg<float, 256, 2, 1, 4, false>{}) : f(WinRowsCfg<float, 256, 1, 1, 4, false>{});
  }
  if (tile_rows == 16 && head_dim <= 128) {
    if (head_dim == 64) return f(WinRowsCfg<B16, 64, 1, 2, 8, true>{});
    if (head_dim < 64) return f(WinRowsCfg<B16, 64, 1, 2, 8, false>{});
    return head_dim == 128 ? f(WinRowsCfg<B16, 128, 1, 2, 8, true>{}) : f(WinRowsCfg<B16, 128, 1, 2, 8, false>{});
  }
  if (head_dim == 64) return tile_rows == 64 ? f(WinRowsCfg<B16, 64, 4, 2, 8, true>{}) : f(WinRowsCfg<B16, 64, 2, 2, 8, true>{});
  if (head_dim < 64) return tile_rows == 64 ? f(WinRowsCfg<B16, 64, 4, 2, 8, false>{}) : f(WinRowsCfg<B16, 64, 2, 2, 8, false>{});
  if (head_dim == 128) return tile_rows == 64 ? f(WinRowsCfg<B16, 128, 4, 2, 4, true>{}) : f(WinRowsCfg<B16, 128, 2, 2, 8, true>{});
  if (head_dim < 128) return tile_rows == 64 ? f(WinRowsCfg<B16, 128, 4, 2, 4, false>{}) : f(WinRowsCfg<B16, 128, 2, 2, 8, false>{});
  if (head_dim == 256) return tile_rows == 32 ? f(WinRowsCfg<B16, 256, 2, 2, 4, true>{}) : f(WinRowsCfg<B16, 256, 1, 2, 4, true>{});
  return tile_rows == 32 ? f(WinRowsCfg<B16, 256, 2, 2, 4, false>{}) : f(WinRowsCfg<B16, 256, 1, 2, 4, false>{});
}

}  // namespace rows

hipError_t attn_window_prepare(int dtype, int head_dim, int tile_rows) {
  return rows::with_window_cfg(dtype, head_dim, tile_rows, [](auto cfg) {
    typedef decltype(cfg) C;
    return hipFuncSetAttribute((const void*)rows::attn_rows_kernel<C>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES);
  });
}

hipError_t launch_attn_window(const WinParams& p, int dtype, int tile_rows, int n_items, const int32_t* split_tiles, int n_split_tiles,
                              hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const unsigned grid = (unsigned)n_items * (unsigned)p.n_kv_heads;
  return rows::with_window_cfg(dtype, p.head_dim, tile_rows, [&](auto cfg) {
    return rows::launch_window<decltype(cfg)>(p, grid, split_tiles, n_split_tiles, stream);
  });
}

}  // namespace calvo
