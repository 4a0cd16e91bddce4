// Host-side planning of an attention launch with a window and first tokens: which tiles, which of a tile's keys, how many pieces.
// No device types here.
#pragma once
#include <cstdint>
#include <vector>

#include "attn_plan.h"

namespace calvo {

struct WindowLens {
  int32_t n_cached, n_new;
};

// A piece of a tile; see WinItem (calvo_internal.h)
struct WindowPiece {
  int32_t req, tile, sub_begin, sub_end, n_splits, first_item, first_subs, gap;
};

struct WindowPlan {
  RowsShape shape{};
  int part_width = 0;                    // floats of a row of partial results
  std::vector<WindowPiece> items;
  std::vector<int32_t> split_tiles;      // first item of every cut tile
};

// The keys that rows at positions [pos_min, pos_max] see, as 32-key sub-tiles: first_subs from position 0 on, then those from
// first_subs + gap on, n of both.
struct WindowKeys {
  int32_t first_subs, gap, n;
};
WindowKeys window_keys(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first);

void plan_window(bool f32, int head_dim, int group, int n_kv_heads, int n_cus, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first,
                 int force_splits, int force_tile, WindowPlan& out);

}  // namespace calvo
