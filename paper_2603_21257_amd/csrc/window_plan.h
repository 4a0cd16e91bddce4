// Host-side planning of an attention launch with a window and first tokens: which kernel, which tiles, which of a tile's keys, how many
// pieces.  No device types here.
#pragma once
#include <cstdint>
#include <vector>

#include "attn_plan.h"

namespace calvo {

struct WindowLens {
  int32_t n_cached, n_new;
};

// A tile's keys as a list of 32-key sub-tiles, in the words of WinItem (calvo_internal.h); n: of the whole list
struct WindowKeys {
  int32_t first_subs = 0, gap = 0, n = 0;
  int32_t n_full = 0, n_part = 0, edge = 0, n_edge = 0, diag = 0;
};
// for rows at positions [pos_min, pos_max]: in the order of the context (packed rows; unit: keys of a sub-tile) ...
WindowKeys window_keys(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first, int unit = 32);
// ... and with those that every row sees in full in front (pipelined kernels)
WindowKeys window_keys_full_first(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first);

struct WindowPiece {
  int32_t req, tile, sub_begin, sub_end, n_splits, first_item;
  WindowKeys keys;
};

constexpr int kWindowRows = -1;          // the packed-rows kernel; else kAttnPipe or kAttnDuo

struct WindowPlan {
  int variant = kWindowRows;
  int tile_rows = 0;                     // packed rows: the tiling
  int tile_tokens = 0;                   // pipelined: tokens of a tile
  int heads_per_wg = 1;                  // pipelined
  bool single_tiles = false;             // packed rows: no request has more than one tile
  bool one_launch = false;               // single_tiles with at most one row for each wave of a workgroup
  int64_t part_rows = 0, part_width = 0; // rows of partial results that a work item leaves over all heads, floats of one
  std::vector<WindowPiece> items;
  std::vector<int32_t> split_tiles;      // first item of every cut tile
  int64_t n_parts = 0;                   // items up to the last one of a cut tile: those that partial results have room for
};

constexpr int kFewRows = 16;             // tile_rows for single tokens

struct WindowShape {
  bool f32;
  int head_dim, n_q_heads, n_kv_heads, n_cus;
  int force_splits, force_tile, force_variant;   // test knobs: 0 = automatic
  bool e4m3 = false;                             // 8-bit pool: packed rows count 64-key steps
};
constexpr int kE4m3Keys = 64;            // keys of a step of its packed rows
void plan_window(const WindowShape& s, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, WindowPlan& out);

// ---- gathered weights: key tiles of tile_keys tokens, and parts of the rows that see one

struct MassPiece {
  int32_t req, tile, begin, end, part;   // see MassItem (calvo_internal.h)
};
struct MassTile {
  int32_t req, tile, part, n_parts;
};
struct MassPlan {
  std::vector<MassPiece> items;
  std::vector<MassTile> adds;            // tiles with several items
  int32_t n_parts = 0;
};
void plan_mass(int group, int n_kv_heads, int n_cus, int tile_keys, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, MassPlan& out);

}  // namespace calvo
