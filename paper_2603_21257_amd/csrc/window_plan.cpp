// Planning of an attention launch with a window and first tokens (window_plan.h).  A tile meets only the sub-tiles that some of its
// rows see; from there on the launch is cut and replayed like a causal one (attn_plan.cpp).
#include "window_plan.h"

#include <algorithm>

namespace calvo {

WindowKeys window_keys(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first) {
  const int64_t lo = std::max<int64_t>(0, pos_min + 1 - window);      // earliest key of the earliest row's window
  const int32_t lo_sub = (int32_t)(lo / 32), end_sub = (int32_t)(pos_max / 32 + 1);
  const int32_t first = (int32_t)std::min<int64_t>(((int64_t)n_first + 31) / 32, lo_sub);
  return {first, lo_sub - first, first + end_sub - lo_sub};
}

namespace {

// most pieces x heads x rows of partial results (34 MB at 128-wide heads)
constexpr int64_t kMostSlots = 2048;

struct Candidate {
  RowsShape shape{};
  std::vector<PlanTile> tiles;
  int want = 1;
};

void make_tiles(const std::vector<WindowLens>& lens, int group, int tile_rows, int32_t window, int32_t n_first, std::vector<PlanTile>& tiles) {
  for (size_t r = 0; r < lens.size(); r++) {
    const int64_t rows = (int64_t)lens[r].n_new * group;
    for (int64_t t = 0; t * tile_rows < rows; t++) {
      const int64_t pos_min = lens[r].n_cached + t * tile_rows / group, pos_max = lens[r].n_cached + (std::min((t + 1) * tile_rows, rows) - 1) / group;
      tiles.push_back({(int32_t)r, (int32_t)t, window_keys(pos_min, pos_max, window, n_first).n});
    }
  }
  std::stable_sort(tiles.begin(), tiles.end(), [](const PlanTile& a, const PlanTile& b) { return a.n_sub > b.n_sub; });
}

}  // namespace

void plan_window(bool f32, int head_dim, int group, int n_kv_heads, int n_cus, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first,
                 int force_splits, int force_tile, WindowPlan& out) {
  out = WindowPlan();
  Candidate best;
  PlanCost best_cost;
  for (const bool large : {false, true}) {
    if (large && (!attn_rows_has_large(f32, head_dim) || force_tile == 1)) break;
    Candidate c;
    c.shape = attn_rows_shape(f32, head_dim, large);
    make_tiles(lens, group, c.shape.tile_rows, window, n_first, c.tiles);
    PlanCost cost;
    c.want = c.tiles.empty() ? 1
                             : plan_pieces(c.tiles, rows_plan_params(c.shape, n_kv_heads, n_cus, force_splits), kMostSlots / c.shape.slots, &cost);
    if (!large || force_tile == 2 || 2. * cost.span + cost.load < 0.97 * (2. * best_cost.span + best_cost.load)) {
      best = std::move(c);
      best_cost = cost;
    }
  }
  out.shape = best.shape;
  out.part_width = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  if (best.tiles.empty()) return;
  const PlanItems pi = plan_items(best.tiles, best.want, rows_plan_params(best.shape, n_kv_heads, n_cus, force_splits));
  out.split_tiles = pi.split_tiles;
  out.items.reserve(pi.items.size());
  for (const WorkItem& x : pi.items) {
    const WindowLens& l = lens[(size_t)x.req];
    const int64_t tr = best.shape.tile_rows, rows = (int64_t)l.n_new * group;
    const WindowKeys k = window_keys(l.n_cached + x.q_tile * tr / group, l.n_cached + (std::min((x.q_tile + 1) * tr, rows) - 1) / group, window, n_first);
    out.items.push_back({x.req, x.q_tile, x.sub_begin, x.sub_end, x.n_splits, x.first_item, k.first_subs, k.gap});
  }
}

}  // namespace calvo
