// Planning of an attention launch with a window and first tokens (window_plan.h).  A tile meets only the sub-tiles that some of its
// rows see; from there on the launch is cut and replayed like a causal one (attn_plan.cpp).
#include "window_plan.h"

#include <algorithm>

namespace calvo {

WindowKeys window_keys(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first, int unit) {
  const int64_t lo = std::max<int64_t>(0, pos_min + 1 - window);      // earliest key of the earliest row's window
  const int32_t lo_sub = (int32_t)(lo / unit), end = (int32_t)(pos_max / unit + 1);
  WindowKeys k;
  k.first_subs = (int32_t)std::min<int64_t>(((int64_t)n_first + unit - 1) / unit, lo_sub);
  k.gap = lo_sub - k.first_subs;
  k.n = k.first_subs + end - lo_sub;
  return k;
}

WindowKeys window_keys_full_first(int64_t pos_min, int64_t pos_max, int32_t window, int32_t n_first) {
  WindowKeys k;
  const bool all = n_first > pos_max - window;                         // nothing lies between the first tokens and the windows
  const int64_t lo = all ? 0 : std::max<int64_t>(0, pos_min + 1 - window);
  const int32_t lo_sub = (int32_t)(lo / 32), end = (int32_t)(pos_max / 32 + 1);
  const int32_t full_end = (int32_t)((pos_min + 1) / 32), full_begin = all || pos_max < window ? 0 : (int32_t)((pos_max - window) / 32 + 1);
  k.first_subs = std::min(n_first / 32, lo_sub);
  k.n_part = n_first % 32 != 0 && n_first / 32 < lo_sub ? 1 : 0;
  k.n_full = k.first_subs;
  k.edge = lo_sub;
  k.n_edge = end - lo_sub;
  int32_t n_diag = 0;
  if (full_begin < full_end) {
    k.gap = full_begin - k.first_subs;
    k.n_full += full_end - full_begin;
    k.n_edge = full_begin - lo_sub;
    k.diag = full_end;
    n_diag = end - full_end;
  }
  k.n = k.n_full + k.n_part + k.n_edge + n_diag;
  return k;
}

namespace {

// most partial results of a launch, in slots of 32 rows of 128 floats (34 MB)
constexpr int64_t kMostSlots = 2048;

struct Candidate {
  int variant = kWindowRows;
  int unit = 32;                         // packed rows: keys of a sub-tile
  RowsShape shape{};                     // packed rows
  int tile_tokens = 0;                   // pipelined
  PlanParams params{};
  std::vector<PlanTile> tiles;
  int want = 1;
  PlanCost cost;
};

WindowKeys tile_keys(const Candidate& c, const WindowLens& l, int64_t tile, int group, int32_t window, int32_t n_first) {
  if (c.variant == kWindowRows) {
    const int64_t rows = (int64_t)l.n_new * group, tr = c.shape.tile_rows;
    return window_keys(l.n_cached + tile * tr / group, l.n_cached + (std::min((tile + 1) * tr, rows) - 1) / group, window, n_first, c.unit);
  }
  const int64_t tt = c.tile_tokens;
  return window_keys_full_first(l.n_cached + tile * tt, l.n_cached + std::min<int64_t>((tile + 1) * tt, l.n_new) - 1, window, n_first);
}

void make_tiles(Candidate& c, const std::vector<WindowLens>& lens, int group, int32_t window, int32_t n_first) {
  for (size_t r = 0; r < lens.size(); r++) {
    const int64_t per = c.variant == kWindowRows ? c.shape.tile_rows : c.tile_tokens;
    const int64_t rows = c.variant == kWindowRows ? (int64_t)lens[r].n_new * group : lens[r].n_new;
    for (int64_t t = 0; t * per < rows; t++) c.tiles.push_back({(int32_t)r, (int32_t)t, tile_keys(c, lens[r], t, group, window, n_first).n});
  }
  std::stable_sort(c.tiles.begin(), c.tiles.end(), [](const PlanTile& a, const PlanTile& b) { return a.n_sub > b.n_sub; });
}

// In the units of attn_rows_shape.  A step of 16 bf16 rows costs more where single tokens leave most of the chip idle, because nothing hides its reads; with the dearer
// one batches that leave half of it idle are cut (us a call, 32Q/8KV D = 128 behind 1024: 4 requests 14.4 / 10.9, 8 14.5 / 12.2, 40 of 5000 to 9000
// tokens behind 4096 153 / 143; the other way only 16Q/4KV D = 64, 48 requests behind 4096 32.2 / 33.4; 60 others within 2 %).
RowsShape few_rows_shape(bool f32, int head_dim, bool single_tokens) {
  if (f32) return {kFewRows, head_dim <= 64 ? 14 : 28, 60, 1};
  return {kFewRows, head_dim <= 64 ? (single_tokens ? 7 : 5) : single_tokens ? 12 : 8, 60, 1};
}

// bf16 arithmetic and 128-wide heads: one of the pipelined kernels in place of the packed rows, of which the replay makes rows_us microseconds
void choose_pipelined(const WindowShape& s, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, double rows_us, Candidate& best) {
  const int group = s.n_q_heads / s.n_kv_heads;
  const int hw = attn_heads_per_wg(s.n_q_heads, s.n_kv_heads), head_groups = s.n_q_heads / hw;
  Candidate pipe, duo;
  for (Candidate* c : {&pipe, &duo}) {
    c->variant = c == &pipe ? kAttnPipe : kAttnDuo;
    c->tile_tokens = attn_mfma_tile_tokens(c->variant, hw);
    c->params = {head_groups, s.n_cus * (8 / attn_mfma_row_blocks(c->variant)), 48, 30, s.force_splits, false, 0, c->variant == kAttnDuo ? s.n_cus : 0};
    make_tiles(*c, lens, group, window, n_first);
    c->want = plan_pieces(c->tiles, c->params, kMostSlots / attn_mfma_row_blocks(c->variant), &c->cost);
  }
  // What the replays make of a launch, in us: packed rows 3 and 1.2 times their tenths, the pipelined kernels 0.6 to 0.8 a step, the larger tiles
  // the more the shorter the launch.  us a call of one caller, 32Q/8KV, packed rows / kAttnDuo / kAttnPipe:
  //   window 1024   4096+1 17.3 / 28.3 / 35.9      4096+64 21.4 / 30.8 / 46.1    4096+256 23.4 / 30.7 / 46.4    4096+1024 59.1 / 36.3 / 50.9
  //   window 16384  20000+1 24.9 / 26.6 / 30.7     20000+64 51.1 / 37.5 / 47.8   20000+256 142 / 79.1 / 81.1    20000+1024 504 / 250 / 242
  //   window 256    0+500 20.5 / 20.6 / 31.5       0+2000 71.9 / 32.0 / 39.2     0+8192 253 / 93.5 / 135
  // Among the pipelined ones the larger tiles read K and V half as often, the smaller ones have two workgroups on a CU whose starts, ends and sub-tiles
  // outside the steady loop hide each other.  Those sub-tiles grow with the tokens of a tile (64, 128 or 256 at four, two or one query heads to a workgroup):
  // the sides cross where a list has some two sub-tiles for every token.  kAttnPipe / kAttnDuo, us a call of one caller, 16384+2048 tokens and 0+16384
  // behind 2048, 4096, 8192, 16384:
  //   32Q/8KV  76.3 / 76.2  122 / 128   214 / 232   403 / 449      569 / 541   861 / 847    1300 / 1330  1634 / 1710
  //   16Q/8KV  63.2 / 53.1  86.4 / 83.0 133 / 140   227 / 254      305 / 271   470 / 443    664 / 698    836 / 881
  //   40Q/8KV  (320 workgroups on 256 CUs: 740 / 622 at 16384)     779 / 717   1138 / 1077  1679 / 1655  2073 / 2130
  // Short launches are the smaller tiles' (20000+700 behind 4096 71.8 / 71.3, 20000+64 behind 16384 47.8 / 37.5), and so are those that fill the last round
  // of CUs badly, where a workgroup of the smaller tiles has its CU to itself.
  constexpr double kSubsPerToken = 1.9, kLongLaunch = 140., kFilled = 0.9;
  int64_t subs = 0;
  for (const PlanTile& t : pipe.tiles) subs += t.n_sub;
  const bool larger = s.force_variant ? s.force_variant == kAttnPipe
                                      : (double)subs >= kSubsPerToken * pipe.tile_tokens * (double)pipe.tiles.size() && pipe.cost.span >= kLongLaunch &&
                                            pipe.cost.load >= kFilled * pipe.cost.span && pipe.cost.span <= 1.03 * duo.cost.span;
  if (s.force_variant || rows_us >= 0.6 * duo.cost.span) best = std::move(larger ? pipe : duo);
}

// Packed rows over an 8-bit pool, in the units of attn_rows_shape: a step is 64 keys, a workgroup has four waves.  A step of single tokens is the latency of
// its reads (1.3 us while they leave the memory's rate alone), and the last piece of a tile to arrive merges them in 1.7 us a round of 32.  us a call of
// one caller, 32Q/8KV, D = 128, with launches of half, one and two workgroups to a CU in mind: 8 requests of 500 to 20000 behind 4096 17.8 / 13.1 / 13.8,
// four of 4096 12.9 / 10.5 / 12.0, 32 of 300 to 33000 138.7 / 112.3 / 109.9, 60000+1 28.1 / 25.2 / 25.2, 24 of 3000 40.4 / 37.1 / 40.4.
constexpr int kMostMerged = 32, kMergedAlong = 4;              // pieces; rows, a wave each
RowsShape e4m3_shape(int head_dim, bool few, bool large, bool along) {
  const int step = head_dim <= 64 ? 8 : head_dim <= 128 ? 13 : 24;
  // A merge in a launch of its own costs twice as much (20 / 40: 7524+1 and seven shorter behind 528, 16Q/2KV, D = 96 9.6 / 7.5, 20 + 1 to 34792 + 1 behind 316, 40Q/8KV,
  // D = 128 9.0 / 7.6)
  if (few) return {kFewRows, step, along ? 20 : 40, 1};
  // Wider heads are cut earlier (60 / 45, D = 256: 700+60 tokens, 8Q/2KV 13.5 / 12.0, 500+33, 4Q/4KV 12.1 / 11.4, nine other shapes the same); with 45
  // 128-wide ones would stay on packed rows too rarely (4096+64 behind 1024, 32Q/8KV 10.0 / 14.7).  Their tiles of 32 rows cost little more a step, whose time goes
  // to widening, and more to end (16 / 32 rows, D = 256: 8192+1024, 32Q/8KV 662 / 389, 2000+200, 8Q/2KV 22.0 / 21.0, 5000+30 15.3 / 17.8, 700+60 12.0 / 15.2)
  if (head_dim > 128) return large ? RowsShape{32, 29, 75, 1} : RowsShape{kFewRows, step, 45, 1};
  if (large) return {32, step + step / 2, 60, 1};
  // Tiles of 16 rows of narrow heads have 126 registers: four workgroups to a CU, whose steps take the longer.  us a call of one caller, D = 64, as two at 8 and 60 /
  // as four at 15 and 45: 787+7218 behind 24, 32Q/8KV 71.1 / 51.5, 257+1643 behind 41, 64Q/8KV 33.0 / 25.5, 0+1032, 40Q/8KV 21.1 / 18.6, 4142+24 with 207+633, 16Q/4KV 12.8 / 12.7
  if (head_dim <= 64) return {kFewRows, 15, 45, 1};
  return {kFewRows, step, head_dim < 128 ? 50 : 60, 1};
}

// The launch of the chosen candidate; a packed-rows workgroup merges at most merge_rows rows along (plan_window)
void make_plan(const WindowShape& s, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, const Candidate& best, int merge_rows, WindowPlan& out) {
  const int group = s.n_q_heads / s.n_kv_heads;
  const int hw = attn_heads_per_wg(s.n_q_heads, s.n_kv_heads), head_groups = s.n_q_heads / hw;
  out.variant = best.variant;
  out.heads_per_wg = hw;
  if (best.variant == kWindowRows) {
    out.tile_rows = best.shape.tile_rows;
    out.single_tiles = true;
    for (const WindowLens& l : lens) out.single_tiles &= (int64_t)l.n_new * group <= best.shape.tile_rows;
    out.one_launch = out.single_tiles && best.shape.tile_rows == kFewRows;
    for (const WindowLens& l : lens) out.one_launch &= (int64_t)l.n_new * group <= merge_rows;
    out.part_rows = (int64_t)s.n_kv_heads * best.shape.tile_rows;
    out.part_width = s.head_dim <= 64 ? 64 : s.head_dim <= 128 ? 128 : 256;
  } else {
    out.tile_tokens = best.tile_tokens;
    out.part_rows = (int64_t)head_groups * attn_mfma_row_blocks(best.variant) * 32;
    out.part_width = 128;
  }
  const PlanItems pi = plan_items(best.tiles, best.want, best.params);
  out.split_tiles = pi.split_tiles;
  if (!pi.split_tiles.empty()) out.n_parts = pi.split_tiles.back() + pi.items[(size_t)pi.split_tiles.back()].n_splits;   // the longest tiles come first
  out.items.reserve(pi.items.size());
  for (const WorkItem& x : pi.items)
    out.items.push_back({x.req, x.q_tile, x.sub_begin, x.sub_end, x.n_splits, x.first_item,
                         tile_keys(best, lens[(size_t)x.req], x.q_tile, group, window, n_first)});
}

void plan_window_e4m3(const WindowShape& s, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, WindowPlan& out) {
  const int group = s.n_q_heads / s.n_kv_heads;
  bool few = s.force_tile == 0, along = true;
  for (const WindowLens& l : lens) {
    few &= (int64_t)l.n_new * group <= kFewRows;
    along &= (int64_t)l.n_new * group <= kMergedAlong;
  }
  Candidate best;
  for (const bool large : {false, true}) {
    if (large && (few || s.force_tile == 1)) break;
    Candidate c;
    c.unit = kE4m3Keys;
    c.shape = e4m3_shape(s.head_dim, few, large, along);
    const int per_cu = few || s.head_dim > 128 ? 1 : s.head_dim <= 64 && !large ? 4 : 2;
    c.params = rows_plan_params(c.shape, s.n_kv_heads, per_cu * s.n_cus, s.force_splits);
    if (per_cu == 4) c.params.alone = s.n_cus;               // 2737+113 behind 1500, 32Q/8KV: without / with 14.0 / 8.4
    // 24 single tokens, 32Q/8KV, D = 128, of which one has 47862 cached tokens and most have few: pieces counted as if all were cut / as many as come of it
    // 60.6 / 36.0 us a call; 8Q/8KV, D = 96, 46902 39.7 / 24.5; 53091+1 with 0+817, 16Q/4KV, D = 64 53.6 / 15.4; even batches the same
    c.params.most = kMostMerged;
    make_tiles(c, lens, group, window, n_first);
    c.want = plan_pieces(c.tiles, c.params, kMostSlots / c.shape.slots, &c.cost);
    if (best.tiles.empty() || (large && s.force_tile == 2) || c.cost.span < best.cost.span) best = std::move(c);
  }
  // Where the replays' lengths differ by 2.4 (packed rows in tenths of a microsecond, the pipelined kernels in steps) the two take the same time, but for 9 us that
  // the start, end and merge of the latter take more.  us a call of one caller, 32Q/8KV, packed rows / kAttnDuo, and that quotient: 4096+64 behind 1024
  // 10.1 / 25.0 (2.4), 1000+100 10.5 / 26.1 (2.3), 60000+5 36.2 / 41.4 (2.1), 20000+16 35.2 / 23.5 (2.7), 20000+64 44.2 / 35.7 (3.9), 4096+256 44.8 / 34.3 (3.7);
  // few heads or long and short requests in one batch: 0+1015 and 45+1, 8Q/8KV 12.0 / 25.4, 1543+435, 6Q/3KV 14.1 / 23.4, 330+259 and 413+215 14.7 / 18.6.
  constexpr double kPipelinedStart = 9.;
  if (s.head_dim == 128 && s.force_variant != 5 && !few) choose_pipelined(s, lens, window, n_first, 0.248 * best.cost.span - kPipelinedStart, best);
  make_plan(s, lens, window, n_first, best, kMergedAlong, out);
}

}  // namespace

void plan_window(const WindowShape& s, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, WindowPlan& out) {
  out = WindowPlan();
  const int group = s.n_q_heads / s.n_kv_heads;
  int64_t total = 0;
  for (const WindowLens& l : lens) total += l.n_new;
  if (total == 0) return;
  if (s.e4m3) return plan_window_e4m3(s, lens, window, n_first, out);

  // Up to 128-wide heads there is a tiling of 16 rows as well.  Single tokens take it: it leaves the combination of the waves half as long (us a call of
  // one caller, 32 / 16 rows, 32Q/8KV: 4096+1 behind 4096 15.4 / 14.0, 20000+1 behind 16384 23.3 / 20.7), and none of the others is looked at
  // (planning 32 requests takes 40 us, 5 this way).
  const bool has_few = s.force_tile == 0 && s.head_dim <= 128;
  bool few = has_few && s.force_variant == 0, one_tile = true;
  for (const WindowLens& l : lens) {
    few &= (int64_t)l.n_new * group <= kFewRows;
    one_tile &= (int64_t)l.n_new * group <= attn_rows_shape(s.f32, s.head_dim, false).tile_rows;
  }
  // Batches that leave most of the chip idle take it where the replay is shorter (one caller, 32 / 16 rows: fp32 D = 64 8Q/2KV 1000+128 behind 300 15.8 /
  // 12.7, bf16 1000+64 14.4 / 13.1, 32Q/8KV 4000+100 behind 1024 14.9 / 14.1; not 16Q/4KV 4111+300 behind 2048 21.2 / 30.4, fp32 8Q/2KV 4000+200
  // 30.0 / 33.8), and where that does not cost the launch that stores the new rows (one_tile); from four workgroups per CU on they are not
  // replayed (of 100000 drawn batches 109 would have taken it).
  Candidate best;
  for (const int kind : {0, 1, 2}) {
    if (kind == 1 && (!has_few || (one_tile && !few) || (int64_t)best.tiles.size() * s.n_kv_heads > 4 * (int64_t)s.n_cus)) continue;
    if (kind == 2 && (few || !attn_rows_has_large(s.f32, s.head_dim) || s.force_tile == 1)) break;
    if (kind == 0 && few) continue;
    Candidate c;
    c.shape = kind == 1 ? few_rows_shape(s.f32, s.head_dim, few) : attn_rows_shape(s.f32, s.head_dim, kind == 2);
    c.params = rows_plan_params(c.shape, s.n_kv_heads, s.n_cus, s.force_splits);
    make_tiles(c, lens, group, window, n_first);
    c.want = plan_pieces(c.tiles, c.params, kMostSlots / c.shape.slots, &c.cost);
    if (best.tiles.empty() || (kind == 2 && s.force_tile == 2) || 2. * c.cost.span + c.cost.load < 0.97 * (2. * best.cost.span + best.cost.load)) best = std::move(c);
  }
  if (!s.f32 && s.head_dim == 128 && s.force_variant != 5 && !few) choose_pipelined(s, lens, window, n_first, 3. + 0.12 * best.cost.span, best);
  // At most one row for each wave of a workgroup: then the last piece of a tile merges them (attn_rows_body.h).  us a call of one caller, by a launch
  // behind / by the last piece: bf16 D = 128, 32Q/8KV, 4096+1 behind 1024 10.9 / 8.9, four such requests 11.5 / 9.2, 64Q/8KV 12.4 / 12.3 behind 4096; 32Q/4KV
  // 11.6 / 12.0; D = 64, 16Q/4KV 11.6 / 9.6; D = 256, 16Q/4KV 14.4 / 14.5, 8Q/8KV 15.0 / 14.7; fp32 D = 128, 32Q/8KV 15.0 / 14.8, 32Q/4KV 13.9 / 14.0.  Two rows
  // a wave and more: 64Q/4KV 12.5 / 16.9, 16Q/1KV 11.7 / 15.9, D = 256 32Q/4KV 14.4 / 20.4, 64Q/4KV 15.1 / 30.4.
  make_plan(s, lens, window, n_first, best, s.head_dim <= 128 ? 8 : 4, out);
}

// Rows that a workgroup takes at least: below, its start and the addition of the parts cost more than the rows
constexpr int64_t kChunkRows = 256;

void plan_mass(int group, int n_kv_heads, int n_cus, int tile_keys, const std::vector<WindowLens>& lens, int32_t window, int32_t n_first, MassPlan& out) {
  out = MassPlan();
  // the new tokens [i0, i1) that see some key of a tile
  auto seen_by = [&](const WindowLens& l, int64_t tile, int64_t& i0, int64_t& i1) {
    const int64_t k0 = tile * tile_keys, k1 = std::min<int64_t>(k0 + tile_keys, (int64_t)l.n_cached + l.n_new);
    i0 = std::max<int64_t>(0, k0 - l.n_cached);
    i1 = k0 < n_first ? l.n_new : std::max<int64_t>(i0, std::min<int64_t>(l.n_new, k1 - 1 + window - l.n_cached));
  };
  int64_t rows = 0;
  auto tiles_of = [&](const WindowLens& l) { return ((int64_t)l.n_cached + l.n_new + tile_keys - 1) / tile_keys; };
  for (const WindowLens& l : lens)
    for (int64_t t = 0, i0, i1; t < tiles_of(l); t++) {
      seen_by(l, t, i0, i1);
      rows += (i1 - i0) * group;
    }
  // Eight workgroups per CU where there are rows enough.  The tokens are cut at the same places for every tile, and the tiles that meet the same tokens
  // follow each other: what runs at a time shares its rows in the L2.
  const int64_t share = std::max(kChunkRows, rows * n_kv_heads / (8 * (int64_t)n_cus));
  const int64_t chunk = std::max<int64_t>(16, (std::min<int64_t>(share, 1 << 19) / group + 15) / 16 * 16);
  for (size_t r = 0; r < lens.size(); r++) {
    const int64_t n_tiles = tiles_of(lens[r]), n_chunks = std::max<int64_t>(1, (lens[r].n_new + chunk - 1) / chunk);
    std::vector<MassTile> tiles((size_t)n_tiles);
    for (int64_t t = 0, i0, i1; t < n_tiles; t++) {
      seen_by(lens[r], t, i0, i1);
      const int32_t n = i1 > i0 ? (int32_t)((i1 - 1) / chunk - i0 / chunk + 1) : 1;
      tiles[(size_t)t] = {(int32_t)r, (int32_t)t, n > 1 ? out.n_parts : -1, n};
      if (n > 1) {
        out.adds.push_back(tiles[(size_t)t]);
        out.n_parts += n;
      }
    }
    for (int64_t k = 0; k < n_chunks; k++)
      for (int64_t t = 0, i0, i1; t < n_tiles; t++) {
        seen_by(lens[r], t, i0, i1);
        const int64_t b = std::max(i0, k * chunk), e = std::min(i1, (k + 1) * chunk);
        const MassTile& m = tiles[(size_t)t];
        if (i1 > i0 ? b < e : k == 0) out.items.push_back({(int32_t)r, (int32_t)t, (int32_t)b, (int32_t)std::max(b, e), m.part < 0 ? -1 : m.part + (int32_t)(k - i0 / chunk)});
      }
  }
}

}  // namespace calvo
