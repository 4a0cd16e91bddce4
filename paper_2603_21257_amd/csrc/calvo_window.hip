// Host side of the operators that keep a request's cache bounded: attention with a sliding window and first tokens, gathered
// weights, eviction (include/calvo.h).  Validation, the plan of a batch and its description to the device, the launches.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <new>

#include "calvo_ctx.h"
#include "window_plan.h"

using namespace calvo;
using namespace calvo::host;

// A batch of calvo_window_prepare
struct calvo_window {
  calvo_ctx* c = nullptr;
  int n_reqs = 0, total = 0;            // total: new tokens
  int32_t window = 0, n_first = 0;
  int64_t longest = 0;                  // most tokens of a request, new ones included
  int max_mass_row = -1;
  bool mass_rows_differ = true;
  WindowPlan plan;
  MassPlan mass;
  StepBuf buf;
  // 32-bit words from the beginning of buf.d
  size_t items_at = 0, split_at = 0, arrived_at = 0, mass_at = 0, add_at = 0, append_at = 0, touched_at = 0, tables_at = 0, offs_at = 0;
  int n_touched = 0;                    // blocks that new tokens go to
  size_t part_o_at = 0, part_ml_at = 0, part_mass_at = 0; // floats, behind them
};

namespace {

// Calls run on the context's device whatever the caller's current one is.
class OnDevice {
 public:
  explicit OnDevice(int device) {
    if (hipGetDevice(&was_) != hipSuccess) { (void)hipGetLastError(); was_ = -1; }
    if (was_ != device) { status_ = hipSetDevice(device); moved_ = status_ == hipSuccess; }
  }
  ~OnDevice() {
    if (moved_ && was_ >= 0) (void)hipSetDevice(was_);
  }
  hipError_t status() const { return status_; }

 private:
  int was_ = -1;
  bool moved_ = false;
  hipError_t status_ = hipSuccess;
};
#define ON_DEVICE(c)             \
  const OnDevice on_device_((c)->device); \
  HIP_TRY(on_device_.status())

bool capturing(calvo_ctx* c) {
  hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(c->s_compute, &s) != hipSuccess) { (void)hipGetLastError(); return false; }
  return s != hipStreamCaptureStatusNone;
}

// ---- descriptor buffers (step_bufs.h)
struct StepDev {
  calvo_ctx* c;
  int make(StepBuf& b) {
    HIP_TRY(hipMalloc((void**)&b.d, b.d_bytes));
    HIP_TRY(hipHostMalloc((void**)&b.h, b.h_bytes, hipHostMallocMapped | hipHostMallocCoherent));
    HIP_TRY(hipEventCreateWithFlags(&b.read, hipEventDisableTiming));
    return CALVO_OK;
  }
  // behind everything that was queued with it
  void free(StepBuf& b) {
    (void)hipStreamSynchronize(c->s_compute);
    if (b.d) (void)hipFree(b.d);
    if (b.h) (void)hipHostFree(b.h);
    if (b.read) (void)hipEventDestroy(b.read);
    (void)hipGetLastError();
    b = StepBuf();
  }
  bool was_read(StepBuf& b) {
    if (hipEventQuery(b.read) == hipSuccess) return true;
    (void)hipGetLastError();
    return false;
  }
  int wait(StepBuf& b) {
    HIP_TRY(hipEventSynchronize(b.read));
    return CALVO_OK;
  }
};

// After an error the caller frees what was made.
int take_buf(calvo_ctx* c, size_t d_bytes, size_t h_bytes, StepBuf& out) {
  StepDev dev{c};
  return c->step_bufs.take(dev, d_bytes, h_bytes, out);
}

void free_buf(calvo_ctx* c, StepBuf& b) {
  if (b.d || b.h || b.read) StepDev{c}.free(b);
}

void give_buf(calvo_ctx* c, StepBuf& b) {
  if (!b.d || !b.h || !b.read || !c->step_bufs.give(b)) free_buf(c, b);
}

int upload(calvo_ctx* c, StepBuf& b, size_t words) {
  if (words == 0) return CALVO_OK;
  HIP_TRY(launch_upload_words(b.h, b.d, words, c->s_compute));
  HIP_TRY(hipEventRecord(b.read, c->s_compute));
  b.pending = true;
  return CALVO_OK;
}

// Slots of a table get `mark`; one that has it already is refused.
int mark_table(const calvo_config& cf, SlotMarks& marks, const int32_t* table, int64_t n, uint32_t mark, const char* what, int r) {
  for (int64_t j = 0; j < n; j++) {
    const int32_t s = table[j];
    if (s < 0 || s >= cf.pool_blocks)
      return fail(CALVO_EINVAL, "request %d: slot %d at %s[%lld] is outside the pool (not allocated)", r, s, what, (long long)j);
    if (marks.of[s] == mark) return fail(CALVO_EINVAL, "request %d: slot %d appears twice in %s", r, s, what);
    marks.of[s] = mark;
  }
  return CALVO_OK;
}

// n marks that no slot carries; returns the first
uint32_t new_marks(const calvo_config& cf, SlotMarks& marks, uint32_t n) {
  if (marks.of.empty()) marks.of.assign((size_t)cf.pool_blocks, 0);
  if (marks.next > UINT32_MAX - n) {
    std::fill(marks.of.begin(), marks.of.end(), 0);
    marks.next = 1;
  }
  const uint32_t first = marks.next;
  marks.next += n;
  return first;
}

int64_t blocks_of(int64_t tokens) { return (tokens + kBlockTokens - 1) / kBlockTokens; }

struct Range {
  uintptr_t at;
  size_t bytes;
  const char* name;
};
int apart(const Range& a, const Range& b) {
  if (!a.at || !b.at || a.at >= b.at + b.bytes || b.at >= a.at + a.bytes) return CALVO_OK;
  return fail(CALVO_EINVAL, "%s overlaps %s", a.name, b.name);
}

float scale_of(const calvo_ctx* c, float scale) { return scale > 0.f ? scale : 1.0f / sqrtf((float)c->cfg.head_dim); }

constexpr int64_t kMostTokens = INT32_MAX - 65536;     // positions and their sums with tile sizes stay within 32 bits
constexpr int64_t kMostThreads = UINT32_MAX;           // of a launch

int check_window_requests(const calvo_config& cf, SlotMarks& marks, const calvo_window_request* reqs, int n_reqs, int32_t window, int32_t n_first,
                          int64_t* total) {
  if (window < 1) return fail(CALVO_EINVAL, "window must be positive");
  if (n_first < 0) return fail(CALVO_EINVAL, "n_first must not be negative");
  if (n_reqs < 0) return fail(CALVO_EINVAL, "n_reqs is negative");
  if (n_reqs > 0 && !reqs) return fail(CALVO_EINVAL, "reqs is NULL");
  *total = 0;
  int64_t blocks = 0;
  for (int r = 0; r < n_reqs; r++) {
    const calvo_window_request& q = reqs[r];
    if (q.n_cached < 0 || q.n_new < 0) return fail(CALVO_EINVAL, "request %d: negative token count", r);
    const int64_t tokens = (int64_t)q.n_cached + q.n_new;
    if (tokens > kMostTokens) return fail(CALVO_EINVAL, "request %d: context too long", r);
    if (blocks_of(tokens) > cf.pool_blocks)
      return fail(CALVO_ENOMEM, "request %d needs %lld slots, the pool has %lld", r, (long long)blocks_of(tokens), (long long)cf.pool_blocks);
    if (tokens > 0 && !q.block_table) return fail(CALVO_EINVAL, "request %d: block_table is NULL", r);
    if (q.reserved != 0) return fail(CALVO_EINVAL, "request %d: reserved must be 0", r);
    *total += q.n_new;
    blocks += blocks_of(tokens);
  }
  if (*total * (cf.n_q_heads / cf.n_kv_heads) > INT32_MAX - 4096) return fail(CALVO_EINVAL, "too many new tokens");
  if (blocks + (int64_t)n_reqs * (kTablePad + 2) > INT32_MAX) return fail(CALVO_EINVAL, "too many tokens in the batch");   // places in its tables are 32 bits wide
  // every table by itself, then the slots that new tokens go to: they are in no other table
  const uint32_t mark = new_marks(cf, marks, (uint32_t)n_reqs + 1), stored = mark + (uint32_t)n_reqs;
  for (int r = 0; r < n_reqs; r++) {
    const int rc = mark_table(cf, marks, reqs[r].block_table, blocks_of((int64_t)reqs[r].n_cached + reqs[r].n_new), mark + (uint32_t)r, "block_table", r);
    if (rc != CALVO_OK) return rc;
  }
  for (int pass = 0; pass < 2 && n_reqs > 1; pass++)
    for (int r = 0; r < n_reqs; r++) {
      const int64_t n_tab = blocks_of((int64_t)reqs[r].n_cached + reqs[r].n_new), own = reqs[r].n_new ? reqs[r].n_cached / kBlockTokens : n_tab;
      // first the blocks that take new tokens, then those that are only read
      for (int64_t j = pass ? 0 : own; j < (pass ? own : n_tab); j++) {
        uint32_t& m = marks.of[reqs[r].block_table[j]];
        if (m == stored) return fail(CALVO_EINVAL, "request %d: slot %d takes new tokens of another request", r, reqs[r].block_table[j]);
        if (!pass) m = stored;
      }
    }
  return CALVO_OK;
}

int check_evict_requests(const calvo_config& cf, SlotMarks& marks, const calvo_evict_request* reqs, int n_reqs, int32_t mass_rows) {
  if (n_reqs < 0 || n_reqs > 65535) return fail(CALVO_EINVAL, "n_reqs outside [0, 65535]");
  if (n_reqs > 0 && !reqs) return fail(CALVO_EINVAL, "reqs is NULL");
  if (mass_rows < 0) return fail(CALVO_EINVAL, "mass_rows must not be negative");
  std::vector<int32_t> used;
  int64_t words = 0;
  for (int r = 0; r < n_reqs; r++) {
    const calvo_evict_request& q = reqs[r];
    if (q.n_tokens < 0 || q.n_keep < 0 || q.n_first < 0 || q.n_last < 0) return fail(CALVO_EINVAL, "request %d: negative token count", r);
    if (q.n_tokens > kMostTokens) return fail(CALVO_EINVAL, "request %d: context too long", r);
    if (q.n_keep > q.n_tokens) return fail(CALVO_EINVAL, "request %d: keeps %d of %d tokens", r, q.n_keep, q.n_tokens);
    if ((int64_t)q.n_first + q.n_last > q.n_keep) return fail(CALVO_EINVAL, "request %d: n_first + n_last is more than n_keep", r);
    if (q.reserved != 0) return fail(CALVO_EINVAL, "request %d: reserved must be 0", r);
    if (q.n_keep == 0) continue;
    const int64_t slots = blocks_of(q.n_tokens) + blocks_of(q.n_keep);
    if (slots > cf.pool_blocks)
      return fail(CALVO_ENOMEM, "request %d needs %lld slots, the pool has %lld", r, (long long)slots, (long long)cf.pool_blocks);
    if (!q.src_table || !q.dst_table) return fail(CALVO_EINVAL, "request %d: a table is NULL", r);
    if (q.mass_row < 0 || q.mass_row >= mass_rows) return fail(CALVO_EINVAL, "request %d: mass_row %d outside [0, %d)", r, q.mass_row, mass_rows);
    used.push_back(q.mass_row);
    words += slots;
  }
  if (words > INT32_MAX) return fail(CALVO_EINVAL, "too many tokens in the call");
  std::sort(used.begin(), used.end());
  if (std::adjacent_find(used.begin(), used.end()) != used.end()) return fail(CALVO_EINVAL, "the requests' mass_row must differ");
  // sources: distinct inside a request.  Destinations: distinct over the call, and no request's source.
  const uint32_t mark = new_marks(cf, marks, (uint32_t)n_reqs + 1), dst = mark + (uint32_t)n_reqs;
  int rc;
  for (int r = 0; r < n_reqs; r++)
    if (reqs[r].n_keep && (rc = mark_table(cf, marks, reqs[r].src_table, blocks_of(reqs[r].n_tokens), mark + (uint32_t)r, "src_table", r)) != CALVO_OK) return rc;
  for (int r = 0; r < n_reqs; r++)
    if (reqs[r].n_keep && (rc = mark_table(cf, marks, reqs[r].dst_table, blocks_of(reqs[r].n_keep), dst, "dst_table", r)) != CALVO_OK) return rc;
  for (int r = 0; r < n_reqs; r++)
    for (int64_t j = 0; reqs[r].n_keep && j < blocks_of(reqs[r].n_tokens); j++)
      if (marks.of[reqs[r].src_table[j]] == dst) return fail(CALVO_EINVAL, "request %d: slot %d of src_table is in a dst_table", r, reqs[r].src_table[j]);
  return CALVO_OK;
}

// CALVO_ATTN_VARIANT, read for every plan: 3 or 4 as for the causal kernels, 5 the packed rows
int forced_variant() {
  const char* e = getenv("CALVO_ATTN_VARIANT");
  return e && e[0] >= '3' && e[0] <= '5' && e[1] == 0 ? e[0] - '0' : 0;
}

int window_prepare(calvo_ctx* c, const calvo_window_request* reqs, int n_reqs, int32_t window, int32_t n_first, calvo_window* w) {
  int64_t total = 0;
  int rc = check_window_requests(c->cfg, c->marks, reqs, n_reqs, window, n_first, &total);
  if (rc != CALVO_OK) return rc;
  const calvo_config& cf = c->cfg;
  w->c = c; w->n_reqs = n_reqs; w->total = (int)total; w->window = window; w->n_first = n_first;

  std::vector<WindowLens> lens((size_t)n_reqs);
  std::vector<int32_t> rows_used;
  int64_t table_words = 0;
  for (int r = 0; r < n_reqs; r++) {
    lens[r] = {reqs[r].n_cached, reqs[r].n_new};
    const int64_t tokens = (int64_t)reqs[r].n_cached + reqs[r].n_new;
    w->longest = std::max(w->longest, tokens);
    table_words += (tokens + kBlockTokens - 1) / kBlockTokens + 1;
    if (tokens > 0) rows_used.push_back(reqs[r].mass_row);
  }
  std::sort(rows_used.begin(), rows_used.end());
  w->mass_rows_differ = std::adjacent_find(rows_used.begin(), rows_used.end()) == rows_used.end() && (rows_used.empty() || rows_used.front() >= 0);
  w->max_mass_row = rows_used.empty() ? -1 : rows_used.back();

  plan_window({cf.dtype == CALVO_F32, cf.head_dim, cf.n_q_heads, cf.n_kv_heads, c->n_cus, c->force_splits, c->force_rows_tile, forced_variant(), cf.dtype == CALVO_E4M3}, lens,
              window, n_first, w->plan);
  const bool e4m3 = cf.dtype == CALVO_E4M3;
  const int tile_keys = attn_mass_tile_keys(cf.dtype, cf.head_dim);
  if (w->mass_rows_differ && !e4m3)                // else calvo_attn_mass refuses the plan (32 requests of 300 to 33000 tokens: 28 us with it, 21 without)
    plan_mass(cf.n_q_heads / cf.n_kv_heads, cf.n_kv_heads, c->n_cus, tile_keys, lens, window, n_first, w->mass);
  const size_t n_mass = w->mass.items.size();
  if ((int64_t)n_mass * cf.n_kv_heads * std::max(256, tile_keys) > kMostThreads) return fail(CALVO_EINVAL, "too many tokens in the batch");
  const bool rows = w->plan.variant == kWindowRows;
  const size_t n_items = w->plan.items.size();
  if ((int64_t)n_items * (rows ? cf.n_kv_heads : cf.n_q_heads / w->plan.heads_per_wg) * 512 > kMostThreads) return fail(CALVO_EINVAL, "too many new tokens");

  // ---- words: work items, first items of cut tiles, the same of the gathered weights, requests for the append, tables; pipelined kernels: the blocks'
  // offsets in a layer, even blocks first, padded as in the causal batches (kTablePad)
  constexpr size_t kItem = sizeof(WinItem) / 4, kMass = sizeof(MassItem) / 4, kAdd = sizeof(MassAdd) / 4, kApp = sizeof(ReqDesc) / 4;
  auto pad4 = [](size_t n) { return (n + 3) / 4 * 4; };
  w->items_at = 0;
  w->split_at = n_items * kItem;
  w->arrived_at = w->split_at + w->plan.split_tiles.size();
  const size_t n_arrived = w->plan.one_launch ? n_items * (size_t)cf.n_kv_heads : 0;
  w->mass_at = pad4(w->arrived_at + n_arrived);
  w->add_at = w->mass_at + n_mass * kMass;
  w->append_at = w->add_at + w->mass.adds.size() * kAdd;
  w->touched_at = pad4(w->append_at + (size_t)n_reqs * kApp);
  for (int r = 0; r < n_reqs && e4m3; r++)
    if (reqs[r].n_new) w->n_touched += (int)(blocks_of((int64_t)reqs[r].n_cached + reqs[r].n_new) - reqs[r].n_cached / kBlockTokens);
  w->tables_at = w->touched_at + (size_t)w->n_touched * (sizeof(TouchedBlock) / 4);
  w->offs_at = pad4(w->tables_at + (size_t)table_words);
  auto offs_of = [](int64_t n_tab) { return n_tab + kTablePad + (n_tab & 1); };
  size_t n_offs = 0;
  for (int r = 0; r < n_reqs && !rows; r++) n_offs += (size_t)offs_of(((int64_t)reqs[r].n_cached + reqs[r].n_new + kBlockTokens - 1) / kBlockTokens);
  const size_t words = pad4(w->offs_at + 2 * n_offs);
  const size_t pieces = (size_t)w->plan.n_parts * (size_t)w->plan.part_rows;
  w->part_o_at = (words + 63) / 64 * 64;
  w->part_ml_at = w->part_o_at + pieces * (size_t)w->plan.part_width;
  w->part_mass_at = w->part_ml_at + pieces * 2;
  const size_t floats = w->part_mass_at + (size_t)w->mass.n_parts * (size_t)cf.n_kv_heads * (size_t)tile_keys;
  if ((rc = take_buf(c, floats * 4, words * 4, w->buf)) != CALVO_OK) return rc;

  int32_t* h = w->buf.h;
  std::vector<int32_t> table_off((size_t)n_reqs), mass_table((size_t)n_reqs), q_off((size_t)n_reqs);
  int64_t* offs = (int64_t*)(h + w->offs_at);
  TouchedBlock* touched = (TouchedBlock*)(h + w->touched_at);
  size_t at = 0, offs_at = 0;
  int32_t q = 0;
  for (int r = 0; r < n_reqs; r++) {
    const int64_t tokens = (int64_t)reqs[r].n_cached + reqs[r].n_new;
    const size_t n_tab = (size_t)((tokens + kBlockTokens - 1) / kBlockTokens);
    table_off[r] = (int32_t)(rows ? at : offs_at);
    mass_table[r] = (int32_t)at;
    q_off[r] = q;
    if (!rows && n_tab) {
      const size_t n = (size_t)offs_of((int64_t)n_tab);
      for (size_t b = 0; b < n; b++)
        offs[offs_at + (b & 1) * (n / 2) + b / 2] = (int64_t)reqs[r].block_table[std::min(b, n_tab - 1)] * (int64_t)c->blk_bytes;
      offs_at += n;
    }
    if (n_tab) memcpy(h + w->tables_at + at, reqs[r].block_table, n_tab * 4);
    h[w->tables_at + at + n_tab] = n_tab ? reqs[r].block_table[n_tab - 1] : 0;
    const ReqDesc a = {(int32_t)at, reqs[r].n_cached, reqs[r].n_new, q};
    memcpy(h + w->append_at + (size_t)r * kApp, &a, sizeof a);
    for (size_t b = (size_t)reqs[r].n_cached / kBlockTokens; e4m3 && reqs[r].n_new && b < n_tab; b++) {
      const int32_t from = std::max(reqs[r].n_cached, (int32_t)b * kBlockTokens), to = (int32_t)std::min<int64_t>(tokens, (int64_t)(b + 1) * kBlockTokens);
      const int32_t first = (int32_t)b * kBlockTokens;
      *touched++ = {reqs[r].block_table[b], q + from - reqs[r].n_cached, from, (from - first) | (to - first) << 8};
    }
    at += n_tab + 1;
    q += reqs[r].n_new;
  }
  for (size_t i = 0; i < n_items; i++) {
    const WindowPiece& x = w->plan.items[i];
    const WinItem d = {x.tile, x.sub_begin, x.sub_end, x.n_splits, x.first_item, table_off[x.req], reqs[x.req].n_cached, reqs[x.req].n_new,
                       q_off[x.req], x.keys.first_subs, x.keys.gap, x.keys.n_full, x.keys.n_part, x.keys.edge, x.keys.n_edge, x.keys.diag};
    memcpy(h + i * kItem, &d, sizeof d);
  }
  for (size_t i = 0; i < n_mass; i++) {
    const MassPiece& x = w->mass.items[i];
    const MassItem d = {mass_table[x.req], reqs[x.req].n_cached, reqs[x.req].n_new, q_off[x.req], reqs[x.req].mass_row, x.tile, x.begin, x.end, x.part, {0, 0, 0}};
    memcpy(h + w->mass_at + i * kMass, &d, sizeof d);
  }
  for (size_t i = 0; i < w->mass.adds.size(); i++) {
    const MassTile& x = w->mass.adds[i];
    const MassAdd d = {reqs[x.req].n_cached, reqs[x.req].n_cached + reqs[x.req].n_new, reqs[x.req].mass_row, x.tile, x.part, x.n_parts, {0, 0}};
    memcpy(h + w->add_at + i * kAdd, &d, sizeof d);
  }
  std::fill_n(h + w->arrived_at, n_arrived, 0);
  if (!w->plan.split_tiles.empty()) memcpy(h + w->split_at, w->plan.split_tiles.data(), w->plan.split_tiles.size() * 4);
  return upload(c, w->buf, words);
}

int check_layer(const calvo_ctx* c, int layer) {
  if (layer < 0 || layer >= c->cfg.n_layers) return fail(CALVO_EINVAL, "layer %d outside [0, %d)", layer, c->cfg.n_layers);
  return CALVO_OK;
}

// The append's launch: q, k, v, their rows and the rotation are in p
int queue_append(calvo_window* w, KvAppendParams& p, unsigned char* pool_layer) {
  calvo_ctx* c = w->c;
  const calvo_config& cf = c->cfg;
  const int32_t* d = w->buf.d;
  if (((int64_t)w->n_touched * ((cf.n_kv_heads + 1) / 2) + w->total) * 256 > kMostThreads) return fail(CALVO_EINVAL, "too many new tokens");
  p.pool_layer = pool_layer;
  p.reqs = (const ReqDesc*)(d + w->append_at); p.touched = (const TouchedBlock*)(d + w->touched_at); p.tables = d + w->tables_at;
  p.n_reqs = w->n_reqs; p.total_tokens = w->total; p.n_touched = w->n_touched;
  p.n_q_heads = cf.n_q_heads; p.n_kv_heads = cf.n_kv_heads; p.head_dim = cf.head_dim;
  HIP_TRY(launch_kv_append(p, cf.dtype, c->n_cus, c->s_compute));
  return CALVO_OK;
}

int kv_append(calvo_window* w, int layer, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
              void* q_out, const calvo_rope* rope) {
  calvo_ctx* c = w->c;
  const calvo_config& cf = c->cfg;
  int rc = check_layer(c, layer);
  if (rc != CALVO_OK) return rc;
  unsigned char* pool_layer = (unsigned char*)cf.pool + (int64_t)layer * c->layer_bytes;
  KvAppendParams p{};
  if (rope) {
    if (rope->reserved != 0) return fail(CALVO_EINVAL, "rope: reserved must be 0");
    if (rope->rot_dim < 2 || rope->rot_dim > cf.head_dim || rope->rot_dim % 2) return fail(CALVO_EINVAL, "rope: rot_dim must be even and in [2, head_dim]");
    if (rope->interleaved != 0 && rope->interleaved != 1) return fail(CALVO_EINVAL, "rope: interleaved must be 0 or 1");
    if (w->total > 0 && !rope->inv_freq) return fail(CALVO_EINVAL, "rope: inv_freq is NULL");
    if ((((uintptr_t)rope->inv_freq | (uintptr_t)rope->positions) & 3) != 0) return fail(CALVO_EINVAL, "rope: inv_freq and positions must be 4-byte aligned");
    p.rope = {rope->inv_freq, rope->positions, rope->rot_dim, rope->rot_dim / 2, rope->interleaved};
  }
  if ((k_new == nullptr) != (v_new == nullptr)) return fail(CALVO_EINVAL, "k_new and v_new must both be given or both be NULL");
  if ((q == nullptr) != (q_out == nullptr)) return fail(CALVO_EINVAL, "q and q_out must both be given or both be NULL");
  if ((((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k_new | (uintptr_t)v_new) & 15) != 0)
    return fail(CALVO_EINVAL, "q, q_out, k_new and v_new must be 16-byte aligned");
  const int64_t kv_row = (int64_t)cf.n_kv_heads * cf.head_dim, q_row = (int64_t)cf.n_q_heads * cf.head_dim, unit = 16 / (int64_t)c->elt;
  struct { const void* at; int64_t given, row; int64_t* bytes; const char* name; } in[] = {
      {k_new, k_stride, kv_row, &p.k_row, "k_new"}, {v_new, v_stride, kv_row, &p.v_row, "v_new"}, {q, q_stride, q_row, &p.q_row, "q"}};
  for (const auto& x : in) {
    if (!x.at) continue;
    const int64_t s = x.given ? x.given : x.row;
    if (s < x.row || s % unit != 0 || s > ((int64_t)1 << 40))
      return fail(CALVO_EINVAL, "the stride of %s must be 0 or a multiple of %d from %lld on", x.name, (int)unit, (long long)x.row);
    *x.bytes = s * (int64_t)c->elt;
  }
  p.q = q; p.k = k_new; p.v = v_new; p.q_out = q_out;
  if (w->total > 0) {
    auto extent = [&](const void* at, int64_t row_bytes, int64_t row, const char* name) {
      return Range{(uintptr_t)at, (size_t)((w->total - 1) * row_bytes + row * (int64_t)c->elt), name};
    };
    const Range to[] = {{(uintptr_t)q_out, (size_t)(w->total * q_row) * c->elt, "q_out"}, {(uintptr_t)pool_layer, (size_t)c->layer_bytes, "the pool"}};
    const Range from[] = {extent(k_new, p.k_row, kv_row, "k_new"), extent(v_new, p.v_row, kv_row, "v_new"), extent(q, p.q_row, q_row, "q"),
                          {(uintptr_t)p.rope.inv_freq, (size_t)p.rope.half * 4, "rope: inv_freq"},
                          {(uintptr_t)p.rope.positions, (size_t)w->total * 4, "rope: positions"}};
    if ((rc = apart(to[0], to[1])) != CALVO_OK) return rc;
    for (const Range& a : to)
      for (const Range& b : from)
        if ((rc = apart(a, b)) != CALVO_OK) return rc;
  }
  ON_DEVICE(c);
  if ((rc = queue_behind_layer(c, layer)) != CALVO_OK) return rc;
  return w->total > 0 ? queue_append(w, p, pool_layer) : CALVO_OK;
}

int window_attn(calvo_window* w, int layer, const void* q, const void* k_new, const void* v_new, void* out, float* lse, float scale) {
  calvo_ctx* c = w->c;
  const calvo_config& cf = c->cfg;
  int rc = check_layer(c, layer);
  if (rc != CALVO_OK) return rc;
  unsigned char* pool_layer = (unsigned char*)cf.pool + (int64_t)layer * c->layer_bytes;
  if (w->total > 0) {
    if (!q || !out) return fail(CALVO_EINVAL, "q or out is NULL");
    if ((k_new == nullptr) != (v_new == nullptr)) return fail(CALVO_EINVAL, "k_new and v_new must both be given or both be NULL");
    if ((((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_new | (uintptr_t)v_new) & 15) != 0)
      return fail(CALVO_EINVAL, "q, k_new, v_new and out must be 16-byte aligned");
    if (((uintptr_t)lse & 3) != 0) return fail(CALVO_EINVAL, "lse must be 4-byte aligned");
    const size_t row = (size_t)w->total * cf.head_dim * c->elt;
    const Range to[] = {{(uintptr_t)out, row * cf.n_q_heads, "out"}, {(uintptr_t)lse, (size_t)w->total * cf.n_q_heads * 4, "lse"},
                        {(uintptr_t)pool_layer, (size_t)c->layer_bytes, "the pool"}};
    const Range from[] = {{(uintptr_t)q, row * cf.n_q_heads, "q"}, {(uintptr_t)k_new, row * cf.n_kv_heads, "k_new"},
                          {(uintptr_t)v_new, row * cf.n_kv_heads, "v_new"}};
    for (const Range& a : to) {
      for (const Range& b : from)
        if ((rc = apart(a, b)) != CALVO_OK) return rc;
      for (const Range& b : to)
        if (&a < &b && (rc = apart(a, b)) != CALVO_OK) return rc;
    }
  }
  ON_DEVICE(c);
  if ((rc = queue_behind_layer(c, layer)) != CALVO_OK) return rc;
  if (w->total == 0) return CALVO_OK;
  const int32_t* d = w->buf.d;
  // The attention launch stores the new rows itself where every request is one tile of packed rows (decoding) and a head's row is whole cache
  // lines: one launch less.
  const bool e4m3 = cf.dtype == CALVO_E4M3;
  if (k_new && e4m3) {
    KvAppendParams app{};
    app.k = k_new; app.v = v_new;
    app.k_row = app.v_row = (int64_t)cf.n_kv_heads * cf.head_dim * (int64_t)c->elt;
    if ((rc = queue_append(w, app, pool_layer)) != CALVO_OK) return rc;
  }
  const bool along = !e4m3 && k_new && w->plan.single_tiles && (size_t)cf.head_dim * c->elt % 128 == 0;
  if (k_new && !along && !e4m3) {
    AppendParams app{};
    app.k_suffix = k_new; app.v_suffix = v_new; app.pool_layer = pool_layer;
    app.reqs = (const ReqDesc*)(d + w->append_at); app.tables = d + w->tables_at;
    app.n_reqs = w->n_reqs; app.total_tokens = w->total;
    app.row_chunks = (int32_t)((size_t)cf.n_kv_heads * cf.head_dim * c->elt / 16);
    HIP_TRY(launch_suffix_append(app, c->s_compute));
  }
  WinParams p{};
  p.q = q; p.out = out; p.lse = lse; p.pool_layer = pool_layer;
  if (along) { p.k_new = k_new; p.v_new = v_new; }
  p.items = (const WinItem*)(d + w->items_at); p.tables = d + w->tables_at;
  p.blk_offs = (const int64_t*)(d + w->offs_at);
  p.n_q_heads = cf.n_q_heads; p.n_kv_heads = cf.n_kv_heads; p.head_dim = cf.head_dim;
  p.group = (uint32_t)(cf.n_q_heads / cf.n_kv_heads);
  p.window = w->window; p.n_first = w->n_first;
  p.scale = scale_of(c, scale);
  p.part_o = (float*)d + w->part_o_at; p.part_ml = (float*)d + w->part_ml_at;
  const int n_items = (int)w->plan.items.size(), n_cut = (int)w->plan.split_tiles.size();
  if (w->plan.variant == kWindowRows) {
    if (w->plan.one_launch) p.arrived = w->buf.d + w->arrived_at;
    if (e4m3) HIP_TRY(launch_attn_e4m3(p, w->plan.tile_rows, n_items, d + w->split_at, p.arrived ? 0 : n_cut, c->s_compute));
    else HIP_TRY(launch_attn_window(p, cf.dtype, w->plan.tile_rows, n_items, d + w->split_at, p.arrived ? 0 : n_cut, c->s_compute));
  } else {
    p.heads_per_wg = w->plan.heads_per_wg;
    p.row_blocks_per_wg = attn_mfma_row_blocks(w->plan.variant);
    if (e4m3) HIP_TRY(launch_attn_e4m3_pipe(p, w->plan.variant, n_items, d + w->split_at, n_cut, c->s_compute));
    else HIP_TRY(launch_attn_window_pipe(p, w->plan.variant, n_items, d + w->split_at, n_cut, c->s_compute));
  }
  return CALVO_OK;
}

int attn_mass(calvo_window* w, int layer, const void* q, const float* lse, const float* mass_in, float* mass_out, int32_t mass_rows,
              int64_t mass_stride, int32_t last_rows, float scale) {
  calvo_ctx* c = w->c;
  const calvo_config& cf = c->cfg;
  int rc = check_layer(c, layer);
  if (rc != CALVO_OK) return rc;
  if ((rc = not_for_e4m3(cf, "calvo_attn_mass")) != CALVO_OK) return rc;
  if (cf.n_q_heads / cf.n_kv_heads > 4096) return fail(CALVO_EINVAL, "more than 4096 query heads to a KV head");
  if (mass_rows < 0 || last_rows < 0) return fail(CALVO_EINVAL, "mass_rows and last_rows must not be negative");
  if (w->longest > 0) {
    if (!mass_out) return fail(CALVO_EINVAL, "mass_out is NULL");
    if (w->total > 0 && (!q || !lse)) return fail(CALVO_EINVAL, "q or lse is NULL");
    if (((uintptr_t)q & 15) != 0) return fail(CALVO_EINVAL, "q must be 16-byte aligned");
    if ((((uintptr_t)lse | (uintptr_t)mass_in | (uintptr_t)mass_out) & 3) != 0) return fail(CALVO_EINVAL, "lse and the weights must be 4-byte aligned");
    if (mass_stride < w->longest) return fail(CALVO_EINVAL, "mass_stride %lld is smaller than a request's %lld tokens", (long long)mass_stride, (long long)w->longest);
    if (mass_stride > ((int64_t)1 << 40)) return fail(CALVO_EINVAL, "mass_stride out of range");
    if (!w->mass_rows_differ) return fail(CALVO_EINVAL, "the requests' mass_row must differ and not be negative");
    if (w->max_mass_row >= mass_rows) return fail(CALVO_EINVAL, "mass_row %d outside [0, %d)", w->max_mass_row, mass_rows);
    const size_t bytes = (size_t)mass_rows * cf.n_kv_heads * (size_t)mass_stride * 4;
    const Range to = {(uintptr_t)mass_out, bytes, "mass_out"};
    const Range from[] = {{(uintptr_t)q, (size_t)w->total * cf.n_q_heads * cf.head_dim * c->elt, "q"}, {(uintptr_t)lse, (size_t)w->total * cf.n_q_heads * 4, "lse"},
                          {(uintptr_t)cf.pool, (size_t)c->layer_bytes * cf.n_layers, "the pool"}};
    for (const Range& b : from)
      if ((rc = apart(to, b)) != CALVO_OK) return rc;
    if (mass_in != mass_out && (rc = apart(to, {(uintptr_t)mass_in, bytes, "mass_in"})) != CALVO_OK) return rc;
  }
  ON_DEVICE(c);
  if ((rc = queue_behind_layer(c, layer)) != CALVO_OK) return rc;
  MassParams p{};
  p.q = q; p.lse = lse; p.mass_in = mass_in; p.mass_out = mass_out;
  p.pool_layer = (const unsigned char*)cf.pool + (int64_t)layer * c->layer_bytes;
  p.items = (const MassItem*)(w->buf.d + w->mass_at); p.tables = w->buf.d + w->tables_at;
  p.part = (float*)w->buf.d + w->part_mass_at;
  p.mass_stride = mass_stride; p.n_items = (int32_t)w->mass.items.size();
  p.n_q_heads = cf.n_q_heads; p.n_kv_heads = cf.n_kv_heads; p.head_dim = cf.head_dim;
  p.group = (uint32_t)(cf.n_q_heads / cf.n_kv_heads);
  p.window = w->window; p.n_first = w->n_first; p.last_rows = last_rows;
  p.scale = scale_of(c, scale);
  HIP_TRY(launch_attn_mass(p, cf.dtype, (const MassAdd*)(w->buf.d + w->add_at), (int)w->mass.adds.size(), c->s_compute));
  return CALVO_OK;
}

int kv_evict(calvo_ctx* c, const calvo_evict_request* reqs, int n_reqs, int layer_begin, int layer_end, const float* mass, int32_t mass_rows,
             int64_t mass_stride, int32_t* kept, int64_t kept_stride, float* mass_out, int64_t out_stride) {
  const calvo_config& cf = c->cfg;
  if (layer_begin < 0 || layer_end > cf.n_layers || layer_begin > layer_end)
    return fail(CALVO_EINVAL, "layers [%d, %d) outside [0, %d)", layer_begin, layer_end, cf.n_layers);
  int rc = not_for_e4m3(cf, "calvo_kv_evict");
  if (rc != CALVO_OK) return rc;
  const int n_layers = layer_end - layer_begin;
  if (n_layers > 65535) return fail(CALVO_EINVAL, "more than 65535 layers");
  if ((rc = check_evict_requests(cf, c->marks, reqs, n_reqs, mass_rows)) != CALVO_OK) return rc;
  int64_t table_words = 0, longest = 0;
  int32_t max_keep = 0;
  for (int r = 0; r < n_reqs; r++) {
    if (reqs[r].n_keep == 0) continue;
    table_words += blocks_of(reqs[r].n_tokens) + blocks_of(reqs[r].n_keep);
    max_keep = std::max(max_keep, reqs[r].n_keep);
    longest = std::max<int64_t>(longest, reqs[r].n_tokens);
  }
  if (max_keep > 0 && n_layers > 0) {
    if (!mass || !kept) return fail(CALVO_EINVAL, "mass or kept is NULL");
    if ((((uintptr_t)mass | (uintptr_t)mass_out | (uintptr_t)kept) & 3) != 0) return fail(CALVO_EINVAL, "mass, mass_out and kept must be 4-byte aligned");
    if (mass_stride < longest) return fail(CALVO_EINVAL, "mass_stride is smaller than a request's %lld tokens", (long long)longest);
    if (kept_stride < max_keep) return fail(CALVO_EINVAL, "kept_stride is smaller than a request's %d kept tokens", max_keep);
    if (mass_out && out_stride < max_keep) return fail(CALVO_EINVAL, "out_stride is smaller than a request's %d kept tokens", max_keep);
    if (std::max(mass_stride, std::max(kept_stride, mass_out ? out_stride : 0)) > ((int64_t)1 << 40)) return fail(CALVO_EINVAL, "a stride is out of range");
    const size_t heads = (size_t)n_layers * cf.n_kv_heads * 4;
    const Range x[] = {{(uintptr_t)mass, heads * (size_t)mass_rows * (size_t)mass_stride, "mass"}, {(uintptr_t)kept, heads * (size_t)n_reqs * (size_t)kept_stride, "kept"},
                       {(uintptr_t)mass_out, heads * (size_t)mass_rows * (size_t)out_stride, "mass_out"},
                       {(uintptr_t)cf.pool, (size_t)c->layer_bytes * cf.n_layers, "the pool"}};
    for (const Range& a : x)
      for (const Range& b : x)
        if (&a < &b && (rc = apart(a, b)) != CALVO_OK) return rc;
    if ((int64_t)n_layers * n_reqs * cf.n_kv_heads * 1024 > kMostThreads || blocks_of(max_keep) * 256 > kMostThreads)
      return fail(CALVO_EINVAL, "too many requests, layers or kept tokens in a call");
  }
  ON_DEVICE(c);
  if (capturing(c)) return fail(CALVO_EINVAL, "calvo_kv_evict cannot be captured: its tables are read from the host");
  for (int l = layer_begin; l < layer_end; l++)
    if ((rc = queue_behind_layer(c, l)) != CALVO_OK) return rc;
  if (max_keep == 0 || n_layers == 0) return CALVO_OK;

  constexpr size_t kReq = sizeof(EvictDesc) / 4;
  const size_t words = ((size_t)n_reqs * kReq + (size_t)table_words + 3) / 4 * 4;
  const bool in_args = words <= (size_t)kEvictArgWords;
  int32_t args[kEvictArgWords];
  StepBuf buf;
  if (!in_args && (rc = take_buf(c, words * 4, words * 4, buf)) != CALVO_OK) { free_buf(c, buf); return rc; }
  int32_t* const h = in_args ? args : buf.h;
  int32_t at = 0;
  int32_t* tables = h + (size_t)n_reqs * kReq;
  for (int r = 0; r < n_reqs; r++) {
    const calvo_evict_request& q = reqs[r];
    const int32_t ns = q.n_keep ? (int32_t)blocks_of(q.n_tokens) : 0, nd = (int32_t)blocks_of(q.n_keep);
    const EvictDesc d = {at, at + ns, q.n_keep ? q.n_tokens : 0, q.n_keep, q.n_first, q.n_last, q.n_keep ? q.mass_row : 0, 0};
    memcpy(h + (size_t)r * kReq, &d, sizeof d);
    if (ns) memcpy(tables + at, q.src_table, (size_t)ns * 4);
    if (nd) memcpy(tables + at + ns, q.dst_table, (size_t)nd * 4);
    at += ns + nd;
  }
  const int n_words = (int)((size_t)n_reqs * kReq) + at;
  if (!in_args && (rc = upload(c, buf, words)) != CALVO_OK) { free_buf(c, buf); return rc; }   // it may be under way, without an event behind it
  EvictParams p{};
  p.pool = (unsigned char*)cf.pool + (int64_t)layer_begin * c->layer_bytes;
  p.reqs = (const EvictDesc*)buf.d; p.tables = in_args ? nullptr : buf.d + (size_t)n_reqs * kReq;
  p.mass = mass; p.mass_out = mass_out; p.kept = kept;
  p.layer_bytes = c->layer_bytes;
  p.mass_stride = mass_stride; p.mass_layer = (int64_t)mass_rows * cf.n_kv_heads * mass_stride;
  p.out_stride = out_stride; p.out_layer = (int64_t)mass_rows * cf.n_kv_heads * out_stride;
  p.kept_stride = kept_stride;
  p.n_reqs = n_reqs; p.n_layers = n_layers; p.n_kv_heads = cf.n_kv_heads;
  p.row_chunks = (int32_t)((size_t)cf.head_dim * c->elt / 16);
  p.max_tokens = (int32_t)longest;
  p.max_keep = max_keep;
  hipError_t e = launch_evict_select(p, in_args ? args : nullptr, n_words, c->s_compute);
  if (e == hipSuccess) e = launch_evict_move(p, in_args ? args : nullptr, n_words, c->s_compute);
  if (e != hipSuccess) rc = fail_hip(e, "launch of calvo_kv_evict");
  if (!in_args) give_buf(c, buf);
  return rc;
}

}  // namespace

extern "C" {

int calvo_window_prepare(calvo_ctx* c, const calvo_window_request* reqs, int n_reqs, int32_t window, int32_t n_first, calvo_window** out) {
  if (!out) return fail(CALVO_EINVAL, "out is NULL");
  *out = nullptr;
  if (!c) return fail(CALVO_EINVAL, "ctx is NULL");
  calvo_window* w = new (std::nothrow) calvo_window();
  if (!w) return fail(CALVO_ENOMEM, "out of host memory");
  int rc = CALVO_OK;
  try {
    const OnDevice dev(c->device);
    if (dev.status() != hipSuccess) rc = fail_hip(dev.status(), "hipSetDevice");
    else if (capturing(c)) rc = fail(CALVO_EINVAL, "calvo_window_prepare cannot be captured: its tables are read from the host");
    else if ((rc = window_kernels_ready(c)) == CALVO_OK) rc = window_prepare(c, reqs, n_reqs, window, n_first, w);
    if (rc != CALVO_OK) free_buf(c, w->buf);
  } catch (const std::bad_alloc&) {
    free_buf(c, w->buf);
    rc = fail(CALVO_ENOMEM, "out of host memory");
  }
  if (rc != CALVO_OK) { delete w; return rc; }
  *out = w;
  return CALVO_OK;
}

int calvo_window_destroy(calvo_window* w) {
  if (!w) return fail(CALVO_EINVAL, "window is NULL");
  {
    const OnDevice dev(w->c->device);
    give_buf(w->c, w->buf);
  }
  delete w;
  return CALVO_OK;
}

int calvo_window_plan(const calvo_config* cfg, int32_t n_cus, const calvo_window_request* reqs, int32_t n_reqs, int32_t window, int32_t n_first,
                      int32_t* kernel, int32_t* entries, int32_t capacity, int32_t* n_entries) {
  if (!cfg || n_cus <= 0 || capacity < 0 || (capacity > 0 && !entries) || !n_entries) return fail(CALVO_EINVAL, "bad argument");
  calvo_config cf = *cfg;
  cf.pool = (void*)16;                         // not looked at
  int rc = validate_config(&cf);
  if (rc != CALVO_OK) return rc;
  try {
    SlotMarks marks;
    int64_t total = 0;
    if ((rc = check_window_requests(cf, marks, reqs, n_reqs, window, n_first, &total)) != CALVO_OK) return rc;
    std::vector<WindowLens> lens((size_t)n_reqs);
    for (int r = 0; r < n_reqs; r++) lens[r] = {reqs[r].n_cached, reqs[r].n_new};
    WindowPlan plan;
    plan_window({cf.dtype == CALVO_F32, cf.head_dim, cf.n_q_heads, cf.n_kv_heads, n_cus, 0, 0, forced_variant(), cf.dtype == CALVO_E4M3}, lens, window, n_first, plan);
    if (kernel) *kernel = plan.variant;
    int32_t n = 0;
    const int group = cf.n_q_heads / cf.n_kv_heads, unit = cf.dtype == CALVO_E4M3 && plan.variant == kWindowRows ? kE4m3Keys / 32 : 1;
    for (const WindowPiece& x : plan.items) {
      const int64_t rows = (int64_t)lens[(size_t)x.req].n_new * group, tr = plan.variant == kWindowRows ? plan.tile_rows : (int64_t)plan.tile_tokens * group;
      // runs of the item's part of the list: where each begins in the list, how many, where in the context
      const WindowKeys& k = x.keys;
      const bool listed = plan.variant != kWindowRows;
      const int32_t runs[5][3] = {{0, k.first_subs, 0},
                                  {k.first_subs, listed ? k.n_full - k.first_subs : k.n - k.first_subs, k.first_subs + k.gap},
                                  {k.n_full, listed ? k.n_part : 0, n_first / 32},
                                  {k.n_full + k.n_part, listed ? k.n_edge : 0, k.edge},
                                  {k.n_full + k.n_part + k.n_edge, listed ? k.n - k.n_full - k.n_part - k.n_edge : 0, k.diag}};
      for (int i = 0; i < 5; i++) {
        const int32_t b = std::max(x.sub_begin, runs[i][0]), e = std::min(x.sub_end, runs[i][0] + runs[i][1]);
        if (b >= e) continue;
        if (n < capacity) {
          int32_t* o = entries + 7 * (int64_t)n;
          o[0] = x.req; o[1] = (int32_t)(x.tile * tr); o[2] = (int32_t)std::min((x.tile + 1) * tr, rows);
          o[3] = unit * (b - runs[i][0] + runs[i][2]); o[4] = unit * (e - runs[i][0] + runs[i][2]);
          o[5] = listed && i < 2; o[6] = x.n_splits;
        }
        n++;
      }
    }
    *n_entries = n;
    return n > capacity ? CALVO_ENOMEM : CALVO_OK;
  } catch (const std::bad_alloc&) {
    return fail(CALVO_ENOMEM, "out of host memory");
  }
}

int calvo_evict_check(const calvo_config* cfg, const calvo_evict_request* reqs, int32_t n_reqs, int32_t mass_rows) {
  if (!cfg) return fail(CALVO_EINVAL, "config is NULL");
  calvo_config cf = *cfg;
  cf.pool = (void*)16;
  int rc = validate_config(&cf);
  if (rc == CALVO_OK) rc = not_for_e4m3(cf, "calvo_kv_evict");
  if (rc != CALVO_OK) return rc;
  try {
    SlotMarks marks;
    return check_evict_requests(cf, marks, reqs, n_reqs, mass_rows);
  } catch (const std::bad_alloc&) {
    return fail(CALVO_ENOMEM, "out of host memory");
  }
}

int calvo_window_attn(calvo_window* w, int layer, const void* q, const void* k_new, const void* v_new, void* out, float* lse, float scale) {
  if (!w) return fail(CALVO_EINVAL, "window is NULL");
  return window_attn(w, layer, q, k_new, v_new, out, lse, scale);
}

int calvo_kv_append(calvo_window* w, int layer, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride, const void* q, int64_t q_stride,
                    void* q_out, const calvo_rope* rope) {
  if (!w) return fail(CALVO_EINVAL, "window is NULL");
  return kv_append(w, layer, k_new, k_stride, v_new, v_stride, q, q_stride, q_out, rope);
}

int calvo_attn_mass(calvo_window* w, int layer, const void* q, const float* lse, const float* mass_in, float* mass_out, int32_t mass_rows,
                    int64_t mass_stride, int32_t last_rows, float scale) {
  if (!w) return fail(CALVO_EINVAL, "window is NULL");
  return attn_mass(w, layer, q, lse, mass_in, mass_out, mass_rows, mass_stride, last_rows, scale);
}

int calvo_kv_evict(calvo_ctx* c, const calvo_evict_request* reqs, int n_reqs, int layer_begin, int layer_end, const float* mass, int32_t mass_rows,
                   int64_t mass_stride, int32_t* kept, int64_t kept_stride, float* mass_out, int64_t out_stride) {
  if (!c) return fail(CALVO_EINVAL, "ctx is NULL");
  try {
    return kv_evict(c, reqs, n_reqs, layer_begin, layer_end, mass, mass_rows, mass_stride, kept, kept_stride, mass_out, out_stride);
  } catch (const std::bad_alloc&) {
    return fail(CALVO_ENOMEM, "out of host memory");
  }
}

}  // extern "C"
