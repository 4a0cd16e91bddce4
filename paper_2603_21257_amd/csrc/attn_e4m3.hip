// Attention over a pool of 8-bit floats with a scale for each block and head (calvo_window_attn on CALVO_E4M3 pools), packed rows: any head width, any
// group size, single tokens to chunks.
//
// out = sum_t exp(s_t - m) V_t / sum_t exp(s_t - m) in one pass with the running maximum m and sum of a row; a tile's rows are the (token, query head) pairs of
// a KV head, 16 or 32 of them.  Both products take bf16 operands: K and V are widened in registers with their scale, which is exact, and weights are rounded
// once to bf16: outputs are 1.64e-3 to 1.76e-3 (2-norm, relative) off 64 bits, of which 1.6e-3 is their own rounding, and the three terms to a weight that the
// packed rows over bf16 pools take would be three products instead of one.  (Products of 8 bits would round q and the weights to four bits.)  A wave takes
// every fourth step of 64 keys of the tile by itself: K and V go from the pool straight to the registers of the lanes whose operands they are, no LDS and no
// barrier until the waves add their rows at the end.
//
// Single tokens are bound by the bytes: 32 requests of 300 to 33000 tokens, 32Q/8KV, D = 128, 477 MB a layer in 90 us, 5.3 TB/s; short contexts by a chain of
// waits (descriptor, table, K, V, the waves' sum, the merge): 4096+1 tokens 7.2 us.  Many rows by the vector ALU, which widens K and V for 32 rows only:
// 16384+2048 tokens with D = 64 387 us, 755 TFLOP/s; 8192+1024 with D = 256 389 us, 752 TFLOP/s (16 rows: 662 us).  128-wide heads with many rows run on
// attn_e4m3_pipe.hip.  Long contexts of few rows are cut into pieces (window_plan.cpp).
#include "attn_rows_body.h"
#include "kv_e4m3.h"

namespace calvo {
namespace e4m3 {

using rows::store_through;

// DP: head_dim rounded up to 64, 128 or 256.  QB: 16-row blocks of a tile.  NW: waves.  FULL: head_dim == DP.
template <int DP_, int QB_, int NW_, bool FULL_>
struct Cfg {
  static constexpr int DP = DP_, QB = QB_, NW = NW_;
  static constexpr bool FULL = FULL_;
  static constexpr int KJ = DP / 64;                           // 16-byte chunks of a key that a lane reads
  static constexpr int DB = DP / 16;                           // blocks of 16 d
  static constexpr int ROWS = 16 * QB;
  static constexpr int UNITS = QB * DB;
  // Steps whose K and V are on their way.  Two where two waves to a SIMD leave registers for it and a wave has many steps (us a call of one caller, one / two:
  // D = 64, 32Q/8KV 16384+2048 tokens 415 / 391, 8192+512 57.3 / 55.0); not for single tokens, whose waves have one to three (4096+1 behind 1024 7.6 / 8.1)
  static constexpr int AHEAD = QB_ == 2 && DP_ == 64 ? 2 : 1;
  static constexpr int LDS_O = NW * UNITS * 64 * 16;           // all waves' accumulators
  static constexpr int LDS_BYTES = LDS_O + NW * ROWS * 8;
};

// Two waves to a SIMD; wider heads have its 512 registers to themselves
template <class C>
__global__ void __launch_bounds__(64 * C::NW, C::DP > 128 ? 1 : 2) attn_e4m3_kernel(WinParams p) {
  constexpr int DP = C::DP, QB = C::QB, NW = C::NW, KJ = C::KJ, DB = C::DB;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int Hkv = p.n_kv_heads, Hq = p.n_q_heads, D = C::FULL ? DP : p.head_dim;
  const unsigned G = p.group;
  constexpr unsigned RT = C::ROWS;

  // ---- work item; a KV head's workgroups stay on one XCD where the heads divide over the eight
  int it, kv;
  {
    const int bid = blockIdx.x;
    if ((Hkv & 7) == 0) {
      const int per = Hkv >> 3, rest = bid >> 3;
      kv = (bid & 7) * per + rest % per;
      it = rest / per;
    } else {
      kv = bid % Hkv;
      it = bid / Hkv;
    }
  }
  const WinItem wi = load_win_item(p.items, it);
  const int n_splits = wi.n_splits;
  const int P = wi.n_cached, ctx_len = P + wi.n_new;
  const unsigned n_rows = (unsigned)wi.n_new * G, row0 = (unsigned)wi.q_tile * RT;

  int64_t qrow[QB];                                            // row of q / out, in heads
  int posq[QB];
  bool ok[QB];
#pragma unroll
  for (int qb = 0; qb < QB; qb++) {
    const unsigned rho = row0 + 16 * qb + c;
    ok[qb] = rho < n_rows;
    const unsigned rr = ok[qb] ? rho : n_rows - 1, tok = rr / G;
    posq[qb] = P + (int)tok;
    qrow[qb] = (int64_t)(wi.q_off + (int)tok) * Hq + kv * (int)G + (int)(rr - tok * G);
  }
  const int pos_min = __builtin_amdgcn_readfirstlane(posq[0]), pos_max = __builtin_amdgcn_readlane(posq[QB - 1], 15);

  // ---- keys, 64 = four blocks to a step.  Row i of score tile kb is key 16 (i / 4) + 4 kb + i % 4: the four tiles leave lane (c, g) the weights
  // of keys 16g .. 16g + 15, all of one block, and 16 bytes of V^T are these keys for its d.
  const E4m3Block lay = e4m3_block(Hkv, D);
  const unsigned char* pool = (const unsigned char*)p.pool_layer;
  const int32_t* table = p.tables + wi.table_off;
  const int last_blk = (ctx_len + kBlockTokens - 1) / kBlockTokens - 1;
  auto step_at = [&](int st) { return st < wi.first_subs ? st : st + wi.gap; };
  auto hidden = [&](int key, int pos) { return (key > pos) | ((key <= pos - p.window) & (key >= p.n_first)); };
  bool k_ok[KJ];
#pragma unroll
  for (int j = 0; j < KJ; j++) k_ok[j] = C::FULL || 64 * j + 16 * g < D;
  const unsigned k_lane = (unsigned)kv * lay.tile + (c & 3) * D, v_lane = lay.v + (unsigned)kv * lay.tile + 16 * c;
  const int n_db = D / 16;

  int slot_k = 0, slot_v = 0;                                  // of the step that is asked for next
  constexpr int AHEAD = C::AHEAD;
  u32x4 kx[AHEAD][4][KJ], vx[AHEAD][DB];
  float ks[AHEAD], vs[AHEAD];
  const unsigned char* v_next = pool;
  auto look_up = [&](int st) {
    const int b = 4 * step_at(st);
    slot_k = table[min(b + (c >> 2), last_blk)];
    slot_v = table[min(b + g, last_blk)];
  };
  auto load_k = [&](auto at) __attribute__((always_inline)) {
    constexpr int A = decltype(at)::value;
    const unsigned char* kp = pool + (uint64_t)(unsigned)slot_k * lay.bytes;
    v_next = pool + (uint64_t)(unsigned)slot_v * lay.bytes;
    ks[A] = *(const float*)(kp + lay.scales + 4 * kv);
    kp += k_lane;
#pragma unroll
    for (int kb = 0; kb < 4; kb++)
#pragma unroll
      for (int j = 0; j < KJ; j++) kx[A][kb][j] = *(const u32x4*)(kp + 4 * kb * D + (k_ok[j] ? 64 * j + 16 * g : 0));
  };
  auto load_v = [&](auto at) __attribute__((always_inline)) {
    constexpr int A = decltype(at)::value;
    vs[A] = *(const float*)(v_next + lay.scales + 4 * (Hkv + kv));
#pragma unroll
    for (int db = 0; db < DB; db++) vx[A][db] = *(const u32x4*)(v_next + v_lane + 256 * (C::FULL ? db : min(db, n_db - 1)));
  };

  const int st_begin = wi.sub_begin + wave;
  const int st_end = min(wi.sub_end, pos_max / 64 + 1 - wi.gap);
  bf16x8 qx[QB][2 * KJ];
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  f32x4 o[QB][DB];
  float m[QB], l[QB];                                          // running maximum (exponent units); this lane's share of the sum
#pragma unroll
  for (int qb = 0; qb < QB; qb++) {
    m[qb] = -INFINITY;
    l[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; db++) o[qb][db] = zero4;
  }
  const float c2 = p.scale * 1.4426950408889634f;

  unsigned dirty = 0;
  // Steps that every row sees in full spend nothing on masks: in front of them are those with first tokens and those that windows begin in
  const int st_full = (pos_min + 1) / 64 - wi.gap, full_from = max(wi.first_subs, (pos_max - p.window < 0 ? 0 : (pos_max - p.window) / 64 + 1) - wi.gap);

  // Step st, whose K and V are in registers A.  MORE: the wave has a step AHEAD further on, which this one asks for.
  auto step = [&](int st, auto at, auto more_tag) __attribute__((always_inline)) {
    constexpr int A = decltype(at)::value;
    constexpr bool MORE = decltype(more_tag)::value != 0;
    const int k0 = step_at(st) * 64;
    const bool hides = st < full_from || st >= st_full;        // some row does not see all of the keys
    f32x4 s[4][QB];
#pragma unroll
    for (int kb = 0; kb < 4; kb++)
#pragma unroll
      for (int qb = 0; qb < QB; qb++) s[kb][qb] = zero4;
#pragma unroll
    for (int j = 0; j < KJ; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
#pragma unroll
        for (int kb = 0; kb < 4; kb++) {
          const u32x4 x = kx[A][kb][j];
          const bf16x8 a = widen(C::FULL || k_ok[j] ? x[2 * h] : 0u, C::FULL || k_ok[j] ? x[2 * h + 1] : 0u, ks[A]);
#pragma unroll
          for (int qb = 0; qb < QB; qb++) s[kb][qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qx[qb][2 * j + h], s[kb][qb], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);                     // four operands at a time in bf16: more would cost the second wave of a SIMD
      }
    if constexpr (MORE) {
      load_k(at);
      look_up(st + (AHEAD + 1) * NW);                          // clamped to the last block
    }
    if (hides) {
#pragma unroll
      for (int kb = 0; kb < 4; kb++)
#pragma unroll
        for (int qb = 0; qb < QB; qb++)
#pragma unroll
          for (int r = 0; r < 4; r++)
            if (hidden(k0 + 16 * g + 4 * kb + r, posq[qb])) s[kb][qb][r] = -INFINITY;
    }
    bf16x8 pw[QB][2];
    float alpha[QB];
    bool moved = false;
#pragma unroll
    for (int qb = 0; qb < QB; qb++) {
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; kb++)
#pragma unroll
        for (int r = 0; r < 4; r++) mx = fmaxf(mx, s[kb][qb][r]);
      const float mn = fmaxf(m[qb], quad_max(mx) * c2), ref = mn == -INFINITY ? 0.f : mn;   // no key seen yet: all weights are 0
      alpha[qb] = __builtin_amdgcn_exp2f(m[qb] - ref);
      moved |= mn != m[qb];
      m[qb] = mn;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
          w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * h + (e >> 2)][qb][e & 3], c2, -ref));
          sum += w[e];
        }
        pw[qb][h] = __builtin_bit_cast(bf16x8, (u32x4){pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])});
      }
      l[qb] = l[qb] * alpha[qb] + sum;
    }
    if (__builtin_amdgcn_ballot_w64(moved) != 0) {
#pragma unroll
      for (int qb = 0; qb < QB; qb++)
#pragma unroll
        for (int db = 0; db < DB; db++) o[qb][db] *= alpha[qb];
    }
    if (hides) {                                               // NaN or an infinity in V: the product takes weight 0 times it, also for rows that do not see the key
      dirty |= may_not_be_finite(vs[A]) ? 1u : 0u;
#pragma unroll
      for (int db = 0; db < DB; db++)
#pragma unroll
        for (int i = 0; i < 4; i++) dirty |= nan_bytes(vx[A][db][i]);
    }
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int db = 0; db < DB; db++) {
        const bf16x8 a = widen(vx[A][db][2 * h], vx[A][db][2 * h + 1], vs[A]);
#pragma unroll
        for (int qb = 0; qb < QB; qb++) o[qb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pw[qb][h], o[qb][db], 0, 0, 0);
        if (db % 4 == 3) __builtin_amdgcn_sched_barrier(0);
      }
    if constexpr (MORE) load_v(at);
  };

  const int n_steps = st_begin < st_end ? (st_end - st_begin + NW - 1) / NW : 0;
  if (n_steps > 0) {
    look_up(st_begin);
#pragma unroll
    for (int qb = 0; qb < QB; qb++)
#pragma unroll
      for (int j = 0; j < KJ; j++)
#pragma unroll
        for (int h = 0; h < 2; h++)
          qx[qb][2 * j + h] = *(const bf16x8*)((const unsigned char*)p.q + (qrow[qb] * D + (k_ok[j] ? 64 * j + 16 * g + 8 * h : 0)) * 2);
    __builtin_amdgcn_sched_barrier(0);
    load_k(Tag<0>{});
    look_up(st_begin + NW);
    __builtin_amdgcn_sched_barrier(0);
    load_v(Tag<0>{});
    __builtin_amdgcn_sched_barrier(0);
    auto settle_q = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int qb = 0; qb < QB; qb++)
#pragma unroll
        for (int i = 0; i < 2 * KJ; i++) {
          if (!C::FULL && !k_ok[i / 2]) qx[qb][i] = __builtin_bit_cast(bf16x8, (u32x4){0u, 0u, 0u, 0u});
          asm volatile("" : "+v"(qx[qb][i]));
        }
    };
    // No request of a step stands in a condition, and none is for a step that the wave does not have
    int st = st_begin, left = n_steps;
    if constexpr (AHEAD == 1) {
      settle_q();
      for (; left > 1; left--, st += NW) step(st, Tag<0>{}, Tag<1>{});
      step(st, Tag<0>{}, Tag<0>{});
    } else {
      // a single step asks for the context's last block beside its own: a path without it would cost half as many registers again
      load_k(Tag<1>{});
      look_up(st + 2 * NW);
      __builtin_amdgcn_sched_barrier(0);
      load_v(Tag<1>{});
      __builtin_amdgcn_sched_barrier(0);
      settle_q();
      // an odd number of steps asks for the last one again at the end
      for (; left > 2; left -= 2, st += 2 * NW) {
        step(st, Tag<0>{}, Tag<1>{});
        step(st + NW, Tag<1>{}, Tag<1>{});
      }
      step(st, Tag<0>{}, Tag<0>{});
      if (left == 2) step(st + NW, Tag<1>{}, Tag<0>{});
    }
  }
  // With such V (a byte or a scale that is NaN, a scale against which some bytes are infinite) the wave's rows meet its keys again, 16 at a time and V key by key: a row adds weight times V of the keys that it sees and touches no
  // other.  Rare, so it is written for few registers.
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(dirty != 0) != 0, 0)) {
    static_for<0, QB>([&](auto qb_tag) __attribute__((always_inline)) {
      constexpr int qb = decltype(qb_tag)::value;
#pragma unroll
      for (int db = 0; db < DB; db++) o[qb][db] = zero4;
      m[qb] = -INFINITY;
      l[qb] = 0.f;
#pragma unroll 1
      for (int b4 = 0; b4 < 4 * n_steps; b4++) {
        const int key0 = 64 * step_at(st_begin + NW * (b4 >> 2)) + kBlockTokens * (b4 & 3), rest = min(kBlockTokens, ctx_len - key0);
        if (rest <= 0) break;
        const unsigned char* blk = pool + (uint64_t)(unsigned)table[key0 / kBlockTokens] * lay.bytes;
        const float k_scale = *(const float*)(blk + lay.scales + 4 * kv), v_scale = *(const float*)(blk + lay.scales + 4 * (Hkv + kv));
        const unsigned char* kr = blk + (unsigned)kv * lay.tile + min(c, rest - 1) * D;
        f32x4 x = zero4;
#pragma unroll 1
        for (int j = 0; j < KJ; j++)
#pragma unroll
          for (int h = 0; h < 2; h++) {
            const int d = 64 * j + 16 * g + 8 * h;
            u32x2 y = {0u, 0u};
            u32x4 q = {0u, 0u, 0u, 0u};
            if (C::FULL || d < D) {
              y = *(const u32x2*)(kr + d);
              q = *(const u32x4*)((const unsigned char*)p.q + (qrow[qb] * D + d) * 2);
            }
            x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(y[0], y[1], k_scale), __builtin_bit_cast(bf16x8, q), x, 0, 0, 0);
          }
        float mx = -INFINITY, w[4];
#pragma unroll
        for (int r = 0; r < 4; r++) {
          if (hidden(key0 + 4 * g + r, posq[qb])) x[r] = -INFINITY;
          mx = fmaxf(mx, x[r]);
        }
        const float mn = fmaxf(m[qb], quad_max(mx) * c2), ref = mn == -INFINITY ? 0.f : mn, a = __builtin_amdgcn_exp2f(m[qb] - ref);
        m[qb] = mn;
        l[qb] *= a;
#pragma unroll
        for (int db = 0; db < DB; db++) o[qb][db] *= a;
#pragma unroll
        for (int r = 0; r < 4; r++) {
          w[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c2, -ref));
          l[qb] += w[r];
        }
#pragma unroll 1
        for (int t = 0; t < rest; t++) {
          const float mine = t & 2 ? (t & 1 ? w[3] : w[2]) : (t & 1 ? w[1] : w[0]);
          const float wk = __shfl(mine, 16 * (t >> 2) + c);
          const bool sees = !hidden(key0 + t, posq[qb]);
          const unsigned char* v = blk + lay.v + (unsigned)kv * lay.tile + t;
#pragma unroll
          for (int db = 0; db < DB; db++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
              const bf16x2 y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[16 * min(16 * db + 4 * g + r, D - 1)], v_scale, false);
              if (sees) o[qb][db][r] = __builtin_fmaf(wk, (float)y[0], o[qb][db][r]);
            }
        }
      }
    });
  }

  // ---- row sums over the four lanes of a row, then over the waves
  f32x4* const lds_o = (f32x4*)smem;
  float* const lds_ml = (float*)(smem + C::LDS_O);
#pragma unroll
  for (int qb = 0; qb < QB; qb++) {
    l[qb] = quad_sum(l[qb]);
    if (g == 0) *(f32x2*)(lds_ml + (wave * C::ROWS + 16 * qb + c) * 2) = (f32x2){m[qb], l[qb]};
  }
  __syncthreads();
#pragma unroll
  for (int qb = 0; qb < QB; qb++) {
    const f32x2* ml = (const f32x2*)lds_ml + 16 * qb + c;
    f32x2 x[NW];
    float all = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < NW; k++) x[k] = ml[k * C::ROWS];
#pragma unroll
    for (int k = 0; k < NW; k++) all = fmaxf(all, x[k][0]);
    const float ref = all == -INFINITY ? 0.f : all;
    const float a = __builtin_amdgcn_exp2f(m[qb] - ref);
#pragma unroll
    for (int k = 0; k < NW; k++) sum += __builtin_amdgcn_exp2f(x[k][0] - ref) * x[k][1];
    m[qb] = all;
    l[qb] = sum;
#pragma unroll
    for (int db = 0; db < DB; db++) lds_o[(wave * C::UNITS + qb * DB + db) * 64 + lane] = o[qb][db] * a;
  }
  __syncthreads();
  if (p.lse && n_splits == 1 && wave == 0 && g == 0) {
#pragma unroll
    for (int qb = 0; qb < QB; qb++)
      if (ok[qb]) p.lse[qrow[qb]] = log_sum(m[qb], l[qb]);
  }
  const int64_t part = (int64_t)it * Hkv + kv;
  const bool along = p.arrived != nullptr;                     // the tile's last piece merges them
  if (n_splits > 1 && wave == 0 && g == 0) {
#pragma unroll
    for (int qb = 0; qb < QB; qb++) {
      float* pm = p.part_ml + (part * C::ROWS + 16 * qb + c) * 2;
      if (along) store_through(pm, m[qb], l[qb]);
      else *(f32x2*)pm = (f32x2){m[qb], l[qb]};
    }
  }
#pragma unroll
  for (int qb = 0; qb < QB; qb++)
#pragma unroll
    for (int db = 0; db < DB; db++) {
      const int unit = qb * DB + db;
      if (unit % NW != wave) continue;                         // the waves share the stores
      f32x4 x = lds_o[unit * 64 + lane];
#pragma unroll
      for (int k = 1; k < NW; k++) x += lds_o[(k * C::UNITS + unit) * 64 + lane];
      const int d = 16 * db + 4 * g;
      if (n_splits > 1) {
        float* po = p.part_o + (part * C::ROWS + 16 * qb + c) * DP + d;
        if (!along) {
          *(f32x4*)po = x;
        } else if (ok[qb]) {
          store_through(po, x[0], x[1]);
          store_through(po + 2, x[2], x[3]);
        }
      } else if (ok[qb] && (C::FULL || d < D)) {
        const float inv = 1.f / l[qb];
        *(u32x2*)((unsigned short*)p.out + qrow[qb] * D + d) = (u32x2){pack_bf16(x[0] * inv, x[1] * inv), pack_bf16(x[2] * inv, x[3] * inv)};
      }
    }
  if (along && n_splits > 1) {
    // as in attn_rows_body.h
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();                                           // every wave's; and LDS is free
    if (threadIdx.x == 0) {
      int32_t* const count = p.arrived + (int64_t)wi.first_item * Hkv + kv;
      const int before = __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      if (before == n_splits - 1) __hip_atomic_store(count, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      *(int32_t*)smem = before;
    }
    __syncthreads();
    if (*(const int32_t*)smem != n_splits - 1) return;
    // every piece's partial result on its way at once where there are few, else 32 of them: a round of loads through the caches takes 1.5 us
    const int here = (int)min(RT, n_rows - row0);
    auto merge = [&](auto batch) {
      for (int row = wave; row < here; row += NW)
        rows::merge_row<uint16_t, DP, C::ROWS, true, decltype(batch)::value>(p, wi.first_item, n_splits, kv, row, row0 + row, wi.q_off);
    };
    if (n_splits <= 8) merge(Tag<8>{});
    else if (n_splits <= 16 || DP > 128) merge(Tag<16>{});
    else merge(Tag<32>{});
  }
}

// f(configuration) for a head width and tiling
template <typename F>
auto with_cfg(int head_dim, int tile_rows, F&& f) {
  if (head_dim == 128) return tile_rows == 16 ? f(Cfg<128, 1, 4, true>{}) : f(Cfg<128, 2, 4, true>{});
  if (head_dim == 64) return tile_rows == 16 ? f(Cfg<64, 1, 4, true>{}) : f(Cfg<64, 2, 4, true>{});
  if (head_dim < 64) return tile_rows == 16 ? f(Cfg<64, 1, 4, false>{}) : f(Cfg<64, 2, 4, false>{});
  if (head_dim < 128) return tile_rows == 16 ? f(Cfg<128, 1, 4, false>{}) : f(Cfg<128, 2, 4, false>{});
  if (head_dim == 256) return tile_rows == 16 ? f(Cfg<256, 1, 4, true>{}) : f(Cfg<256, 2, 4, true>{});
  return tile_rows == 16 ? f(Cfg<256, 1, 4, false>{}) : f(Cfg<256, 2, 4, false>{});
}

}  // namespace e4m3

hipError_t attn_e4m3_prepare(int head_dim, int tile_rows) {
  return e4m3::with_cfg(head_dim, tile_rows, [](auto cfg) {
    typedef decltype(cfg) C;
    return hipFuncSetAttribute((const void*)e4m3::attn_e4m3_kernel<C>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS_BYTES);
  });
}

hipError_t launch_attn_e4m3(const WinParams& p, int tile_rows, int n_items, const int32_t* split_tiles, int n_split_tiles, hipStream_t stream) {
  if (n_items <= 0) return hipSuccess;
  const unsigned grid = (unsigned)n_items * (unsigned)p.n_kv_heads;
  return e4m3::with_cfg(p.head_dim, tile_rows, [&](auto cfg) {
    typedef decltype(cfg) C;
    hipLaunchKernelGGL(e4m3::attn_e4m3_kernel<C>, dim3(grid), dim3(64 * C::NW), C::LDS_BYTES, stream, p);
    if (n_split_tiles > 0) {
      const unsigned slots = (unsigned)n_split_tiles * (unsigned)p.n_kv_heads;
      hipLaunchKernelGGL((rows::merge_rows_kernel<uint16_t, C::DP, C::ROWS, WinParams>), dim3(slots * (C::ROWS / 4)), dim3(256), 0, stream, p,
                         split_tiles);
    }
    return hipGetLastError();
  });
}

}  // namespace calvo
