// Gathered attention weights (calvo_attn_mass): for every key t of a request and KV head g
//     mass[g][t] += sum over the rows i that see t and the query heads h of g of  exp(scale <q[i][h], K[t][g]> - lse[i][h]).
// The rows' log-sum-exp comes from their attention, so one pass over the scores is enough and nothing is divided.
//
// A wave owns a tile of keys of one KV head and meets the rows that see some of them: every sum has one owner and one order, no
// atomics.  The tile's K stays in registers as the B operand (lane c of 16: key c); packed rows (token * group + head of the group) are the
// A operand, 16 at a time.  In the 16 x 16 result a lane has one key and rows 4g + r, so the sums stay in the lane until the end.
// The four waves of a workgroup own tiles side by side and share the rows, which come straight from memory into LDS (global_load_lds), 16 KiB
// a stage, two stages ahead; 16-byte chunks are XOR-swizzled on the way so that operand reads have no bank conflicts.  Where there are
// many rows a tile is worked on by several workgroups, each with its part of them (MassItem); mass_add_kernel adds their sums in order.
//
// What bounds it (32Q/8KV, D = 128, bf16).  Few rows: reading K.  One new token each of 8 requests of 4096 to 20000 tokens 39 us, 4.9 TB/s, what
// a large copy reaches.  Many: a score costs the vector ALU a fused multiply-add, an exponential and an addition, and the clock falls to 1.98 GHz under the
// power of both units.  0+8192 tokens 313 us and 4.6 of addition, 880 TFLOP/s (960 between the ends); the ALU issues in 72 % of the cycles (what
// the others wait for was not found: other orders of the instructions changed nothing).  Rows straight from memory to registers instead of through LDS: 548 us.
// Sums are fp32, a lane's in the order of its rows, the parts' behind each other: 0+8192 tokens 1.6e-7 from 64 bits (2-norm, relative); weights in
// 32 bits, summed in 64, would leave 2.5e-8.
#include "attn_common.h"
#include "../../include/calvo.h"

namespace calvo {
namespace mass {

using namespace attn;

// T_: storage.  DP: head_dim rounded up to 64, 128 or 256.  KT: 16-key blocks of a wave's tile.
template <typename T_, int DP_, int KT_, bool FULL_>
struct MassCfg {
  typedef T_ T;
  static constexpr int DP = DP_, KT = KT_, E = sizeof(T_), NW = 4;
  static constexpr bool F32 = sizeof(T_) == 4, FULL = FULL_;
  static constexpr int KJ = F32 ? DP / 16 : DP / 32;           // 16-byte operand chunks of a K or Q row per lane
  static constexpr int KEYS = 16 * KT;                         // of a wave
  static constexpr int CPR = DP * E / 16;                      // chunks of a row
  static constexpr int SR = 1024 / CPR;                        // rows of a stage
  static constexpr int RPI = 64 / CPR;                         // rows of one request instruction (1 KiB)
  static constexpr int NI = SR / (NW * RPI);                   // such instructions of a wave per stage: four
  static constexpr int STAGES = 3;
  static constexpr int LDS_LSE = STAGES * 16384, LDS_BYTES = LDS_LSE + STAGES * SR * 4;
};

constexpr unsigned kPastEnd = 0xfffff000u, kBufferWord3 = 0x00020000u;
constexpr float kLog2e = 1.4426950408889634f;
__device__ inline float as_float(unsigned x) { return __builtin_bit_cast(float, x); }

__device__ inline MassItem load_mass_item(const MassItem* items, int i) {
  const const_i32p w = (const_i32p)(uintptr_t)(items + i);
  return {w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7], w[8], {0, 0, 0}};
}

// 64 lanes x 16 (or 4) bytes from their addresses to LDS at lds_addr (uniform) + 16 (4) * lane; lanes that are off write nothing
__device__ inline void to_lds_16(const void* from, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(lds_addr));
}
__device__ inline void to_lds_4(const void* from, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(from), "s"(lds_addr));
}

template <class C>
__global__ void __launch_bounds__(256, 3) attn_mass_kernel(MassParams p) {
  constexpr int KT = C::KT, KJ = C::KJ, E = C::E, KEYS = C::KEYS, NW = C::NW, CPR = C::CPR, SR = C::SR, RPI = C::RPI, NI = C::NI;
  constexpr bool F32 = C::F32, FULL = C::FULL;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const lds_u8* lds = (const lds_u8*)smem;
  const unsigned lds0 = (unsigned)(size_t)lds;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int Hkv = p.n_kv_heads, Hq = p.n_q_heads, D = p.head_dim;
  const unsigned G = p.group;

  // ---- a KV head's workgroups stay on one XCD where the heads divide over the eight
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
  const MassItem mi = load_mass_item(p.items, it);
  const int n_cached = mi.n_cached, n_new = mi.n_new, ctx = n_cached + n_new;
  const const_i32p table = (const_i32p)(uintptr_t)(p.tables + mi.table_off);
  const int t0 = mi.tile * (NW * KEYS) + wave * KEYS, t1 = min(t0 + KEYS, ctx);
  const bool live = t0 < ctx;                                  // the last tile's waves past the context only help to load

  // ---- the item's rows, in stages of SR
  const unsigned row_begin = (unsigned)max(mi.begin, p.last_rows ? n_new - p.last_rows : 0) * G, row_end = (unsigned)mi.end * G;
  const int n_stages = row_begin < row_end ? (int)((row_end - row_begin + SR - 1) / SR) : 0;
  // Row rel of the item is head rel % G of token rel / G behind the item's first.  rel is below 2^20 and G at most 4096 (plan_mass, calvo_attn_mass): the
  // product with 2^32 / G, rounded up, has the quotient in its upper half.
  const int64_t q_base = ((int64_t)mi.q_off + row_begin / G) * Hq + kv * (int)G;
  const unsigned recip = G == 1 ? 0 : 0xffffffffu / G + 1, last_rel = max(row_end - row_begin, 1u) - 1;
  auto row_of = [&](unsigned rel) {
    rel = min(rel, last_rel);                                  // past the end the last row
    const unsigned tok = G == 1 ? rel : __umulhi(rel, recip);
    return q_base + (int64_t)tok * Hq + (rel - tok * G);
  };
  int q_off[NI];                                               // the chunk of its row that a lane asks for, in bytes
#pragma unroll
  for (int h = 0; h < NI; h++) q_off[h] = (((lane % CPR) ^ ((wave * (NI * RPI) + h * RPI + lane / CPR) & 15)) & (CPR - 1)) * 16;
  auto request = [&](int st, int slot) {
    const unsigned rel0 = (unsigned)st * SR + wave * (SR / NW);
    const unsigned char* from0 = (const unsigned char*)p.q + row_of(rel0 + lane / CPR) * (D * E);
    // whole tokens from one instruction to the next: no division for each
    const bool even = RPI % G == 0 && rel0 + SR / NW - 1 <= last_rel;
    const unsigned step = RPI / G * (unsigned)(Hq * D * E);
#pragma unroll
    for (int h = 0; h < NI; h++) {
      const unsigned char* row = from0 + h * step;
      if (h > 0 && !even) row = (const unsigned char*)p.q + row_of(rel0 + h * RPI + lane / CPR) * (D * E);
      if (FULL || q_off[h] < D * E) to_lds_16(row + q_off[h], lds0 + slot * 16384 + (wave * NI + h) * 1024);
    }
    const float* from = p.lse + row_of(rel0 + lane);
    if (lane < SR / NW) to_lds_4(from, lds0 + C::LDS_LSE + (slot * SR + wave * (SR / NW)) * 4);
  };
  if (!FULL) {
    // chunks past the head stay zero
    for (int i = threadIdx.x; i < C::LDS_LSE / 16; i += 256) *(u32x4*)(smem + 16 * i) = (u32x4){0u, 0u, 0u, 0u};
    __syncthreads();
  }
  if (n_stages > 0) request(0, 0);

  // ---- K of the tile: what lies past the context or the head reads zeros
  const unsigned rs = (unsigned)(Hkv * D * E), half = kBlockTokens * rs;
  u32x4 kreg[KT][KJ];
  int slot[KT];
  if (n_stages > 0) {                                          // else no row counts: 0+32768 tokens, the last 32 of them counted, 38 / 29 us
#pragma unroll
    for (int kt = 0; kt < KT; kt++) slot[kt] = table[min(t0 / kBlockTokens + kt, (ctx - 1) / kBlockTokens)];
#pragma unroll
    for (int kt = 0; kt < KT; kt++) {
      const int rows = max(0, min(kBlockTokens, ctx - t0 - kBlockTokens * kt));
      const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>((const unsigned char*)p.pool_layer + (uint64_t)(unsigned)slot[kt] * 2 * half),
                                                         0, (unsigned)rows * rs, kBufferWord3);
#pragma unroll
      for (int j = 0; j < KJ; j++) {
        const int d = F32 ? 16 * j + 4 * g : 32 * j + 8 * g;
        kreg[kt][j] = __builtin_amdgcn_raw_buffer_load_b128(buf, FULL || d < D ? (unsigned)((kv * D + d) * E) + c * rs : kPastEnd, 0, 0);
      }
    }
    // in registers before a stage is waited for by count
#pragma unroll
    for (int kt = 0; kt < KT; kt++)
#pragma unroll
      for (int j = 0; j < KJ; j++) asm volatile("" : "+v"(kreg[kt][j]));
    if (n_stages > 1) request(1, 1);
  }

  const float c2 = p.scale * kLog2e;
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  float acc[KT];
#pragma unroll
  for (int kt = 0; kt < KT; kt++) acc[kt] = 0.f;
  // Blocks whose rows all see every key of the wave's tile: those from the last key's row on, up to the rows whose window begins behind the first
  const int64_t from = (int64_t)max(0, t1 - 1 - n_cached) * G, to = t1 <= p.n_first ? row_end : max<int64_t>(0, (int64_t)t0 + p.window - n_cached) * G;
  const unsigned full_from = (unsigned)min<int64_t>(from, row_end), full_to = (unsigned)min<int64_t>(to, row_end);
  // ... and those whose rows see some of them: from the first key's row on, up to the rows whose window begins behind the last
  const int64_t some = (int64_t)max(0, t0 - n_cached) * G, none = t0 < p.n_first ? row_end : max<int64_t>(0, (int64_t)t1 - 1 + p.window - n_cached) * G;
  const unsigned see_from = (unsigned)min<int64_t>(some, row_end), see_to = (unsigned)min<int64_t>(none, row_end);

  const lds_u8* q_addr[KJ];                                    // this lane's operand chunks of a block in LDS
#pragma unroll
  for (int j = 0; j < KJ; j++) q_addr[j] = lds + c * (CPR * 16) + (((4 * j + g) ^ c) & (CPR - 1)) * 16;
  auto block = [&](unsigned row0, const lds_u8* const (&qa)[KJ], const lds_u8* la, auto masked) {
    constexpr bool MASKED = decltype(masked)::value != 0;
    u32x4 q[KJ];
#pragma unroll
    for (int j = 0; j < KJ; j++) q[j] = *(const __attribute__((address_space(3))) u32x4*)qa[j];
    f32x4 L = *(const __attribute__((address_space(3))) f32x4*)la;
    L *= -kLog2e;
    // a row sees the keys from lo on, `many` of them, and the first ones; a row past the end none
    unsigned lo[4], many[4], first[4];
    if constexpr (MASKED) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const unsigned rel = row0 + 4 * g + i - row_begin, tok = G == 1 ? rel : __umulhi(rel, recip);
        const int pos = n_cached + (int)(row_begin / G + tok);
        const bool ok = rel <= last_rel;
        lo[i] = (unsigned)max(0, pos - p.window + 1);
        many[i] = ok ? (unsigned)pos + 1 - lo[i] : 0;
        first[i] = ok ? (unsigned)min(p.n_first, pos + 1) : 0;
      }
    }
    // The scores of the next 16 keys are under way while the weights of these are computed
    f32x4 s[2];
    auto scores = [&](int kt) {
      f32x4& y = s[kt & 1];
      y = zero4;
#pragma unroll
      for (int j = 0; j < KJ; j++) {
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 4; i++) y = __builtin_amdgcn_mfma_f32_16x16x4f32(as_float(q[j][i]), as_float(kreg[kt][j][i]), y, 0, 0, 0);
        } else {
          y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, q[j]), __builtin_bit_cast(bf16x8, kreg[kt][j]), y, 0, 0, 0);
        }
      }
    };
    scores(0);
#pragma unroll
    for (int kt = 0; kt < KT; kt++) {
      if (kt + 1 < KT) scores(kt + 1);
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt & 1][i], c2, L[i]));
      if constexpr (MASKED) {
        const unsigned key = (unsigned)(t0 + 16 * kt + c);
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = (key - lo[i] < many[i]) | (key < first[i]) ? w[i] : 0.f;
      }
      acc[kt] += (w[0] + w[1]) + (w[2] + w[3]);
    }
  };
  int ring = 0;
  for (int st = 0; st < n_stages; st++) {
    if (st + 1 < n_stages) wait_vm<NI + 1>();                  // all but the stage behind this one
    else wait_vm<0>();
    __syncthreads();                                           // ... for every wave; and everyone is done with the stage before
    if (st + 2 < n_stages) request(st + 2, ring == 0 ? 2 : ring - 1);
    const unsigned row_st = row_begin + (unsigned)st * SR;
    const lds_u8* qs[KJ];
    const lds_u8* ls = lds + C::LDS_LSE + ring * (SR * 4) + 16 * g;
#pragma unroll
    for (int j = 0; j < KJ; j++) qs[j] = q_addr[j] + ring * 16384;
    constexpr int kBlock = 16 * CPR * 16;                      // bytes of a block of 16 rows
    if (live && row_st >= full_from && row_st + SR <= full_to) {
      // the whole stage: operands of the next block are on their way during this one
#pragma unroll
      for (int b = 0; b < SR / 16; b++) {
        const lds_u8* qa[KJ];
#pragma unroll
        for (int j = 0; j < KJ; j++) qa[j] = qs[j] + b * kBlock;
        block(row_st + 16 * b, qa, ls + 64 * b, Tag<0>{});
      }
    } else if (live && row_st + SR > see_from && row_st < see_to) {
#pragma unroll 1
      for (int b = 0; b < SR / 16; b++) {
        const unsigned row0 = row_st + 16 * b;
        if (row0 + 16 <= see_from) continue;
        if (row0 >= see_to) break;
        const lds_u8* qa[KJ];
#pragma unroll
        for (int j = 0; j < KJ; j++) qa[j] = qs[j] + b * kBlock;
        block(row0, qa, ls + 64 * b, Tag<1>{});
      }
    }
    ring = ring == 2 ? 0 : ring + 1;
  }
  if (!live) return;

  // ---- over the four lanes of a key
  float x[KT];
#pragma unroll
  for (int kt = 0; kt < KT; kt++) x[kt] = quad_sum(acc[kt]);
  if (g == 0) {
    if (mi.part < 0) {
      const int64_t at = ((int64_t)mi.mass_row * Hkv + kv) * p.mass_stride + t0 + c;
#pragma unroll
      for (int kt = 0; kt < KT; kt++) {
        const int t = t0 + 16 * kt + c;
        if (t < t1) p.mass_out[at + 16 * kt] = x[kt] + (t < n_cached && p.mass_in ? p.mass_in[at + 16 * kt] : 0.f);
      }
    } else {
      float* part = p.part + ((int64_t)mi.part * Hkv + kv) * (C::NW * KEYS) + wave * KEYS + c;
#pragma unroll
      for (int kt = 0; kt < KT; kt++) part[16 * kt] = x[kt];
    }
  }
}

// The sums of the tiles that several workgroups worked on.  64 keys to a workgroup of one wave, eight parts on their way at a time.
__global__ void __launch_bounds__(64) mass_add_kernel(MassParams p, const MassAdd* adds, int wg_keys) {
  const int Hkv = p.n_kv_heads, per = wg_keys / 64;
  const int i = blockIdx.x % per * 64 + threadIdx.x, rest = blockIdx.x / per;
  const int kv = rest % Hkv;
  const const_i32p a = (const_i32p)(uintptr_t)(adds + rest / Hkv);
  const int n_cached = a[0], n_tokens = a[1], mass_row = a[2], tile = a[3], first = a[4], n_parts = a[5];
  const int t = tile * wg_keys + i;
  if (t >= n_tokens) return;
  const float* part = p.part + ((int64_t)first * Hkv + kv) * wg_keys + i;
  const int64_t step = (int64_t)Hkv * wg_keys, at = ((int64_t)mass_row * Hkv + kv) * p.mass_stride + t;
  const float before = t < n_cached && p.mass_in ? p.mass_in[at] : 0.f;
  float x = 0.f;
  for (int k0 = 0; k0 < n_parts; k0 += 8) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; k++) v[k] = part[min(k0 + k, n_parts - 1) * step];
#pragma unroll
    for (int k = 0; k < 8; k++)
      if (k0 + k < n_parts) x += v[k];
  }
  p.mass_out[at] = x + before;
}

// K of a wave's tile in at most 64 registers, so that three waves share a SIMD.  0+8192 tokens (bf16, D = 128) at 8, 6, 5, 4, 3, 2 blocks of keys:
// 352, 345, 322, 320, 324, 361 us; single tokens of 8 requests 44.6, 45.4, 44.7, 40.0, 41.3, 44.4.
template <typename F>
auto with_cfg(int dtype, int head_dim, F&& f) {
  if (dtype == CALVO_F32) {
    if (head_dim == 64) return f(MassCfg<float, 64, 4, true>{});
    if (head_dim < 64) return f(MassCfg<float, 64, 4, false>{});
    if (head_dim == 128) return f(MassCfg<float, 128, 2, true>{});
    if (head_dim < 128) return f(MassCfg<float, 128, 2, false>{});
    return f(MassCfg<float, 256, 1, false>{});
  }
  if (head_dim == 64) return f(MassCfg<uint16_t, 64, 4, true>{});
  if (head_dim < 64) return f(MassCfg<uint16_t, 64, 4, false>{});
  if (head_dim == 128) return f(MassCfg<uint16_t, 128, 4, true>{});
  if (head_dim < 128) return f(MassCfg<uint16_t, 128, 4, false>{});
  return f(MassCfg<uint16_t, 256, 2, false>{});
}

}  // namespace mass

int attn_mass_tile_keys(int dtype, int head_dim) {
  return mass::with_cfg(dtype, head_dim, [](auto cfg) { return decltype(cfg)::NW * decltype(cfg)::KEYS; });
}

hipError_t launch_attn_mass(const MassParams& p, int dtype, const MassAdd* adds, int n_adds, hipStream_t stream) {
  if (p.n_items <= 0) return hipSuccess;
  const unsigned grid = (unsigned)p.n_items * (unsigned)p.n_kv_heads;
  return mass::with_cfg(dtype, p.head_dim, [&](auto cfg) {
    typedef decltype(cfg) C;
    hipLaunchKernelGGL(mass::attn_mass_kernel<C>, dim3(grid), dim3(64 * C::NW), C::LDS_BYTES, stream, p);
    if (n_adds > 0)
      hipLaunchKernelGGL(mass::mass_add_kernel, dim3((unsigned)n_adds * (unsigned)p.n_kv_heads * (C::NW * C::KEYS / 64)), dim3(64), 0,
                         stream, p, adds, C::NW * C::KEYS);
    return hipGetLastError();
  });
}

}  // namespace calvo
