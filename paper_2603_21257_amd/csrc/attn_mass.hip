// Gathered attention weights (calvo_attn_mass): for every key t of a request and KV head g
//     mass[g][t] += sum over the rows i that see t and the query heads h of g of  exp(scale <q[i][h], K[t][g]> - lse[i][h]).
// The rows' log-sum-exp comes from their attention, so one pass over the scores is enough and nothing is divided.
//
// A workgroup owns a tile of keys of one KV head and meets all rows that see some of them: every sum has one owner and one order, no
// atomics.  The tile's K stays in registers as the B operand (lane c of 16: key c), packed rows (token * group + head of the group) stream
// through as the A operand, 16 at a time: in the 16 x 16 result a lane has one key and rows 4g + r, so the sums stay in the lane
// until the end.  The waves take alternate blocks of rows and are added through LDS in a fixed order.
#include "attn_common.h"
#include "../../include/calvo.h"

namespace calvo {
namespace mass {

using namespace attn;

// T_: storage.  DP: head_dim rounded up to 64, 128 or 256.  KT: 16-key blocks of a tile.  NW: waves.
template <typename T_, int DP_, int KT_, int NW_>
struct MassCfg {
  typedef T_ T;
  static constexpr int DP = DP_, KT = KT_, NW = NW_, E = sizeof(T_);
  static constexpr bool F32 = sizeof(T_) == 4;
  static constexpr int KJ = F32 ? DP / 16 : DP / 32;           // 16-byte operand chunks of a K or Q row per lane
};

constexpr unsigned kPastEnd = 0xfffff000u, kBufferWord3 = 0x00020000u;
__device__ inline float as_float(unsigned x) { return __builtin_bit_cast(float, x); }

template <class C>
__global__ void __launch_bounds__(64 * C::NW) attn_mass_kernel(MassParams p) {
  constexpr int KT = C::KT, NW = C::NW, KJ = C::KJ, E = C::E, KEYS = 16 * KT;
  constexpr bool F32 = C::F32;
  __shared__ float sums[NW][KEYS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, g = lane >> 4;
  const int Hkv = p.n_kv_heads, Hq = p.n_q_heads, D = p.head_dim;
  const unsigned G = p.group;

  // ---- a KV head's workgroups stay on one XCD where the heads divide over the eight
  int tile, kv;
  {
    const int bid = blockIdx.x;
    if ((Hkv & 7) == 0) {
      const int per = Hkv >> 3, rest = bid >> 3;
      kv = (bid & 7) * per + rest % per;
      tile = rest / per;
    } else {
      kv = bid % Hkv;
      tile = bid / Hkv;
    }
  }
  const const_i32p reqs = (const_i32p)(uintptr_t)p.reqs;
  constexpr int kReq = sizeof(WinReq) / 4;
  int r = 0;                                                   // the last request that begins at or before the tile
  for (int end = p.n_reqs; end - r > 1;) {
    const int mid = (r + end) / 2;
    if (tile >= reqs[kReq * mid + 5]) r = mid;
    else end = mid;
  }
  const const_i32p rq = reqs + kReq * r;
  const int n_cached = rq[1], n_new = rq[2], q_off = rq[3], mass_row = rq[4];
  const const_i32p table = (const_i32p)(uintptr_t)(p.tables + rq[0]);
  const int ctx = n_cached + n_new;
  const int t0 = (tile - rq[5]) * KEYS, t1 = min(t0 + KEYS, ctx);

  // ---- K of the tile: what lies past the context or the head reads zeros
  const unsigned rs = (unsigned)(Hkv * D * E), half = kBlockTokens * rs;
  u32x4 kreg[KT][KJ];
  bool d_ok[KJ];
  unsigned d_off[KJ];
#pragma unroll
  for (int j = 0; j < KJ; j++) {
    const int d = F32 ? 16 * j + 4 * g : 32 * j + 8 * g;
    d_ok[j] = d < D;
    d_off[j] = (unsigned)((d_ok[j] ? d : 0) * E);
  }
#pragma unroll
  for (int kt = 0; kt < KT; kt++) {
    const int b = t0 / kBlockTokens + kt;
    const int rows = max(0, min(kBlockTokens, ctx - kBlockTokens * b));
    const int slot = table[min(b, (ctx - 1) / kBlockTokens)];
    const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>((const unsigned char*)p.pool_layer + (uint64_t)(unsigned)slot * 2 * half),
                                                       0, (unsigned)rows * rs, kBufferWord3);
#pragma unroll
    for (int j = 0; j < KJ; j++)
      kreg[kt][j] = __builtin_amdgcn_raw_buffer_load_b128(buf, d_ok[j] ? (unsigned)(kv * D * E) + c * rs + d_off[j] : kPastEnd, 0, 0);
  }

  // ---- rows that see some key of the tile
  int i0 = max(0, t0 - n_cached);
  if (p.last_rows) i0 = max(i0, n_new - p.last_rows);
  int i1 = n_new;
  if (t0 >= p.n_first) i1 = (int)min((int64_t)n_new, (int64_t)t1 - 1 + p.window - n_cached);
  const unsigned row_begin = (unsigned)i0 * G, row_end = (unsigned)max(i1, i0) * G;
  const float c2 = p.scale * 1.4426950408889634f;
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  float acc[KT];
#pragma unroll
  for (int kt = 0; kt < KT; kt++) acc[kt] = 0.f;

  for (unsigned row0 = row_begin + 16 * wave; row0 < row_end; row0 += 16 * NW) {
    u32x4 qreg[KJ];
    const unsigned rho = min(row0 + c, row_end - 1), tok = rho / G;
    const unsigned char* qp = (const unsigned char*)p.q + ((int64_t)(q_off + (int)tok) * Hq + kv * (int)G + (int)(rho - tok * G)) * (D * E);
#pragma unroll
    for (int j = 0; j < KJ; j++) {
      qreg[j] = *(const u32x4*)(qp + d_off[j]);
      if (!d_ok[j]) qreg[j] = (u32x4){0u, 0u, 0u, 0u};
    }
    float L[4];
    int pos[4];
    bool ok[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const unsigned x = row0 + 4 * g + i, xr = min(x, row_end - 1), t = xr / G;
      ok[i] = x < row_end;
      pos[i] = n_cached + (int)t;
      L[i] = p.lse[(int64_t)(q_off + (int)t) * Hq + kv * (int)G + (int)(xr - t * G)] * 1.4426950408889634f;
    }
    // every row of the block sees every key of the tile
    const int pos_min = n_cached + (int)(row0 / G), pos_max = n_cached + (int)(min(row0 + 15, row_end - 1) / G);
    const bool full = row0 + 16 <= row_end && pos_min >= t1 - 1 && (t1 <= p.n_first || pos_max - p.window < t0);
#pragma unroll
    for (int kt = 0; kt < KT; kt++) {
      f32x4 s = zero4;
#pragma unroll
      for (int j = 0; j < KJ; j++) {
        if constexpr (F32) {
#pragma unroll
          for (int i = 0; i < 4; i++) s = __builtin_amdgcn_mfma_f32_16x16x4f32(as_float(qreg[j][i]), as_float(kreg[kt][j][i]), s, 0, 0, 0);
        } else {
          s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, qreg[j]), __builtin_bit_cast(bf16x8, kreg[kt][j]), s, 0, 0, 0);
        }
      }
      float w[4];
#pragma unroll
      for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c2, -L[i]));
      if (!full) {
        const int key = t0 + 16 * kt + c;
#pragma unroll
        for (int i = 0; i < 4; i++)
          if (!ok[i] || key > pos[i] || (key <= pos[i] - p.window && key >= p.n_first)) w[i] = 0.f;
      }
      acc[kt] += (w[0] + w[1]) + (w[2] + w[3]);
    }
  }

  // ---- the four lanes of a key, then the waves
#pragma unroll
  for (int kt = 0; kt < KT; kt++) {
    const float x = quad_sum(acc[kt]);
    if (g == 0) sums[wave][16 * kt + c] = x;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < t1 - t0; i += 64 * NW) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < NW; w++) x += sums[w][i];
    const int64_t at = ((int64_t)mass_row * Hkv + kv) * p.mass_stride + t0 + i;
    if (t0 + i < n_cached && p.mass_in) x += p.mass_in[at];
    p.mass_out[at] = x;
  }
}

template <typename F>
auto with_cfg(int dtype, int head_dim, F&& f) {
  if (dtype == CALVO_F32) {
    if (head_dim <= 64) return f(MassCfg<float, 64, 4, 4>{});
    if (head_dim <= 128) return f(MassCfg<float, 128, 4, 4>{});
    return f(MassCfg<float, 256, 2, 4>{});
  }
  if (head_dim <= 64) return f(MassCfg<uint16_t, 64, 4, 4>{});
  if (head_dim <= 128) return f(MassCfg<uint16_t, 128, 4, 4>{});
  return f(MassCfg<uint16_t, 256, 4, 4>{});
}

}  // namespace mass

int attn_mass_tile_keys(int dtype, int head_dim) {
  return mass::with_cfg(dtype, head_dim, [](auto cfg) { return 16 * decltype(cfg)::KT; });
}

hipError_t launch_attn_mass(const MassParams& p, int dtype, hipStream_t stream) {
  if (p.n_tiles <= 0) return hipSuccess;
  const unsigned grid = (unsigned)p.n_tiles * (unsigned)p.n_kv_heads;
  return mass::with_cfg(dtype, p.head_dim, [&](auto cfg) {
    typedef decltype(cfg) C;
    hipLaunchKernelGGL(mass::attn_mass_kernel<C>, dim3(grid), dim3(64 * C::NW), 0, stream, p);
    return hipGetLastError();
  });
}

}  // namespace calvo
