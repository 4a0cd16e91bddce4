// New tokens into the paged pool, Q and K rotated by position on the way (calvo_kv_append).
//
// Rotation of a head x at position p: a_i = p f_i for i < R / 2, and for every pair (x, y) of elements - i and i + R / 2, or 2i and 2i + 1 -
//     x' = x cos a_i - y sin a_i,   y' = y cos a_i + x sin a_i;
// elements from R on stay.  Far positions lose an angle in 32 bits (at position 10^6 the fastest pair would be off by 0.03 of a radian): it is made in 64
// bits as a number of turns, whose fraction is exact enough in 32.  One rounding at the end, of the sum.
#include "../../include/calvo.h"
#include "kv_e4m3.h"

namespace calvo {
namespace append {

using namespace attn;
using e4m3::bits_of;
using e4m3::float_of;

// the last request that begins at or before a token (halving: append_suffix, attn_common.h)
__device__ inline int request_of(const ReqDesc* reqs, int n_reqs, int tok) {
  int r = 0;
  for (int end = n_reqs; end - r > 1;) {
    const int mid = (r + end) / 2;
    if (tok >= reqs[mid].q_off) r = mid;
    else end = mid;
  }
  return r;
}

__device__ inline f32x2 cos_sin(const RopeParams& rope, int pos, int i) {
  const double turns = (double)pos * ((double)rope.inv_freq[i] * 0.15915494309189533577);
  float s, c;
  sincospif((float)(2. * (turns - __builtin_rint(turns))), &s, &c);
  return (f32x2){c, s};
}

// 16 bytes of a head's row as numbers, and back
template <typename T>
struct Chunk;
template <>
struct Chunk<uint16_t> {
  static constexpr int N = 8;
  static __device__ void read(const unsigned char* a, float (&x)[8]) {
    const u32x4 v = *(const u32x4*)a;
#pragma unroll
    for (int i = 0; i < 8; i++) x[i] = float_of(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16);
  }
  static __device__ float one(const unsigned char* row, int d) { return float_of((unsigned)((const unsigned short*)row)[d] << 16); }
  static __device__ u32x4 packed(const float (&x)[8]) { return (u32x4){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}; }
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ void read(const unsigned char* a, float (&x)[4]) {
    const f32x4 v = *(const f32x4*)a;
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = v[i];
  }
  static __device__ float one(const unsigned char* row, int d) { return ((const float*)row)[d]; }
  static __device__ u32x4 packed(const float (&x)[4]) { return (u32x4){bits_of(x[0]), bits_of(x[1]), bits_of(x[2]), bits_of(x[3])}; }
};

// Chunk ch of a head's row, rotated.  cs: (cos, sin) of the token's pairs.
template <typename T>
__device__ inline void rotated(const RopeParams& rope, const unsigned char* row, int ch, const f32x2* cs, float (&x)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
  const int d0 = ch * N;
  Chunk<T>::read(row + 16 * ch, x);
  if (d0 >= rope.rot) return;
  if (rope.interleaved) {
#pragma unroll
    for (int i = 0; i < N; i += 2)
      if (d0 + i < rope.rot) {
        const f32x2 t = cs[(d0 + i) >> 1];
        const float a = x[i], b = x[i + 1];
        x[i] = a * t[0] - b * t[1];
        x[i + 1] = b * t[0] + a * t[1];
      }
  } else if (rope.half % N == 0) {
    const bool lower = d0 < rope.half;
    float y[N];
    Chunk<T>::read(row + 16 * ch + (lower ? rope.half : -rope.half) * (int)sizeof(T), y);
    const f32x2* t = cs + (lower ? d0 : d0 - rope.half);
#pragma unroll
    for (int i = 0; i < N; i++) x[i] = x[i] * t[i][0] + (lower ? -y[i] : y[i]) * t[i][1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int d = d0 + i;
      if (d >= rope.rot) continue;
      const bool lower = d < rope.half;
      const f32x2 t = cs[lower ? d : d - rope.half];
      const float y = Chunk<T>::one(row, lower ? d + rope.half : d - rope.half);
      x[i] = x[i] * t[0] + (lower ? -y : y) * t[1];
    }
  }
}

constexpr int kThreads = 256;

// Rows of tokens [t0, t0 + n): q -> q_out, and where the pool holds the same type k and v -> pool.  cs: room for n * rot / 2 pairs.
template <typename T, bool KV>
__device__ inline void move_rows(const KvAppendParams& p, int t0, int n, f32x2* cs) {
  constexpr int N = Chunk<T>::N;
  const int half = p.rope.half;
  for (int i = threadIdx.x; i < n * half; i += kThreads) {
    const int tok = t0 + i / half;
    int pos;
    if (p.rope.positions) {
      pos = p.rope.positions[tok];
    } else {
      const ReqDesc rd = p.reqs[request_of(p.reqs, p.n_reqs, tok)];
      pos = rd.prefix_len + tok - rd.q_off;
    }
    cs[i] = cos_sin(p.rope, pos, i % half);
  }
  __syncthreads();
  const int chunks = p.head_dim / N, row_chunks = p.n_kv_heads * chunks;
  const int nq = p.q ? p.n_q_heads * chunks : 0, nk = KV && p.k ? row_chunks : 0;
  const int all = nq + 2 * nk;
  for (int i = threadIdx.x; i < n * all; i += kThreads) {
    const int t = i / all, j = i - t * all, tok = t0 + t;
    if (j < nq) {
      float x[N];
      rotated<T>(p.rope, (const unsigned char*)p.q + tok * p.q_row + (j / chunks) * p.head_dim * (int)sizeof(T), j % chunks, cs + t * half, x);
      ((u32x4*)p.q_out)[(int64_t)tok * nq + j] = Chunk<T>::packed(x);
    } else if constexpr (KV) {
      const int r = request_of(p.reqs, p.n_reqs, tok);
      const ReqDesc rd = p.reqs[r];
      const int pos = rd.prefix_len + (tok - rd.q_off), k = j - nq;
      const int64_t slot = p.tables[rd.table_off + pos / kBlockTokens];
      u32x4* dst = (u32x4*)p.pool_layer + (slot * 2 * kBlockTokens + pos % kBlockTokens) * row_chunks;
      if (k < nk) {
        float x[N];
        rotated<T>(p.rope, (const unsigned char*)p.k + tok * p.k_row + (k / chunks) * p.head_dim * (int)sizeof(T), k % chunks, cs + t * half, x);
        dst[k] = Chunk<T>::packed(x);
      } else {
        dst[kBlockTokens * row_chunks + k - nk] = *(const u32x4*)((const unsigned char*)p.v + tok * p.v_row + 16 * (k - nk));
      }
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) append_kernel(KvAppendParams p, int tokens_per_wg) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int t0 = blockIdx.x * tokens_per_wg;
  move_rows<T, true>(p, t0, min(tokens_per_wg, p.total_tokens - t0), (f32x2*)smem);
}

// ---- pools of 8-bit floats

// Biased exponent of the scale for values of at most `top` (its bits; more than those of an infinity: NaN): the smallest 2^e with top <= 448 2^e = 1.75 * 2^(e + 8)
__device__ inline int scale_exponent(unsigned top) {
  if (top >= 0x7f800000u) return 255;
  return max((int)((top + 0x1fffffu) >> 23) - 8, 1);
}
__device__ inline unsigned wave_max(unsigned x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, (unsigned)__shfl_xor((int)x, o));
  return x;
}
__device__ inline float scale_of(int e) { return e == 255 ? __builtin_nanf("") : float_of((unsigned)e << 23); }
// four bytes times 2^-shift, rounded
__device__ inline unsigned rescaled(unsigned x, int shift) {
  float v[4];
  v[0] = __builtin_amdgcn_cvt_f32_fp8((int)x, 0);
  v[1] = __builtin_amdgcn_cvt_f32_fp8((int)x, 1);
  v[2] = __builtin_amdgcn_cvt_f32_fp8((int)x, 2);
  v[3] = __builtin_amdgcn_cvt_f32_fp8((int)x, 3);
#pragma unroll
  for (int i = 0; i < 4; i++) v[i] = __builtin_amdgcn_ldexpf(v[i], -shift);
  return e4m3::pack4(v[0], v[1], v[2], v[3]);
}

// One (block, head) at a time for a wave.  Tokens [a, e) of the block are new, those in front of a stay (at the larger scale), those behind e become zeros.
template <int DP>
__device__ inline void block_k(const KvAppendParams& p, const unsigned char* src, unsigned char* tile, float* scale, int a, int e, const f32x2* cs) {
  constexpr int NC = DP / 64;                                  // pairs of 8-element chunks that a lane has
  const int lane = threadIdx.x & 63, t = lane >> 2, D = p.head_dim;
  const bool is_new = t >= a && t < e;
  float x[NC][2][8];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < NC; i++)
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int ch = 8 * i + 2 * (lane & 3) + h;
#pragma unroll
      for (int k = 0; k < 8; k++) x[i][h][k] = 0.f;
      if (is_new && 8 * ch < D) rotated<uint16_t>(p.rope, src + (t - a) * p.k_row, ch, cs + (t - a) * p.rope.half, x[i][h]);
#pragma unroll
      for (int k = 0; k < 8; k++) top = max(top, bits_of(x[i][h][k]) & 0x7fffffffu);
    }
  int ex = scale_exponent(wave_max(top)), before = 0;
  if (a > 0) {
    before = (int)(bits_of(*scale) >> 23) & 255;
    ex = max(ex, before);
  }
#pragma unroll
  for (int i = 0; i < NC; i++) {
    const int d = 64 * i + 16 * (lane & 3);
    if (d >= D) continue;
    u32x4* at = (u32x4*)(tile + t * D + d);
    u32x4 y = {0u, 0u, 0u, 0u};
    if (ex != 255) {
      if (is_new) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; k++) v[k] = __builtin_amdgcn_ldexpf(x[i][h][k], 127 - ex);
          y[2 * h] = e4m3::pack4(v[0], v[1], v[2], v[3]);
          y[2 * h + 1] = e4m3::pack4(v[4], v[5], v[6], v[7]);
        }
      } else if (t < a) {
        y = *at;
        if (ex != before) {
#pragma unroll
          for (int k = 0; k < 4; k++) y[k] = rescaled(y[k], ex - before);
        }
      }
    }
    *at = y;
  }
  if (lane == 0) *scale = scale_of(ex);
}

template <int DP>
__device__ inline void block_v(const KvAppendParams& p, const unsigned char* src, unsigned char* tile, float* scale, int a, int e) {
  constexpr int ND = (DP + 127) / 128;                         // pairs of neighbouring d that a lane has
  const int lane = threadIdx.x & 63, D = p.head_dim;
  unsigned x[ND][16];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < ND; i++)
#pragma unroll
    for (int t = 0; t < 16; t++) {
      const int d = 128 * i + 2 * lane;
      x[i][t] = t >= a && t < e && d < D ? *(const unsigned*)(src + (t - a) * p.v_row + 2 * d) : 0u;
    }
#pragma unroll
  for (int i = 0; i < ND; i++)
#pragma unroll
    for (int t = 0; t < 16; t++) top = max(max(top, x[i][t] & 0x7fff0000u), x[i][t] << 16 & 0x7fff0000u);
  int ex = scale_exponent(wave_max(top)), before = 0;
  if (a > 0) {
    before = (int)(bits_of(*scale) >> 23) & 255;
    ex = max(ex, before);
  }
#pragma unroll
  for (int i = 0; i < ND; i++) {
    const int d = 128 * i + 2 * lane;
    if (d >= D) continue;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      u32x4* at = (u32x4*)(tile + 16 * (d + h));
      u32x4 y = {0u, 0u, 0u, 0u}, old = y;
      if (a > 0) old = *at;
      if (ex != 255) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; j++) v[j] = __builtin_amdgcn_ldexpf(float_of(h ? x[i][4 * k + j] & 0xffff0000u : x[i][4 * k + j] << 16), 127 - ex);
          const unsigned now = e4m3::pack4(v[0], v[1], v[2], v[3]);
          const int n_old = min(max(a - 4 * k, 0), 4);         // of these four
          unsigned was = old[k];
          if (ex != before && n_old) was = rescaled(was, ex - before);
          const unsigned keep = n_old == 4 ? 0xffffffffu : (1u << 8 * n_old) - 1;
          y[k] = (was & keep) | (now & ~keep);
        }
      }
      *at = y;
    }
  }
  if (lane == 0) *scale = scale_of(ex);
}

template <int DP>
__global__ void __launch_bounds__(kThreads) append_e4m3_kernel(KvAppendParams p, int kv_wgs, int heads_per_wg, int tokens_per_wg) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  f32x2* const cs = (f32x2*)smem;
  if ((int)blockIdx.x >= kv_wgs) {
    const int t0 = ((int)blockIdx.x - kv_wgs) * tokens_per_wg;
    move_rows<uint16_t, false>(p, t0, min(tokens_per_wg, p.total_tokens - t0), cs);
    return;
  }
  const int groups = (p.n_kv_heads + heads_per_wg - 1) / heads_per_wg;
  const int blk = blockIdx.x / groups, h0 = (blockIdx.x % groups) * heads_per_wg;
  int r = 0;                                                   // the last request that writes a block at or before this one
  for (int end = p.n_reqs; end - r > 1;) {
    const int mid = (r + end) / 2;
    if (blk >= p.touched[mid]) r = mid;
    else end = mid;
  }
  const ReqDesc rd = p.reqs[r];
  const int b = rd.prefix_len / kBlockTokens + blk - p.touched[r];
  const int first = max(rd.prefix_len, kBlockTokens * b), a = first - kBlockTokens * b;
  const int e = min(kBlockTokens, rd.prefix_len + rd.suffix_len - kBlockTokens * b);
  const int tok = rd.q_off + first - rd.prefix_len, half = p.rope.half;
  for (int i = threadIdx.x; i < (e - a) * half; i += kThreads) {
    const int t = i / half;
    cs[i] = cos_sin(p.rope, p.rope.positions ? p.rope.positions[tok + t] : first + t, i - t * half);
  }
  __syncthreads();
  const E4m3Block lay = e4m3_block(p.n_kv_heads, p.head_dim);
  unsigned char* const at = p.pool_layer + (uint64_t)(unsigned)p.tables[rd.table_off + b] * lay.bytes;
  float* const scales = (float*)(at + lay.scales);
  const unsigned char *k = (const unsigned char*)p.k + tok * p.k_row, *v = (const unsigned char*)p.v + tok * p.v_row;
  for (int h = h0 + (int)(threadIdx.x >> 6); h < min(h0 + heads_per_wg, p.n_kv_heads); h += kThreads / 64) {
    block_k<DP>(p, k + 2 * h * p.head_dim, at + h * lay.tile, scales + h, a, e, cs);
    block_v<DP>(p, v + 2 * h * p.head_dim, at + lay.v + h * lay.tile, scales + p.n_kv_heads + h, a, e);
  }
}

}  // namespace append

hipError_t launch_kv_append(const KvAppendParams& p, int dtype, int n_cus, hipStream_t stream) {
  using namespace append;
  if (p.total_tokens <= 0 || (!p.q && !p.k)) return hipSuccess;
  const int half = p.rope.half;
  // a workgroup's tokens share their angles' start-up; few tokens are spread over the chip
  const int tokens_per_wg = p.total_tokens >= 16 * n_cus ? 4 : 1;
  const unsigned row_wgs = (unsigned)((p.total_tokens + tokens_per_wg - 1) / tokens_per_wg);
  if (dtype != CALVO_E4M3) {
    const size_t lds = (size_t)tokens_per_wg * half * sizeof(attn::f32x2);
    if (dtype == CALVO_F32) hipLaunchKernelGGL(append_kernel<float>, dim3(row_wgs), dim3(kThreads), lds, stream, p, tokens_per_wg);
    else hipLaunchKernelGGL(append_kernel<uint16_t>, dim3(row_wgs), dim3(kThreads), lds, stream, p, tokens_per_wg);
    return hipGetLastError();
  }
  const int heads_per_wg = 4;
  const int groups = (p.n_kv_heads + heads_per_wg - 1) / heads_per_wg;
  const int kv_wgs = p.k ? p.n_touched * groups : 0;
  const unsigned grid = (unsigned)kv_wgs + (p.q ? row_wgs : 0);
  const size_t lds = (size_t)kBlockTokens * half * sizeof(attn::f32x2);
  if (p.head_dim <= 64) hipLaunchKernelGGL(append_e4m3_kernel<64>, dim3(grid), dim3(kThreads), lds, stream, p, kv_wgs, heads_per_wg, tokens_per_wg);
  else if (p.head_dim <= 128) hipLaunchKernelGGL(append_e4m3_kernel<128>, dim3(grid), dim3(kThreads), lds, stream, p, kv_wgs, heads_per_wg, tokens_per_wg);
  else hipLaunchKernelGGL(append_e4m3_kernel<256>, dim3(grid), dim3(kThreads), lds, stream, p, kv_wgs, heads_per_wg, tokens_per_wg);
  return hipGetLastError();
}

}  // namespace calvo
