// New tokens into the paged pool, Q and K rotated by position on the way (calvo_kv_append).
//
// Rotation of a head x at position p: a_i = p f_i for i < R / 2, and for every pair (x, y) of elements - i and i + R / 2, or 2i and 2i + 1 -
//     x' = x cos a_i - y sin a_i,   y' = y cos a_i + x sin a_i;
// elements from R on stay.  Far positions lose an angle in 32 bits (at position 10^6 the fastest pair would be off by 0.03 of a radian): it is made in 64
// bits as a number of turns, whose fraction is exact enough in 32.  One rounding at the end, of the sum.
//
// Bound by the bytes of the rows, and for few tokens by a chain of waits (launch, a token's place, angles, store: 3.8 us).  Rows of K, V and q are moved in chunks
// of 16 bytes a lane, a workgroup to a token or four, whose angles it makes once into LDS.  Into an 8-bit pool a block is written whole, since its scale
// depends on all of its tokens: a wave has K or V of one (block, head) in registers, finds the largest value, and stores bytes in the order that attention
// reads (K by token; V by element, so that a lane has two elements of all 16 tokens and turns nothing around).  What a block holds already is asked for with the
// new values.  us of a call, 32Q/8KV, D = 128, all of a head rotated: 8000 tokens bf16 31.7 (6.2 TB/s), fp32 74.6 (5.3), 8 bits 31.5 (5.7); 32 requests of one
// token 4.6, a single one 4.6 (of the kernel 4.5 and 3.8).
#include "../../include/calvo.h"
#include "kv_e4m3.h"

namespace calvo {
namespace append {

using namespace attn;
using e4m3::bits_of;
using e4m3::float_of;

// The last of n requests whose entry is at or below x (entries ascend, the first is): 64 of them at a time, for a whole wave
template <typename F>
__device__ inline int last_at_or_below(int n, int x, F&& entry) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int stride = (n + 63) / 64, i = lane * stride;
    const int c = __popcll(__builtin_amdgcn_ballot_w64(i < n && entry(lo + min(i, n - 1)) <= x));
    const int skip = (c - 1) * stride;
    lo += skip;
    n = min(stride, n - skip);
  }
  return lo;
}

__device__ inline f32x2 cos_sin(const RopeParams& rope, int pos, int i) {
  const double turns = (double)pos * ((double)rope.inv_freq[i] * 0.15915494309189533577);
  float s, c;
  sincospif((float)(2. * (turns - __builtin_rint(turns))), &s, &c);
  return (f32x2){c, s};
}

// Where pair i of a token is in LDS, and pairs from one token to the next.  Lanes that read at once have four chunks of a row 128 bytes apart and some tokens:
// rows of whole bank sets would put all of these on one bank (8000 tokens into an 8-bit pool, 32Q/8KV, D = 128: the blocks' launch 20.7 / 12.8 us).  An
// element more for every 32 and rows of 2 mod 4 elements spread them.
__host__ __device__ inline int angle_at(int i) { return i + (i >> 5); }
__host__ __device__ inline int angle_row(int half) { return (half + (half >> 5) + 1) / 4 * 4 + 2; }

// Where element d's partner is, of pairs (i, i + half); an element that is not rotated is its own
__device__ inline int partner(const RopeParams& rope, int d) { return d < rope.half ? d + rope.half : d < rope.rot ? d - rope.half : d; }

// 16 bytes of a head's row as numbers, and back
template <typename T>
struct Chunk;
template <>
struct Chunk<uint16_t> {
  static constexpr int N = 8;
  static __device__ float number(const u32x4& v, int k) { return float_of(k & 1 ? v[k >> 1] & 0xffff0000u : v[k >> 1] << 16); }
  // the partners of chunk elements d0 ...; two at a time where halves are even
  static __device__ u32x4 partners(const RopeParams& rope, const unsigned char* row, int d0) {
    u32x4 y;
    const unsigned short* x = (const unsigned short*)row;
    if (rope.half % 2 == 0) {
#pragma unroll
      for (int i = 0; i < 4; i++) y[i] = *(const unsigned*)(x + partner(rope, d0 + 2 * i));
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) y[i] = x[partner(rope, d0 + 2 * i)] | (unsigned)x[partner(rope, d0 + 2 * i + 1)] << 16;
    }
    return y;
  }
  static __device__ u32x4 packed(const float (&x)[8]) { return (u32x4){pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])}; }
};
template <>
struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ float number(const u32x4& v, int k) { return float_of(v[k]); }
  static __device__ u32x4 partners(const RopeParams& rope, const unsigned char* row, int d0) {
    u32x4 y;
#pragma unroll
    for (int i = 0; i < 4; i++) y[i] = ((const unsigned*)row)[partner(rope, d0 + i)];
    return y;
  }
  static __device__ u32x4 packed(const float (&x)[4]) { return (u32x4){bits_of(x[0]), bits_of(x[1]), bits_of(x[2]), bits_of(x[3])}; }
};

// How pairs lie in 16-byte chunks: none is rotated, a pair's elements are in the same places of two chunks, those two belong to one lane (of a block in 8 bits),
// they are neighbours, or anywhere
enum { kNone, kHalves, kWhole, kNeighbours, kAnywhere };

// Chunk ch of a head's row, rotated.  cs: (cos, sin) of the token's pairs.  Both elements of its pairs are asked for before either is waited for.
template <typename T, int MODE>
__device__ inline void rotated(const RopeParams& rope, const unsigned char* row, int ch, const f32x2* cs, float (&x)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
  const int d0 = ch * N;
  const bool lower = d0 < rope.half;
  const u32x4 own = *(const u32x4*)(row + 16 * ch);
  u32x4 other = own;
  if (MODE == kHalves && d0 < rope.rot) other = *(const u32x4*)(row + 16 * ch + (lower ? rope.half : -rope.half) * (int)sizeof(T));
  if (MODE == kAnywhere && d0 < rope.rot) other = Chunk<T>::partners(rope, row, d0);
#pragma unroll
  for (int i = 0; i < N; i++) x[i] = Chunk<T>::number(own, i);
  if (MODE == kNone || d0 >= rope.rot) return;
  if constexpr (MODE == kNeighbours) {
    const f32x2* t = cs + angle_at(d0 >> 1);
#pragma unroll
    for (int i = 0; i < N; i += 2)
      if (d0 + i < rope.rot) {
        const float a = x[i], b = x[i + 1];
        x[i] = a * t[i >> 1][0] - b * t[i >> 1][1];
        x[i + 1] = b * t[i >> 1][0] + a * t[i >> 1][1];
      }
  } else if constexpr (MODE == kHalves) {
    const f32x2* t = cs + angle_at(lower ? d0 : d0 - rope.half);
#pragma unroll
    for (int i = 0; i < N; i++) {
      const float o = Chunk<T>::number(other, i);
      x[i] = x[i] * t[i][0] + (lower ? -o : o) * t[i][1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i++) {
      const int d = d0 + i;
      const bool first = d < rope.half;
      const f32x2 t = cs[angle_at(min(first ? d : d - rope.half, rope.half - 1))];
      const float o = Chunk<T>::number(other, i);
      if (d < rope.rot) x[i] = x[i] * t[0] + (first ? -o : o) * t[1];
    }
  }
}

constexpr int kThreads = 256, kMostTokens = 4;       // of a workgroup: one wave finds the place of each

// Rows of tokens [t0, t0 + n): q -> q_out, and where the pool holds the same type k and v -> pool.  cs: room for n rows of angles.
template <typename T, bool KV, int MODE>
__device__ inline void move_rows(const KvAppendParams& p, int t0, int n, f32x2* cs) {
  constexpr int N = Chunk<T>::N;
  __shared__ int pos_of[kMostTokens];
  __shared__ int64_t row_of[kMostTokens];                      // of the pool, in tokens from its first one (K of a block, then its V)
  const int half = p.rope.half, wave = threadIdx.x >> 6;
  if (wave < n) {
    const int tok = t0 + wave;
    const ReqDesc rd = p.reqs[last_at_or_below(p.n_reqs, tok, [&](int r) { return p.reqs[r].q_off; })];
    const int pos = rd.prefix_len + (tok - rd.q_off);
    if ((threadIdx.x & 63) == 0) {
      pos_of[wave] = p.rope.positions ? p.rope.positions[tok] : pos;
      if constexpr (KV) row_of[wave] = (int64_t)p.tables[rd.table_off + pos / kBlockTokens] * 2 * kBlockTokens + pos % kBlockTokens;
    }
  }
  __syncthreads();
  const int cs_row = angle_row(half);
  if constexpr (MODE != kNone) {
    for (int i = threadIdx.x; i < n * half; i += kThreads) cs[i / half * cs_row + angle_at(i % half)] = cos_sin(p.rope, pos_of[i / half], i % half);
    __syncthreads();
  }
  const int chunks = p.head_dim / N, row_chunks = p.n_kv_heads * chunks;
  const int nq = p.q ? p.n_q_heads * chunks : 0, nk = KV && p.k ? row_chunks : 0;
  const int all = nq + 2 * nk;
  for (int i = threadIdx.x; i < n * all; i += kThreads) {
    const int t = i / all, j = i - t * all, tok = t0 + t;
    if (j < nq) {
      float x[N];
      rotated<T, MODE>(p.rope, (const unsigned char*)p.q + tok * p.q_row + (j / chunks) * p.head_dim * (int)sizeof(T), j % chunks, cs + t * cs_row, x);
      ((u32x4*)p.q_out)[(int64_t)tok * nq + j] = Chunk<T>::packed(x);
    } else if constexpr (KV) {
      const int k = j - nq;
      u32x4* dst = (u32x4*)p.pool_layer + row_of[t] * row_chunks;
      if (k < nk) {
        float x[N];
        rotated<T, MODE>(p.rope, (const unsigned char*)p.k + tok * p.k_row + (k / chunks) * p.head_dim * (int)sizeof(T), k % chunks, cs + t * cs_row, x);
        dst[k] = Chunk<T>::packed(x);
      } else {
        dst[kBlockTokens * row_chunks + k - nk] = *(const u32x4*)((const unsigned char*)p.v + tok * p.v_row + 16 * (k - nk));
      }
    }
  }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(kThreads) append_kernel(KvAppendParams p, int tokens_per_wg) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int t0 = blockIdx.x * tokens_per_wg;
  move_rows<T, true, MODE>(p, t0, min(tokens_per_wg, p.total_tokens - t0), (f32x2*)smem);
}

template <int MODE>
__global__ void __launch_bounds__(kThreads) append_q_kernel(KvAppendParams p, int tokens_per_wg) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int t0 = blockIdx.x * tokens_per_wg;
  move_rows<uint16_t, false, MODE>(p, t0, min(tokens_per_wg, p.total_tokens - t0), (f32x2*)smem);
}

// ---- pools of 8-bit floats

// Biased exponent of the scale for values of at most `top` (its bits; more than those of an infinity: NaN): the smallest 2^e with top <= 448 2^e = 1.75 * 2^(e + 8)
__device__ inline int scale_exponent(unsigned top) {
  if (top >= 0x7f800000u) return 255;
  return max((int)((top + 0x1fffffu) >> 23) - 8, 1);
}
// largest of the wave's (of each of 16 lanes by rotations in the vector ALU, then of the four rows)
__device__ inline unsigned wave_max(unsigned x) {
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));   // row_ror:1, 2, 4, 8
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));
  unsigned a = x, b = x;
  row_swap(a, b);
  a = b = max(a, b);
  float fa = float_of(a), fb = float_of(b);
  half_swap(fa, fb);
  return max(bits_of(fa), bits_of(fb));
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

__device__ inline float number(const u32x4& v, int k) { return Chunk<uint16_t>::number(v, k); }

// K or V of one (block, head) for a wave.  Tokens [a, e) of the block are new, those in front of a stay (at the larger scale), those behind e become
// zeros.  What the block holds is asked for first: it is there when the new values' scale is known.
template <int DP, int MODE>
struct BlockK {
  static constexpr int NC = DP / 64;                           // pairs of 8-element chunks that a lane has
  u32x4 y[NC], own[NC][2], other[NC][2];
  float old_scale;

  __device__ void ask(const KvAppendParams& p, const unsigned char* src, const unsigned char* tile, const float* scale, int a, int e) {
    const int lane = threadIdx.x & 63, t = lane >> 2, D = p.head_dim, rot = p.rope.rot, half = p.rope.half;
    const unsigned char* row = src + (t - a) * p.k_row;
    old_scale = a > 0 ? *scale : 0.f;
#pragma unroll
    for (int i = 0; i < NC; i++) {
      const int d = 64 * i + 16 * (lane & 3);
      y[i] = (u32x4){0u, 0u, 0u, 0u};
      if (t < a && d < D) y[i] = *(const u32x4*)(tile + t * D + d);
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int d0 = d + 8 * h;
        own[i][h] = other[i][h] = (u32x4){0u, 0u, 0u, 0u};
        if (t >= a && t < e && d < D) {
          own[i][h] = *(const u32x4*)(row + 2 * d0);
          if (MODE == kHalves && d0 < rot) other[i][h] = *(const u32x4*)(row + 2 * (d0 < half ? d0 + half : d0 - half));
          if (MODE == kAnywhere && d0 < rot) other[i][h] = Chunk<uint16_t>::partners(p.rope, row, d0);
        }
      }
    }
  }

  __device__ void store(const KvAppendParams& p, unsigned char* tile, float* scale, int a, int e, const f32x2* cs) {
    const int lane = threadIdx.x & 63, t = lane >> 2, D = p.head_dim, rot = p.rope.rot, half = p.rope.half;
    const bool is_new = t >= a && t < e;
    const f32x2* my_cs = cs + (t - a) * angle_row(half);
    float x[NC][2][8];
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < NC; i++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int d0 = 64 * i + 16 * (lane & 3) + 8 * h;
#pragma unroll
        for (int k = 0; k < 8; k++) x[i][h][k] = number(own[i][h], k);
        if (MODE != kNone && is_new && d0 < rot) {
          const bool lower = d0 < half;
          if constexpr (MODE == kHalves || MODE == kWhole) {
            const f32x2* c2 = my_cs + angle_at(lower ? d0 : d0 - half);
#pragma unroll
            for (int k = 0; k < 8; k++) {
              const float o = number(MODE == kWhole ? own[(i + NC / 2) % NC][h] : other[i][h], k);
              x[i][h][k] = x[i][h][k] * c2[k][0] + (lower ? -o : o) * c2[k][1];
            }
          } else if constexpr (MODE == kNeighbours) {
            const f32x2* c2 = my_cs + angle_at(d0 >> 1);
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
              const float u = x[i][h][k], v = x[i][h][k + 1];
              if (d0 + k < rot) {
                x[i][h][k] = u * c2[k >> 1][0] - v * c2[k >> 1][1];
                x[i][h][k + 1] = v * c2[k >> 1][0] + u * c2[k >> 1][1];
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < 8; k++) {
              const int d = d0 + k;
              const bool first = d < half;
              const f32x2 c = my_cs[angle_at(min(first ? d : d - half, half - 1))];
              const float o = number(other[i][h], k);
              if (d < rot) x[i][h][k] = x[i][h][k] * c[0] + (first ? -o : o) * c[1];
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 8; k++) top = max(top, bits_of(x[i][h][k]) & 0x7fffffffu);
        __builtin_amdgcn_sched_barrier(0);
      }
    const int before = (int)(bits_of(old_scale) >> 23) & 255, ex = max(scale_exponent(wave_max(top)), before);
#pragma unroll
    for (int i = 0; i < NC; i++) {
      const int d = 64 * i + 16 * (lane & 3);
      if (is_new) {
#pragma unroll
        for (int h = 0; h < 2; h++) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 8; k++) v[k] = __builtin_amdgcn_ldexpf(x[i][h][k], 127 - ex);
          y[i][2 * h] = e4m3::pack4(v[0], v[1], v[2], v[3]);
          y[i][2 * h + 1] = e4m3::pack4(v[4], v[5], v[6], v[7]);
        }
      } else if (t < a && ex != before) {
#pragma unroll
        for (int k = 0; k < 4; k++) y[i][k] = rescaled(y[i][k], ex - before);
      }
      if (ex == 255) y[i] = (u32x4){0u, 0u, 0u, 0u};
      if (d < D) *(u32x4*)(tile + t * D + d) = y[i];
    }
    if (lane == 0) *scale = scale_of(ex);
  }
};

template <int DP>
struct BlockV {
  static constexpr int ND = (DP + 127) / 128;                  // pairs of neighbouring d that a lane has
  u32x4 old[ND][2];
  unsigned x[ND][16];
  float old_scale;

  __device__ void ask(const KvAppendParams& p, const unsigned char* src, const unsigned char* tile, const float* scale, int a, int e) {
    const int lane = threadIdx.x & 63, D = p.head_dim;
    old_scale = a > 0 ? *scale : 0.f;
#pragma unroll
    for (int i = 0; i < ND; i++) {
      const int d = 128 * i + 2 * lane;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        old[i][h] = (u32x4){0u, 0u, 0u, 0u};
        if (a > 0 && d < D) old[i][h] = *(const u32x4*)(tile + 16 * (d + h));
      }
#pragma unroll
      for (int t = 0; t < 16; t++) x[i][t] = t >= a && t < e && d < D ? *(const unsigned*)(src + (t - a) * p.v_row + 2 * d) : 0u;
    }
  }

  __device__ void store(const KvAppendParams& p, unsigned char* tile, float* scale, int a) {
    const int lane = threadIdx.x & 63, D = p.head_dim;
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < ND; i++)
#pragma unroll
      for (int t = 0; t < 16; t++) top = max(max(top, x[i][t] & 0x7fff0000u), x[i][t] << 16 & 0x7fff0000u);
    const int before = (int)(bits_of(old_scale) >> 23) & 255, ex = max(scale_exponent(wave_max(top)), before);
#pragma unroll
    for (int i = 0; i < ND; i++) {
      const int d = 128 * i + 2 * lane;
      if (d >= D) continue;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        u32x4 y;
#pragma unroll
        for (int k = 0; k < 4; k++) {
          float v[4];
#pragma unroll
          for (int j = 0; j < 4; j++) v[j] = __builtin_amdgcn_ldexpf(float_of(h ? x[i][4 * k + j] & 0xffff0000u : x[i][4 * k + j] << 16), 127 - ex);
          const int n_old = min(max(a - 4 * k, 0), 4);           // of these four
          unsigned was = old[i][h][k];
          if (ex != before && n_old) was = rescaled(was, ex - before);
          const unsigned keep = n_old == 4 ? 0xffffffffu : (1u << 8 * n_old) - 1;
          y[k] = ex == 255 ? 0u : (was & keep) | (e4m3::pack4(v[0], v[1], v[2], v[3]) & ~keep);
        }
        *(u32x4*)(tile + 16 * (d + h)) = y;
      }
    }
    if (lane == 0) *scale = scale_of(ex);
  }
};

// as many as leave every instantiation its registers
constexpr int waves_per_simd(int dp, int mode) {
  if (dp > 128) return mode == kHalves || mode == kAnywhere ? 1 : 2;
  return mode == kAnywhere ? 2 : mode == kHalves && dp > 64 ? 3 : 4;
}

// The workgroups of the first kv_wgs take a touched block and heads_per_wg heads each, a wave K or V of a head at a time; the others rows of q.
template <int DP, int MODE>
__global__ void __launch_bounds__(kThreads, waves_per_simd(DP, MODE)) append_e4m3_kernel(KvAppendParams p, int kv_wgs, int heads_per_wg, int tokens_per_wg) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  f32x2* const cs = (f32x2*)smem;
  if ((int)blockIdx.x >= kv_wgs) {
    const int t0 = ((int)blockIdx.x - kv_wgs) * tokens_per_wg;
    move_rows<uint16_t, false, MODE == kWhole ? (int)kHalves : MODE>(p, t0, min(tokens_per_wg, p.total_tokens - t0), cs);
    return;
  }
  const int groups = (p.n_kv_heads + heads_per_wg - 1) / heads_per_wg;
  const int h0 = (blockIdx.x % groups) * heads_per_wg;
  const const_i32p item = (const_i32p)(uintptr_t)(p.touched + blockIdx.x / groups);
  const int slot = item[0], tok = item[1], first = item[2], a = item[3] & 255, e = item[3] >> 8;
  const E4m3Block lay = e4m3_block(p.n_kv_heads, p.head_dim);
  unsigned char* const at = p.pool_layer + (uint64_t)(unsigned)slot * lay.bytes;
  float* const scales = (float*)(at + lay.scales);
  const unsigned char *k = (const unsigned char*)p.k + tok * p.k_row, *v = (const unsigned char*)p.v + tok * p.v_row;
  const int u0 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = p.rope.half;
  // All waves meet once, before they part for K and V.  (A barrier in either part, behind the first unit's loads: 8000 tokens, 32Q/8KV, D = 128 32.2 / 31.5 us, a
  // single token's kernel 3.6 / 3.8, 32 requests' 4.5 / 4.5)
  for (int i = threadIdx.x; MODE != kNone && i < (e - a) * half; i += kThreads) {
    const int t = i / half, j = i - t * half;
    cs[t * angle_row(half) + angle_at(j)] = cos_sin(p.rope, p.rope.positions ? p.rope.positions[tok + t] : first + t, j);
  }
  __syncthreads();
  // unit u: K (u even) or V of head h0 + u / 2; a wave has units of one kind.  The next one's values are on their way while one is stored.
  const int units = 2 * (min(h0 + heads_per_wg, p.n_kv_heads) - h0);
  auto all_units = [&](auto&& here, auto&& next, auto&& ask, auto&& store) {
    if (u0 < units) ask(here, h0 + (u0 >> 1));
    for (int u = u0; u < units; u += kThreads / 64) {
      const bool more = u + kThreads / 64 < units;
      if (more) ask(next, h0 + (u >> 1) + kThreads / 128);
      store(here, h0 + (u >> 1));
      if (more) here = next;
    }
  };
  if (u0 & 1) {
    BlockV<DP> here, next;
    all_units(here, next, [&](auto& x, int h) { x.ask(p, v + 2 * h * p.head_dim, at + lay.v + h * lay.tile, scales + p.n_kv_heads + h, a, e); },
              [&](auto& x, int h) { x.store(p, at + lay.v + h * lay.tile, scales + p.n_kv_heads + h, a); });
  } else {
    BlockK<DP, MODE> here, next;
    all_units(here, next, [&](auto& x, int h) { x.ask(p, k + 2 * h * p.head_dim, at + h * lay.tile, scales + h, a, e); },
              [&](auto& x, int h) { x.store(p, at + h * lay.tile, scales + h, a, e, cs); });
  }
}

}  // namespace append

hipError_t launch_kv_append(const KvAppendParams& p, int dtype, int n_cus, hipStream_t stream) {
  using namespace append;
  if (p.total_tokens <= 0 || (!p.q && !p.k)) return hipSuccess;
  const int half = p.rope.half, per_chunk = dtype == CALVO_F32 ? 4 : 8;
  // Several tokens share a workgroup's start where there are many and their rows leave its threads few chunks each.  One / four to a workgroup, us of the launch:
  // bf16, 8000 tokens, 8Q/8KV, D = 64 13.8 / 11.6, 32Q/8KV 20.4 / 18.6, D = 128 32.5 / 33.0, D = 256 76.5 / 83.7; 600 tokens, D = 128 6.1 / 10.6
  const bool many = p.total_tokens >= 16 * n_cus;
  const int row_chunks = ((p.q ? p.n_q_heads : 0) + (p.k && dtype != CALVO_E4M3 ? 2 * p.n_kv_heads : 0)) * p.head_dim / per_chunk;
  const int tokens_per_wg = many && row_chunks <= 2 * kThreads ? kMostTokens : 1;
  const unsigned row_wgs = (unsigned)((p.total_tokens + tokens_per_wg - 1) / tokens_per_wg);
  const size_t angles = (size_t)angle_row(half) * sizeof(attn::f32x2);
  const int mode = p.rope.rot == 0 ? kNone : p.rope.interleaved ? kNeighbours : half % per_chunk ? kAnywhere : kHalves;
  auto with_mode = [&](auto&& f) {
    if (mode == kNone) f(attn::Tag<kNone>{});
    else if (mode == kHalves) f(attn::Tag<kHalves>{});
    else if (mode == kNeighbours) f(attn::Tag<kNeighbours>{});
    else f(attn::Tag<kAnywhere>{});
  };
  if (dtype != CALVO_E4M3) {
    with_mode([&](auto m) {
      constexpr int M = decltype(m)::value;
      if (dtype == CALVO_F32) hipLaunchKernelGGL((append_kernel<float, M>), dim3(row_wgs), dim3(kThreads), tokens_per_wg * angles, stream, p, tokens_per_wg);
      else hipLaunchKernelGGL((append_kernel<uint16_t, M>), dim3(row_wgs), dim3(kThreads), tokens_per_wg * angles, stream, p, tokens_per_wg);
    });
    return hipGetLastError();
  }
  // a wave for each K and V of a head where blocks are few; else a block's angles are made once for eight heads (two / eight, 32Q/8KV, D = 128: 1 token 4.0 / 7.4,
  // 1000 8.3 / 11.2, 4000 23.7 / 20.4; 8Q/8KV, D = 64, 2000 tokens 7.2 / 9.8)
  const int heads_per_wg = (int64_t)p.n_touched * p.n_kv_heads <= 4 * n_cus ? 2 : 8;
  const int groups = (p.n_kv_heads + heads_per_wg - 1) / heads_per_wg;
  const int kv_wgs = p.k ? p.n_touched * groups : 0;
  // Many wide rows of q go by themselves: beside the blocks of such heads they would have two waves to a SIMD (8000 tokens, 32Q/8KV, a launch of their own / one
  // launch: D = 256 83 / 114, D = 128 36.5 / 33.9, D = 64 24.8 / 19.4)
  const bool apart = p.q && kv_wgs && many && p.head_dim > 128;
  if (apart)
    with_mode([&](auto m) {
      hipLaunchKernelGGL(append_q_kernel<decltype(m)::value>, dim3(row_wgs), dim3(kThreads), tokens_per_wg * angles, stream, p, tokens_per_wg);
    });
  const unsigned grid = (unsigned)kv_wgs + (p.q && !apart ? row_wgs : 0);
  auto launch = [&](auto dp, auto m) {
    hipLaunchKernelGGL((append_e4m3_kernel<decltype(dp)::value, decltype(m)::value>), dim3(grid), dim3(kThreads), kBlockTokens * angles, stream, p, kv_wgs,
                       heads_per_wg, tokens_per_wg);
  };
  auto with_width = [&](auto dp) {
    if constexpr (decltype(dp)::value > 64) {                  // a lane of narrower heads has no chunk of its other half
      if (mode == kHalves && half == decltype(dp)::value / 2) return launch(dp, attn::Tag<kWhole>{});
    }
    with_mode([&](auto m) { launch(dp, m); });
  };
  if (p.head_dim <= 64) with_width(attn::Tag<64>{});
  else if (p.head_dim <= 128) with_width(attn::Tag<128>{});
  else with_width(attn::Tag<256>{});
  return hipGetLastError();
}

}  // namespace calvo
