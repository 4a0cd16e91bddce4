// The pool of CALVO_E4M3: where things are in a block, and its numbers on the device.
#pragma once
#include <stdint.h>

#include "attn_common.h"

namespace calvo {

// A block: K [heads][16][D] bytes, V [heads][D][16] bytes, scales fp32 [K, V][heads], up to a whole cache line.  V lies with a d's tokens side by
// side because that is the operand order of the product weights x V, in which a lane holds one d and several keys: 16 bytes of V are 16 keys for a
// lane, and nothing has to be transposed between the pool and the matrix pipes.  K's operand has a key per lane and several d.
struct E4m3Block {
  uint32_t tile;      // bytes of one head's K or V
  uint32_t v;         // where V begins
  uint32_t scales;
  uint64_t bytes;
};
__host__ __device__ inline E4m3Block e4m3_block(int n_kv_heads, int head_dim) {
  const uint32_t tile = 16u * (uint32_t)head_dim, half = (uint32_t)n_kv_heads * tile;
  return {tile, half, 2 * half, ((uint64_t)2 * half + 8u * (uint32_t)n_kv_heads + 127) / 128 * 128};
}

namespace e4m3 {
using namespace attn;

// by value: __builtin_bit_cast applied to an element of a vector reads element 0 with this compiler
__device__ inline unsigned bits_of(float x) { return __builtin_bit_cast(unsigned, x); }
__device__ inline float float_of(unsigned x) { return __builtin_bit_cast(float, x); }

// Eight bytes times 2^(exponent of s), exact in bf16, whose eight significant bits hold four, but for values below its normal range or beyond its
// largest.  An exponent of ones makes NaN of every byte.
__device__ inline bf16x8 widen(unsigned a, unsigned b, float s) {
  const unsigned x[4] = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true))};
  return __builtin_bit_cast(bf16x8, (u32x4){x[0], x[1], x[2], x[3]});
}

// four numbers of at most 448, rounded to nearest even
__device__ inline unsigned pack4(float a, float b, float c, float d) {
  int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
}

// bytes that are NaN (0x7f, 0xff), marked in their upper bits
__device__ inline unsigned nan_bytes(unsigned x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// scales from 2^120 on, against which bytes of 256 and more are infinite in bf16, and those that are NaN themselves
__device__ inline bool may_not_be_finite(float s) { return (bits_of(s) & 0x7f800000u) >= (247u << 23); }

}  // namespace e4m3
}  // namespace calvo
