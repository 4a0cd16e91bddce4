// Eviction from the paged cache by gathered attention weight (calvo_kv_evict): per layer, request and KV head the first n_first and
// the last n_last tokens stay, and of the others those of largest weight, ties to the lower position; the kept tokens' K and V move, in
// order, to the slots of another table.
//
// Selection: one workgroup per (layer, request, KV head).  Weights are compared as integers of the same order (a NaN below every
// number, -0 as 0).  The weight of the last token that stays is found digit by digit: a histogram of eight bits in LDS, the digit in
// which the wanted rank falls, then the next eight bits of the weights that share the digits so far.  A wave then owns a run of positions,
// so that one exchange of counts tells every wave where its kept tokens go.
// Move: one workgroup per destination block, bytes in, bytes out.
#include "attn_common.h"

namespace calvo {
namespace evict {

using namespace attn;

__device__ inline uint32_t rank_of(float x) {
  if (x != x) return 0u;
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);    // -0 as 0
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

constexpr int kThreads = 1024, kWaves = kThreads / 64;

__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictParams p) {
  __shared__ int hist[256];
  __shared__ int pick[2];                                      // digit, rank that is left inside it
  __shared__ int counts[kWaves][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = blockIdx.x % p.n_kv_heads, r = blockIdx.x / p.n_kv_heads % p.n_reqs, layer = blockIdx.x / p.n_kv_heads / p.n_reqs;
  const EvictDesc d = p.reqs[r];
  const float* mass = p.mass + layer * p.mass_layer + ((int64_t)d.mass_row * p.n_kv_heads + g) * p.mass_stride;
  int32_t* kept = p.kept + (((int64_t)layer * p.n_reqs + r) * p.n_kv_heads + g) * p.kept_stride;
  float* out = p.mass_out ? p.mass_out + layer * p.out_layer + ((int64_t)d.mass_row * p.n_kv_heads + g) * p.out_stride : nullptr;
  const int begin = d.n_first, end = d.n_tokens - d.n_last;    // positions that are chosen from
  int want = d.n_keep - d.n_first - d.n_last;

  // ---- the rank of the last chosen token, and how many of equal rank are chosen
  uint32_t found = 0xffffffffu;                                // nothing is above it
  int ties = 0;
  if (want > 0) {
    found = 0;
    ties = want;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      for (int i = begin + tid; i < end; i += kThreads) {
        const uint32_t x = rank_of(mass[i]);
        if (shift == 24 || (x ^ found) >> (shift + 8) == 0) atomicAdd(&hist[x >> shift & 255], 1);
      }
      __syncthreads();
      if (wave == 0) {
        // lane i: digits 255 - 4i down to 252 - 4i
        int n[4], sum = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) { n[k] = hist[255 - 4 * lane - k]; sum += n[k]; }
        int before = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int x = __shfl_up(before, o);
          if (lane >= o) before += x;
        }
        before -= sum;
#pragma unroll
        for (int k = 0; k < 4; k++) {
          if (before < ties && ties <= before + n[k]) { pick[0] = 255 - 4 * lane - k; pick[1] = ties - before; }
          before += n[k];
        }
      }
      __syncthreads();
      found |= (uint32_t)pick[0] << shift;
      ties = pick[1];
    }
  }

  // ---- the wave's run of positions
  const int run = (d.n_tokens + kThreads - 1) / kThreads * 64;
  const int from = min(wave * run, d.n_tokens), to = min(from + run, d.n_tokens);
  auto classify = [&](int i, bool& above, bool& equal, float& x) {
    const bool in = i < to;
    x = in ? mass[i] : 0.f;
    const bool safe = i < begin || i >= end;
    const uint32_t k = rank_of(x);
    above = in && (safe || (want > 0 && k > found));
    equal = in && !safe && want > 0 && k == found;
  };
  int n_above = 0, n_equal = 0;
  for (int i0 = from; i0 < to; i0 += 64) {
    bool above, equal;
    float x;
    classify(i0 + lane, above, equal, x);
    n_above += __popcll(__ballot(above));
    n_equal += __popcll(__ballot(equal));
  }
  if (lane == 0) { counts[wave][0] = n_above; counts[wave][1] = n_equal; }
  __syncthreads();
  int above0 = 0, equal0 = 0;
  for (int w = 0; w < wave; w++) { above0 += counts[w][0]; equal0 += counts[w][1]; }
  const uint64_t below = (1ull << lane) - 1;
  for (int i0 = from; i0 < to; i0 += 64) {
    bool above, equal;
    float x;
    classify(i0 + lane, above, equal, x);
    const uint64_t ma = __ballot(above), me = __ballot(equal);
    const int rank = equal0 + __popcll(me & below);
    const int at = above0 + __popcll(ma & below) + min(rank, ties);
    if (above || (equal && rank < ties)) {
      kept[at] = i0 + lane;
      if (out) out[at] = x;
    }
    above0 += __popcll(ma);
    equal0 += __popcll(me);
  }
}

__global__ void __launch_bounds__(256) evict_move_kernel(EvictParams p) {
  const EvictDesc d = p.reqs[blockIdx.y];
  const int block = blockIdx.x;
  const int rows = min(kBlockTokens, d.n_keep - block * kBlockTokens);   // of the destination block
  if (rows <= 0) return;
  const int64_t half = (int64_t)kBlockTokens * p.n_kv_heads * p.row_chunks;   // 16-byte chunks of a block's K (or V)
  u32x4* pool = (u32x4*)(p.pool + blockIdx.z * p.layer_bytes);
  const int32_t* kept = p.kept + ((int64_t)blockIdx.z * p.n_reqs + blockIdx.y) * p.n_kv_heads * p.kept_stride + block * kBlockTokens;
  const int32_t* src = p.tables + d.src_off;
  const int64_t dst = (int64_t)p.tables[d.dst_off + block] * 2 * half;
  const int per_row = p.n_kv_heads * p.row_chunks, n = rows * per_row;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int j = i / per_row, in_row = i - j * per_row, g = in_row / p.row_chunks;
    const int pos = kept[g * p.kept_stride + j];
    const int64_t at = (int64_t)src[pos / kBlockTokens] * 2 * half + (int64_t)(pos % kBlockTokens) * per_row + in_row;
    const u32x4 k = pool[at], v = pool[at + half];
    pool[dst + i] = k;
    pool[dst + i + half] = v;
  }
}

}  // namespace evict

hipError_t launch_evict_select(const EvictParams& p, hipStream_t stream) {
  const unsigned grid = (unsigned)p.n_layers * (unsigned)p.n_reqs * (unsigned)p.n_kv_heads;
  if (grid == 0) return hipSuccess;
  hipLaunchKernelGGL(evict::evict_select_kernel, dim3(grid), dim3(evict::kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_evict_move(const EvictParams& p, hipStream_t stream) {
  if (p.max_keep <= 0 || p.n_reqs <= 0 || p.n_layers <= 0) return hipSuccess;
  const unsigned blocks = (unsigned)(p.max_keep + kBlockTokens - 1) / kBlockTokens;
  hipLaunchKernelGGL(evict::evict_move_kernel, dim3(blocks, (unsigned)p.n_reqs, (unsigned)p.n_layers), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace calvo
