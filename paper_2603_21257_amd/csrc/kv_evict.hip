// Eviction from the paged cache by gathered attention weight (calvo_kv_evict): per layer, request and KV head the first n_first and
// the last n_last tokens stay, and of the others those of largest weight, ties to the lower position; the kept tokens' K and V move, in
// order, to the slots of another table.
//
// Selection: one workgroup of 16 waves per (layer, request, KV head), a wave per run of positions.  Weights are compared as integers of the same
// order (a NaN below every number, -0 as 0), which stay in registers where 32 a lane are enough (32768 tokens); longer rows are read again for
// every step.  The weight of the last token that stays lies between the smallest and the largest; a step cuts that range into 512 bins, counts the
// weights in each in LDS, and goes on with the bin that the wanted rank falls into, until that is wanted as a whole or holds one number.  Bins
// of the range that there is, not of the leading bits: those of weights are few, and lanes that count on one word wait for each other.
// Then one exchange of counts tells every wave where its kept tokens go.  256 rows of 16384 tokens: 20 us (bins of the leading eight bits 27;
// the rank found bit by bit, tokens counted in the waves' masks, 37).
// Move: one workgroup per destination block, bytes in, bytes out, at the rate of a large copy (32 layers of 8 heads, 2048 tokens each, bf16 D = 128: 113 us,
// 4.75 TB/s of reads and writes).
#include <cstring>
#include <type_traits>

#include "attn_common.h"

namespace calvo {
namespace evict {

using namespace attn;

// what the order of the weights is as that of integers; 0 and kSafe are left free
constexpr uint32_t kNobody = 0, kNaN = 1, kSafe = 0xffffffffu;
__device__ inline uint32_t rank_of(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.f);    // -0 as 0
  const uint32_t k = b & 0x80000000u ? ~b : b | 0x80000000u;
  return x != x ? kNaN : k;
}

// Descriptors and tables: in device memory, or for small calls in the launch's arguments, which saves the upload in front of it and its event (one
// request of 2011 tokens, 4 layers, fp32: 18.3 -> 12.7 us a call)
struct NoWords {};
struct ArgWords {
  int32_t w[kEvictArgWords];
};
constexpr int kDescWords = sizeof(EvictDesc) / 4;
template <typename W>
__device__ inline EvictDesc desc_of(const EvictParams& p, const W& words, int r) {
  if constexpr (std::is_same<W, NoWords>::value) return p.reqs[r];
  else {
    const int32_t* w = words.w + kDescWords * r;
    return {w[0], w[1], w[2], w[3], w[4], w[5], w[6], 0};
  }
}
template <typename W>
__device__ inline int32_t table_at(const EvictParams& p, const W& words, int i) {
  if constexpr (std::is_same<W, NoWords>::value) return p.tables[i];
  else return words.w[kDescWords * p.n_reqs + i];
}

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 512;

// V: steps of 64 positions of a wave whose weights are in registers at a time.  No branch stands between their loads (one for each step made
// them wait for one another: 16384 tokens 61 us).
template <int V, typename W>
__global__ void __launch_bounds__(kThreads) evict_select_kernel(EvictParams p, W words) {
  __shared__ int hist[kBins];
  __shared__ uint32_t ends[kWaves][2];                         // smallest and largest rank of a wave
  __shared__ int pick[3];                                      // bin, rank that is left inside it, weights in it
  __shared__ int places[kWaves][2];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % p.n_kv_heads, r = blockIdx.x / p.n_kv_heads % p.n_reqs, layer = blockIdx.x / p.n_kv_heads / p.n_reqs;
  const EvictDesc d = desc_of(p, words, r);
  if (d.n_keep == 0) return;                                   // then its counts are 0: there is no position to read at
  const float* mass = p.mass + layer * p.mass_layer + ((int64_t)d.mass_row * p.n_kv_heads + g) * p.mass_stride;
  int32_t* kept = p.kept + (((int64_t)layer * p.n_reqs + r) * p.n_kv_heads + g) * p.kept_stride;
  float* out = p.mass_out ? p.mass_out + layer * p.out_layer + ((int64_t)d.mass_row * p.n_kv_heads + g) * p.out_stride : nullptr;
  const int n = d.n_tokens, begin = d.n_first, end = n - d.n_last;   // positions that are chosen from

  // ---- the wave's run of positions, 64 a step
  const int steps = (n + kThreads - 1) / kThreads;
  const int64_t from = (int64_t)wave * steps * 64 + lane;
  const bool stays = steps <= V;
  // a lane's ranks: kSafe of a token that stays anyway, kNobody past the end
  uint32_t x[V];
  // the weights themselves: a buffer of those that are there, past its end a load reads 0 without a branch.  The step is in the vector offset, which is
  // what is compared with the end; a scalar offset is not.
  auto read = [&](int s0, uint32_t (&w)[V]) {
    const int64_t at = (int64_t)wave * steps * 64 + 64 * s0;
    const int here = (int)max((int64_t)0, min((int64_t)n - at, (int64_t)64 * min(V, steps - s0)));
    const auto buf = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(mass + min(at, (int64_t)n)), 0, 4 * here, 0x00020000u);
#pragma unroll
    for (int j0 = 0; j0 < V; j0 += 16) {
      int off = 4 * lane + 256 * j0;                           // one for 16 steps, the rest is immediate: of its own each takes a register
      asm volatile("" : "+v"(off));
#pragma unroll
      for (int j = j0; j < min(V, j0 + 16); j++) w[j] = __builtin_amdgcn_raw_buffer_load_b32(buf, off + 256 * (j - j0), 0, 0);
    }
  };
  auto load = [&](int s0) {
    read(s0, x);
    const int64_t at = (int64_t)wave * steps * 64 + 64 * s0;
    const int here = (int)max((int64_t)0, min((int64_t)n - at, (int64_t)64 * min(V, steps - s0)));
    const int lo = (int)max((int64_t)0, min(begin - at, (int64_t)here)), hi = (int)max((int64_t)0, min(end - at, (int64_t)here));
#pragma unroll
    for (int j = 0; j < V; j++) {
      const int i = 64 * j + lane;
      const uint32_t k = rank_of(__builtin_bit_cast(float, x[j]));
      x[j] = i >= here ? kNobody : (i < lo) | (i >= hi) ? kSafe : k;
    }
  };
  // f(step, rank), in order
  auto each = [&](auto&& f) {
    for (int s0 = 0; s0 < steps; s0 += V) {
      if (!stays) load(s0);
#pragma unroll
      for (int j = 0; j < V; j++) f(s0 + j, x[j]);
    }
  };
  if (stays) load(0);

  // ---- tokens above `found` stay, and the first `ties` of those that are equal to it
  uint32_t found = kSafe - 1;
  int ties = 0;
  if (d.n_keep == n) {
    found = kNobody;
  } else if (d.n_keep > d.n_first + d.n_last) {
    uint32_t lo = kSafe, hi = kNobody;
    each([&](int, uint32_t k) {
      lo = min(lo, k - 1 < kSafe - 1 ? k : kSafe);             // neither kNobody nor kSafe
      hi = max(hi, k == kSafe ? kNobody : k);
    });
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      lo = min(lo, (uint32_t)__shfl_xor((int)lo, o));
      hi = max(hi, (uint32_t)__shfl_xor((int)hi, o));
    }
    if (lane == 0) { ends[wave][0] = lo; ends[wave][1] = hi; }
    if (tid < kBins) hist[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
      lo = min(lo, ends[w][0]);
      hi = max(hi, ends[w][1]);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    ties = d.n_keep - d.n_first - d.n_last;
    for (;;) {
      // the wanted rank is that of the ties-th largest in [lo, hi]
      const uint32_t span = hi - lo;
      const int shift = max(0, 32 - __builtin_clz(span | 1) - 9);
      each([&](int, uint32_t k) {
        if (k - lo <= span) atomicAdd(&hist[(k - lo) >> shift], 1);
      });
      __syncthreads();
      if (wave == 0) {
        // lane i: bins 511 - 8i down to 504 - 8i
        int c[8], sum = 0;
#pragma unroll
        for (int k = 0; k < 8; k++) { c[k] = hist[kBins - 1 - 8 * lane - k]; sum += c[k]; }
#pragma unroll
        for (int k = 0; k < 8; k++) hist[kBins - 1 - 8 * lane - k] = 0;
        int before = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(before, o);
          if (lane >= o) before += y;
        }
        before -= sum;
#pragma unroll
        for (int k = 0; k < 8; k++) {
          if (before < ties && ties <= before + c[k]) { pick[0] = kBins - 1 - 8 * lane - k; pick[1] = ties - before; pick[2] = c[k]; }
          before += c[k];
        }
      }
      __syncthreads();
      lo += (uint32_t)pick[0] << shift;
      ties = pick[1];
      const int in_bin = pick[2];
      // all of the bin are wanted: what is above the largest number below it (ranks begin behind kNobody)
      if (ties == in_bin) { found = lo - 1; ties = 0; break; }
      if (shift == 0) { found = lo; break; }
      hi = min(hi, lo + (1u << shift) - 1);
      __syncthreads();                                         // pick is read
    }
  }

  // ---- where the wave's kept tokens go
  int n_above = 0, n_equal = 0;
  each([&](int, uint32_t k) {
    n_above += __popcll(__ballot(k > found));
    n_equal += __popcll(__ballot(k == found));
  });
  if (lane == 0) { places[wave][0] = n_above; places[wave][1] = n_equal; }
  __syncthreads();
  int above0 = 0, equal0 = 0;
  for (int w = 0; w < wave; w++) { above0 += places[w][0]; equal0 += places[w][1]; }
  const uint64_t below = (1ull << lane) - 1;
  for (int s0 = 0; s0 < steps; s0 += V) {
    uint32_t w[V];
    read(s0, w);                                               // again, all at once: a load for each step in the loop takes 15 us at 16384 tokens
    if (!stays) load(s0);
#pragma unroll
    for (int j = 0; j < V; j++) {
      const uint32_t k = x[j];
      const bool above = k > found;
      const uint64_t ma = __ballot(above), me = __ballot(k == found);
      const int rank = equal0 + __popcll(me & below);
      if (above || (k == found && rank < ties)) {
        const int at = above0 + __popcll(ma & below) + min(rank, ties);
        kept[at] = (int)(from + 64 * (s0 + j));
        if (out) out[at] = __builtin_bit_cast(float, w[j]);
      }
      above0 += __popcll(ma);
      equal0 += __popcll(me);
    }
  }
}

template <typename W>
__global__ void __launch_bounds__(256) evict_move_kernel(EvictParams p, W words) {
  const EvictDesc d = desc_of(p, words, blockIdx.y);
  const int block = blockIdx.x;
  const int rows = min(kBlockTokens, d.n_keep - block * kBlockTokens);   // of the destination block
  if (rows <= 0) return;
  const int64_t half = (int64_t)kBlockTokens * p.n_kv_heads * p.row_chunks;   // 16-byte chunks of a block's K (or V)
  u32x4* pool = (u32x4*)(p.pool + blockIdx.z * p.layer_bytes);
  const int32_t* kept = p.kept + ((int64_t)blockIdx.z * p.n_reqs + blockIdx.y) * p.n_kv_heads * p.kept_stride + block * kBlockTokens;
  const int64_t dst = (int64_t)table_at(p, words, d.dst_off + block) * 2 * half;
  const int per_row = p.n_kv_heads * p.row_chunks, n = rows * per_row;
  for (int i = threadIdx.x; i < n; i += 256) {
    const int j = i / per_row, in_row = i - j * per_row, g = in_row / p.row_chunks;
    const int pos = kept[g * p.kept_stride + j];
    const int64_t at = (int64_t)table_at(p, words, d.src_off + pos / kBlockTokens) * 2 * half + (int64_t)(pos % kBlockTokens) * per_row + in_row;
    const u32x4 k = pool[at], v = pool[at + half];
    pool[dst + i] = k;
    pool[dst + i + half] = v;
  }
}

template <typename F>
hipError_t with_words(const int32_t* words, int n_words, F&& launch) {
  if (words) {
    ArgWords a;
    std::memcpy(a.w, words, (size_t)n_words * 4);
    launch(a);
  } else {
    launch(NoWords{});
  }
  return hipGetLastError();
}

}  // namespace evict

hipError_t launch_evict_select(const EvictParams& p, const int32_t* words, int n_words, hipStream_t stream) {
  using namespace evict;
  const unsigned grid = (unsigned)p.n_layers * (unsigned)p.n_reqs * (unsigned)p.n_kv_heads;
  if (grid == 0) return hipSuccess;
  const int64_t steps = ((int64_t)p.max_tokens + kThreads - 1) / kThreads;
  return with_words(words, n_words, [&](const auto& w) {
    typedef typename std::decay<decltype(w)>::type W;
    if (steps <= 4) hipLaunchKernelGGL((evict_select_kernel<4, W>), dim3(grid), dim3(kThreads), 0, stream, p, w);
    else if (steps <= 16) hipLaunchKernelGGL((evict_select_kernel<16, W>), dim3(grid), dim3(kThreads), 0, stream, p, w);
    else hipLaunchKernelGGL((evict_select_kernel<32, W>), dim3(grid), dim3(kThreads), 0, stream, p, w);
  });
}

hipError_t launch_evict_move(const EvictParams& p, const int32_t* words, int n_words, hipStream_t stream) {
  using namespace evict;
  if (p.max_keep <= 0 || p.n_reqs <= 0 || p.n_layers <= 0) return hipSuccess;
  const unsigned blocks = (unsigned)(p.max_keep + kBlockTokens - 1) / kBlockTokens;
  return with_words(words, n_words, [&](const auto& w) {
    typedef typename std::decay<decltype(w)>::type W;
    hipLaunchKernelGGL(evict_move_kernel<W>, dim3(blocks, (unsigned)p.n_reqs, (unsigned)p.n_layers), dim3(256), 0, stream, p, w);
  });
}

}  // namespace calvo
