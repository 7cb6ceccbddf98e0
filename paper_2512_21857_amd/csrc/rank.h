// Selection by rank within one workgroup: the `need` largest of a row of unsigned keys, found by
// radix (eight bits a pass, from the top, ending early once a digit's keys are just those still
// needed), and written out in index order.  Ties go to the lower index.
#pragma once

#include "common.h"

namespace adt {

template <int THREADS>
struct RankScratch {
  uint32_t hist[256];
  uint32_t wave_n[2][THREADS / WAVE];
  uint32_t pick[3];     // digit, keys above it, whether the digit's keys are just those needed
};

// Keys with (key & mask) > prefix are selected, and of those with (key & mask) == prefix the
// first `need`.
template <typename K>
struct RankCut {
  K prefix = 0, mask = 0;
  int need = 0;
};

// The cut that selects `need` (0 <= need <= hi - lo) of key(lo) .. key(hi - 1).  Called by every
// thread of the workgroup; ends with a barrier.
template <typename K, int THREADS, class F>
__device__ __forceinline__ RankCut<K> rank_cut(F key, int lo, int hi, int need, RankScratch<THREADS>& sh) {
  static_assert(THREADS >= 256, "a thread per digit");
  RankCut<K> cut;
  cut.need = need;
  const int tid = threadIdx.x, lane = tid % WAVE;
  bool all_equal = need == 0;                           // every key with this prefix is selected
  for (int shift = 8 * (int)sizeof(K) - 8; shift >= 0 && !all_equal; shift -= 8) {
    if (tid < 256) sh.hist[tid] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += THREADS) {
      const K k = key(i);
      if ((k & cut.mask) == cut.prefix) atomicAdd(&sh.hist[(int)(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (tid < WAVE) {
      // lane l holds the digits 255 - 4 l .. 252 - 4 l, so a prefix sum over lanes counts from the top
      uint32_t c[4], sum = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += c[j] = sh.hist[255 - 4 * lane - j];
      uint32_t incl = sum;
#pragma unroll
      for (int o = 1; o < WAVE; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o, WAVE);
        if (lane >= o) incl += up;
      }
      uint32_t above = incl - sum;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (above < (uint32_t)cut.need && above + c[j] >= (uint32_t)cut.need) {
          sh.pick[0] = 255 - 4 * lane - j;
          sh.pick[1] = above;
          sh.pick[2] = above + c[j] == (uint32_t)cut.need;
        }
        above += c[j];
      }
    }
    __syncthreads();
    cut.prefix |= (K)sh.pick[0] << shift;
    cut.mask |= (K)255 << shift;
    cut.need -= sh.pick[1];
    all_equal = sh.pick[2];
    __syncthreads();
  }
  return cut;
}

// Calls out(rank, i), in rank order, for every i of [0, n) that is outside [lo, hi) or selected by
// the cut (none of [lo, hi) if `none`).  Called by every thread of the workgroup.
template <typename K, int THREADS, class F, class O>
__device__ __forceinline__ void rank_emit(F key, int n, int lo, int hi, bool none, const RankCut<K>& cut,
                                          RankScratch<THREADS>& sh, O out) {
  const int tid = threadIdx.x, wave = tid / WAVE, lane = tid % WAVE;
  const uint64_t below = (1ull << lane) - 1;
  uint32_t done = 0, equal_n = 0;
  for (int base = 0; base < n; base += THREADS) {
    const int i = base + tid;
    bool stays = i < lo || (i >= hi && i < n), equal = false;
    if (i >= lo && i < hi && !none) {
      const K k = key(i);
      stays = (k & cut.mask) > cut.prefix;
      equal = (k & cut.mask) == cut.prefix;
    }
    const uint64_t eq = __ballot(equal);
    if (lane == 0) sh.wave_n[0][wave] = __popcll(eq);
    __syncthreads();
    uint32_t rank = equal_n + __popcll(eq & below);
#pragma unroll
    for (int v = 0; v < THREADS / WAVE; ++v) {
      const uint32_t c = sh.wave_n[0][v];
      if (v < wave) rank += c;
      equal_n += c;
    }
    stays = stays || (equal && rank < (uint32_t)cut.need);
    const uint64_t st = __ballot(stays);
    if (lane == 0) sh.wave_n[1][wave] = __popcll(st);
    __syncthreads();
    uint32_t at = done + __popcll(st & below);
#pragma unroll
    for (int v = 0; v < THREADS / WAVE; ++v) {
      const uint32_t c = sh.wave_n[1][v];
      if (v < wave) at += c;
      done += c;
    }
    if (stays) out((int)at, i);
  }
}

}  // namespace adt
