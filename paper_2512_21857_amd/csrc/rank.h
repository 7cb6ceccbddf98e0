// Selection by rank within one workgroup: the `need` largest of a row of unsigned keys, found by
// radix from the top digit down (ending early once a digit's keys are just those still needed), and
// their indices written out in order.  Ties go to the lower index.
#pragma once

#include "common.h"

namespace adt {

// THREADS threads, V keys each per round, digits of BITS bits counted in COPIES histograms side by
// side (neighbouring lanes count in different ones: keys that agree in a digit, as many do in the
// first, queue for one counter).  ONE: rows have at most THREADS * V keys.
template <int THREADS_, int V_, int BITS_, int COPIES_, bool ONE_>
struct RankShape {
  static constexpr bool ONE = ONE_;
  static constexpr int THREADS = THREADS_, V = V_, BITS = BITS_, COPIES = COPIES_;
  static constexpr int BINS = 1 << BITS, WAVES = THREADS / WAVE, ROUND = THREADS * V;
  static_assert(BINS % THREADS == 0, "bins per thread");
  struct Scratch {
    uint32_t hist[COPIES * (BINS + 1)];       // (a digit's copies lie in different banks)
    uint32_t wave_n[2][WAVES];
    uint32_t pick[3];                         // digit, keys above it, whether the digit's keys are just those needed
  };
};

// One row of n keys.  The workgroup goes through it in rounds of THREADS * V: wave w of a round holds
// the 64 V keys from 64 V w on, V a lane, 64 apart.  A row of ONE round is read once and stays in
// registers; a longer one is read anew in every pass.  value(i) gives what is read, key(value) its
// key.  Both methods are called by every thread of the workgroup.
template <typename K, class S, class VF, class KF>
struct RankRow {
  static constexpr int V = S::V;
  VF value;
  KF key;
  int n, rounds;
  typename S::Scratch& sh;
  K k[V];
  // keys with (key & mask) > prefix are selected, and of those with (key & mask) == prefix the first `need`
  // (settled: all of those)
  K prefix = 0, mask = 0;
  uint32_t need = 0;
  bool settled = false;

  __device__ __forceinline__ RankRow(VF value, KF key, int n, typename S::Scratch& sh)
      : value(value), key(key), n(n), rounds(S::ONE ? 1 : (n + S::ROUND - 1) / S::ROUND), sh(sh) {}

  // index of this lane's key j of a round: first(round) + 64 j
  __device__ __forceinline__ int first(int round) const {
    return round * S::ROUND + (int)threadIdx.x / WAVE * WAVE * V + (int)threadIdx.x % WAVE;
  }
  // All values are requested before the first is used.  Places past the end get key 0: no key is
  // less, and of equal keys those before them go first, so none of them is ever selected (and the
  // loops over keys need no test for the end, whose V masks would fill the scalar registers).
  __device__ __forceinline__ void load(int round) {
    decltype(value(0)) x[V];
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = value(min(first(round) + j * WAVE, n - 1));
#pragma unroll
    for (int j = 0; j < V; ++j) k[j] = first(round) + j * WAVE < n ? key(x[j]) : 0;
  }

  // Finds the cut that selects `count` (0 < count <= n) keys.
  __device__ __forceinline__ void cut(int count) {
    need = count;
    const int tid = threadIdx.x, lane = tid % WAVE, wave = tid / WAVE;
    uint32_t* mine = sh.hist + tid % S::COPIES * (S::BINS + 1);
    if (S::ONE) load(0);
    for (int top = 8 * (int)sizeof(K); top > 0 && !settled; top -= S::BITS) {
      const int shift = top > S::BITS ? top - S::BITS : 0, digit = (1 << (top - shift)) - 1;
      for (int i = tid; i < S::COPIES * (S::BINS + 1); i += S::THREADS) sh.hist[i] = 0;
      __syncthreads();
      for (int r = 0; r < rounds; ++r) {
        if (!S::ONE) load(r);
        int left = (n - first(r) + WAVE - 1) / WAVE;     // (they are not counted: one counter would take them all)
        asm volatile("" : "+v"(left));
#pragma unroll
        for (int j = 0; j < V; ++j) {
          if (j < left && (k[j] & mask) == prefix) atomicAdd(&mine[(int)(k[j] >> shift) & digit], 1u);
          __builtin_amdgcn_sched_barrier(0);         // (or the compares of all V pile up in scalar registers)
        }
      }
      __syncthreads();
      // thread t holds the digits B t .. B t + B - 1 from the top; sums of all digits above, then its own
      constexpr int B = S::BINS / S::THREADS;
      uint32_t c[B], sum = 0;
#pragma unroll
      for (int j = 0; j < B; ++j) {
        c[j] = 0;
#pragma unroll
        for (int u = 0; u < S::COPIES; ++u) c[j] += sh.hist[u * (S::BINS + 1) + S::BINS - 1 - (tid * B + j)];
        sum += c[j];
      }
      const uint32_t incl = wave_prefix_sum(sum);
      if (lane == WAVE - 1) sh.wave_n[0][wave] = incl;
      __syncthreads();
      uint32_t above = incl - sum;
      for (int w = 0; w < wave; ++w) above += sh.wave_n[0][w];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (above < need && above + c[j] >= need) {
          sh.pick[0] = S::BINS - 1 - (tid * B + j);
          sh.pick[1] = above;
          sh.pick[2] = above + c[j] == need;
        }
        above += c[j];
      }
      __syncthreads();
      prefix |= (K)sh.pick[0] << shift;
      mask |= (K)digit << shift;
      need -= sh.pick[1];
      settled = sh.pick[2] && prefix != 0;          // (places past the end have key 0 as well: by the tie rule)
    }
  }

  // Calls out(rank, i), in rank order, for every key i that the cut selects.  A wave counts its
  // selected keys, and once all waves have, writes from where those before it end.
  template <class O>
  __device__ __forceinline__ void emit(O out) {
    if (settled) emit_as<true>(out);
    else emit_as<false>(out);
  }
  template <bool SETTLED, class O>
  __device__ __forceinline__ void emit_as(O out) {
    const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
    const uint64_t below = (1ull << lane) - 1;
    uint32_t done = 0, equal_done = 0;
    for (int r = 0; r < rounds; ++r) {
      if (!S::ONE) load(r);
      uint32_t n_in = 0, n_equal = 0;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const K m = k[j] & mask;
        n_in += __popcll(__ballot(SETTLED ? m >= prefix : m > prefix));
        if (!SETTLED) n_equal += __popcll(__ballot(m == prefix));
        __builtin_amdgcn_sched_barrier(0);
      }
      // (what lane 0 stores is counted above, key by key: sunk into its branch, V masks would wait for it)
      asm volatile("" : "+v"(n_in), "+v"(n_equal));
      __syncthreads();
      if (lane == 0) {
        sh.wave_n[0][wave] = n_in;
        sh.wave_n[1][wave] = n_equal;
      }
      __syncthreads();
      // of the equal keys before this wave's, the first `need` are selected
      uint32_t in0 = 0, equal0 = 0, in_all = 0, equal_all = 0;
#pragma unroll
      for (int w = 0; w < S::WAVES; ++w) {
        if (w == wave) {
          in0 = in_all;
          equal0 = equal_all;
        }
        in_all += sh.wave_n[0][w];
        equal_all += sh.wave_n[1][w];
      }
      uint32_t eq = equal_done + equal0, at = done + in0 + min(eq, need) - min(equal_done, need);
      int i0 = first(r);
      K low = prefix;
      asm volatile("" : "+v"(i0), "+v"(low));      // (or V indices and V compares from above are kept for here)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const K m = k[j] & mask;
        bool in = SETTLED ? m >= low : m > low;
        if (!SETTLED) {
          const bool equal = m == low;
          const uint64_t eqs = __ballot(equal);
          in = in || (equal && eq + __popcll(eqs & below) < need);
          eq += __popcll(eqs);
        }
        const uint64_t ins = __ballot(in);
        if (in) out((int)(at + __popcll(ins & below)), i0 + j * WAVE);
        at += __popcll(ins);
        __builtin_amdgcn_sched_barrier(0);
      }
      done += in_all + min(equal_done + equal_all, need) - min(equal_done, need);
      equal_done += equal_all;
    }
  }
};

template <typename K, class S, class VF, class KF>
__device__ __forceinline__ RankRow<K, S, VF, KF> rank_row(VF value, KF key, int n, typename S::Scratch& sh) {
  return RankRow<K, S, VF, KF>(value, key, n, sh);
}

// Which of 256 counters in LDS (a wave's own), counted from the top, the `need`-th key falls in; need
// becomes its rank there, count the counter's value.
__device__ __forceinline__ uint32_t digit_of_rank(const uint32_t* hist, uint32_t& need, uint32_t& count) {
  // lane l holds the digits 255 - 4 l down to 252 - 4 l
  const uint4 c = reinterpret_cast<const uint4*>(hist)[WAVE - 1 - threadIdx.x % WAVE];
  const uint32_t sum = c.x + c.y + c.z + c.w, incl = wave_prefix_sum(sum), above = incl - sum;
  const int at = __ffsll((unsigned long long)__ballot(above < need && incl >= need)) - 1;
  // within that lane's four digits, from the top
  auto of_lane = [&](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, at); };
  const uint32_t rest = need - of_lane(above), w = of_lane(c.w), z = of_lane(c.z), y = of_lane(c.y), x = of_lane(c.x);
  uint32_t digit = 255 - 4 * at, over = 0;
  count = w;
  if (rest > w) { digit -= 1; over = w; count = z; }
  if (rest > w + z) { digit -= 1; over = w + z; count = y; }
  if (rest > w + z + y) { digit -= 1; over = w + z + y; count = x; }
  need = rest - over;
  return digit;
}

// The same for one wave and keys in LDS, by eight-bit digits: calls out(rank, i), in order, for the
// `need` (0 < need <= n) largest of key[0] .. key[n - 1].  hist: 256 counters of LDS of the wave's own.
template <class O>
__device__ __forceinline__ void wave_radix_select(const uint64_t* key, int n, uint32_t need, uint32_t* hist, O out) {
  const int lane = threadIdx.x % WAVE;
  uint64_t prefix = 0, mask = 0;
  bool settled = false;
  for (int shift = 56; shift >= 0 && !settled; shift -= 8) {
    reinterpret_cast<uint4*>(hist)[lane] = make_uint4(0, 0, 0, 0);
    wave_lds_fence();
    for (int i = lane; i < n; i += WAVE) {
      const uint64_t k = key[i];
      if ((k & mask) == prefix) atomicAdd(&hist[(int)(k >> shift) & 255], 1u);
    }
    wave_lds_fence();
    uint32_t count;
    const uint32_t digit = digit_of_rank(hist, need, count);
    settled = count == need;
    prefix |= (uint64_t)digit << shift;
    mask |= 255ull << shift;
    wave_lds_fence();
  }
  const uint64_t below = (1ull << lane) - 1;
  uint32_t done = 0, eq = 0;
  for (int base = 0; base < n; base += WAVE) {
    const int i = base + lane;
    const uint64_t m = i < n ? key[i] & mask : 0;
    const bool equal = i < n && m == prefix;
    const uint64_t eqs = __ballot(equal);
    const bool in = i < n && (m > prefix || (equal && eq + __popcll(eqs & below) < need));
    eq += __popcll(eqs);
    const uint64_t ins = __ballot(in);
    if (in) out((int)(done + __popcll(ins & below)), i);
    done += __popcll(ins);
  }
}

// The same for keys of doubles (value(key): the double as a float, rounded; the order of keys is the
// doubles').  One pass counts the keys in 256 even steps between the least and the greatest value: a
// monotone rule, whatever it rounds, so the keys of the steps above the `need`-th key's are selected,
// those below are not, and of the few in its step each lane ranks one.  (Digits from the top would
// first tell signs and exponents, which nearly all keys share.)  The keys are read once, 64 V of them at
// the most; where there are more, the values' range is none, or the step holds more keys than the wave
// has lanes, it goes by digits after all.
template <int V, class VF, class O>
__device__ __forceinline__ void wave_select_in(const uint64_t* key, int n, uint32_t need_, uint32_t* hist, VF value, O out) {
  const int lane = threadIdx.x % WAVE;
  const uint64_t below = (1ull << lane) - 1;
  uint32_t need = need_;
  uint64_t k[V];
#pragma unroll
  for (int j = 0; j < V; ++j) k[j] = key[min(j * WAVE + lane, n - 1)];
  float f[V], lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    f[j] = value(k[j]);
    lo = fminf(lo, f[j]);                        // (places past the end repeat the last key)
    hi = fmaxf(hi, f[j]);
  }
  lo = -wave_max_dpp(-lo);
  hi = wave_max_dpp(hi);
  const float range = hi - lo, per = 256.f / range;
  if (!(range > 0.f) || !(range < INFINITY)) return wave_radix_select(key, n, need, hist, out);
  reinterpret_cast<uint4*>(hist)[lane] = make_uint4(0, 0, 0, 0);
  wave_lds_fence();
  int step[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    // (a value that is no number gives step 0; its key is below all others there too)
    const bool in = j * WAVE + lane < n;
    step[j] = in ? (int)fminf(fmaxf((f[j] - lo) * per, 0.f), 255.f) : -1;
    if (in) atomicAdd(&hist[step[j]], 1u);
  }
  wave_lds_fence();
  uint32_t count;
  const int last = digit_of_rank(hist, need, count);     // the step that decides
  if (count > WAVE && count != need) return wave_radix_select(key, n, need_, hist, out);
  wave_lds_fence();
  uint64_t chosen = ~0ull;                               // of that step's keys, in order
  if (count != need) {
    uint64_t* mine = reinterpret_cast<uint64_t*>(hist);
    uint32_t at = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const uint64_t ins = __ballot(step[j] == last);
      if (step[j] == last) mine[at + __popcll(ins & below)] = k[j];
      at += __popcll(ins);
    }
    wave_lds_fence();
    const uint64_t own = mine[min(lane, (int)count - 1)];
    uint32_t rank = 0;
    for (int j = 0; j < (int)count; ++j) {
      const uint64_t o = mine[j];
      rank += (o > own) | ((o == own) & (j < lane));
    }
    chosen = __ballot(lane < (int)count && rank < need);
  }
  uint32_t done = 0, at = 0;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const uint64_t eqs = __ballot(step[j] == last);
    const bool in = step[j] > last || (step[j] == last && (count == need || (chosen >> (at + __popcll(eqs & below)) & 1)));
    at += __popcll(eqs);
    const uint64_t ins = __ballot(in);
    if (in) out((int)(done + __popcll(ins & below)), j * WAVE + lane);
    done += __popcll(ins);
  }
}
template <class VF, class O>
__device__ __forceinline__ void wave_select(const uint64_t* key, int n, int need, uint32_t* hist, VF value, O out) {
  if (n <= 2 * WAVE) wave_select_in<2>(key, n, need, hist, value, out);
  else if (n <= 8 * WAVE) wave_select_in<8>(key, n, need, hist, value, out);
  else if (n <= 16 * WAVE) wave_select_in<16>(key, n, need, hist, value, out);
  else wave_radix_select(key, n, need, hist, out);
}

}  // namespace adt
