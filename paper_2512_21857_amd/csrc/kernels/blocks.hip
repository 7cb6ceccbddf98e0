// Blocks of cache slots and what a query thinks of them: the mean key of every block of the
// prefix, kept beside the cache, and for every query row the blocks it will attend to.
#include <algorithm>

#include "../launch.h"
#include "../rank.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(blocks)

constexpr int BK_WAVES = 4;

// Mean key of one block per wave: a row takes DH * sizeof(T) / 16 lanes of 16 bytes, so the wave
// reads several rows at once, every 16 bytes of the keys once; sums in fp32, slots in order
// within a lane, then across the lanes of a column.  Bound by the read of the keys: 906 MB of sixteen
// caches in 151 us, 6.0 TB/s.
template <typename T, int DH>
__global__ __launch_bounds__(BK_WAVES * WAVE) void block_keys_kernel(const T* __restrict__ kc, int64_t stride_b,
                                                                     int64_t stride_h, const int32_t* __restrict__ start,
                                                                     const int32_t* __restrict__ kv_len, int block,
                                                                     int kv_cap, float* __restrict__ means, int64_t mb,
                                                                     int64_t mh) {
  constexpr int V = 16 / sizeof(T), COLS = DH / V, ROWS = WAVE / COLS;
  const int h = blockIdx.y, b = blockIdx.z;
  const int L = max(0, min(kv_len[b], kv_cap));
  if (kv_len[b] > kv_cap && threadIdx.x == 0 && blockIdx.x == 0) dev_fail(DEVINV_KV_RANGE);
  const int j = blockIdx.x * BK_WAVES + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  const int j0 = start ? max(0, start[b]) / block : 0;
  const int n = min(block, L - j * block);             // slots of the block in the prefix
  if (j < j0 || n <= 0) return;
  const int c = lane % COLS * V, r0 = lane / COLS;
  const T* base = kc + b * stride_b + h * stride_h + (int64_t)j * block * DH + c;
  float sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) sum[e] = 0.f;
  constexpr int UN = 8;                                // rows in flight per lane
  for (int r = r0; r < n; r += ROWS * UN) {
    u16x8 x[UN];
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (r + u * ROWS < n)
        x[u] = __builtin_nontemporal_load(reinterpret_cast<const u16x8*>(base + (int64_t)(r + u * ROWS) * DH));
#pragma unroll
    for (int u = 0; u < UN; ++u)
      if (r + u * ROWS < n) {
        const T* t = reinterpret_cast<const T*>(&x[u]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += Elem<T>::load(t, e);
      }
  }
#pragma unroll
  for (int o = COLS; o < WAVE; o <<= 1)
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] += __shfl_xor(sum[e], o, WAVE);
  if (r0 == 0) {
    float* out = means + b * mb + h * mh + (int64_t)j * DH + c;
#pragma unroll
    for (int e = 0; e < V; e += 4)
      *reinterpret_cast<float4*>(out + e) = make_float4(sum[e] / n, sum[e + 1] / n, sum[e + 2] / n, sum[e + 3] / n);
  }
}

// Scores are products of the rows' queries, summed over the heads that share the keys, with the mean
// keys.  In double, where the sum of 128 products is off by 2^-50 or so of its terms: a choice between
// two blocks then depends on the inputs alone, not on the order of a sum (in float, one choice in
// some ten thousand would).
//
// On the fp64 MFMA, 16 blocks and 16 query rows per wave: A = mean keys (lane (l, g): block l, dims
// 16 d + 4 g + e), B = the rows' sums, so lane (l, g) gets blocks 4 r + g of row l.  Bound by latency: 61
// rows of 32 heads against 73 blocks 8.0 us, sixteen sequences' 16 rows of 8 heads against 320 each 13.0.
typedef double f64x4 __attribute__((ext_vector_type(4)));
template <int DH>
constexpr int SUM_PITCH = DH + 2;           // a row of sums in LDS, padded: 16 rows at one dim on distinct banks
// rows i0 .. i0 + rows - 1 (zero from nq on), four dims per thread and turn; no barrier
template <typename T, int DH, int THREADS>
__device__ __forceinline__ void sum_queries(double* sums, const T* q, int i0, int rows, int nq, int h, int64_t row0,
                                            int Hkv, int G) {
  for (int x = threadIdx.x; x < rows * (DH / 4); x += THREADS) {
    const int i = x / (DH / 4), d = x % (DH / 4) * 4;
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    if (i0 + i < nq) {
      const T* qp = q + ((row0 + i0 + i) * Hkv + h) * G * DH + d;
      for (int u0 = 0; u0 < G; u0 += 4) {       // four heads requested at a time
        T t[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          __builtin_memcpy(t[u], __builtin_assume_aligned(qp + (int64_t)min(u0 + u, G - 1) * DH, 4 * sizeof(T)),
                           4 * sizeof(T));
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u0 + u < G)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += (double)Elem<T>::load(t[u], e);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[i * SUM_PITCH<DH> + d + e] = s[e];
  }
}
// sums: of 16 rows; mean: lane (l, g)'s block's mean key + 4 g
template <int DH>
__device__ __forceinline__ f64x4 tile_scores(const double* sums, const float* mean, int l, int g) {
  f32x4 m[DH / 16];
#pragma unroll
  for (int d = 0; d < DH / 16; ++d) m[d] = *reinterpret_cast<const f32x4*>(mean + 16 * d);
  f64x4 acc{0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int e = 0; e < DH / 4; ++e)
    acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)m[e / 4][e % 4],
                                               sums[l * SUM_PITCH<DH> + e / 4 * 16 + 4 * g + e % 4], acc, 0, 0, 0);
  return acc;
}

// Scores to memory; also clears the blocks' row marks and the pair's count of arrivals for the selection
// that follows.
constexpr int SC_WAVES = 4, SC_TILES = 2;      // waves, and 16-block tiles per wave
template <typename T, int DH>
__global__ __launch_bounds__(SC_WAVES * WAVE) void block_score_kernel(const T* __restrict__ q,
                                                                      const float* __restrict__ means, int64_t mb,
                                                                      int64_t mh, const int32_t* __restrict__ kv_len,
                                                                      const int32_t* __restrict__ n_q, int Hkv, int G,
                                                                      int nq_max, int kv_cap, int block, int n_blk,
                                                                      double* __restrict__ score,
                                                                      uint64_t* __restrict__ marks,
                                                                      uint32_t* __restrict__ arrived) {
  __shared__ __attribute__((aligned(16))) double sums[16 * SUM_PITCH<DH>];
  const int h = blockIdx.z % Hkv, b = blockIdx.z / Hkv;
  const int L = max(0, min(kv_len[b], kv_cap)), live = (L + block - 1) / block;
  const int first = blockIdx.x * SC_WAVES * SC_TILES * 16, i0 = blockIdx.y * 16;
  if (first == 0 && i0 == 0 && threadIdx.x == 0) arrived[blockIdx.z] = 0;
  if (first >= live) return;
  if (i0 == 0 && (int)threadIdx.x < SC_WAVES * SC_TILES * 16 && first + (int)threadIdx.x < n_blk) {
    uint64_t* mk = marks + ((int64_t)blockIdx.z * n_blk + first + threadIdx.x) * ADT_MASK_WORDS;
    mk[0] = 0;
    mk[1] = 0;
  }
  const int nq = min(n_q[b], nq_max);
  if (i0 >= nq) return;
  sum_queries<T, DH, SC_WAVES * WAVE>(sums, q, i0, 16, nq, h, (int64_t)b * nq_max, Hkv, G);
  __syncthreads();
  const int lane = threadIdx.x % WAVE, l = lane & 15, g = lane >> 4;
#pragma unroll
  for (int t = 0; t < SC_TILES; ++t) {
    const int j0 = first + (threadIdx.x / WAVE * SC_TILES + t) * 16;
    if (j0 >= live) break;
    const f64x4 acc = tile_scores<DH>(sums, means + b * mb + h * mh + (int64_t)min(j0 + l, live - 1) * DH + 4 * g, l, g);
    if (i0 + l >= nq) continue;
    double* out = score + ((int64_t)blockIdx.z * nq_max + i0 + l) * n_blk + j0;
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (j0 + 4 * r + g < live) out[4 * r + g] = acc[r];
  }
}

// The blocks j < live with a mark (w0(j), w1(j)), in order, into the pair's list.  Called by every
// thread of the workgroup; scratch: an int of LDS per wave.
template <int THREADS, class F>
__device__ __forceinline__ void list_marked(const BlockLists& lists, int64_t pair, int n_blk, int live, int* scratch,
                                            F mark) {
  const int wave = threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
  uint16_t* blocks = lists.blocks + pair * n_blk;
  uint64_t* marks = lists.marks + pair * n_blk * ADT_MASK_WORDS;
  int n = 0;
  for (int base = 0; base < live; base += THREADS) {
    const int j = base + threadIdx.x;
    uint64_t w0 = 0, w1 = 0;
    if (j < live) mark(j, w0, w1);
    const bool on = (w0 | w1) != 0;
    const uint64_t bal = __ballot(on);
    if (lane == 0) scratch[wave] = __popcll(bal);
    __syncthreads();
    int at = n + __popcll(bal & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < THREADS / WAVE; ++w) {
      const int c = scratch[w];
      if (w < wave) at += c;
      n += c;
    }
    if (on) {
      blocks[at] = (uint16_t)j;
      marks[2 * at] = w0;
      marks[2 * at + 1] = w1;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    lists.count[pair] = n;
    lists.arrived[pair] = 0;
  }
}

// Scores in an unsigned order: larger score, larger key; -0 equals +0; NaN below all.  key_score: back again.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 0;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

__device__ __forceinline__ float key_score(uint64_t k) {
  return (float)__builtin_bit_cast(double, k >> 63 ? k & ~(1ull << 63) : ~k);
}

// The n_sel blocks of one query row and key-value head: the first and last, and the best of those
// between by radix selection; written in order, and the row marked in each of them.
struct BlockPick {
  int live, n_sel, n_first, n_last;
  int32_t* out;                       // the row's list, or null
  unsigned long long* marks;          // the row's word of the first block's mark
  unsigned long long bit;
  __device__ __forceinline__ void take(int at, int j) const {
    atomicOr(marks + (int64_t)j * ADT_MASK_WORDS, bit);
    if (out) out[at] = j;
  }
  // what the scores do not decide, by `n` threads of which this is number t; whether they decide the rest
  __device__ __forceinline__ bool ends(int t, int n) const {
    if (live <= n_sel) {
      for (int j = t; j < live; j += n) take(j, j);
      for (int j = live + t; out && j < n_sel; j += n) out[j] = -1;
      return false;
    }
    for (int m = t; m < n_first; m += n) take(m, m);
    for (int m = t; m < n_last; m += n) take(n_sel - n_last + m, live - n_last + m);
    return n_sel > n_first + n_last;
  }
};
struct BlockRows {
  const double* score;                // [B][Hkv][nq_max][n_blk]
  const int32_t *kv_len, *n_q;
  int Hkv, nq_max, kv_cap, block, n_blk, n_sel, n_first, n_last;
  unsigned long long* marks;          // [B][Hkv][n_blk][ADT_MASK_WORDS], zero before
  uint32_t* arrived;                  // [B][Hkv], zero before
  BlockLists lists;
  int32_t* sel;
  // The last workgroup of a pair to get here lists the marked blocks: marks are set by atomics, complete
  // at the agent's coherence point (waited for) before the arrival counts, and read past the local caches.
  template <int THREADS>
  __device__ __forceinline__ void finish(int h, int b, int* scratch) const {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int64_t pair = (int64_t)b * Hkv + h;
    if (threadIdx.x == 0)
      scratch[0] = __hip_atomic_fetch_add(arrived + pair, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1 == gridDim.x;
    __syncthreads();
    const int last = scratch[0];
    __syncthreads();
    if (!last) return;
    const int L = max(0, min(kv_len[b], kv_cap));
    const unsigned long long* mk = marks + pair * n_blk * ADT_MASK_WORDS;
    list_marked<THREADS>(lists, pair, n_blk, (L + block - 1) / block, scratch, [&](int j, uint64_t& w0, uint64_t& w1) {
      w0 = __hip_atomic_load(mk + 2 * (int64_t)j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      w1 = __hip_atomic_load(mk + 2 * (int64_t)j + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
  }
  __device__ __forceinline__ BlockPick pick(int i, int h, int b) const {
    const int L = max(0, min(kv_len[b], kv_cap));
    return BlockPick{(L + block - 1) / block, n_sel, n_first, n_last,
                     sel ? sel + (((int64_t)b * nq_max + i) * Hkv + h) * n_sel : nullptr,
                     marks + ((int64_t)b * Hkv + h) * n_blk * ADT_MASK_WORDS + i / 64, 1ull << (i & 63)};
  }
  __device__ __forceinline__ const double* row(int i, int h, int b) const {
    return score + (((int64_t)b * Hkv + h) * nq_max + i) * n_blk;
  }
};

// A wave per row, keys in LDS (n_blk a wave).
constexpr int BS_THREADS = 256, BS_WAVES = BS_THREADS / WAVE;
constexpr int BS_WAVE_KEYS = 1024;
__global__ __launch_bounds__(BS_THREADS) void block_select_wave_kernel(BlockRows a) {
  extern __shared__ uint64_t keys[];
  __shared__ __attribute__((aligned(16))) uint32_t hist[BS_WAVES][256];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
  const int i = blockIdx.x * BS_WAVES + wave, h = blockIdx.y, b = blockIdx.z;
  if (i < min(a.n_q[b], a.nq_max)) {
    const BlockPick p = a.pick(i, h, b);
    if (p.ends(lane, WAVE)) {
      const double* row = a.row(i, h, b) + p.n_first;
      uint64_t* k = keys + wave * a.n_blk;
      const int n = p.live - p.n_first - p.n_last;
      for (int j = lane; j < n; j += WAVE) k[j] = score_key(row[j]);
      wave_lds_fence();
      wave_select(k, n, p.n_sel - p.n_first - p.n_last, hist[wave], key_score,
                  [&](int at, int j) { p.take(p.n_first + at, p.n_first + j); });
    }
  }
  a.finish<BS_THREADS>(h, b, (int*)hist);
}

// A workgroup per row, for rows of more blocks; the keys are read anew in every pass.
__global__ __launch_bounds__(BS_THREADS) void block_select_kernel(BlockRows a) {
  typedef RankShape<BS_THREADS, 8, 8, 1, false> Rank;
  __shared__ typename Rank::Scratch sh;
  const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  if (i < min(a.n_q[b], a.nq_max)) {
    const BlockPick p = a.pick(i, h, b);
    if (p.ends(threadIdx.x, BS_THREADS)) {
      const double* row = a.row(i, h, b) + p.n_first;
      auto ranked = rank_row<uint64_t, Rank>([&](int j) { return row[j]; }, [](double s) { return score_key(s); },
                                             p.live - p.n_first - p.n_last, sh);
      ranked.cut(p.n_sel - p.n_first - p.n_last);
      ranked.emit([&](int at, int j) { p.take(p.n_first + at, p.n_first + j); });
    }
  }
  a.finish<BS_THREADS>(h, b, (int*)&sh);
}

// Score and selection in one launch for up to BC_ROWS query rows: a workgroup of 16 waves per key-value
// head, whose 16-lane groups take a block each (a lane DH / 16 dims, the row's sum over the lanes by
// rotations within the group), leave the keys in LDS, and whose first waves then select for a row each;
// the rows' marks meet in LDS, so the pair's list is written without another workgroup's.  It saves a
// launch where one row leaves it little to do, and breaks even at two to four: whole calls of one row over
// 511 blocks of 8 key-value heads 19.3 us against 24.9 in two launches, of 128 heads 41 against 50, over 74
// of 32 heads 16.9 against 21.4, over 141 of 512 heads 110 against 111; of four rows 33.4 against 33.0, 86
// against 89, 20.9 against 22.1, 188 against 187, and over 74 of 512 heads 78 against 75.  More rows take two launches at any number of heads.
// One launch by matrix products, a form of its own, was no gain for them all round: 21.7 us for 16 rows
// of 128 heads over 320 blocks against 23.2 in two, but 20.4 for 61 rows of 32 heads over 73 against 16.5.
constexpr int BC_THREADS = 1024;
constexpr int BC_ROWS = 4;
constexpr int BC_LDS_BYTES = 144 * 1024;
static size_t choose_lds_bytes(int nq_max, int n_blk) {
  return (size_t)n_blk * (nq_max * sizeof(uint64_t) + sizeof(uint32_t));
}
static bool choose_at_once(int nq_max, int n_blk) {
  return nq_max <= BC_ROWS && choose_lds_bytes(nq_max, n_blk) <= BC_LDS_BYTES;
}

// x + x of the lane C places on, round the 16 lanes of a row
template <int C>
__device__ __forceinline__ double add_rotated(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, 0x120 + C, 0xf, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), 0x120 + C, 0xf, 0xf, false);
  return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

template <typename T, int DH, int R>
__global__ __launch_bounds__(BC_THREADS) void block_choose_kernel(
    const T* __restrict__ q, const float* __restrict__ means, int64_t mb, int64_t mh, const int32_t* __restrict__ kv_len,
    const int32_t* __restrict__ n_q, int Hkv, int G, int nq_max, int kv_cap, int block, int n_blk, int n_sel, int n_first,
    int n_last, BlockLists lists, int32_t* __restrict__ sel) {
  constexpr int PER = DH / 16, GROUPS = BC_THREADS / 16, UN = 4;
  extern __shared__ uint64_t keys[];                      // [nq_max][n_blk], then the row bits of each block
  __shared__ double qs[R][DH];
  __shared__ __attribute__((aligned(16))) uint32_t hist[R][256];
  uint32_t* bits = reinterpret_cast<uint32_t*>(keys + (size_t)nq_max * n_blk);
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int L = max(0, min(kv_len[b], kv_cap)), live = (L + block - 1) / block, nq = min(n_q[b], nq_max);
  // the first blocks' means, requested ahead of the queries' sums
  const int c = tid % 16 * PER;
  const float* mp = means + b * mb + h * mh + c;
  f32x4 m[UN][PER / 4];
  auto request = [&](int j0) {
#pragma unroll
    for (int u = 0; u < UN; ++u)
#pragma unroll
      for (int e = 0; e < PER / 4; ++e)
        m[u][e] = *reinterpret_cast<const f32x4*>(mp + (int64_t)min(j0 + u * GROUPS, live - 1) * DH + 4 * e);
  };
  if (live > n_sel) request(tid / 16);
  for (int j = tid; j < live; j += BC_THREADS) bits[j] = 0;
  for (int x = tid; x < R * DH; x += BC_THREADS) {
    const int i = x / DH, d = x % DH;
    double s = 0.0;
    if (i < nq) {
      const T* qp = q + (((int64_t)b * nq_max + i) * Hkv + h) * G * DH + d;
      for (int u0 = 0; u0 < G; u0 += 4) {         // four heads requested at a time
        float t[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) t[u] = Elem<T>::load(qp, (int64_t)min(u0 + u, G - 1) * DH);
#pragma unroll
        for (int u = 0; u < 4; ++u) s += u0 + u < G ? (double)t[u] : 0.0;
      }
    }
    qs[i][d] = s;
  }
  __syncthreads();
  if (live > n_sel) {
    double x[R][PER];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int e = 0; e < PER; ++e) x[i][e] = qs[i][c + e];
    for (int j0 = tid / 16; j0 < live; j0 += GROUPS * UN) {
      if (j0 >= GROUPS * UN) request(j0);
#pragma unroll
      for (int u = 0; u < UN; ++u)
#pragma unroll
        for (int i = 0; i < R; ++i) {
          double s = 0.0;
#pragma unroll
          for (int e = 0; e < PER; ++e) s = fma((double)m[u][e / 4][e % 4], x[i][e], s);
          s = add_rotated<8>(s);
          s = add_rotated<4>(s);
          s = add_rotated<2>(s);
          s = add_rotated<1>(s);
          if (tid % 16 == i && i < nq && j0 + u * GROUPS < live) keys[(size_t)i * n_blk + j0 + u * GROUPS] = score_key(s);
        }
    }
  }
  __syncthreads();
  const int i = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  if (i < nq) {
    int32_t* out = sel ? sel + (((int64_t)b * nq_max + i) * Hkv + h) * n_sel : nullptr;
    auto take = [&](int at, int j) {
      atomicOr(&bits[j], 1u << i);
      if (out) out[at] = j;
    };
    if (live <= n_sel) {
      for (int j = lane; j < live; j += WAVE) take(j, j);
      for (int j = live + lane; out && j < n_sel; j += WAVE) out[j] = -1;
    } else {
      const int lo = n_first, hi = live - n_last, need = n_sel - n_first - n_last;
      for (int m = lane; m < lo; m += WAVE) take(m, m);
      for (int m = lane; m < n_last; m += WAVE) take(n_sel - n_last + m, hi + m);
      if (need > 0)
        wave_select(keys + (size_t)i * n_blk + lo, hi - lo, need, hist[i], key_score,
                    [&](int at, int j) { take(lo + at, lo + j); });
    }
  }
  __syncthreads();
  list_marked<BC_THREADS>(lists, (int64_t)b * Hkv + h, n_blk, live, (int*)hist, [&](int j, uint64_t& w0, uint64_t&) { w0 = bits[j]; });
}

// Scratch: scores, marks, arrivals.
size_t block_select_ws_bytes(int B, int Hkv, int nq_max, int n_blk) {
  if (choose_at_once(nq_max, n_blk)) return 0;
  const size_t pairs = (size_t)B * Hkv;
  return pairs * n_blk * ((size_t)nq_max * sizeof(double) + ADT_MASK_WORDS * sizeof(uint64_t)) + pairs * sizeof(uint32_t);
}

adt_status launch_block_select(const void* q, const float* means, int64_t mb, int64_t mh, const int32_t* kv_len,
                               const int32_t* n_q, int B, int Hkv, int G, int Dh, int nq_max, int kv_cap, int block,
                               int n_sel, int n_first, int n_last, int dtype, void* ws, const BlockLists& lists,
                               int32_t* sel, hipStream_t st) {
  const int n_blk = (kv_cap + block - 1) / block;
  if (choose_at_once(nq_max, n_blk)) {
#define ADT_BC(TV, DHV, RV)                                                                                             \
  block_choose_kernel<TV, DHV, RV><<<dim3(Hkv, B), BC_THREADS, choose_lds_bytes(nq_max, n_blk), st>>>(                  \
      (const TV*)q, means, mb, mh, kv_len, n_q, Hkv, G, nq_max, kv_cap, block, n_blk, n_sel, n_first, n_last, lists, sel)
#define ADT_BCR(TV, DHV)                       \
  if (nq_max == 1) ADT_BC(TV, DHV, 1);         \
  else ADT_BC(TV, DHV, BC_ROWS)
    if (dtype == ADT_BF16) {
      if (Dh == 128) { ADT_BCR(uint16_t, 128); }
      else { ADT_BCR(uint16_t, 64); }
    } else {
      if (Dh == 128) { ADT_BCR(float, 128); }
      else { ADT_BCR(float, 64); }
    }
#undef ADT_BCR
#undef ADT_BC
    ADT_LAUNCH_CHECK();
    return ADT_OK;
  }
  const size_t pairs = (size_t)B * Hkv;
  double* score = (double*)ws;
  uint64_t* marks = (uint64_t*)(score + pairs * nq_max * n_blk);
  uint32_t* arrived = (uint32_t*)(marks + pairs * n_blk * ADT_MASK_WORDS);
  const int per = 16 * SC_WAVES * SC_TILES;
  const dim3 grid((n_blk + per - 1) / per, (nq_max + 15) / 16, B * Hkv);
#define ADT_SC(TV, DHV)                                                                                            \
  block_score_kernel<TV, DHV><<<grid, SC_WAVES * WAVE, 0, st>>>((const TV*)q, means, mb, mh, kv_len, n_q, Hkv, G,  \
                                                                nq_max, kv_cap, block, n_blk, score, marks,      \
                                                                arrived)
  if (dtype == ADT_BF16) {
    if (Dh == 128) ADT_SC(uint16_t, 128);
    else ADT_SC(uint16_t, 64);
  } else {
    if (Dh == 128) ADT_SC(float, 128);
    else ADT_SC(float, 64);
  }
#undef ADT_SC
  ADT_LAUNCH_CHECK();
  const BlockRows rows{score, kv_len, n_q, Hkv, nq_max, kv_cap, block, n_blk, n_sel, n_first, n_last,
                       (unsigned long long*)marks, arrived, lists, sel};
  if (n_blk <= BS_WAVE_KEYS)
    block_select_wave_kernel<<<dim3((nq_max + BS_WAVES - 1) / BS_WAVES, Hkv, B), BS_THREADS,
                               BS_WAVES * n_blk * sizeof(uint64_t), st>>>(rows);
  else
    block_select_kernel<<<dim3(nq_max, Hkv, B), BS_THREADS, 0, st>>>(rows);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

adt_status launch_block_keys(const void* k, int64_t sb, int64_t sh, const int32_t* start, const int32_t* kv_len, int B,
                             int Hkv, int Dh, int block, int kv_cap, float* means, int64_t mb, int64_t mh, int dtype,
                             hipStream_t st) {
  const int n_blk = (kv_cap + block - 1) / block;
  const dim3 grid((n_blk + BK_WAVES - 1) / BK_WAVES, Hkv, B);
#define ADT_BK(TV, DHV)                                                                                           \
  block_keys_kernel<TV, DHV><<<grid, BK_WAVES * WAVE, 0, st>>>((const TV*)k, sb, sh, start, kv_len, block, kv_cap, \
                                                               means, mb, mh)
  if (dtype == ADT_BF16) {
    if (Dh == 128) ADT_BK(uint16_t, 128);
    else ADT_BK(uint16_t, 64);
  } else {
    if (Dh == 128) ADT_BK(float, 128);
    else ADT_BK(float, 64);
  }
#undef ADT_BK
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

}  // namespace adt
