// Blocks of cache slots and what a query thinks of them: the mean key of every block of the
// prefix, kept beside the cache, and for every query row the blocks it will attend to.
#include "../launch.h"
#include "../rank.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(blocks)

constexpr int BK_WAVES = 4;

// Mean key of one block per wave: a row takes DH * sizeof(T) / 16 lanes of 16 bytes, so the wave
// reads several rows at once, every 16 bytes of the keys once; sums in fp32, slots in order
// within a lane, then across the lanes of a column.  Bound by the read of the keys.
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

// Scores of 16 blocks for 16 query rows per wave on the fp64 MFMA: A = mean keys (lane (l, g): block
// l, dims 16 j + 4 g + e), B = the rows' queries summed over the heads that share the keys, so
// lane (l, g) gets blocks 4 r + g of row l.  In double, where the sum of 128 products is off by
// 2^-50 or so of its terms: a choice between two blocks then depends on the inputs alone, not on
// the order of a sum (in float, one choice in some ten thousand would).  Also clears the blocks'
// row marks for the selection that follows.
typedef double f64x4 __attribute__((ext_vector_type(4)));
constexpr int SC_WAVES = 4;
template <typename T, int DH>
__global__ __launch_bounds__(SC_WAVES * WAVE) void block_score_kernel(const T* __restrict__ q,
                                                                      const float* __restrict__ means, int64_t mb,
                                                                      int64_t mh, const int32_t* __restrict__ kv_len,
                                                                      const int32_t* __restrict__ n_q, int Hkv, int G,
                                                                      int nq_max, int kv_cap, int block, int n_blk,
                                                                      double* __restrict__ score,
                                                                      uint64_t* __restrict__ marks) {
  const int h = blockIdx.z % Hkv, b = blockIdx.z / Hkv;
  const int L = max(0, min(kv_len[b], kv_cap)), live = (L + block - 1) / block;
  const int j0 = (blockIdx.x * SC_WAVES + threadIdx.x / WAVE) * 16, i0 = blockIdx.y * 16;
  if (j0 >= live) return;
  const int lane = threadIdx.x % WAVE, lq = lane & 15, g = lane >> 4;
  if (i0 == 0 && lane < 32) {
    const int j = j0 + lane / 2;
    if (j < n_blk) marks[((int64_t)blockIdx.z * n_blk + j) * ADT_MASK_WORDS + (lane & 1)] = 0;
  }
  const int nq = min(n_q[b], nq_max);
  if (i0 >= nq) return;
  const bool row = i0 + lq < nq;
  const T* qp = q + (((int64_t)b * nq_max + min(i0 + lq, nq - 1)) * Hkv + h) * G * DH + 4 * g;
  const float* mp = means + b * mb + h * mh + (int64_t)min(j0 + lq, live - 1) * DH + 4 * g;
  f64x4 acc{0.0, 0.0, 0.0, 0.0};
#pragma unroll
  for (int d = 0; d < DH; d += 16) {
    const f32x4 m = *reinterpret_cast<const f32x4*>(mp + d);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    for (int u = 0; u < G; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += (double)Elem<T>::load(qp + (int64_t)u * DH + d, e);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)m[e], row ? s[e] : 0.0, acc, 0, 0, 0);
  }
  if (!row) return;
  double* out = score + ((int64_t)blockIdx.z * nq_max + i0 + lq) * n_blk + j0;
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (j0 + 4 * r + g < live) out[4 * r + g] = acc[r];
}

// Scores in an unsigned order: larger score, larger key; -0 equals +0; NaN below all.
__device__ __forceinline__ uint64_t score_key(double s) {
  if (s != s) return 0;
  const uint64_t u = __builtin_bit_cast(uint64_t, s + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}

// The n_sel blocks of one query row and key-value head per workgroup: the first and last, and the
// best of those between by radix selection; written in order, and the row marked in each of them.
// The keys are held in LDS, or, where there are more than BS_LDS_KEYS, read anew in every pass.
constexpr int BS_THREADS = 256;
constexpr int BS_LDS_KEYS = 4096;
template <bool LDS>
__global__ __launch_bounds__(BS_THREADS) void block_select_kernel(const double* __restrict__ score,
                                                                  const int32_t* __restrict__ kv_len,
                                                                  const int32_t* __restrict__ n_q, int Hkv, int nq_max,
                                                                  int kv_cap, int block, int n_blk, int n_sel,
                                                                  int n_first, int n_last,
                                                                  unsigned long long* __restrict__ marks,
                                                                  int32_t* __restrict__ sel) {
  extern __shared__ uint64_t keys[];
  typedef RankShape<BS_THREADS, BS_LDS_KEYS / BS_THREADS, 8, 1, LDS> BlockRank;
  __shared__ typename BlockRank::Scratch sh;
  const int i = blockIdx.x, h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  if (i >= min(n_q[b], nq_max)) return;
  const int L = max(0, min(kv_len[b], kv_cap)), live = (L + block - 1) / block;
  const int64_t pair = (int64_t)b * Hkv + h;
  unsigned long long* mk = marks + pair * n_blk * ADT_MASK_WORDS + i / 64;
  const unsigned long long bit = 1ull << (i & 63);
  int32_t* out = sel ? sel + (((int64_t)b * nq_max + i) * Hkv + h) * n_sel : nullptr;
  auto take = [&](int at, int j) {
    atomicOr(mk + (int64_t)j * ADT_MASK_WORDS, bit);
    if (out) out[at] = j;
  };
  if (live <= n_sel) {
    for (int j = tid; j < live; j += BS_THREADS) take(j, j);
    for (int j = live + tid; out && j < n_sel; j += BS_THREADS) out[j] = -1;
    return;
  }
  const double* row = score + (pair * nq_max + i) * n_blk;
  if (LDS) {
    for (int j = tid; j < live; j += BS_THREADS) keys[j] = score_key(row[j]);
    __syncthreads();
  }
  const int lo = n_first, hi = live - n_last, need = n_sel - n_first - n_last;
  // the ends, then the blocks between them that the scores select
  for (int m = tid; m < lo; m += BS_THREADS) take(m, m);
  for (int m = tid; m < n_last; m += BS_THREADS) take(n_sel - n_last + m, hi + m);
  if (need == 0) return;
  auto value = [&](int j) { return LDS ? keys[lo + j] : score_key(row[lo + j]); };
  auto ranked = rank_row<uint64_t, BlockRank>(value, [](uint64_t k) { return k; }, hi - lo, sh);
  ranked.cut(need);
  ranked.emit([&](int at, int j) { take(lo + at, lo + j); });
}

size_t block_select_ws_bytes(int B, int Hkv, int nq_max, int n_blk) {
  return (size_t)B * Hkv * nq_max * n_blk * sizeof(double);
}

adt_status launch_block_select(const void* q, const float* means, int64_t mb, int64_t mh, const int32_t* kv_len,
                               const int32_t* n_q, int B, int Hkv, int G, int Dh, int nq_max, int kv_cap, int block,
                               int n_sel, int n_first, int n_last, int dtype, double* score, uint64_t* marks,
                               int32_t* sel, hipStream_t st) {
  const int n_blk = (kv_cap + block - 1) / block;
  const dim3 grid((n_blk + 16 * SC_WAVES - 1) / (16 * SC_WAVES), (nq_max + 15) / 16, B * Hkv);
#define ADT_SC(TV, DHV)                                                                                            \
  block_score_kernel<TV, DHV><<<grid, SC_WAVES * WAVE, 0, st>>>((const TV*)q, means, mb, mh, kv_len, n_q, Hkv, G,  \
                                                                nq_max, kv_cap, block, n_blk, score, marks)
  if (dtype == ADT_BF16) {
    if (Dh == 128) ADT_SC(uint16_t, 128);
    else ADT_SC(uint16_t, 64);
  } else {
    if (Dh == 128) ADT_SC(float, 128);
    else ADT_SC(float, 64);
  }
#undef ADT_SC
  ADT_LAUNCH_CHECK();
  const dim3 rows(nq_max, Hkv, B);
#define ADT_BS(LDSV, BYTES)                                                                                            \
  block_select_kernel<LDSV><<<rows, BS_THREADS, BYTES, st>>>(score, kv_len, n_q, Hkv, nq_max, kv_cap, block, n_blk,    \
                                                             n_sel, n_first, n_last, (unsigned long long*)marks, sel)
  if (n_blk <= BS_LDS_KEYS) ADT_BS(true, n_blk * sizeof(uint64_t));
  else ADT_BS(false, 0);
#undef ADT_BS
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
