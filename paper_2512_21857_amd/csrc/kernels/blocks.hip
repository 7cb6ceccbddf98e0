// Blocks of cache slots and what a query thinks of them: the mean key of every block of the
// prefix, kept beside the cache.
#include "../launch.h"

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
