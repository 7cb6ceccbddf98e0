// Eviction from a cache by accumulated attention weight: of every (sequence, slice) the first and
// last slots and, between them, the slots of the largest weights stay, in their order, moved
// together; and the weights of an accepted path, moved as the path's keys and values are.
//
// Two launches.  evict_select_kernel, a workgroup per slice, finds the smallest weight that stays
// by radix selection on the weights' bits and writes the kept slots in order; evict_move_kernel
// moves the rows.  Selecting is bound by its passes over the weights (they stay in the L2), moving
// by memory: the kept rows are read once and written once.
#include "../launch.h"
#include "../rank.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(evict)

constexpr int SEL_THREADS = 1024;

// Weights in an unsigned order: larger weight, larger key; -0 equals +0; NaN below all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(const float* __restrict__ w, int64_t stride_wb,
                                                                   int64_t stride_ws, const int32_t* __restrict__ kv_len,
                                                                   int kv_cap, int slices, int budget, int n_first,
                                                                   int n_last, int32_t* __restrict__ kept) {
  __shared__ RankScratch<SEL_THREADS> sh;
  const int s = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int L = max(0, min(kv_len[b], kv_cap));
  if (kv_len[b] > kv_cap && tid == 0) dev_fail(DEVINV_KV_RANGE);
  int32_t* out = kept + ((int64_t)b * slices + s) * budget;
  if (L <= budget) {
    for (int m = tid; m < L; m += SEL_THREADS) out[m] = m;
    return;
  }
  const float* row = w + b * stride_wb + s * stride_ws;
  const int lo = n_first, hi = L - n_last;              // budget < L, so the middle is not empty
  const int need = budget - n_first - n_last;
  auto key = [&](int i) { return weight_key(row[i]); };
  const RankCut<uint32_t> cut = rank_cut<uint32_t, SEL_THREADS>(key, lo, hi, need, sh);
  rank_emit(key, L, lo, hi, need == 0, cut, sh, [&](int at, int i) { out[at] = i; });
}

// Rows of the kept slots of one slice to its first slots: a workgroup takes a stripe of STRIPE
// bytes of every key row or of every value row, in rounds of as many rows as its threads hold.
// In place a round's rows are all read before any is written; a later round's sources lie at or
// after its own destinations, which the earlier rounds have not reached.
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_ROUND = 4;      // rows in flight per thread

template <int STRIPE>
__global__ __launch_bounds__(MOVE_THREADS) void evict_move_kernel(EvictMove a) {
  constexpr int PER = STRIPE / 16, ROWS = MOVE_THREADS / PER;
  const int s = blockIdx.x, b = blockIdx.z;
  const int stripes = a.row_bytes / STRIPE, part = blockIdx.y;      // stripes of K, of V, then the weights
  // (min(kv_len, budget) is the same before and after new_len, which may be kv_len, is written)
  const int n = max(0, min(min(a.kv_len[b], a.kv_cap), a.budget));
  const int32_t* kept = a.kept + ((int64_t)b * a.slices + s) * a.budget;
  if (part == 2 * stripes) {
    const float* src = a.w + b * a.stride_wb + s * a.stride_ws;
    float* dst = a.w_out + b * a.ostride_wb + s * a.ostride_ws;
    for (int base = 0; base < n; base += MOVE_THREADS) {
      const int m = base + threadIdx.x;
      const float x = m < n ? src[kept[m]] : 0.f;
      __syncthreads();
      if (m < n) dst[m] = x;
    }
    if (s == 0 && threadIdx.x == 0) a.new_len[b] = n;
    return;
  }
  const bool value = part >= stripes;
  const int off = (value ? part - stripes : part) * STRIPE + threadIdx.x % PER * 16;
  const char* src = (const char*)(value ? a.v : a.k) + b * a.stride_b + s * a.stride_s + off;
  char* dst = (char*)(value ? a.v_out : a.k_out) + b * a.ostride_b + s * a.ostride_s + off;
  for (int base = 0; base < n; base += ROWS * MOVE_ROUND) {
    u16x8 x[MOVE_ROUND];
#pragma unroll
    for (int j = 0; j < MOVE_ROUND; ++j) {
      const int m = base + j * ROWS + threadIdx.x / PER;
      if (m < n) x[j] = *reinterpret_cast<const u16x8*>(src + (int64_t)kept[m] * a.row_bytes);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < MOVE_ROUND; ++j) {
      const int m = base + j * ROWS + threadIdx.x / PER;
      if (m < n) *reinterpret_cast<u16x8*>(dst + (int64_t)m * a.row_bytes) = x[j];
    }
  }
}

adt_status launch_kv_evict(const EvictMove& a, int B, int n_first, int n_last, hipStream_t st) {
  evict_select_kernel<<<dim3(a.slices, B), SEL_THREADS, 0, st>>>(a.w, a.stride_wb, a.stride_ws, a.kv_len, a.kv_cap,
                                                                 a.slices, a.budget, n_first, n_last, a.kept);
  ADT_LAUNCH_CHECK();
  if (a.row_bytes % 128 == 0)
    evict_move_kernel<128><<<dim3(a.slices, 2 * (a.row_bytes / 128) + 1, B), MOVE_THREADS, 0, st>>>(a);
  else
    evict_move_kernel<16><<<dim3(a.slices, 2 * (a.row_bytes / 16) + 1, B), MOVE_THREADS, 0, st>>>(a);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

// Weights of the accepted path's slots, as kv_compact moves their rows: one workgroup per
// (sequence, slice), a path entry per thread, all read before any is written.
__global__ __launch_bounds__(ADT_MAX_NODES) void weights_compact_kernel(float* __restrict__ w, int64_t stride_wb,
                                                                        int64_t stride_ws,
                                                                        const int32_t* __restrict__ kv_len, int kv_cap,
                                                                        const int32_t* __restrict__ path,
                                                                        int path_stride,
                                                                        const int32_t* __restrict__ n_acc, int a_max) {
  const int s = blockIdx.x, b = blockIdx.y, m = threadIdx.x + 1;
  const int64_t L = kv_len[b];
  float* row = w + b * stride_wb + s * stride_ws + L;
  const bool live = m <= min(n_acc[b], a_max);
  const int src = live ? path[(int64_t)b * path_stride + m] : -1;
  const bool in_tree = src >= m && src < ADT_MAX_NODES, ok = in_tree && L >= 0 && L + src < kv_cap;
  if (live && !in_tree) dev_fail(DEVINV_PATH);
  if (in_tree && !ok) dev_fail(DEVINV_KV_RANGE);
  const float x = ok ? row[src] : 0.f;
  __syncthreads();
  if (ok) row[m] = x;
}

adt_status launch_weights_compact(float* w, int B, int slices, int64_t stride_wb, int64_t stride_ws,
                                  const int32_t* kv_len, int kv_cap, const int32_t* path, int path_stride,
                                  const int32_t* n_acc, int a_max, hipStream_t st) {
  weights_compact_kernel<<<dim3(slices, B), ADT_MAX_NODES, 0, st>>>(w, stride_wb, stride_ws, kv_len, kv_cap, path,
                                                                   path_stride, n_acc, a_max);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

}  // namespace adt
