// Eviction from a cache by accumulated attention weight: of every (sequence, slice) the first and
// last slots and, between them, the slots of the largest weights stay, in their order, moved
// together; and the weights of an accepted path, moved as the path's keys and values are.
//
// Two launches.  evict_select_kernel, a workgroup per slice, finds the smallest weight that stays
// by radix selection on the weights' bits and writes the kept slots in order; evict_copy_kernel, or
// in place evict_place_kernel, moves the rows.  Selecting is bound by one CU's passes over its slice's
// weights (65321 of them 28 us, 2400 of each of 1024 slices 11; more than 65536 are read anew in every pass,
// 131000 of them 84), moving by memory: the kept rows are read once and written once (1024 of 1024 slices,
// 1.07 GB in all, 202 us, 5.3 TB/s; in place 211).  In place few slices are bound by latency, a workgroup
// for each 128 bytes of a slice's rows going through its rounds one by one: 8192 rows of 8 slices 54 us,
// 13 into another cache.
#include <algorithm>

#include "../launch.h"
#include "../rank.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(evict)

// Weights in an unsigned order: larger weight, larger key; -0 equals +0; NaN below all.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <class S>
__global__ __launch_bounds__(S::THREADS) void evict_select_kernel(const float* __restrict__ w, int64_t stride_wb,
                                                                  int64_t stride_ws, const int32_t* __restrict__ kv_len,
                                                                  int kv_cap, int slices, int budget, int n_first,
                                                                  int n_last, int32_t* __restrict__ kept) {
  __shared__ typename S::Scratch sh;
  const int s = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int L = max(0, min(kv_len[b], kv_cap));
  if (kv_len[b] > kv_cap && tid == 0) dev_fail(DEVINV_KV_RANGE);
  int32_t* out = kept + ((int64_t)b * slices + s) * budget;
  if (L <= budget) {
    for (int m = tid; m < L; m += S::THREADS) out[m] = m;
    return;
  }
  // the ends, then the slots between them that the weights select (budget < L, so there are some)
  const int lo = n_first, hi = L - n_last, need = budget - n_first - n_last;
  for (int m = tid; m < lo; m += S::THREADS) out[m] = m;
  for (int m = tid; m < n_last; m += S::THREADS) out[budget - n_last + m] = hi + m;
  if (need == 0) return;
  const float* row = w + b * stride_wb + s * stride_ws + lo;
  auto ranked = rank_row<uint32_t, S>([&](int i) { return row[i]; }, [](float x) { return weight_key(x); }, hi - lo, sh);
  ranked.cut(need);
  ranked.emit([&](int at, int i) { out[lo + at] = lo + i; });
}

// Rows of the kept slots of one slice to its first slots, into memory apart from it: a workgroup
// takes MOVE_ROWS of the slice's rows, of keys and values, in 16-byte pieces with MOVE_UN in flight
// per thread, and their weights.
constexpr int MOVE_THREADS = 256;
constexpr int MOVE_ROWS = 128;
constexpr int MOVE_UN = 8;
__global__ __launch_bounds__(MOVE_THREADS) void evict_copy_kernel(EvictMove a) {
  const int s = blockIdx.x, b = blockIdx.z;
  // (min(kv_len, budget) is the same before and after new_len, which may be kv_len, is written)
  const int n = max(0, min(min(a.kv_len[b], a.kv_cap), a.budget));
  if (s == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.new_len[b] = n;
  __shared__ int32_t from[MOVE_ROWS];
  for (int m0 = blockIdx.y * MOVE_ROWS; m0 < n; m0 += gridDim.y * MOVE_ROWS) {
    const int rows = min(MOVE_ROWS, n - m0);
    if (m0 >= (int)gridDim.y * MOVE_ROWS) __syncthreads();      // (the piece before has been moved)
    const int32_t* kept = a.kept + ((int64_t)b * a.slices + s) * a.budget + m0;
    if ((int)threadIdx.x < rows) {
      const int i = kept[threadIdx.x];
      from[threadIdx.x] = i;
      a.w_out[b * a.ostride_wb + s * a.ostride_ws + m0 + threadIdx.x] = a.w[b * a.stride_wb + s * a.stride_ws + i];
    }
    __syncthreads();
    const int per = a.row_bytes / 16, pieces = rows * per;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const char* src = (const char*)(part ? a.v : a.k) + b * a.stride_b + s * a.stride_s;
      char* dst = (char*)(part ? a.v_out : a.k_out) + b * a.ostride_b + s * a.ostride_s + (int64_t)m0 * a.row_bytes;
      for (int p0 = threadIdx.x; p0 < pieces; p0 += MOVE_THREADS * MOVE_UN) {
        u16x8 x[MOVE_UN];
#pragma unroll
        for (int j = 0; j < MOVE_UN; ++j) {
          const int p = min(p0 + j * MOVE_THREADS, pieces - 1), m = p / per;
          x[j] = __builtin_nontemporal_load(
              reinterpret_cast<const u16x8*>(src + (int64_t)from[m] * a.row_bytes + (p - m * per) * 16));
        }
#pragma unroll
        for (int j = 0; j < MOVE_UN; ++j) {
          const int p = p0 + j * MOVE_THREADS;
          if (p < pieces) __builtin_nontemporal_store(x[j], reinterpret_cast<u16x8*>(dst + (int64_t)p * 16));
        }
      }
    }
  }
}

// The same in place: a workgroup takes a stripe of STRIPE bytes of every key row or of every value
// row, in rounds of as many rows as its threads hold.  A round's rows are all read before any is
// written; a later round's sources lie at or after its own destinations, which the earlier rounds
// have not reached.  Rows that stay where they are, those before the first slot that went, are left.
constexpr int PLACE_THREADS = 512;
constexpr int PLACE_UN = 8;        // rows in flight per thread
template <int STRIPE>
__global__ __launch_bounds__(PLACE_THREADS) void evict_place_kernel(EvictMove a) {
  constexpr int PER = STRIPE / 16, ROWS = PLACE_THREADS / PER;
  const int s = blockIdx.x, b = blockIdx.z;
  const int stripes = a.row_bytes / STRIPE, part = blockIdx.y;      // stripes of K, of V, then the weights
  const int n = max(0, min(min(a.kv_len[b], a.kv_cap), a.budget));
  const int32_t* kept = a.kept + ((int64_t)b * a.slices + s) * a.budget;
  if (part == 2 * stripes) {
    float* w = a.w_out + b * a.ostride_wb + s * a.ostride_ws;
    for (int base = 0; base < n; base += PLACE_THREADS) {
      const int m = base + threadIdx.x;
      const float x = m < n ? w[kept[m]] : 0.f;
      __syncthreads();
      if (m < n) w[m] = x;
    }
    if (s == 0 && threadIdx.x == 0) a.new_len[b] = n;
    return;
  }
  const bool value = part >= stripes;
  char* at = (char*)(value ? a.v_out : a.k_out) + b * a.ostride_b + s * a.ostride_s +
             (value ? part - stripes : part) * STRIPE + threadIdx.x % PER * 16;
  for (int base = 0; base < n; base += ROWS * PLACE_UN) {
    u16x8 x[PLACE_UN];
    int from[PLACE_UN];
#pragma unroll
    for (int j = 0; j < PLACE_UN; ++j) {
      const int m = base + j * ROWS + threadIdx.x / PER;
      from[j] = m < n ? kept[m] : m;
    }
#pragma unroll
    for (int j = 0; j < PLACE_UN; ++j) {
      const int m = base + j * ROWS + threadIdx.x / PER;
      if (from[j] != m) x[j] = *reinterpret_cast<const u16x8*>(at + (int64_t)from[j] * a.row_bytes);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < PLACE_UN; ++j) {
      const int m = base + j * ROWS + threadIdx.x / PER;
      if (from[j] != m) *reinterpret_cast<u16x8*>(at + (int64_t)m * a.row_bytes) = x[j];
    }
  }
}

adt_status launch_kv_evict(const EvictMove& a, int B, int n_first, int n_last, hipStream_t st) {
  const dim3 grid(a.slices, B);
#define ADT_ES(...)                                                                                                 \
  evict_select_kernel<RankShape<__VA_ARGS__>><<<grid, RankShape<__VA_ARGS__>::THREADS, 0, st>>>(                    \
      a.w, a.stride_wb, a.stride_ws, a.kv_len, a.kv_cap, a.slices, a.budget, n_first, n_last, a.kept)
  if (a.kv_cap <= 4096) ADT_ES(256, 16, 8, 1, true);
  else if (a.kv_cap <= 16384) ADT_ES(1024, 16, 11, 2, true);
  else if (a.kv_cap <= 65536) ADT_ES(1024, 64, 11, 2, true);
  else ADT_ES(1024, 16, 11, 2, false);
#undef ADT_ES
  ADT_LAUNCH_CHECK();
  if (a.k_out != a.k) {
    const int most = std::min(a.kv_cap, a.budget);
    // (65535: the most workgroups that a launch may have in its second dimension)
    const int pieces = std::min((most + MOVE_ROWS - 1) / MOVE_ROWS, 65535);
    evict_copy_kernel<<<dim3(a.slices, pieces, B), MOVE_THREADS, 0, st>>>(a);
  } else if (a.row_bytes % 128 == 0) {
    evict_place_kernel<128><<<dim3(a.slices, 2 * (a.row_bytes / 128) + 1, B), PLACE_THREADS, 0, st>>>(a);
  } else {
    evict_place_kernel<16><<<dim3(a.slices, 2 * (a.row_bytes / 16) + 1, B), PLACE_THREADS, 0, st>>>(a);
  }
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
