// Rotary positions of a batch of rows and their append to the caches: queries and keys are
// rotated, pair by pair, by the angle position x frequency, and keys and values go to the slots
// after each sequence's prefix.  Positions are an input of their own (after an eviction a row's
// slot says nothing about its position).
//
// Bound by memory: every value is read once and written once, three flops each.  A workgroup
// takes one row (all its heads), or a part of one row's heads where there are few rows, and first
// makes the row's rot / 2 sines and cosines, in LDS; the heads then share them.  4096 rows of 32 + 8 + 8
// heads of 128: 18.5 us, 5.4 TB/s, in fp32 31.6; one row 3 us.  Where the rotated part is not whole 16-byte pieces
// (in the half layout, of each half) the call goes value by value: 24 of 96 dims 38.5 us, 32 of 96 15.7.
#include <algorithm>

#include "../launch.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(rope)

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MAX_PAIRS = 128;   // Dh <= 256

// (cos, sin) of pos * freq.  The angle may be millions of turns' worth of radians, of which only
// the part of a quarter turn decides: it is reduced in double, where 2^20 positions leave an error
// near 1e-10 turns (a float angle would be off by 0.06 radians), and the remainder, at most half
// a quarter turn, enters the float functions with a rounding of 2^-25 quarter turns.
__device__ __forceinline__ float2 turn(double pos, double freq) {
  const double quarters = pos * freq * 0x1.45f306dc9c883p-1;   // 2 / pi
  const double n = rint(quarters);
  float s, c;
  sincospif((float)(quarters - n) * 0.5f, &s, &c);
  const int k = (int)((long long)n & 3);
  const float2 cs = k & 1 ? make_float2(-s, c) : make_float2(c, s);
  return k & 2 ? make_float2(-cs.x, -cs.y) : cs;
}

template <typename T, int N, int ALIGN>
struct alignas(ALIGN) Pack {
  T v[N];
};

// One row's work is numbered in units of VEC neighbouring values, or of VEC pairs whose halves lie
// apart (half layout): of every query head, then of every key head, then of every value head.  VEC
// values are 16 bytes where the sizes and addresses allow it, else one value (interleaved: a pair).
template <typename T, int VEC, bool INTER>
__global__ __launch_bounds__(ROPE_THREADS) void rope_append_kernel(RopeRows a, const double* __restrict__ freq,
                                                                   float gain) {
  __shared__ float2 cs[ROPE_MAX_PAIRS];
  const int i = a.row0 + blockIdx.x, b = blockIdx.z;
  if (i >= min(a.n_rows[b], a.n_max)) return;
  const int64_t row = (int64_t)b * a.n_max + i;
  const int rot = a.rot, half = rot / 2, DH = a.Dh;
  for (int p = threadIdx.x; p < half; p += ROPE_THREADS) {
    const float2 t = turn((double)a.pos[row], freq[p]);
    cs[p] = make_float2(t.x * gain, t.y * gain);
  }
  __syncthreads();
  const int64_t slot = (int64_t)a.kv_len[b] + i;
  const bool store_kv = a.kv_len[b] >= 0 && slot < a.kv_cap;
  if (!store_kv && threadIdx.x == 0 && blockIdx.y == 0) dev_fail(DEVINV_KV_RANGE);
  constexpr int W = INTER && VEC == 1 ? 2 : VEC;       // values per unit and half
  const int turned = INTER ? rot / W : half / W;       // rotating units per head
  const int units = turned + (DH - rot) / W;           // per query or key head
  const int v_units = DH / W;
  const int nq = a.H * units, nk = a.Hkv * units, total = nq + nk + a.Hkv * v_units;
  typedef Pack<T, W, VEC == 1 ? sizeof(T) : 16> P;
  for (int u = blockIdx.y * ROPE_THREADS + threadIdx.x; u < total; u += gridDim.y * ROPE_THREADS) {
    if (u >= nq + nk) {
      if (!store_kv) continue;
      const int h = (u - nq - nk) / v_units, d = (u - nq - nk) % v_units * W;
      *reinterpret_cast<P*>((T*)a.vc + b * a.stride_b + h * a.stride_h + slot * DH + d) =
          *reinterpret_cast<const P*>((const T*)a.v + row * a.ldv + (int64_t)h * DH + d);
      continue;
    }
    const bool key = u >= nq;
    const int h = (key ? u - nq : u) / units, w = (key ? u - nq : u) % units;
    const T* src = key ? (const T*)a.k + row * a.ldk + (int64_t)h * DH : (const T*)a.q + row * a.ldq + (int64_t)h * DH;
    T* dst = key ? (T*)a.kc + b * a.stride_b + h * a.stride_h + slot * DH
                 : (T*)a.q_out + (row * a.H + h) * (int64_t)DH;
    if (key && !store_kv) continue;
    if (w >= turned) {
      const int d = rot + (w - turned) * W;
      *reinterpret_cast<P*>(dst + d) = *reinterpret_cast<const P*>(src + d);
    } else if constexpr (INTER) {
      const int d = w * W;
      P x = *reinterpret_cast<const P*>(src + d);
#pragma unroll
      for (int e = 0; e < W; e += 2) {
        const float2 t = cs[(d + e) / 2];
        const float x0 = Elem<T>::load(x.v, e), x1 = Elem<T>::load(x.v, e + 1);
        Elem<T>::store(x.v, e, x0 * t.x - x1 * t.y);
        Elem<T>::store(x.v, e + 1, x0 * t.y + x1 * t.x);
      }
      *reinterpret_cast<P*>(dst + d) = x;
    } else {
      const int d = w * W;
      P x = *reinterpret_cast<const P*>(src + d), y = *reinterpret_cast<const P*>(src + half + d);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float2 t = cs[d + e];
        const float x0 = Elem<T>::load(x.v, e), x1 = Elem<T>::load(y.v, e);
        Elem<T>::store(x.v, e, x0 * t.x - x1 * t.y);
        Elem<T>::store(y.v, e, x0 * t.y + x1 * t.x);
      }
      *reinterpret_cast<P*>(dst + d) = x;
      *reinterpret_cast<P*>(dst + half + d) = y;
    }
  }
}

template <typename T>
static adt_status rope_append(RopeRows a, int B, const double* freq, float gain, bool inter, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int64_t lds[] = {a.ldq, a.ldk, a.ldv, a.stride_b, a.stride_h};
  const void* ptrs[] = {a.q, a.k, a.v, a.q_out, a.kc, a.vc};
  bool wide = a.Dh % V == 0 && a.rot % (inter ? V : 2 * V) == 0;
  for (int64_t l : lds) wide = wide && l % V == 0;
  for (const void* p : ptrs) wide = wide && (uintptr_t)p % 16 == 0;
  // few rows: a row's units over several workgroups (a unit a thread) until some 1024 are there
  const int width = wide ? V : 1;
  const int units = (a.H + 2 * a.Hkv) * a.Dh / width;
  int parts = (units + ROPE_THREADS - 1) / ROPE_THREADS;
  const int64_t rows = (int64_t)B * a.n_max;
  parts = (int)std::min<int64_t>(parts, std::max<int64_t>(1, 1024 / rows));
  // (a launch has fewer than 2^32 threads in a dimension, or it wraps: more rows take several)
  constexpr int MOST = 1 << 23;
#define ADT_ROPE(VECV, INTERV) rope_append_kernel<T, VECV, INTERV><<<grid, ROPE_THREADS, 0, st>>>(a, freq, gain)
  for (int64_t r0 = 0; r0 < a.n_max; r0 += MOST) {
    a.row0 = (int)r0;
    const dim3 grid((unsigned)std::min<int64_t>(MOST, a.n_max - r0), parts, B);
    if (wide) {
      if (inter) ADT_ROPE(V, true);
      else ADT_ROPE(V, false);
    } else {
      if (inter) ADT_ROPE(1, true);
      else ADT_ROPE(1, false);
    }
    ADT_LAUNCH_CHECK();
  }
#undef ADT_ROPE
  return ADT_OK;
}

adt_status launch_rope_append(RopeRows a, int B, const double* freq, float gain, bool inter, int dtype,
                              hipStream_t st) {
  return dtype == ADT_BF16 ? rope_append<uint16_t>(a, B, freq, gain, inter, st)
                           : rope_append<float>(a, B, freq, gain, inter, st);
}

}  // namespace adt
