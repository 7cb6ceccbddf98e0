// Rows on their way into, out of and within a cache of any type: norms of queries and keys with the
// rotation and the append, conversion between plain and eight-bit caches, and the moves of an
// accepted path.
//
// All are bound by memory: a value is read once and written once.  A head's row of Dh values goes to a
// group of neighbouring lanes, a 16-byte piece each, so that its sum of squares and its largest size
// are a few lane exchanges away and every access is whole lines.
//
// Measured (a 4 GiB copy reads and writes 4.68 TB/s): 4001 rows of 32 query and 8 + 8 key and value heads
// of 128 dims into int8, half of each head rotated, 26.9 us (3.3 TB/s); 61 rows of 32 heads into e4m3 5.7 us (latency);
// sixteen e4m3 caches of 512 to 4096 slots of 8 heads read back 48-52 us (a copy's rate); 1100 slots of 32
// heads put in int8 12 us (2.3 TB/s), read back 7.0 (3.9); 12 rows of each of 1024 slices moved 4.9 us (latency).
#include <algorithm>

#include "../eight_bit.h"
#include "../launch.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(kv_rows)

constexpr int KR_THREADS = 256;
constexpr int KR_MAX_PAIRS = 128;     // Dh <= 256

template <typename T, int N, int ALIGN>
struct alignas(ALIGN) RowPack {
  T v[N];
};

// (cos, sin) of pos * freq in double: the angle less whole quarter turns (pi / 2 in two parts, so far
// positions lose nothing), then the Taylor sums to r^18 and r^17, whose next terms are below 2^-56 for
// |r| <= pi / 4.
__device__ __forceinline__ double2 turn64(double pos, double freq) {
  const double angle = pos * freq;
  const double n = rint(angle * 0x1.45f306dc9c883p-1);     // 2 / pi
  double r = fma(-n, 0x1.921fb54442d18p+0, angle);
  r = fma(-n, 0x1.1a62633145c07p-54, r);
  const double z = r * r;
  double c = -1.0 / 6402373705728000.0;
  c = fma(c, z, 1.0 / 20922789888000.0);
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  double s = 1.0 / 355687428096000.0;
  s = fma(s, z, -1.0 / 1307674368000.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  const int k = (int)((long long)n & 3);
  const double2 t = k & 1 ? make_double2(-s, c) : make_double2(c, s);
  return k & 2 ? make_double2(-t.x, -t.y) : t;
}

// Sum and maximum over groups of `lanes` (a power of two) neighbouring lanes, all of which take part.
template <typename R>
__device__ __forceinline__ R group_sum(R v, int lanes) {
  for (int o = lanes / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}
__device__ __forceinline__ float group_max(float v, int lanes) {
  for (int o = lanes / 2; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
  return v;
}

// A row's values of this lane, N pieces of VEC of them, into an eight-bit cache row: the group agrees
// on the scale first.  piece(j): the first dim of piece j; dims from Dh on are none (values 0).
template <typename C, int VEC, int N, typename R, class F>
__device__ __forceinline__ void store_codes(const R (&y)[N][VEC], int lanes, bool first, int Dh, C* row, float* scale,
                                            F piece) {
  float largest = 0.f, odd = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float f = (float)y[j][e];
      largest = fmaxf(largest, fabsf(f));
      odd += f * 0.f;               // NaN if any value is not finite
    }
  largest = group_max(odd != odd ? INFINITY : largest, lanes);
  double inverse;
  const float s = row_scale<C>(largest, inverse);
  if (first) *scale = s;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int d = piece(j);
    if (d >= Dh) continue;
    float t[VEC];
    // (a row that is not finite has inverse 0 and codes 0)
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = s == s ? (float)((double)y[j][e] * inverse) : 0.f;
    if constexpr (VEC == 1) {
      reinterpret_cast<uint8_t*>(row)[d] = (uint8_t)encode4<C>(t[0], 0.f, 0.f, 0.f);
    } else {
      RowPack<uint32_t, VEC / 4, VEC> p;
#pragma unroll
      for (int e = 0; e < VEC; e += 4) p.v[e / 4] = encode4<C>(t[e], t[e + 1], t[e + 2], t[e + 3]);
      *reinterpret_cast<decltype(p)*>(row + d) = p;
    }
  }
}

// A workgroup takes ROWS rows, all their heads or a part of them; a group of `lanes` lanes takes a head, and
// others after it, whose values are requested HEADS heads of all rows at once, the first ones before the
// rows' sines and cosines are made (in LDS): the two waits pass together.  Many rows go two to a
// workgroup, which then starts half as often and reads a head's gains for two; few rows one, with
// three heads requested at once.  VEC values are 16 bytes where sizes and addresses allow it (N = 1 piece
// a lane), else one value (a wave a head, N = 4).  A pair's other half is read from memory beside it (the
// same lines).
template <typename T, typename C, int VEC, bool INTER, int HEADS, int ROWS>
__global__ __launch_bounds__(KR_THREADS) void norm_rope_kernel(NormRopeRows a, int lanes) {
  constexpr int N = VEC == 1 ? 4 : 1;
  constexpr bool MATES = !INTER || VEC == 1;      // the other half of a pair lies outside the piece
  __shared__ double2 cs[ROWS][KR_MAX_PAIRS];
  __shared__ float2 cs32[ROWS][KR_MAX_PAIRS];
  const int b = blockIdx.z;
  const int n_rows = min(a.n_rows[b], a.n_max), kv_len = a.kv_len[b];
  const int64_t i0 = a.row0 + (int64_t)blockIdx.x * ROWS;
  if (i0 >= n_rows) return;
  const int count = (int)min((int64_t)ROWS, n_rows - i0);
  const int64_t row0 = (int64_t)b * a.n_max + i0, slot0 = kv_len + i0;
  const int rot = a.rot, half = rot / 2, DH = a.c.Dh, H = a.H, Hkv = a.c.heads, heads = H + 2 * Hkv;
  // rows whose slots lie in the cache: [0, kept) of the `count` (a negative length has none)
  const int kept = kv_len < 0 ? 0 : (int)max((int64_t)0, min((int64_t)count, a.c.cap - slot0));
  if (kept < count && threadIdx.x == 0 && blockIdx.y == 0) dev_fail(DEVINV_KV_RANGE);
  const int per = KR_THREADS / lanes, sub = threadIdx.x / lanes, l = threadIdx.x % lanes;
  const int first = blockIdx.y * per + sub, step = gridDim.y * per;
  typedef RowPack<T, VEC, VEC == 1 ? sizeof(T) : 16> P;
  // this lane's pieces: first dim, and that of the other half of its pairs (itself, if it is not rotated)
  auto piece = [&](int j) { return (l + j * lanes) * VEC; };
  auto mate = [&](int j) {
    const int d = piece(j);
    return d >= rot ? d : INTER ? d ^ 1 : d < half ? d + half : d - half;
  };
  P own[HEADS][ROWS][N], other[HEADS][ROWS][N];
  auto request = [&](int h0) {
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
      const int hd = h0 + u * step;
      if (hd >= heads) break;
      const bool query = hd < H, key = !query && hd < H + Hkv;
      const int64_t ld = query ? a.ldq : key ? a.ldk : a.ldv;
      const T* src = (const T*)(query ? a.q : key ? a.k : a.v) + row0 * ld + (int64_t)(query ? hd : key ? hd - H : hd - H - Hkv) * DH;
#pragma unroll
      for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int j = 0; j < N; ++j) {
          const T* at = src + min(r, count - 1) * ld;
          own[u][r][j] = P{};
          if (piece(j) < DH) own[u][r][j] = *reinterpret_cast<const P*>(at + piece(j));
          if constexpr (MATES) {
            other[u][r][j] = P{};
            if (piece(j) < DH && (query || key)) other[u][r][j] = *reinterpret_cast<const P*>(at + mate(j));
          }
        }
    }
  };
  request(first);
  for (int x = threadIdx.x; x < count * half; x += KR_THREADS) {
    const int r = x / half, p = x % half;
    const double2 t = turn64((double)a.pos[row0 + r], a.freq[p]);
    cs[r][p] = make_double2(t.x * a.gain, t.y * a.gain);
    cs32[r][p] = make_float2((float)(t.x * a.gain), (float)(t.y * a.gain));
  }
  __syncthreads();
  // y = x c + other s, s with the sign that the half has
  auto turn_of = [&](auto zero, int r, int j, int e) {
    const int d = piece(j) + e;
    const bool second = INTER ? d & 1 : d >= half;
    const int p = INTER ? d / 2 : second ? d - half : d;
    struct {
      decltype(zero) x, y;
    } t;
    if constexpr (sizeof(zero) == 8) t.x = cs[r][p].x, t.y = cs[r][p].y;
    else t.x = cs32[r][p].x, t.y = cs32[r][p].y;
    if (!second) t.y = -t.y;
    return t;
  };

  // a head's gains at this lane's dims, and at their mates where those lie outside the piece (none: 1)
  float gain[N][VEC], mate_gain[N][VEC];
  auto gains = [&](const float* g) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      typedef RowPack<float, VEC, VEC == 1 ? 4 : 16> G;
      G x, y;
#pragma unroll
      for (int e = 0; e < VEC; ++e) x.v[e] = y.v[e] = 1.f;
      if (g && piece(j) < DH) {
        if constexpr (VEC == 1) {
          x.v[0] = g[piece(j)];
          y.v[0] = g[mate(j)];
        } else {
#pragma unroll
          for (int e = 0; e < VEC; ++e) x.v[e] = g[piece(j) + e];
          if constexpr (MATES) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) y.v[e] = g[mate(j) + e];
          }
        }
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        gain[j][e] = x.v[e];
        if constexpr (MATES) mate_gain[j][e] = y.v[e];
      }
    }
  };
  // Sum of squares of a row's values times `unit`.
  auto squares = [&](auto unit, const P (&mine)[N]) {
    decltype(unit) ss = 0;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const auto x = (decltype(unit))Elem<T>::load(mine[j].v, e) * unit;
        ss += x * x;
      }
    return group_sum(ss, lanes);
  };
  // This lane's values of a row, times `first` and `second` before anything else and `last` after, with the gains and
  // the turns between them.
  auto turned = [&](const P (&mine)[N], const P (&mates)[N], int r, auto first, auto second, auto last, auto& y) {
    typedef decltype(first) R;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      R x[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[e] = (R)Elem<T>::load(mine[j].v, e) * first * second * (R)gain[j][e];
      // (a piece is rotated as a whole, or not: a dim that is not takes nothing of another)
      const bool whole = piece(j) < rot;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        y[j][e] = x[e] * last;
        if (!whole) continue;
        const R w = MATES ? (R)Elem<T>::load(mates[j].v, e) * first * second * (R)mate_gain[j][e] : x[e ^ 1];
        const auto t = turn_of(first, r, j, e);
        y[j][e] = last * (x[e] * t.x + w * t.y);
      }
    }
  };
  // one head of a row, queries in fp32 and keys in double
  auto made = [&](auto zero, const P (&mine)[N], const P (&mates)[N], int r, bool norm, auto store) {
    typedef decltype(zero) R;
    R y[N][VEC];
    if constexpr (sizeof(R) == 8) {
      turned(mine, mates, r, 1.0, 1.0, norm ? 1.0 / sqrt(squares(1.0, mine) / (double)DH + (double)a.eps) : 1.0, y);
    } else {
      // the factor of a row's values times `unit` (the hardware's reciprocal root of an fp32 number is within its
      // last bit)
      auto factor = [&](float ss, float unit) { return __builtin_amdgcn_rsqf(ss * (1.f / (float)DH) + a.eps * unit * unit); };
      const float ss = norm ? squares(1.f, mine) : 0.f;
      const bool past = !(ss <= 3.402823466e38f);
      bool again = past;
      if (!past) {
        turned(mine, mates, r, 1.f, 1.f, norm ? factor(ss, 1.f) : 1.f, y);
        float odd = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) odd += y[j][e] * 0.f;        // NaN if any is not finite
        again = odd != odd;
      }
      if (again) {
        // Squares, or products with gains and turns, left fp32: the row's factor comes before those.  Values whose squares
        // are too large are made 2^70 times smaller for them, and half of that goes to the factor, so that neither they nor it
        // leave fp32 at its lower end; values that have no factor are made as much smaller until the end.
        float first = 1.f, second = 1.f;
        if (!norm) first = 0x1p-70f;
        else if (past) first = 0x1p-35f, second = 0x1p-35f * factor(squares(0x1p-70f, mine), 0x1p-70f);
        else second = factor(ss, 1.f);
        // (a value that was finite stays: what is small beside a large one would be lost)
        float z[N][VEC];
        turned(mine, mates, r, first, second, norm ? 1.f : 0x1p70f, z);
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) y[j][e] = past || !(fabsf(y[j][e]) <= 3.402823466e38f) ? z[j][e] : y[j][e];
      }
    }
    store(y);
  };
  auto plain = [&](const auto& y, T* dst) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (piece(j) >= DH) continue;
      P p;
#pragma unroll
      for (int e = 0; e < VEC; ++e) Elem<T>::store(p.v, e, (float)y[j][e]);
      *reinterpret_cast<P*>(dst + piece(j)) = p;
    }
  };
  auto take = [&](int u, int hd) {
    const bool query = hd < H, key = !query && hd < H + Hkv;
    const int h = query ? hd : key ? hd - H : hd - H - Hkv;
    const float* g = query ? a.q_norm : a.k_norm;
    // (queries that share their gains keep them from one head to the next)
    if ((query || key) && (!query || a.norm_step || hd == first)) gains(g ? g + (int64_t)h * a.norm_step : nullptr);
    C* to = (C*)(key ? a.c.k : a.c.v) + b * a.c.stride_b + h * a.c.stride_h + slot0 * DH;
    float* scale = (key ? a.c.k_scale : a.c.v_scale) + (int64_t)b * a.c.scale_b + h * a.c.scale_h + slot0;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      if (query) {
        if (r < count)
          made(0.f, own[u][r], other[u][r], r, g != nullptr,
               [&](const auto& y) { plain(y, (T*)a.q_out + ((row0 + r) * H + h) * (int64_t)DH); });
        continue;
      }
      if (r >= kept) continue;
      auto store = [&](const auto& y) {
        if constexpr (EIGHT<C>) store_codes<C, VEC, N>(y, lanes, l == 0, DH, to + r * DH, scale + r, piece);
        else plain(y, (T*)to + r * DH);
      };
      if (key) {
        made(0.0, own[u][r], other[u][r], r, g != nullptr, store);
      } else {
        float y[N][VEC];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
          for (int e = 0; e < VEC; ++e) y[j][e] = Elem<T>::load(own[u][r][j].v, e);
        store(y);
      }
    }
  };
  for (int h0 = first; h0 < heads; h0 += HEADS * step) {
    if (h0 != first) request(h0);
#pragma unroll
    for (int u = 0; u < HEADS; ++u)
      if (h0 + u * step < heads) take(u, h0 + u * step);
  }
}

// Rows from which on they go two to a workgroup.  One, two and four to a workgroup, 32 + 8 + 8 heads of 128
// dims into int8, rotated in halves: 1000 rows 11.8, 13.3, 18.8 us; 1536 16.8, 15.1; 4001 35.4, 29.9, 38.2; 8000 64.8, 53.7,
// 58.7; half of each head in neighbouring pairs: 1250 rows 11.5, 12.8; 1536 13.2, 13.8; 1750 16.9, 15.3; fp32 into
// fp32: 1250 17.7, 19.3; 1750 24.9, 20.9; 4001 45.7, 38.7, 35.7.  (Four hold so many registers that few
// workgroups share a CU.)
constexpr int KR_MANY = 1536;

static int pow2_at_least(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

template <typename T, typename C>
static adt_status norm_rope(NormRopeRows a, bool inter, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  const int64_t strides[] = {a.ldq, a.ldk, a.ldv}, cache[] = {a.c.stride_b, a.c.stride_h};
  const int code = EIGHT<C> ? V : 16 / (int)sizeof(C);     // elements a cache row's piece is aligned to
  bool wide = a.c.Dh % V == 0 && a.rot % (inter ? V : 2 * V) == 0 && (uintptr_t)a.q % 16 == 0 && (uintptr_t)a.k % 16 == 0 &&
              (uintptr_t)a.v % 16 == 0 && (uintptr_t)a.q_out % 16 == 0 && (uintptr_t)a.c.k % 16 == 0 &&
              (uintptr_t)a.c.v % 16 == 0;
  for (int64_t s : strides) wide = wide && s % V == 0;
  for (int64_t s : cache) wide = wide && s % code == 0;
  const int lanes = wide ? pow2_at_least(a.c.Dh / V) : WAVE;
  const int per = KR_THREADS / lanes;
  int parts = (a.H + 2 * a.c.heads + per - 1) / per;
  const int64_t rows = (int64_t)a.c.B * a.n_max;
  const bool many = rows >= KR_MANY && a.n_max >= 2;
  // few rows: a row's heads over several workgroups until some 1024 are there
  parts = many ? 1 : (int)std::min<int64_t>(parts, std::max<int64_t>(1, 1024 / rows));
  // (a launch has fewer than 2^32 threads in a dimension, or it wraps: more rows take several)
  constexpr int MOST = 1 << 23;
#define ADT_NR(VECV, INTERV)                                                                        \
  if (many) norm_rope_kernel<T, C, VECV, INTERV, 1, 2><<<grid, KR_THREADS, 0, st>>>(a, lanes);      \
  else norm_rope_kernel<T, C, VECV, INTERV, 3, 1><<<grid, KR_THREADS, 0, st>>>(a, lanes)
  for (int64_t r0 = 0; r0 < a.n_max; r0 += MOST) {
    a.row0 = (int)r0;
    const int64_t left = std::min<int64_t>(MOST, a.n_max - r0);
    const dim3 grid((unsigned)(many ? (left + 1) / 2 : left), parts, a.c.B);
    if (wide) {
      if (inter) { ADT_NR(V, true); }
      else { ADT_NR(V, false); }
    } else {
      if (inter) { ADT_NR(1, true); }
      else { ADT_NR(1, false); }
    }
    ADT_LAUNCH_CHECK();
  }
#undef ADT_NR
  return ADT_OK;
}

adt_status launch_norm_rope_append(NormRopeRows a, bool inter, int dtype, hipStream_t st) {
  if (dtype == ADT_BF16) {
    if (a.c.type == ADT_E4M3) return norm_rope<uint16_t, E4M3>(a, inter, st);
    if (a.c.type == ADT_I8) return norm_rope<uint16_t, I8>(a, inter, st);
    return norm_rope<uint16_t, uint16_t>(a, inter, st);
  }
  if (a.c.type == ADT_E4M3) return norm_rope<float, E4M3>(a, inter, st);
  if (a.c.type == ADT_I8) return norm_rope<float, I8>(a, inter, st);
  return norm_rope<float, float>(a, inter, st);
}

// ---------------------------------------------------------------------------- conversion
struct ConvertArgs {
  adt_kv_cache src, dst;
  const int32_t *length, *src_start, *dst_start;
  int n_max;
};
// The rows of sequence b: first slots on either side, and how many; rows outside either cache go.
struct ConvertSpan {
  int64_t s0, d0;
  int first, end;
};
__device__ __forceinline__ ConvertSpan convert_span(const ConvertArgs& a, int b, bool check) {
  ConvertSpan c;
  c.s0 = a.src_start ? a.src_start[b] : 0;
  c.d0 = a.dst_start ? a.dst_start[b] : 0;
  const int64_t n = min(a.length[b], a.n_max);
  const int64_t first = max((int64_t)0, max(-c.s0, -c.d0));
  const int64_t end = min(n, min((int64_t)a.src.cap - c.s0, (int64_t)a.dst.cap - c.d0));
  if (check && n > 0 && (first > 0 || end < n)) dev_fail(DEVINV_KV_RANGE);
  c.first = (int)min(first, (int64_t)a.n_max);
  c.end = (int)max(end, (int64_t)0);
  return c;
}

// Codes to values: a group of lanes a row, 16 codes a lane (or one, and up to four pieces).  A lane takes one
// row at a time; four in flight were no faster.
template <typename C, typename T, int VEC>
__global__ __launch_bounds__(KR_THREADS) void cache_read_kernel(ConvertArgs a, int lanes) {
  constexpr int N = VEC == 1 ? 4 : 1;
  const int b = blockIdx.z, h = blockIdx.y >> 1, DH = a.src.Dh;
  const bool key = !(blockIdx.y & 1);
  const ConvertSpan c = convert_span(a, b, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0);
  const C* src = (const C*)(key ? a.src.k : a.src.v) + b * a.src.stride_b + h * a.src.stride_h + c.s0 * DH;
  T* dst = (T*)(key ? a.dst.k : a.dst.v) + b * a.dst.stride_b + h * a.dst.stride_h + c.d0 * DH;
  const float* scale = (key ? a.src.k_scale : a.src.v_scale) + b * a.src.scale_b + h * a.src.scale_h + c.s0;
  const int per = KR_THREADS / lanes, sub = threadIdx.x / lanes, l = threadIdx.x % lanes;
  for (int64_t i = c.first + (int64_t)blockIdx.x * per + sub; i < c.end; i += (int64_t)gridDim.x * per) {
    const float s = scale[i];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int d = (l + j * lanes) * VEC;
      if (d >= DH) continue;
      const int64_t at = i * DH + d;
      if constexpr (VEC == 1) {
        Elem<T>::store(dst, at, decode4<C>(reinterpret_cast<const uint8_t*>(src)[at]).x * s);
      } else {
        const uint4 w = *reinterpret_cast<const uint4*>(src + at);
        const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float4 f = decode4<C>(q[u]);
          store4(dst + at + 4 * u, f.x * s, f.y * s, f.z * s, f.w * s);
        }
      }
    }
  }
}

// Values to codes: a group of lanes a row.
template <typename T, typename C, int VEC>
__global__ __launch_bounds__(KR_THREADS) void cache_write_kernel(ConvertArgs a, int lanes) {
  constexpr int N = VEC == 1 ? 4 : 1;
  const int b = blockIdx.z, h = blockIdx.y >> 1, DH = a.src.Dh;
  const bool key = !(blockIdx.y & 1);
  const ConvertSpan c = convert_span(a, b, threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0);
  const T* src = (const T*)(key ? a.src.k : a.src.v) + b * a.src.stride_b + h * a.src.stride_h + c.s0 * DH;
  C* dst = (C*)(key ? a.dst.k : a.dst.v) + b * a.dst.stride_b + h * a.dst.stride_h + c.d0 * DH;
  float* scale = (key ? a.dst.k_scale : a.dst.v_scale) + b * a.dst.scale_b + h * a.dst.scale_h + c.d0;
  const int per = KR_THREADS / lanes, sub = threadIdx.x / lanes, l = threadIdx.x % lanes;
  auto piece = [&](int j) { return (l + j * lanes) * VEC; };
  typedef RowPack<T, VEC, VEC == 1 ? sizeof(T) : 16> P;
  for (int64_t i = c.first + (int64_t)blockIdx.x * per + sub; i < c.end; i += (int64_t)gridDim.x * per) {
    float y[N][VEC];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      P p{};
      if (piece(j) < DH) p = *reinterpret_cast<const P*>(src + i * DH + piece(j));
#pragma unroll
      for (int e = 0; e < VEC; ++e) y[j][e] = Elem<T>::load(p.v, e);
    }
    store_codes<C, VEC, N>(y, lanes, l == 0, DH, dst + i * DH, scale + i, piece);
  }
}

// Workgroups along the slots: one step each, unless that were more than a launch may have.
constexpr int64_t KR_GRID = 1 << 20;

template <typename C, typename T>
static adt_status cache_read(const ConvertArgs& a, hipStream_t st) {
  bool wide = a.src.Dh % 16 == 0 && (uintptr_t)a.src.k % 16 == 0 && (uintptr_t)a.src.v % 16 == 0 &&
              (uintptr_t)a.dst.k % 16 == 0 && (uintptr_t)a.dst.v % 16 == 0;
  const int64_t strides[] = {a.src.stride_b, a.src.stride_h, a.dst.stride_b, a.dst.stride_h};
  for (int64_t s : strides) wide = wide && s % 16 == 0;
  const int lanes = wide ? pow2_at_least(a.src.Dh / 16) : WAVE;
  const int64_t steps = ((int64_t)a.n_max * lanes + KR_THREADS - 1) / KR_THREADS;
  const dim3 grid((unsigned)std::min<int64_t>(KR_GRID, steps), 2 * a.src.heads, a.src.B);
  if (wide) cache_read_kernel<C, T, 16><<<grid, KR_THREADS, 0, st>>>(a, lanes);
  else cache_read_kernel<C, T, 1><<<grid, KR_THREADS, 0, st>>>(a, lanes);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

template <typename T, typename C>
static adt_status cache_write(const ConvertArgs& a, hipStream_t st) {
  constexpr int V = 16 / sizeof(T);
  bool wide = a.src.Dh % V == 0 && (uintptr_t)a.src.k % 16 == 0 && (uintptr_t)a.src.v % 16 == 0 &&
              (uintptr_t)a.dst.k % V == 0 && (uintptr_t)a.dst.v % V == 0;
  const int64_t strides[] = {a.src.stride_b, a.src.stride_h, a.dst.stride_b, a.dst.stride_h};
  for (int64_t s : strides) wide = wide && s % V == 0;
  const int lanes = wide ? pow2_at_least(a.src.Dh / V) : WAVE;
  const int64_t steps = ((int64_t)a.n_max * lanes + KR_THREADS - 1) / KR_THREADS;
  const dim3 grid((unsigned)std::min<int64_t>(KR_GRID, steps), 2 * a.src.heads, a.src.B);
  if (wide) cache_write_kernel<T, C, V><<<grid, KR_THREADS, 0, st>>>(a, lanes);
  else cache_write_kernel<T, C, 1><<<grid, KR_THREADS, 0, st>>>(a, lanes);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

adt_status launch_cache_convert(const adt_kv_cache& src, const adt_kv_cache& dst, const int32_t* length, int n_max,
                                const int32_t* src_start, const int32_t* dst_start, hipStream_t st) {
  const ConvertArgs a{src, dst, length, src_start, dst_start, n_max};
  if (src.type == ADT_E4M3)
    return dst.type == ADT_BF16 ? cache_read<E4M3, uint16_t>(a, st) : cache_read<E4M3, float>(a, st);
  if (src.type == ADT_I8) return dst.type == ADT_BF16 ? cache_read<I8, uint16_t>(a, st) : cache_read<I8, float>(a, st);
  if (dst.type == ADT_E4M3)
    return src.type == ADT_BF16 ? cache_write<uint16_t, E4M3>(a, st) : cache_write<float, E4M3>(a, st);
  return src.type == ADT_BF16 ? cache_write<uint16_t, I8>(a, st) : cache_write<float, I8>(a, st);
}

// ---------------------------------------------------------------------------- accepted path
// A workgroup takes whole slices: it reads every row that moves into registers, with its scales, and
// writes after a barrier, as a destination may be another row's source.
template <int RM>
__global__ __launch_bounds__(KR_THREADS) void cache_compact_kernel(adt_kv_cache c, int row_bytes,
                                                                   const int32_t* __restrict__ kv_len,
                                                                   const int32_t* __restrict__ path, int path_stride,
                                                                   const int32_t* __restrict__ n_acc, int a_max,
                                                                   int slices_each) {
  const int b = blockIdx.y, s0 = blockIdx.x * slices_each;
  const int acc = min(n_acc[b], a_max);
  const int64_t L = kv_len[b];
  const int per_row = row_bytes / 16, per_slice = a_max * per_row, total = slices_each * per_slice;
  const int64_t es = row_bytes / c.Dh;
  u16x8 kr[RM], vr[RM];
  float ks[RM], vs[RM];
  // piece p: slice, rank on the path, 16 bytes of the row; false where nothing moves
  struct Move {
    int slice, piece;
    int64_t from, to;
  };
  auto move = [&](int it, Move& m) {
    const int p = threadIdx.x + it * KR_THREADS;
    if (p >= total) return false;
    m.slice = s0 + p / per_slice;
    const int w = p % per_slice, rank = w / per_row + 1;
    m.piece = w % per_row;
    if (m.slice >= c.heads || rank > acc) return false;
    const int node = path[(int64_t)b * path_stride + rank];
    m.from = L + node;
    m.to = L + rank;
    if (node < rank || node >= ADT_MAX_NODES) {
      dev_fail(DEVINV_PATH);
      return false;
    }
    if (L < 0 || m.from >= c.cap) {
      dev_fail(DEVINV_KV_RANGE);
      return false;
    }
    return true;
  };
#pragma unroll
  for (int it = 0; it < RM; ++it) {
    Move m;
    if (!move(it, m)) continue;
    const int64_t at = (b * c.stride_b + m.slice * c.stride_h + m.from * c.Dh) * es;
    kr[it] = reinterpret_cast<const u16x8*>((const char*)c.k + at)[m.piece];
    vr[it] = reinterpret_cast<const u16x8*>((const char*)c.v + at)[m.piece];
    if (c.k_scale && m.piece == 0) {
      const int64_t sc = b * c.scale_b + m.slice * c.scale_h + m.from;
      ks[it] = c.k_scale[sc];
      vs[it] = c.v_scale[sc];
    }
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < RM; ++it) {
    Move m;
    if (!move(it, m)) continue;
    const int64_t at = (b * c.stride_b + m.slice * c.stride_h + m.to * c.Dh) * es;
    reinterpret_cast<u16x8*>((char*)c.k + at)[m.piece] = kr[it];
    reinterpret_cast<u16x8*>((char*)c.v + at)[m.piece] = vr[it];
    if (c.k_scale && m.piece == 0) {
      const int64_t sc = b * c.scale_b + m.slice * c.scale_h + m.to;
      c.k_scale[sc] = ks[it];
      c.v_scale[sc] = vs[it];
    }
  }
}

adt_status launch_cache_compact(const adt_kv_cache& c, const int32_t* kv_len, const int32_t* path, int path_stride,
                                const int32_t* n_acc, int a_max, hipStream_t st) {
  const int es = c.type == ADT_F32 ? 4 : c.type == ADT_BF16 ? 2 : 1, row_bytes = c.Dh * es;
  const int pieces = a_max * (row_bytes / 16);      // of a slice: at most 127 * 64
  const int rm = pieces <= 2 * KR_THREADS ? 2 : pieces <= 8 * KR_THREADS ? 8 : 32;
  const int each = std::max(1, std::min(c.heads, rm * KR_THREADS / pieces));
  const dim3 grid((c.heads + each - 1) / each, c.B);
#define ADT_CC(RM) \
  cache_compact_kernel<RM><<<grid, KR_THREADS, 0, st>>>(c, row_bytes, kv_len, path, path_stride, n_acc, a_max, each)
  if (rm == 2) ADT_CC(2);
  else if (rm == 8) ADT_CC(8);
  else ADT_CC(32);
#undef ADT_CC
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

}  // namespace adt
