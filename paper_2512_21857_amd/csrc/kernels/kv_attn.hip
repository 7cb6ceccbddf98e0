// Tree attention over caches of any type, and behind a prefix that groups of sequences share.
//
// A row's context has up to two parts: the prefix of its group and the cache of its sequence.  Softmax
// over both is the merge of softmax over each: a part gives the row's maximum m, sum l and
// unnormalised output o, and
//   out = sum of 2^(m_i - M) o_i / sum of 2^(m_i - M) l_i,  M the largest m_i.
// So a group's prefix is one attention of all the group's rows, wherever their trees are, over keys
// that are read once for 128 of them; a sequence's own slots are another, with the tree's mask.  Both
// are jobs of one launch: (part, group or sequence, key-value head, block of rows, range of keys).
// Their results meet in a second launch, always in one order; where a row's keys are all in one job,
// that job writes the output.
//
// Eight-bit keys are codes kc with a scale each, so  q . k = scale (q . kc),  p v = (p scale) vc:  bf16
// holds every code exactly, the products take codes as they are, and the scales meet scores and
// probabilities in fp32.
//
// What bounds it, measured (attention + merge; a 4 GiB copy moves 4.68 TB/s, an 8192-cubed bf16 product
// 1242 TFLOP/s): one row of 32 heads on 8 over 65333 int8 slots 36 + 5.2 us, 3.8 TB/s of codes; sixteen ragged
// trees of up to 61 rows of 32 heads over 512 to 2400 e4m3 slots 57-68 us, behind one prefix of 2100 bf16 slots
// 58 + 8.6; one row of each of 64 sequences behind 32700 int8 slots 71 + 7.4: in those with many rows for a key a CU
// holds waves for 66-74 % of the launch, as workgroups are uneven, and within that time the matrix products (14-21 % of
// the launch) and the vector instructions of the softmax and of turning codes into bf16 (26-35 %) overlap only
// in part; 17 rows over 300 slots 7.9, latency.
#include <algorithm>
#include <cstddef>

#include "../eight_bit.h"
#include "../launch.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(kv_attn)

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int KA_WAVES = 4;
constexpr int KA_THREADS = KA_WAVES * WAVE;
constexpr int KA_UNIT = 64;       // keys that a workgroup takes at a time, and that splits are counted in

// How a launch covers rows and keys.  A workgroup holds `tiles` tiles of 32 rows (fp32: one).
struct KvSide {
  int tiles, blocks;              // tiles of a workgroup (1, 2 or 4); workgroups side by side for one head's rows
  int splits, per;                // of the keys; units of a split at least
};
struct KvPlan {
  KvSide own, pre;
  int64_t pre_jobs, jobs;         // the first pre_jobs take prefixes
  int parts;                      // partial results a row may have: own splits, then the prefix's
};

// A job's keys: slots [0, L) and the tail [L, total) of a part, in steps of KT keys that do not straddle
// L, and how many splits share them.
struct Reach {
  int L, total, prefix_steps, steps, units, live;
};
template <int KT>
__device__ __forceinline__ Reach reach_of(int len, int n_tail, int cap, const KvSide& side, int least) {
  Reach r;
  r.L = max(0, min(len, cap));
  r.total = (int)min((int64_t)r.L + max(0, min(n_tail, ADT_MAX_NODES)), (int64_t)cap);
  r.prefix_steps = (r.L + KT - 1) / KT;
  r.steps = r.prefix_steps + (r.total - r.L + KT - 1) / KT;
  r.units = (r.steps + KA_UNIT / KT - 1) / (KA_UNIT / KT);
  r.live = max(least, min(side.splits, (r.units + side.per - 1) / side.per));
  return r;
}
template <int KT>
__device__ __forceinline__ Reach pre_reach(const KvAttn& a, const KvPlan& p, int b) {
  if (!a.groups) return Reach{};
  return reach_of<KT>(a.pre.len[b / a.group], 0, a.pre.cap, p.pre, 0);
}
__device__ __forceinline__ int rows_of(const KvAttn& a, int b) { return max(0, min(a.n_q[b], a.nq_max)) * a.G; }

// What a workgroup does: rows [r0, ...) of the job's `live` rows, split sp of `reach`.
struct Job {
  bool pre, direct;               // a prefix; all keys of the rows are here: the result is the output
  int b, h, r0, live, sp;         // b: sequence, or first sequence of the group
  Reach reach;
  const KvPart* part;
  int64_t cache;                  // sequence or group
};
// first: LDS [group + 1], filled with the rows before each sequence of a group (prefix jobs only).
// false: nothing to do.  Ends with a barrier where it is a prefix job.
template <int KT>
__device__ __forceinline__ bool take_job(const KvAttn& a, const KvPlan& p, int rows_each, int* first, Job& j) {
  uint32_t id = blockIdx.x;
  j.pre = id < (uint32_t)p.pre_jobs;
  if (!j.pre) id -= (uint32_t)p.pre_jobs;
  const KvSide& side = j.pre ? p.pre : p.own;
  j.h = id % (uint32_t)a.Hkv;
  id /= (uint32_t)a.Hkv;
  const int block = id % (uint32_t)side.blocks;
  id /= (uint32_t)side.blocks;
  j.sp = id % (uint32_t)side.splits;
  const int at = id / (uint32_t)side.splits;
  j.cache = at;
  j.part = j.pre ? &a.pre : &a.own;
  j.r0 = block * rows_each;
  if (!j.pre) {
    const int n_q = a.n_q[at], len = a.own.len[at], n_tail = a.n_tail[at];     // (one wait for all)
    const int pre_len = a.groups ? a.pre.len[at / (uint32_t)a.group] : 0;
    j.b = at;
    j.live = max(0, min(n_q, a.nq_max)) * a.G;
    j.reach = reach_of<KT>(len, n_tail, a.own.cap, p.own, 1);
    j.direct = j.reach.live == 1 && pre_len <= 0;
    if (j.r0 >= j.live || j.sp >= j.reach.live) return false;
    if (threadIdx.x == 0 && (int64_t)len + n_tail > a.own.cap) dev_fail(DEVINV_KV_RANGE);
    return true;
  }
  j.direct = false;
  j.b = at * a.group;
  j.reach = pre_reach<KT>(a, p, j.b);
  if (threadIdx.x == 0 && a.pre.len[at] > a.pre.cap) dev_fail(DEVINV_KV_RANGE);
  if (j.sp >= j.reach.live) return false;
  if (threadIdx.x < WAVE) {
    uint32_t before = 0;
    if (threadIdx.x == 0) first[0] = 0;
    for (int s = 0; s < a.group; s += WAVE) {
      const int i = s + threadIdx.x;
      const uint32_t upto = before + wave_prefix_sum(i < a.group ? (uint32_t)rows_of(a, j.b + i) : 0u);
      if (i < a.group) first[i + 1] = (int)upto;
      before = __shfl(upto, WAVE - 1, WAVE);
    }
  }
  __syncthreads();
  j.live = first[a.group];
  return j.r0 < j.live;
}
// A job's row: sequence, node and head of the group; its query and its place among the sequence's rows.
struct RowAt {
  int b, node, u;
  __device__ __forceinline__ int64_t q(const KvAttn& a, int h) const {
    return ((((int64_t)b * a.nq_max + node) * a.Hkv + h) * a.G + u) * a.Dh;
  }
  // its partial result of split `sp`, in rows
  __device__ __forceinline__ int64_t part(const KvAttn& a, const KvPlan& p, int h, int sp) const {
    return (((int64_t)b * a.Hkv + h) * p.parts + sp) * ((int64_t)a.nq_max * a.G) + node * a.G + u;
  }
};
__device__ __forceinline__ RowAt row_at(const KvAttn& a, const Job& j, int row, const int* first) {
  int s = 0;
  if (j.pre) {
    int hi = a.group;
    while (hi - s > 1) {
      const int mid = (s + hi) / 2;
      if (first[mid] <= row) s = mid;
      else hi = mid;
    }
    row -= first[s];
  }
  return RowAt{j.b + s, row / a.G, row % a.G};
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) <= 3.402823466e38f); }

// A row's running maximum (log2 domain) and this lane's share of its sum.  step: the new maximum's
// bound for this step's scores; returns the factor of what was summed before.
struct Softmax {
  float m = -INFINITY, l = 0.f;
  __device__ __forceinline__ float raise(float mx, float& m_use) {
    const float m_new = fmaxf(m, mx);
    m_use = m_new == -INFINITY ? 0.f : m_new;       // nothing seen yet: weights 0, not NaN
    const float alpha = m_new == m ? 1.f : exp2_hw(m - m_use);
    m = m_new;
    return alpha;
  }
};
// What a part (m, l) weighs beside a maximum M of all parts; one that saw nothing weighs 0.  Parts add up whatever they
// weigh: outputs that are not finite make the sum so even times 0, as they would among the keys of one part.
__device__ __forceinline__ float part_weight(float m, float l, float M) {
  return m == -INFINITY && l == 0.f ? 0.f : exp2_hw(m - (M == -INFINITY ? 0.f : M));
}

// ---------------------------------------------------------------------------- rows that left fp32
// Weighted values may add up to more than fp32 holds where it holds their mean: values past 2^120, or past 2^128 over
// their number.  The output is then not finite though the sum of weights is, which every row is tested for where its
// output is written; such a row is made again: by a wave, from all its keys, with sums in double.  (Far slower: a 61-row
// tree of 32 heads over 2300 bf16 slots 0.9 ms in place of 22 us, one row over 65333 17 ms in place of 67 us.)  Where a
// value that the row sees is not finite itself, its outputs stay as they are.

// Whether any of N times four outputs is not finite, though the sum of weights l is.
template <int N>
__device__ __forceinline__ bool left_fp32(const f32x4 (&o)[N], float l) {
  f32x4 x = o[0] * 0.f;
#pragma unroll
  for (int n = 1; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = fmaf(o[n][e], 0.f, x[e]);
  const float sum = (x[0] + x[1]) + (x[2] + x[3]);        // 0, or NaN
  return sum != sum && !not_finite(l);
}
// The values of a lane's piece of a row: 16 bytes, or eight codes.
template <typename C>
constexpr int PIECE = sizeof(C) == 4 ? 4 : 8;
template <typename C>
struct alignas(PIECE<C> * sizeof(C)) Piece {
  uint32_t w[PIECE<C> * sizeof(C) / 4];
  __device__ __forceinline__ void values(float (&f)[PIECE<C>]) const {
#pragma unroll
    for (int i = 0; i < PIECE<C> * (int)sizeof(C) / 4; ++i) {
      if constexpr (EIGHT<C>) {
        const float4 x = decode4<C>(w[i]);
        f[4 * i] = x.x, f[4 * i + 1] = x.y, f[4 * i + 2] = x.z, f[4 * i + 3] = x.w;
      } else if constexpr (sizeof(C) == 2) {
        f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        f[i] = __uint_as_float(w[i]);
      }
    }
  }
};
// Whether any element in 16 bytes is not finite.
__device__ __forceinline__ bool odd_elements(int type, u32x4 w) {
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = w[i] & 0x7fffffffu, low = w[i] & 0x7fffu, none = (w[i] & 0x7f7f7f7fu) ^ 0x7f7f7f7fu;
    if (type == ADT_F32) odd |= x >= 0x7f800000u;
    else if (type == ADT_BF16) odd |= x >= 0x7f800000u || low >= 0x7f80u;
    else if (type == ADT_E4M3) odd |= ((none - 0x01010101u) & ~none & 0x80808080u) != 0;      // a byte of `none` is 0
  }
  return odd;
}
// A structure that lies in constant memory.
typedef const __attribute__((address_space(4))) uint32_t ConstWord;
template <typename S>
__device__ __forceinline__ S read_words(ConstWord* from) {
  struct {
    uint32_t w[sizeof(S) / 4];
  } words;
#pragma unroll
  for (size_t i = 0; i < sizeof(S) / 4; ++i) words.w[i] = from[i];
  return __builtin_bit_cast(S, words);
}
// What the code of this section works with.  A kernel's first argument is `a`: read anew from where it lies, and the lane
// counted anew, they are not kept through the loops before, whose registers they would take.
struct Anew {
  ConstWord* args;
  KvAttn a;
  int lane;
  __device__ __forceinline__ Anew() : args((ConstWord*)__builtin_amdgcn_kernarg_segment_ptr()) {
    asm volatile("" : "+s"(args));
    a = read_words<KvAttn>(args);
    lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
  }
};
// A part of the context of sequence b's rows: L slots that all of them see, and up to `total` a tail.
struct Keys {
  const void *k, *v;
  const float *ks, *vs;
  int L, total;
  int64_t base, scales;
  __device__ __forceinline__ Keys(const Anew& n, bool own, int b, int h) {
    const KvPart p = read_words<KvPart>(n.args + (own ? offsetof(KvAttn, own) : offsetof(KvAttn, pre)) / 4);
    const int64_t of = own ? b : b / n.a.group;
    k = p.k, v = p.v, ks = p.ks, vs = p.vs;
    L = max(0, min(p.len[of], p.cap));
    total = own ? (int)min((int64_t)L + max(0, min(n.a.n_tail[b], ADT_MAX_NODES)), (int64_t)p.cap) : L;
    base = of * p.sb + h * p.sh;
    scales = of * p.ssb + h * p.ssh;
  }
};
// Whether a lane's values of the slots [from, to) are finite, for those that sees(slot) says; the whole wave's lanes take
// all of them, until one is not.
template <class F>
__device__ __forceinline__ bool odd_values(const Anew& n, const Keys& k, int from, int to, F sees) {
  const int type = n.a.type, bytes = type == ADT_F32 ? 4 : type == ADT_BF16 ? 2 : 1, row_log2 = __builtin_ctz(n.a.Dh * bytes);
  const char* v = (const char*)k.v + k.base * bytes;
  const int64_t end = type == ADT_I8 ? 0 : (int64_t)to << row_log2;
  constexpr int AT_ONCE = 4;
  bool odd = false;
#pragma unroll 1
  for (int64_t at0 = (int64_t)from << row_log2; at0 < end; at0 += AT_ONCE * WAVE * 16) {
    u32x4 w[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) w[i] = *reinterpret_cast<const u32x4*>(v + min(at0 + (i * WAVE + n.lane) * 16, end - 16));
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const int64_t at = at0 + (i * WAVE + n.lane) * 16;
      odd |= at < end && odd_elements(type, w[i]) && sees(at >> row_log2);
    }
    if (__any(odd)) return true;
  }
  if (k.vs) {
#pragma unroll 4
    for (int64_t key = from + n.lane; key < to; key += WAVE) odd |= not_finite(k.vs[k.scales + key]) && sees(key);
  }
  return __any(odd);
}
// Whether a value that all rows of sequence b see is not finite: its rows are then left as they are.  Where outputs are
// written over the queries they are not there yet: false.
__device__ __forceinline__ bool odd_for_all(int b, int h) {
  const Anew n;
  if (n.a.out == n.a.q) return false;
#pragma unroll 1
  for (int own = n.a.groups ? 0 : 1; own < 2; ++own) {
    const Keys k(n, own, b, h);
    if (odd_values(n, k, 0, k.L, [](int64_t) { return true; })) return true;
  }
  return false;
}
// Row `row` (node and head of the group) of sequence b; all lanes of the wave take part: a group of lanes a key, a piece
// of it each, AT_ONCE keys in flight; the groups, whose sums are their own, meet at the end.  Outputs are written
// before, unless they are the queries.
template <typename C, int AT_ONCE = 4>
__device__ __forceinline__ void row_again(int b, int h, int row) {
  typedef std::conditional_t<sizeof(C) == 4, float, uint16_t> T;
  constexpr int EPL = PIECE<C>;
  const Anew n;
  const KvAttn& a = n.a;
  const int per = a.Dh / EPL, groups = WAVE / per, group = n.lane / per, dim = n.lane % per * EPL;
  const int64_t at = RowAt{b, row / a.G, row % a.G}.q(a, h) + dim;
  const uint64_t* mask = a.mask + ((int64_t)b * a.nq_max + row / a.G) * ADT_MASK_WORDS;
  auto sees = [&](const Keys& k, int64_t key) {
    const int64_t t = key - k.L;
    return key < k.total && (t < 0 || (mask[t / 64] >> (t % 64) & 1));
  };
  if (a.out != a.q) {
    const Keys k(n, true, b, h);
    if (odd_values(n, k, k.L, k.total, [&](int64_t key) { return sees(k, key); })) return;
  }
  const float scale_log2 = a.scale * LOG2E;
  float q[EPL], m = -INFINITY;
  double o[EPL], l = 0.0;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    q[e] = Elem<T>::load((const T*)a.q, at + e);
    o[e] = 0.0;
  }
#pragma unroll 1
  for (int own = a.groups ? 0 : 1; own < 2; ++own) {
    const Keys p(n, own, b, h);
#pragma unroll 1
    for (int64_t key0 = group; key0 - group < p.total; key0 += groups * AT_ONCE) {
      Piece<C> kr[AT_ONCE], vr[AT_ONCE];
      float by_k[AT_ONCE], by_v[AT_ONCE];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const int64_t key = min(key0 + i * groups, (int64_t)p.total - 1), from = p.base + key * a.Dh + dim;
        kr[i] = *reinterpret_cast<const Piece<C>*>((const C*)p.k + from);
        vr[i] = *reinterpret_cast<const Piece<C>*>((const C*)p.v + from);
        by_k[i] = EIGHT<C> ? p.ks[p.scales + key] * scale_log2 : scale_log2;
        by_v[i] = EIGHT<C> ? p.vs[p.scales + key] : 1.f;
      }
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        const bool seen = sees(p, key0 + i * groups);
        float f[EPL], x = 0.f;
        kr[i].values(f);
#pragma unroll
        for (int e = 0; e < EPL; ++e) x = fmaf(q[e], f[e], x);
        for (int k = per / 2; k >= 1; k /= 2) x += __shfl_xor(x, k, WAVE);
        x = seen ? x * by_k[i] : -INFINITY;
        const float top = fmaxf(m, x), ref = top == -INFINITY ? 0.f : top, down = top == m ? 1.f : exp2_hw(m - ref);
        const double w = seen ? (double)exp2_hw(x - ref) : 0.0, by = seen ? w * (double)by_v[i] : 0.0;
        m = top;
        l = l * (double)down + w;
        vr[i].values(f);
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] = o[e] * (double)down + (seen ? by * (double)f[e] : 0.0);
      }
    }
  }
  float M = m;
  for (int k = per; k < WAVE; k *= 2) M = fmaxf(M, __shfl_xor(M, k, WAVE));
  const double weight = (double)part_weight(m, (float)l, M);
  auto sum = [&](double x) {
    x *= weight;
    for (int k = per; k < WAVE; k *= 2) x += __shfl_xor(x, k, WAVE);
    return x;
  };
  l = sum(l);
  const double inv = l == 0.0 ? 0.0 : 1.0 / l;
  const float most = sizeof(T) == 4 ? 3.402823466e38f : 3.389531389e38f;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    // (a mean of finite values is: where a rounding takes it past the type's largest, it is that)
    const double s = sum(o[e]);
    float y = (float)(s * inv);
    if (fabsf(y) > most && fabs(s) < (double)INFINITY) y = copysignf(most, y);
    if (group == 0) Elem<T>::store((T*)a.out, at + e, y);
  }
}
// Of a wave whose rows have `per` neighbouring lanes each: the lanes of those rows of which one says so.
__device__ __forceinline__ uint64_t rows_lanes(bool left, int per) {
  const uint64_t any = __ballot(left), group = (1ull << per) - 1;
  uint64_t all = 0;
  if (any)
    for (int i = 0; i < WAVE; i += per) all |= any >> i & group ? group << i : 0;
  return all;
}

// Makes the rows of sets of such lanes again; row_of(set, lane): the row.  T: the rows' type.
template <typename T, int N, class F>
__device__ __forceinline__ void lanes_again(const uint64_t (&sets)[N], int type, int b, int h, F row_of, int per) {
  uint64_t any = 0;
#pragma unroll
  for (int y = 0; y < N; ++y) any |= sets[y];
  if (!any) return;
  __threadfence_block();
  if (odd_for_all(b, h)) return;
#pragma unroll 1
  for (int y = 0; y < N; ++y) {
    uint64_t lanes = sets[0];
#pragma unroll
    for (int z = 1; z < N; ++z) lanes = y == z ? sets[z] : lanes;
#pragma unroll 1
    for (int i = 0; i < WAVE; i += per)
      if (lanes >> i & 1) {
        if constexpr (sizeof(T) == 4) row_again<float, 2>(b, h, row_of(y, i));
        else if (type == ADT_BF16) row_again<uint16_t, 2>(b, h, row_of(y, i));
        else if (type == ADT_E4M3) row_again<E4M3, 2>(b, h, row_of(y, i));
        else row_again<I8, 2>(b, h, row_of(y, i));
      }
  }
}

// ---------------------------------------------------------------------------- bf16 rows
// A wave takes a tile of 32 rows through the keys, 32 of them a step:
//   S^T[key][row] = K Q^T  (32 x 32 x 16 MFMA; lane (r, s) = (lane % 32, lane / 32) holds row r's scores of
//                           keys 8 c + 4 s + e, c and e < 4),
//   O^T[dim][row] += V^T P^T  (V by transpose loads from LDS, its keys in the order in which lanes hold P).
// A row's scores lie in two lanes, so its maximum takes one exchange, and 32 rows a wave halve the LDS
// reads that 16 would need.
template <int DH>
struct RowTile {
  static constexpr int KS = DH / 16, OT = DH / 32;
  bf16x8 q[KS];
  f32x16 o[OT];
  float m = -INFINITY, l = 0.f;    // running maximum (log2 domain), this lane's share of the sum
  bool odd = false;                // a value of the tail was not finite
};
// LDS rows, padded so that what half a wave reads at once falls on distinct banks (K: 16 rows of 16
// bytes; V: 4 rows of 64), and every operand lies at a constant distance from one address (swizzled
// rows took some 25 registers of addresses).
template <int DH>
constexpr int K_PITCH = DH * 2 + 16;
template <int DH>
constexpr int V_PITCH = DH * 2 + 64;

template <int N>
__device__ __forceinline__ float max_of(const f32x16 (&x)[N]) {
  float m[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    m[u] = x[0][u];
#pragma unroll
    for (int e = 4 + u; e < 16 * N; e += 4) m[u] = fmaxf(m[u], x[e / 16][e % 16]);
  }
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// A row's reference of the softmax: scores count as 2^(score - m).  It is the maximum of the first scores
// that the row saw, and is raised only where a later one is larger by more than this (in log2), so
// that outputs are hardly ever rescaled; weights then reach 2^8.
constexpr float SLACK = 8.f;

// N steps at once.  k(n, f): the K operands of step n; ks, vs: LDS, the scales of this lane's keys (those of
// the keys times the softmax's, in log2); v: LDS, this lane's first transpose load.  Where not WHOLE: the
// keys that the row sees (bit i: key i), and whether a step is of the tail, whose values alone may be
// kept from a row.
template <typename C, int DH, bool WHOLE, int N, class K, class Then>
__device__ __forceinline__ void take_steps(RowTile<DH>& t, float scale_log2, K k, Then then, const float* ks, const float* vs,
                                           const unsigned char* v, const uint32_t (&seen)[N], const bool (&tail)[N], int s) {
  constexpr int KS = DH / 16, OT = DH / 32, VP = V_PITCH<DH>;
  constexpr bool CODES = EIGHT<C>;
  f32x16 x[N];
#pragma unroll
  for (int n = 0; n < N; ++n) {
    bf16x8 f[KS];
    k(n, f);
#pragma unroll
    for (int e = 0; e < 16; ++e) x[n][e] = 0.f;
#pragma unroll
    for (int i = 0; i < KS; ++i) x[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[i], t.q[i], x[n], 0, 0, 0);
  }
  then();
  // scores less the row's reference, in log2
  const bool fresh = t.m == -INFINITY;
  const float ref = fresh ? 0.f : t.m;
#pragma unroll
  for (int n = 0; n < N; ++n) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      f32x4 by{scale_log2, scale_log2, scale_log2, scale_log2};
      if constexpr (CODES) by = *reinterpret_cast<const f32x4*>(ks + 32 * n + 8 * c);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[n][4 * c + e] = fmaf(x[n][4 * c + e], by[e], -ref);
    }
    if constexpr (!WHOLE) {
      // bit 8 c + e, after the shift: this lane's score 4 c + e
#pragma unroll
      for (int e = 0; e < 16; ++e) x[n][e] = seen[n] >> 4 * s >> (e / 4 * 8 + e % 4) & 1 ? x[n][e] : -INFINITY;
    }
  }
  const float over = xor32_max(max_of(x));
  const bool raise = over > (fresh ? -INFINITY : SLACK);
  if (__any(raise)) {
    // (a row's first scores have nothing to rescale)
    const float up = raise ? over : 0.f, factor = fresh ? 1.f : exp2_hw(-up);
    if (raise) t.m = ref + up;
    t.l *= factor;
#pragma unroll
    for (int d = 0; d < OT; ++d) t.o[d] *= factor;
#pragma unroll
    for (int n = 0; n < N; ++n) x[n] -= up;
  }
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[n][e] = exp2_hw(x[n][e]);
      sum[e % 4] += x[n][e];
    }
  t.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    if constexpr (CODES) {
      // (a slot the row does not see may have any scale)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const f32x4 by = *reinterpret_cast<const f32x4*>(vs + 32 * n + 8 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x[n][4 * c + e] = WHOLE || (seen[n] >> 4 * s >> (8 * c + e) & 1) ? x[n][4 * c + e] * by[e] : 0.f;
      }
    }
    // (rounded to bf16 for the product, as no other operand enters it: 2^-9 of a weight at most, results 0.0024 of
    // their size from 64 bits where the output's own rounding leaves 0.0017; the sum of weights is not rounded)
    bf16x8 pb[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) pb[e / 8][e % 8] = (__bf16)x[n][e];
    // lane i of a 16-lane group that addresses row k0 + i / 4, dims d0 + 4 (i % 4)..+3 gets V[k0 + 0..3][d0 + i]
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int d = 0; d < OT; ++d) {
        v4i16 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(v + (32 * n + 16 * c) * VP + d * 64));
        v4i16 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(v + (32 * n + 16 * c + 8) * VP + d * 64));
        if (!WHOLE && tail[n]) {
          // a value that is not finite may only meet the rows that see it: it is taken out here, and added
          // when all keys are done
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool b0 = (x0[e] & 0x7f80) == 0x7f80, b1 = (x1[e] & 0x7f80) == 0x7f80;
            x0[e] = b0 ? 0 : x0[e];
            x1[e] = b1 ? 0 : x1[e];
            t.odd |= b0 | b1;
          }
        }
        const bf16x8 vf = __builtin_bit_cast(bf16x8, v8i16{x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]});
        t.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pb[c], t.o[d], 0, 0, 0);
      }
    }
  }
}
// This lane's first transpose load of rows that start at `rows`.
template <int DH>
__device__ __forceinline__ const unsigned char* v_operand(const unsigned char* rows, int lane) {
  return rows + (4 * (lane >> 5) + (lane & 15) / 4) * V_PITCH<DH> + (lane >> 4 & 1) * 32 + (lane & 3) * 8;
}

// 16 bytes of a row of K or V into bf16 at `at`.
template <typename C>
__device__ __forceinline__ void put_bf16(unsigned char* at, u32x4 w) {
  if constexpr (EIGHT<C>) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u16x4 lo = decode4_bf16<C>(w[2 * i]), hi = decode4_bf16<C>(w[2 * i + 1]);
      *reinterpret_cast<u16x8*>(at + 16 * i) = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
  } else {
    *reinterpret_cast<u32x4*>(at) = w;
  }
}

// What both forms of the attention work with.
template <typename C, int DH>
struct KeySource {
  const C *k, *v;
  const float *ks, *vs;
  int L, total, prefix_steps, steps, sp, n_live;
  __device__ __forceinline__ KeySource(const Job& j)
      : L(j.reach.L), total(j.reach.total), prefix_steps(j.reach.prefix_steps), steps(j.reach.steps), sp(j.sp),
        n_live(j.reach.live) {
    const KvPart& p = *j.part;
    k = (const C*)p.k + j.cache * p.sb + j.h * p.sh;
    v = (const C*)p.v + j.cache * p.sb + j.h * p.sh;
    ks = EIGHT<C> ? p.ks + j.cache * p.ssb + j.h * p.ssh : nullptr;
    vs = EIGHT<C> ? p.vs + j.cache * p.ssb + j.h * p.ssh : nullptr;
  }
  // A step's first key, and the last key of the prefix or tail that it lies in (a step past the end has none:
  // last < key0).
  struct Span {
    int key0, last;
  };
  __device__ __forceinline__ Span span(int st) const {
    if (st >= steps) return Span{0, -1};
    if (st >= prefix_steps) return Span{L + (st - prefix_steps) * 32, total - 1};
    return Span{st * 32, L - 1};
  }
  // the step's keys that a row of mask `words` sees
  __device__ __forceinline__ uint32_t seen(int st, const uint32_t* words) const {
    const Span at = span(st);
    const int count = at.last - at.key0 + 1;
    const uint32_t have = count >= 32 ? ~0u : (1u << max(count, 0)) - 1;
    return st >= prefix_steps && st < steps ? have & words[st - prefix_steps] : have;
  }
};

// Adds the values of a tail step that are not finite to the rows that see them (whatever its weight, an
// infinite value makes the output infinite, and NaN makes it NaN).
template <typename C, int DH>
__device__ __forceinline__ void add_odd_values(RowTile<DH>& t, const KeySource<C, DH>& src, int st, const uint32_t* words, int s) {
  const auto at = src.span(st);
  for (int key = at.key0; key <= min(at.last, at.key0 + 31); ++key) {
    const bool vis = words[st - src.prefix_steps] >> (key - at.key0) & 1;
#pragma unroll
    for (int d = 0; d < DH / 32; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const C* p = src.v + (int64_t)key * DH + 32 * d + 8 * c + 4 * s;
        f32x4 v;
        if constexpr (EIGHT<C>) v = __builtin_bit_cast(f32x4, decode4<C>(*reinterpret_cast<const uint32_t*>(p)));
        else v = f32x4{bf2f(p[0]), bf2f(p[1]), bf2f(p[2]), bf2f(p[3])};
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (vis && not_finite(v[e])) t.o[d][4 * c + e] += v[e];
      }
  }
}

// a times u and b times v, rounded each: the two parts of a row alike.
__device__ __forceinline__ float both(float a, float u, float b, float v) {
#pragma clang fp contract(off)
  return a * u + b * v;
}
// Where a row's result goes: the output, or a partial result.
__device__ __forceinline__ int64_t row_out(const KvAttn& a, const KvPlan& p, const Job& j, const RowAt& at) {
  return j.direct ? at.q(a, j.h) : at.part(a, p, j.h, j.pre ? p.own.splits + j.sp : j.sp);
}
// Outputs 32 d + 8 c + 4 s.. of a row.
template <int DH>
__device__ __forceinline__ void put_out(const KvAttn& a, bool direct, int64_t to, int dim, f32x4 o, float inv, float* part_o) {
  if (direct) store4((uint16_t*)a.out + to + dim, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  else *reinterpret_cast<f32x4*>(part_o + to * DH + dim) = o;
}

// Many rows: a unit of 64 keys, K and V, comes into LDS once for the workgroup (eight bits turned into
// bf16 on the way), the next P on their way into registers meanwhile; a wave takes its tile through both
// steps of a unit, or, where the job has two tiles only, through one of them.  Returns which of its tile's rows (bits) a
// wave has to make again.
template <typename C, int DH, int TILES>
__device__ __forceinline__ uint32_t attend_shared(const KvAttn& a, const KvPlan& p, const Job& j, const int* first, unsigned char* smem,
                                              float* part_o, float* part_ml) {
  constexpr int KT = 32, KS = DH / 16, OT = DH / 32, KH = KA_WAVES / TILES, N = 2 / KH, KP = K_PITCH<DH>, VP = V_PITCH<DH>;
  constexpr int EPL = 16 / (int)sizeof(C), CPL = DH / EPL;         // elements of a load, loads of a row
  constexpr int LOADS = KA_UNIT * CPL / KA_THREADS;
  constexpr int ROWS = KA_UNIT * (KP + VP), BYTES = ROWS + (EIGHT<C> ? 2 * KA_UNIT * 4 : 0);   // a unit: K, V, scales
  constexpr bool CODES = EIGHT<C>;
  constexpr int P = CODES ? 2 : 1;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  const int r = lane & 31, s = lane >> 5;
  const int tile = wave % TILES, kpart = wave / TILES;
  const KeySource<C, DH> src(j);
  const int n_live = src.n_live;
  const int units = max(0, (j.reach.units - j.sp + n_live - 1) / n_live);   // of this split: sp, sp + n_live, ...
  const float scale_log2 = a.scale * LOG2E;

  // Load x of a unit takes row x / CPL, elements (x % CPL) * EPL..; thread t takes loads y * 256 + t.  Rows
  // past a step's last key read that one, or the head's first row, and are stored as zeros.
  u32x4 kr[P][LOADS], vr[P][LOADS];
  float sc[P];
  auto unit_step = [&](int i) { return i < units ? 2 * (j.sp + n_live * i) : src.steps; };
  auto fetch = [&](int u, int i) {
    const int st = unit_step(i);
    const float* scale = wave ? src.vs : src.ks;       // (the first two waves take the scales)
    if (st + 2 <= src.L / KT) {
      // 64 rows in a row: constant distances from one address
      const char* kp = (const char*)(src.k + (int64_t)st * KT * DH) + tid * 16;
      const char* vp = (const char*)(src.v + (int64_t)st * KT * DH) + tid * 16;
#pragma unroll
      for (int y = 0; y < LOADS; ++y) {
        kr[u][y] = *reinterpret_cast<const u32x4*>(kp + y * KA_THREADS * 16);
        vr[u][y] = *reinterpret_cast<const u32x4*>(vp + y * KA_THREADS * 16);
      }
      if (CODES && wave < 2) sc[u] = scale[(int64_t)st * KT + lane];
      return;
    }
    const auto w0 = src.span(st), w1 = src.span(st + 1);
#pragma unroll
    for (int y = 0; y < LOADS; ++y) {
      const int x = y * KA_THREADS + tid, rx = x / CPL, c = x % CPL;
      const int key = max(0, min((rx < KT ? w0.key0 : w1.key0) + rx % KT, rx < KT ? w0.last : w1.last));
      kr[u][y] = *reinterpret_cast<const u32x4*>(src.k + (int64_t)key * DH + c * EPL);
      vr[u][y] = *reinterpret_cast<const u32x4*>(src.v + (int64_t)key * DH + c * EPL);
    }
    if (CODES && wave < 2) sc[u] = scale[max(0, min((lane < KT ? w0.key0 : w1.key0) + lane % KT, lane < KT ? w0.last : w1.last))];
  };
#pragma unroll
  for (int u = 0; u < P; ++u) {
    fetch(u, u);
    __builtin_amdgcn_sched_barrier(0);     // (in order, or the first one used could be the last to arrive)
  }

  RowTile<DH> t;
  const int row = j.r0 + tile * 32 + r;
  const bool mine = row < j.live, tile_live = j.r0 + tile * 32 < j.live;
  RowAt at{j.b, 0, 0};
  if (mine) at = row_at(a, j, row, first);
#pragma unroll
  for (int i = 0; i < KS; ++i) t.q[i] = bf16x8{};
  if (mine) {
    const uint16_t* q = (const uint16_t*)a.q + at.q(a, j.h) + s * 8;
#pragma unroll
    for (int i = 0; i < KS; ++i) t.q[i] = *reinterpret_cast<const bf16x8*>(q + i * 16);
  }
#pragma unroll
  for (int d = 0; d < OT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) t.o[d][e] = 0.f;
  // the row's mask, 32 tail slots a word: those of a step
  const uint32_t* words = reinterpret_cast<const uint32_t*>(a.mask) + ((int64_t)at.b * a.nq_max + at.node) * 2 * ADT_MASK_WORDS;

  auto store = [&](auto whole_tag, int u, int i) {
    unsigned char* to = smem + (i & 1) * BYTES;
    const auto w0 = src.span(unit_step(i)), w1 = src.span(unit_step(i) + 1);
#pragma unroll
    for (int y = 0; y < LOADS; ++y) {
      const int x = y * KA_THREADS + tid, rx = x / CPL, c = x % CPL;
      if (!decltype(whole_tag)::value && (rx < KT ? w0.key0 : w1.key0) + rx % KT > (rx < KT ? w0.last : w1.last)) vr[u][y] = u32x4{};
      put_bf16<C>(to + rx * KP + c * EPL * 2, kr[u][y]);
      put_bf16<C>(to + KA_UNIT * KP + rx * VP + c * EPL * 2, vr[u][y]);
    }
    if (CODES && wave < 2) {
      const bool none = !decltype(whole_tag)::value && (lane < KT ? w0.key0 : w1.key0) + lane % KT > (lane < KT ? w0.last : w1.last);
      reinterpret_cast<float*>(to + ROWS)[tid] = none ? 0.f : wave ? sc[u] : sc[u] * scale_log2;
    }
  };
  auto compute = [&](auto whole_tag, int buf, const uint32_t (&seen)[N], const bool (&tail)[N]) {
    const unsigned char* base = smem + buf * BYTES;
    const unsigned char* kl = base + (kpart * KT + r) * KP + s * 16;
    const float* sl = reinterpret_cast<const float*>(base + ROWS) + kpart * KT + 4 * s;
    take_steps<C, DH, decltype(whole_tag)::value, N>(
        t, scale_log2,
        [&](int n, bf16x8 (&f)[KS]) {
#pragma unroll
          for (int i = 0; i < KS; ++i) f[i] = *reinterpret_cast<const bf16x8*>(kl + n * KT * KP + i * 32);
          __builtin_amdgcn_sched_barrier(0);       // all of them requested before the first product
        },
        [] {}, sl, sl + KA_UNIT, v_operand<DH>(base + KA_UNIT * KP + kpart * KT * VP, lane), seen, tail, s);
  };

  // (the registers of a unit go by its place in a round of P)
  auto unit = [&](auto whole_tag, int u, int i) {
    // the buffer written here was last read two units ago, before the previous barrier
    store(whole_tag, u, i);
    __syncthreads();
    fetch(u, i + P);
    if (!tile_live) return;
    uint32_t seen[N] = {};
    bool tail[N] = {};
    if constexpr (!decltype(whole_tag)::value) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const int st = unit_step(i) + kpart + n;
        seen[n] = src.seen(st, words);
        tail[n] = st >= src.prefix_steps;
      }
    }
    compute(whole_tag, i & 1, seen, tail);
  };
  // units of whole prefix steps first, then the others, in code of their own: a split's units come in order
  const int whole = max(0, min(units, (src.L / KA_UNIT - j.sp + n_live - 1) / n_live));
  int i = 0;
  auto loop = [&](auto whole_tag, int end) {
    for (;;) {
#pragma unroll
      for (int u = 0; u < P; ++u) {
        if (i >= end) return u;
        unit(whole_tag, u, i++);
      }
    }
  };
  if (loop(std::true_type{}, whole) == 1 && i < units) unit(std::false_type{}, 1, i++);
  loop(std::false_type{}, units);
  if (__any(t.odd)) {
    for (int st = src.prefix_steps; st < src.steps; ++st)
      if (st / 2 % n_live == j.sp && st % 2 % KH == kpart) add_odd_values(t, src, st, words, s);
  }

  t.l = xor32_add(t.l);
  if constexpr (KH > 1) {
    // the second wave of a tile passes its state through LDS to the first
    static_assert(TILES * (OT * 16 + 2) * WAVE * 4 <= 2 * ROWS, "merge area");
    float* mo = reinterpret_cast<float*>(smem) + (size_t)tile * (OT * 16 + 2) * WAVE;
    __syncthreads();
    if (kpart == 1) {
#pragma unroll
      for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) mo[(d * 16 + e) * WAVE + lane] = t.o[d][e];
      mo[OT * 16 * WAVE + lane] = t.m;
      mo[(OT * 16 + 1) * WAVE + lane] = t.l;
    }
    __syncthreads();
    if (kpart == 1) return 0;
    const float m1 = mo[OT * 16 * WAVE + lane], l1 = mo[(OT * 16 + 1) * WAVE + lane], M = fmaxf(t.m, m1);
    const float w0 = part_weight(t.m, t.l, M), w1 = part_weight(m1, l1, M);
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float y = mo[(d * 16 + e) * WAVE + lane];
        t.o[d][e] = both(t.o[d][e], w0, y, w1);
      }
    t.l = both(t.l, w0, l1, w1);
    t.m = M;
  }
  uint32_t which = 0;
  if (j.direct) {
    f32x4 o[4 * OT];
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[4 * d + e / 4][e % 4] = t.o[d][e];
    const uint64_t any = __ballot(mine && left_fp32(o, t.l));
    which = (uint32_t)(any | any >> 32);
  }
  if (!mine || (a.out == a.q && (which >> r & 1))) return which;
  const int64_t to = row_out(a, p, j, at);
  const float inv = t.l == 0.f ? 0.f : 1.f / t.l;
#pragma unroll
  for (int d = 0; d < OT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      put_out<DH>(a, j.direct, to, 32 * d + 8 * c + 4 * s, f32x4{t.o[d][4 * c], t.o[d][4 * c + 1], t.o[d][4 * c + 2], t.o[d][4 * c + 3]}, inv, part_o);
  if (!j.direct && s == 0) *reinterpret_cast<float2*>(part_ml + to * 2) = make_float2(t.m, t.l);
  return which;
}

// Up to 32 rows: the waves take steps of their own, with no barrier between them.  K comes straight into the
// operands' registers (eight bits: 16 codes a load, so that an operand's dims lie in pairs of 8, the
// queries' alike), V through rows of LDS that are the wave's own; P steps are in flight.  The waves'
// results meet in LDS, in their order.  again: LDS, 0.  Returns which of the rows have to be made again.
template <typename C, int DH>
__device__ __forceinline__ uint32_t attend_few(const KvAttn& a, const KvPlan& p, const Job& j, const int* first, unsigned char* smem,
                                           uint32_t* again, float* part_o, float* part_ml) {
  constexpr int KT = 32, KS = DH / 16, OT = DH / 32, VP = V_PITCH<DH>;
  constexpr bool CODES = EIGHT<C>;
  constexpr int P = CODES ? 2 : 1;
  constexpr int EPL = 16 / (int)sizeof(C), CPL = DH / EPL;         // elements of a load, loads of a row
  constexpr int LOADS = KT * CPL / WAVE;                           // of a step, K or V
  constexpr int OWN = KT * VP + 2 * KT * 4;                        // a wave's LDS: V, scales
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  const int r = lane & 31, s = lane >> 5;
  const KeySource<C, DH> src(j);
  const float scale_log2 = a.scale * LOG2E;

  unsigned char* rows = smem + wave * OWN;
  float* sl = reinterpret_cast<float*>(rows + KT * VP);

  u32x4 kr[P][LOADS], vr[P][LOADS];
  float sc[P];
  const int stride = src.n_live * KA_WAVES;
  // (a step past the end reads the head's first row, so the loads in flight are the same on every path)
  const float* scale = s ? src.vs : src.ks;
  auto fetch = [&](int u, int st) {
    if (st < src.L / KT) {
      // 32 rows in a row: constant distances from one address
      const char* kp = (const char*)(src.k + (int64_t)st * KT * DH) + (r * DH + s * EPL) * (int)sizeof(C);
      const char* vp = (const char*)(src.v + (int64_t)st * KT * DH) + lane * 16;
#pragma unroll
      for (int x = 0; x < LOADS; ++x) kr[u][x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + x * 32));
#pragma unroll
      for (int x = 0; x < LOADS; ++x) vr[u][x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + x * WAVE * 16));
      if (CODES) sc[u] = scale[(int64_t)st * KT + r];
      return;
    }
    const auto at = src.span(st);
    const C* kp = src.k + (int64_t)max(0, min(at.key0 + r, at.last)) * DH + s * EPL;
#pragma unroll
    for (int x = 0; x < LOADS; ++x) kr[u][x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + x * 2 * EPL));
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int y = x * WAVE + lane, key = max(0, min(at.key0 + y / CPL, at.last));
      vr[u][x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src.v + (int64_t)key * DH + y % CPL * EPL));
    }
    if (CODES) sc[u] = scale[max(0, min(at.key0 + r, at.last))];
  };
  int st = j.sp * KA_WAVES + wave;
#pragma unroll
  for (int u = 0; u < P; ++u) {
    fetch(u, st + u * stride);
    __builtin_amdgcn_sched_barrier(0);     // (in order, or the first one used could be the last to arrive)
  }

  RowTile<DH> t;
  const int row = j.r0 + r;
  const bool mine = row < j.live;
  RowAt at{j.b, 0, 0};
  if (mine) at = row_at(a, j, row, first);
#pragma unroll
  for (int i = 0; i < KS; ++i) t.q[i] = bf16x8{};
  if (mine) {
    const uint16_t* q = (const uint16_t*)a.q + at.q(a, j.h);
#pragma unroll
    for (int i = 0; i < KS; ++i)
      t.q[i] = *reinterpret_cast<const bf16x8*>(q + (CODES ? i / 2 * 32 + s * 16 + i % 2 * 8 : i * 16 + s * 8));
  }
#pragma unroll
  for (int d = 0; d < OT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) t.o[d][e] = 0.f;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(a.mask) + ((int64_t)at.b * a.nq_max + at.node) * 2 * ADT_MASK_WORDS;
  auto step = [&](auto whole_tag, int u, int st) {
    constexpr bool WHOLE = decltype(whole_tag)::value;
    const auto span = src.span(st);
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int y = x * WAVE + lane;
      if (!WHOLE && span.key0 + y / CPL > span.last) vr[u][x] = u32x4{};
      put_bf16<C>(rows + y / CPL * VP + y % CPL * EPL * 2, vr[u][x]);
    }
    if (CODES) sl[lane] = s ? (WHOLE || span.key0 + r <= span.last ? sc[u] : 0.f) : sc[u] * scale_log2;
    wave_lds_fence();
    const uint32_t seen[1] = {WHOLE ? 0u : src.seen(st, words)};
    const bool tail[1] = {!WHOLE && st >= src.prefix_steps};
    take_steps<C, DH, WHOLE, 1>(
        t, scale_log2,
        [&](int, bf16x8 (&f)[KS]) {
          if constexpr (CODES) {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const u16x4 lo = decode4_bf16<C>(kr[u][x][2 * i]), hi = decode4_bf16<C>(kr[u][x][2 * i + 1]);
                f[2 * x + i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
              }
            }
          } else {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) f[x] = __builtin_bit_cast(bf16x8, kr[u][x]);
          }
        },
        [&] { fetch(u, st + P * stride); }, sl + 4 * s, sl + KT + 4 * s, v_operand<DH>(rows, lane), seen, tail, s);
    wave_lds_fence();
  };

  const int whole = src.L / KT;
  auto loop = [&](auto whole_tag, int end) {
    // (P steps a round: the registers of a step go by its place in the round)
    for (;;) {
#pragma unroll
      for (int u = 0; u < P; ++u) {
        if (st >= end) return u;
        step(whole_tag, u, st);
        st += stride;
      }
    }
  };
  int u = loop(std::true_type{}, whole);
  if constexpr (P == 2) {
    if (u == 1 && st < src.steps) {
      step(std::false_type{}, 1, st);
      st += stride;
    }
  }
  loop(std::false_type{}, src.steps);
  if (__any(t.odd)) {
    for (int x = j.sp * KA_WAVES + wave; x < src.steps; x += stride)
      if (x >= src.prefix_steps) add_odd_values(t, src, x, words, s);
  }

  // merge: wave w takes the outputs 32 w.. of all
  t.l = xor32_add(t.l);
  static_assert(KA_WAVES >= OT, "a wave for each 32 outputs");
  float* mo = reinterpret_cast<float*>(smem);                       // [wave][OT * 16 outputs, m, l][lane]
  constexpr int EACH = (OT * 16 + 2) * WAVE;
  __syncthreads();
#pragma unroll
  for (int d = 0; d < OT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) mo[wave * EACH + (d * 16 + e) * WAVE + lane] = t.o[d][e];
  mo[wave * EACH + OT * 16 * WAVE + lane] = t.m;
  mo[wave * EACH + (OT * 16 + 1) * WAVE + lane] = t.l;
  __syncthreads();
  const bool writes = wave < OT && mine;
  if (!j.direct && !writes) return 0;
  float m[KA_WAVES], l[KA_WAVES], M = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < KA_WAVES; ++w) {
    m[w] = mo[w * EACH + OT * 16 * WAVE + lane];
    l[w] = mo[w * EACH + (OT * 16 + 1) * WAVE + lane];
    M = fmaxf(M, m[w]);
  }
  f32x4 o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (writes) {
#pragma unroll
    for (int w = 0; w < KA_WAVES; ++w) {
      const float wt = part_weight(m[w], l[w], M);
      sum += wt * l[w];
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e / 4][e % 4] += wt * mo[w * EACH + (wave * 16 + e) * WAVE + lane];
    }
  }
  uint32_t which = 0;
  if (j.direct) {
    // (a row's outputs are in several waves: where out is q all of them leave it, or none does)
    const uint64_t any = __ballot(writes && left_fp32(o, sum));
    if (any && lane == 0) atomicOr(again, (uint32_t)(any | any >> 32));
    __syncthreads();
    which = *again;
    if (!writes || (a.out == a.q && (which >> r & 1))) return which;
  }
  const int64_t to = row_out(a, p, j, at);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int c = 0; c < 4; ++c) put_out<DH>(a, j.direct, to, 32 * wave + 8 * c + 4 * s, o[c], inv, part_o);
  if (!j.direct && wave == 0 && s == 0) *reinterpret_cast<float2*>(part_ml + to * 2) = make_float2(M, sum);
  return which;
}

template <typename C, int DH>
constexpr int SHARED_BYTES = 2 * (KA_UNIT * (K_PITCH<DH> + V_PITCH<DH>) + (EIGHT<C> ? 2 * KA_UNIT * 4 : 0));
template <int DH>
constexpr int FEW_BYTES = KA_WAVES * (DH / 2 + 2) * WAVE * 4;      // (the merge takes more than the steps)

template <typename C, int DH>
__global__ __launch_bounds__(KA_THREADS, 2) void kv_attn_kernel(KvAttn a, KvPlan p, float* __restrict__ part_o,
                                                               float* __restrict__ part_ml) {
  static_assert(FEW_BYTES<DH> <= SHARED_BYTES<C, DH> && KA_WAVES * (32 * V_PITCH<DH> + 256) <= FEW_BYTES<DH>, "LDS");
  __shared__ __attribute__((aligned(16))) unsigned char smem[SHARED_BYTES<C, DH>];
  __shared__ uint32_t again;
  extern __shared__ int first[];
  if (threadIdx.x == 0) again = 0;
  Job j;
  const int tiles = (int64_t)blockIdx.x < p.pre_jobs ? p.pre.tiles : p.own.tiles;
  if (!take_job<32>(a, p, 32 * tiles, first, j)) return;
  // (the shared forms' rows are those of the wave's tile)
  uint32_t which;
  if (tiles == 1) which = attend_few<C, DH>(a, p, j, first, smem, &again, part_o, part_ml);
  else if (tiles == 2) which = attend_shared<C, DH, 2>(a, p, j, first, smem, part_o, part_ml);
  else which = attend_shared<C, DH, 4>(a, p, j, first, smem, part_o, part_ml);
  if (!which) return;
  // (the rows are written anew after their outputs are; few rows' by another wave: the bits are the workgroup's)
  if (tiles == 1) __syncthreads();
  else __threadfence_block();
  if (odd_for_all(j.b, j.h)) return;
  const int wave = threadIdx.x / WAVE, row0 = j.r0 + wave % tiles * 32;
#pragma unroll 1
  for (int i = tiles == 1 ? wave : 0; i < 32; i += tiles == 1 ? KA_WAVES : 1)
    if (which >> i & 1) row_again<C>(j.b, j.h, row0 + i);
}

// ---------------------------------------------------------------------------- fp32 rows
// 32 rows a workgroup, in two tiles of 16; the waves take 16 keys of a unit each, straight from memory,
// on the 16x16x4 MFMA (lane (l, g) = (lane % 16, lane / 16) holds row l's scores of keys 4 g + e), and
// merge in LDS.
template <int DH>
__global__ __launch_bounds__(KA_THREADS, 2) void kv_attn_f32_kernel(KvAttn a, KvPlan p, float* __restrict__ part_o,
                                                                   float* __restrict__ part_ml) {
  constexpr int KT = 16, RT = 2, OT = DH / 16, MP = DH + 4;
  __shared__ __attribute__((aligned(16))) float mo[KA_WAVES * 16 * MP];     // [wave][16][MP]
  __shared__ float mml[KA_WAVES * 16 * 2];
  extern __shared__ int first[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  const int l = lane & 15, g = lane >> 4;
  Job j;
  if (!take_job<KT>(a, p, 16 * RT, first, j)) return;
  const int L = j.reach.L, total = j.reach.total, steps = j.reach.steps, n_live = j.reach.live;
  const KvPart& part = *j.part;
  const float* kb = (const float*)part.k + j.cache * part.sb + j.h * part.sh;
  const float* vb = (const float*)part.v + j.cache * part.sb + j.h * part.sh;
  const float scale_log2 = a.scale * LOG2E;

  f32x4 q[RT][DH / 16];
  uint64_t aw0[RT], aw1[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    aw0[t] = aw1[t] = 0;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) q[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int row = j.r0 + t * 16 + l;
    if (row >= j.live) continue;
    const RowAt at = row_at(a, j, row, first);
    const float* src = (const float*)a.q + at.q(a, j.h) + g * 4;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) q[t][i] = *reinterpret_cast<const f32x4*>(src + i * 16);
    if (!j.pre) {
      const uint64_t* mp = a.mask + ((int64_t)at.b * a.nq_max + at.node) * ADT_MASK_WORDS;
      aw0[t] = mp[0];
      aw1[t] = mp[1];
    }
  }
  f32x4 o[RT][OT];
  Softmax sm[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int d = 0; d < OT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  // this wave's steps: those of the split's units that are its own
  const int stride = n_live * (KA_UNIT / KT);
  struct Span {
    int k0, last;
  };
  auto span = [&](int st) {
    const bool tail = st >= j.reach.prefix_steps;
    return Span{tail ? L + (st - j.reach.prefix_steps) * KT : st * KT, (tail ? total : L) - 1};
  };
  // the next step's keys are requested when this one's scores are done, its values when this one's are used
  f32x4 k[DH / 16], v[4][DH / 64];
  auto fetch_k = [&](int st) {
    if (st >= steps) return;
    const Span s = span(st);
    const float* src = kb + (int64_t)min(s.k0 + l, s.last) * DH + g * 4;
#pragma unroll
    for (int i = 0; i < DH / 16; ++i) k[i] = *reinterpret_cast<const f32x4*>(src + i * 16);
  };
  auto fetch_v = [&](int st) {
    if (st >= steps) return;
    const Span s = span(st);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* src = vb + (int64_t)min(s.k0 + 4 * g + e, s.last) * DH + 4 * l;
#pragma unroll
      for (int c = 0; c < DH / 64; ++c) v[e][c] = *reinterpret_cast<const f32x4*>(src + c * 64);
    }
  };
  int st = j.sp * (KA_UNIT / KT) + wave;
  fetch_k(st);
  fetch_v(st);
  for (; st < steps; st += stride) {
    const bool tail = st >= j.reach.prefix_steps;
    const int k0 = span(st).k0, k_last = span(st).last;
    f32x4 x[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      x[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < DH / 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i][e], q[t][i][e], x[t], 0, 0, 0);
    }
    fetch_k(st + stride);
    auto sees = [&](int t, int key) {
      const int n = k0 + key - L;
      return (k0 + key <= k_last) & (!tail | (bool)((n < 64 ? aw0[t] : aw1[t]) >> (n & 63) & 1));
    };
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[t][e] = sees(t, 4 * g + e) ? x[t][e] : -INFINITY;
        mx = fmaxf(mx, x[t][e]);
      }
      mx = xor32_max(xor16_max(mx));
      float m_use;
      const float alpha = sm[t].raise(mx * scale_log2, m_use);
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[t][e] = exp2_hw(fmaf(x[t][e], scale_log2, -m_use));
        sum += x[t][e];
      }
      sm[t].l = sm[t].l * alpha + sum;
      if (!__all(alpha == 1.f)) {
#pragma unroll
        for (int d = 0; d < OT; ++d) o[t][d] *= alpha;
      }
    }
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < DH / 64; ++c) {
        if (k0 + 4 * g + e > k_last) v[e][c] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (tail) {
          // a value that is not finite may only meet the rows that see it: it is taken out here, added below
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (not_finite(v[e][c][i])) v[e][c][i] = 0.f, odd = true;
        }
      }
    odd = __any(odd);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      // output tile 4 c + i takes the dims 64 c + 4 m + i of its rows m
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < OT; ++d) o[t][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][d / 4][d % 4], x[t][e], o[t][d], 0, 0, 0);
      if (odd) {
        for (int key = 0; key < KT; ++key) {
          float have = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) have = key % 4 == e ? x[t][e] : have;
          const float pk = __shfl(have, l + 16 * (key / 4), WAVE);
          const bool vis = sees(t, key);
          const float* src = vb + (int64_t)min(k0 + key, k_last) * DH;
#pragma unroll
          for (int d = 0; d < OT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float f = src[d / 4 * 64 + 16 * g + 4 * e + d % 4];
              if (vis && not_finite(f)) o[t][d][e] += pk * f;
            }
        }
      }
    }
    fetch_v(st + stride);
  }

  constexpr int SETS = DH / 64;
  uint64_t again[RT * SETS] = {};       // lanes whose rows have to be made again
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    sm[t].l = xor32_add(xor16_add(sm[t].l));
    __syncthreads();
    float* mine = mo + (wave * 16 + l) * MP;
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) mine[d / 4 * 64 + 16 * g + 4 * e + d % 4] = o[t][d][e];
    if (g == 0) {
      mml[(wave * 16 + l) * 2] = sm[t].m;
      mml[(wave * 16 + l) * 2 + 1] = sm[t].l;
    }
    __syncthreads();
#pragma unroll
    for (int x0 = 0; x0 < 16 * (DH / 4); x0 += KA_THREADS) {
      const int x = x0 + tid;
      const int i = x / (DH / 4), d = x % (DH / 4) * 4, row = j.r0 + t * 16 + i;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < KA_WAVES; ++w) M = fmaxf(M, mml[(w * 16 + i) * 2]);
      float ls = 0.f;
      f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < KA_WAVES; ++w) {
        const float mw = mml[(w * 16 + i) * 2], lw = mml[(w * 16 + i) * 2 + 1], wt = part_weight(mw, lw, M);
        ls += wt * lw;
        acc += wt * *reinterpret_cast<const f32x4*>(&mo[(w * 16 + i) * MP + d]);
      }
      if (j.direct) {
        const f32x4 outputs[1] = {acc};
        again[t * SETS + x0 / KA_THREADS] = rows_lanes(row < j.live && left_fp32(outputs, ls), DH / 4);
        if (a.out == a.q && (again[t * SETS + x0 / KA_THREADS] >> lane & 1)) continue;
      }
      if (row >= j.live) continue;
      const RowAt at = row_at(a, j, row, first);
      if (j.direct) {
        const float inv = ls == 0.f ? 0.f : 1.f / ls;
        store4((float*)a.out + at.q(a, j.h) + d, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      } else {
        const int64_t to = at.part(a, p, j.h, j.pre ? p.own.splits + j.sp : j.sp);
        *reinterpret_cast<f32x4*>(part_o + to * DH + d) = acc;
        if (d == 0) *reinterpret_cast<float2*>(part_ml + to * 2) = make_float2(M, ls);
      }
    }
  }
  lanes_again<float>(again, a.type, j.b, j.h, [&](int y, int i) { return j.r0 + y / SETS * 16 + (y % SETS * KA_THREADS + wave * WAVE + i) / (DH / 4); },
              DH / 4);
}

// ---------------------------------------------------------------------------- merge
// A row's parts, own splits then the prefix's, in that order: DH / 4 threads take four dims each.  Many
// rows: ROWS of them a thread, two parts of each requested at a time.  Few rows of many parts (ROWS = 1):
// `count` groups of threads deal out the parts, and their sums meet in LDS, in their order.
// (Five waves a SIMD are what the four-row form needs; rows that are made again, two keys at once, fit that.)
template <typename T, int KT, int ROWS>
__global__ __launch_bounds__(KA_THREADS, 5) void kv_merge_kernel(KvAttn a, KvPlan p, int count, const float* __restrict__ part_o,
                                                              const float* __restrict__ part_ml) {
  __shared__ f32x4 so[ROWS == 1 ? KA_THREADS : 1];
  __shared__ float2 sml[ROWS == 1 ? KA_THREADS : 1];
  const int per = a.Dh / 4, b = blockIdx.z, h = blockIdx.y, tid = threadIdx.x;
  const int n_q = a.n_q[b], len = a.own.len[b], n_tail = a.n_tail[b];          // (one wait for all)
  const int n_own = reach_of<KT>(len, n_tail, a.own.cap, p.own, 1).live, n = n_own + pre_reach<KT>(a, p, b).live;
  const int fit = KA_THREADS / per, unit = tid / per, d = tid % per * 4;
  const int grp = ROWS == 1 ? unit % count : 0, step = ROWS == 1 ? count : 1;
  const int each = ROWS == 1 ? fit / count : fit * ROWS, live = max(0, min(n_q, a.nq_max)) * a.G;
  const int row0 = blockIdx.x * each + (ROWS == 1 ? unit / count : unit);
  if (n == 1 || (int)blockIdx.x * each >= live) return;
  // rows row0, row0 + fit, ...; one past the last repeats it
  constexpr int AT_ONCE = ROWS == 1 ? 4 : 2;
  const int64_t rows = (int64_t)a.nq_max * a.G, base = ((int64_t)b * a.Hkv + h) * p.parts * rows;
  float m[ROWS], l[ROWS];
  f32x4 o[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
    o[r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  auto add = [](float pm, float pl, const f32x4& po, float m, float& l, f32x4& o) {       // at the maximum m
    const float wt = part_weight(pm, pl, m);
    l = fmaf(wt, pl, l);
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = fmaf(wt, po[e], o[e]);
  };
  for (int s0 = row0 < live ? grp : n; s0 < n; s0 += AT_ONCE * step) {
    float2 ml[ROWS][AT_ONCE];
    f32x4 x[ROWS][AT_ONCE];
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) {
        ml[r][i] = make_float2(-INFINITY, 0.f);
        const int s = s0 + i * step;
        if (s >= n) continue;
        const int64_t from = base + (s < n_own ? s : p.own.splits + s - n_own) * rows + min(row0 + r * fit, live - 1);
        ml[r][i] = *reinterpret_cast<const float2*>(part_ml + from * 2);
        x[r][i] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(part_o + from * a.Dh + d));
      }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      float M = m[r];
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i) M = fmaxf(M, ml[r][i].x);
      const float down = m[r] == -INFINITY ? 1.f : exp2_hw(m[r] - M);
      m[r] = M;
      l[r] *= down;
      o[r] *= down;
#pragma unroll
      for (int i = 0; i < AT_ONCE; ++i)
        if (s0 + i * step < n) add(ml[r][i].x, ml[r][i].y, x[r][i], m[r], l[r], o[r]);
    }
  }
  if (ROWS == 1 && count > 1) {
    so[tid] = o[0];
    sml[tid] = make_float2(m[0], l[0]);
    __syncthreads();
    const int groups = grp > 0 ? 0 : min(count, n);
    for (int g = 1; g < groups; ++g) m[0] = fmaxf(m[0], sml[tid + g * per].x);
    l[0] = 0.f;
    o[0] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < groups; ++g) add(sml[tid + g * per].x, sml[tid + g * per].y, so[tid + g * per], m[0], l[0], o[0]);
  }
  uint64_t again[ROWS];        // lanes whose rows have to be made again
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const int row = row0 + r * fit;
    const bool writes = row < live && grp == 0;
    const f32x4 outputs[1] = {o[r]};
    again[r] = rows_lanes(writes && left_fp32(outputs, l[r]), per);
    if (!writes || (a.out == a.q && (again[r] >> (tid % WAVE) & 1))) continue;
    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
    store4((T*)a.out + RowAt{b, row / a.G, row % a.G}.q(a, h) + d, o[r][0] * inv, o[r][1] * inv, o[r][2] * inv, o[r][3] * inv);
  }
  lanes_again<T>(again, a.type, b, h, [&](int r, int i) { return __builtin_amdgcn_readlane(row0, i) + r * fit; }, per);
}

// ---------------------------------------------------------------------------- host
// Splits: as many as give the workgroups that the CUs hold at once (two each) equal shares of the keys of
// both parts, by the bounds the launch is given.  At least eight units of 64 keys pay for a split's start
// and end, its partial results and their merge: one row of 32 heads over 300 slots 11.8 us with eight,
// 11.1 + 3.9 (attention + merge) with three, 11.9 with twelve; over 700 slots 12.7 + 4.0, 12.1 + 3.9, 16.2;
// over 8000 13.7 + 3.9, 13.8 + 4.6, 15.6 + 3.8; a 61-row tree of 32 heads over 100 slots 12.1, 13.0 + 3.8;
// over 2300 18.3 + 4.8, 18.6 + 6.6, 19.9 + 3.9.  Shares for 1024 or 1536 workgroups in place of 512 cost more in
// partial results than they even out (sixteen ragged 61-row trees 67 + 0, 68 + 8.7, 69 + 9.7 us).  fp32, whose
// waves take their steps one after the other from memory, at least two: one row over 300 slots 11.7 + 4.0
// with two, 14.4 + 3.9 with three, 19.2 with eight; over 2000 11.8 + 4.0, 14.5 + 3.9, 26.4 + 4.0; over 8000 24.8 +
// 5.2, 25.0 + 5.0, 28.7 + 4.6; a 61-row tree over 2300 45.7 + 4.8, 45.7 + 4.7, 55.5 + 4.8.
// most: the parts that the plans of these bounds and of any smaller ones have at most.  A share is LEAST units or more, and
// one pair's keys of SLOTS shares a SLOTS-th of its side's or more, so a side has at most as many splits as either makes.
static KvPlan kv_plan(const KvAttn& a, int* most = nullptr) {
  KvPlan p{};
  const bool f32 = a.type == ADT_F32;
  auto side = [&](KvSide& s, int64_t rows) {
    s.tiles = f32 || rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    s.blocks = (int)((rows + 32 * s.tiles - 1) / (32 * s.tiles));
  };
  const int64_t rows = (int64_t)a.nq_max * a.G;
  side(p.own, rows);
  const int64_t own_pairs = (int64_t)a.B * a.Hkv * p.own.blocks, own_units = ((int64_t)a.own.cap + KA_UNIT - 1) / KA_UNIT + 1;
  int64_t pre_pairs = 0, pre_units = 0;
  if (a.groups) {
    side(p.pre, rows * a.group);
    pre_pairs = (int64_t)a.groups * a.Hkv * p.pre.blocks;
    pre_units = ((int64_t)a.pre.cap + KA_UNIT - 1) / KA_UNIT;
  }
  const int64_t SLOTS = 512, LEAST = f32 ? 2 : 8;
  const int64_t per = std::max<int64_t>(LEAST, (own_pairs * own_units + pre_pairs * pre_units + SLOTS - 1) / SLOTS);
  auto split = [&](KvSide& s, int64_t pairs, int64_t units) {
    s.per = (int)std::min<int64_t>(per, 1 << 30);
    int64_t n = units <= per + per / 4 ? 1 : (units + per - 1) / per;
    n = std::min<int64_t>(n, std::max<int64_t>(1, 2 * SLOTS / std::max<int64_t>(1, pairs)));
    s.splits = (int)std::min<int64_t>(n, 64);
    int64_t top = units <= LEAST + LEAST / 4 ? 1 : (units + LEAST - 1) / LEAST;
    top = std::min(top, std::max<int64_t>(1, (SLOTS + pairs - 1) / std::max<int64_t>(1, pairs)));
    if (most) *most += (int)std::min<int64_t>(top, 64);
  };
  if (most) *most = 0;
  split(p.own, own_pairs, own_units);
  if (a.groups) split(p.pre, pre_pairs, pre_units);
  p.pre_jobs = pre_pairs * p.pre.splits;
  p.jobs = p.pre_jobs + own_pairs * p.own.splits;
  p.parts = p.own.splits + p.pre.splits;
  return p;
}
static size_t part_rows(const KvAttn& a, int parts) { return parts == 1 ? 0 : (size_t)a.B * a.Hkv * parts * a.nq_max * a.G; }

size_t kv_attn_ws_bytes(const KvAttn& a) {
  int most;
  kv_plan(a, &most);
  return part_rows(a, most) * (a.Dh + 2) * sizeof(float);
}
size_t kv_attn_ws_need(const KvAttn& a) { return part_rows(a, kv_plan(a).parts) * (a.Dh + 2) * sizeof(float); }

adt_status launch_kv_attn(const KvAttn& a, void* ws, hipStream_t st) {
  const KvPlan p = kv_plan(a);
  // (a launch has fewer than 2^32 threads in a dimension)
  ADT_CHECK_ARG(p.jobs < (int64_t)1 << 24, ADT_E_CAPACITY, "cache_tree_attn: %lld workgroups", (long long)p.jobs);
  float *part_o = (float*)ws, *part_ml = part_o + part_rows(a, p.parts) * a.Dh;
  const size_t lds = a.groups ? (size_t)(a.group + 1) * sizeof(int) : 0;
  const unsigned jobs = (unsigned)p.jobs;
#define ADT_KA(CV)                                                                               \
  if (a.Dh == 128) kv_attn_kernel<CV, 128><<<jobs, KA_THREADS, lds, st>>>(a, p, part_o, part_ml); \
  else kv_attn_kernel<CV, 64><<<jobs, KA_THREADS, lds, st>>>(a, p, part_o, part_ml)
  switch (a.type) {
    case ADT_BF16: ADT_KA(uint16_t); break;
    case ADT_E4M3: ADT_KA(E4M3); break;
    case ADT_I8: ADT_KA(I8); break;
    default:
      if (a.Dh == 128) kv_attn_f32_kernel<128><<<jobs, KA_THREADS, lds, st>>>(a, p, part_o, part_ml);
      else kv_attn_f32_kernel<64><<<jobs, KA_THREADS, lds, st>>>(a, p, part_o, part_ml);
  }
#undef ADT_KA
  ADT_LAUNCH_CHECK();
  if (p.parts == 1) return ADT_OK;
  // a thread for every four outputs, or for few outputs of many parts several, or for many outputs one for
  // sixteen: trees of 61 rows of 32 heads of 128 dims, two or three parts, with one row a thread and with
  // four: 4 trees 6.9, 7.9 us, 8 trees 7.9, 7.3, 16 trees 11.6, 7.9, 32 trees 21.1, 14.3
  const int fit = KA_THREADS / (a.Dh / 4), rows = a.nq_max * a.G;
  const int64_t outputs = (int64_t)a.B * a.Hkv * rows * (a.Dh / 4);
  const int count = p.parts > 8 && outputs < 65536 ? fit : 1;
  const bool many = outputs >= 1 << 18;
  const int64_t each = many ? 4 * fit : fit / count;
  const dim3 grid((unsigned)((rows + each - 1) / each), a.Hkv, a.B);
#define ADT_KM(TV, KTV)                                                                                     \
  if (many) kv_merge_kernel<TV, KTV, 4><<<grid, KA_THREADS, 0, st>>>(a, p, count, part_o, part_ml);         \
  else kv_merge_kernel<TV, KTV, 1><<<grid, KA_THREADS, 0, st>>>(a, p, count, part_o, part_ml)
  if (a.type == ADT_F32) { ADT_KM(float, 16); }
  else { ADT_KM(uint16_t, 32); }
#undef ADT_KM
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

}  // namespace adt
