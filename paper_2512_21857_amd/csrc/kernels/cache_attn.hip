// Tree attention over a long cache for grouped heads: over the blocks of the prefix that each query
// row chose, or over all of it with the weight that every slot received.
//
// The query rows of one key-value head, nq * G of them (row = node * G + head of the group), go in
// tiles of 16 through one pass over the keys with the running maximum and sum of a softmax:
//   S^T[key][row] = K[key][:] . Q[row][:]        (A = K rows, B = Q^T)
//   O^T[dim][row] += V^T[dim][key] . P^T[key][row]
// A workgroup holds RT tiles (16 RT rows) in registers; its waves and the other workgroups of the
// same rows (splits) deal the keys out in steps among themselves, each step read by one wave only,
// so K and V come straight from memory into registers and every slot is read once per 16 RT rows.
// What the waves of a workgroup found is merged in LDS, what the splits found by a launch of its own
// (few rows over chosen blocks: by the last split), always in one order.  Steps never straddle the end
// of the prefix: the tree's own slots, which the rows see through their ancestor masks, have steps of
// their own.
//
// bf16 runs on the 16x16x32 MFMA, 32 keys a step, V transposed through LDS, probabilities rounded to
// bf16 for the second product (off by 2^-8 of a term at most, as the output by its own rounding);
// with more than 16 rows in cache_attn_shared_kernel, whose waves share the keys.  fp32 runs on the
// 16x16x4 MFMA, 16 keys a step, without LDS.  Scores, softmax sums and outputs are fp32.
//
// Bound by the read of K and V, in bf16 also at 64 rows a head: one row of 32 heads over 65333 slots of 8
// key-value heads (268 MB) 52-58 us, sixteen trees of up to 61 rows of 32 heads (398 MB) 78 us, 5.1 TB/s;
// the chosen blocks of sixteen 16-row trees (462 MB) 98-102 us.  fp32 keeps up with up to 16 rows a head (one
// row of 32 heads over 65333 slots, 535 MB, 111 us).  More rows are bound by latency: a step's loads start when
// the products of the one before are done, at one wave per SIMD with four tiles, and each 64 rows read the keys
// anew: 61 rows of 32 heads over 2340 slots 43 us (bf16 15), sixteen such trees 331 (78), 16-row trees over chosen
// blocks 457 (99).
//
// A masked score is dropped by selection, so whatever a slot's key holds does not matter to rows
// that do not see it.  Its value does meet their zero weight in the second product, and 0 * inf is
// NaN; a wave whose results come out not finite therefore goes through its steps once more with
// such values taken out of the product and added for the rows that see them only.
#include <algorithm>
#include <type_traits>

#include "../launch.h"

namespace adt {

ADT_DEVICE_ERROR_WORD(cache_attn)

constexpr int CA_WAVES = 4;
constexpr int CA_THREADS = CA_WAVES * WAVE;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool not_finite(float x) { return !(fabsf(x) <= 3.402823466e38f); }

template <bool NT, class V>
__device__ __forceinline__ V load16(const V* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p);
  else return *p;
}

// What the two types differ in.  Lane (l, g) = (lane % 16, lane / 16) holds the scores of row l and
// the KT keys key(sub, r) = 16 sub + 4 g + r of a step, and the outputs dim(t, r) of row l.
template <typename T, int DH>
struct Tile;

template <int DH>
struct Tile<uint16_t, DH> {
  static constexpr int DIM = DH, KT = 32, SUBS = 2, KS = DH / 32, OT = DH / 16, VG = DH / 64;
  static constexpr int VP = DH + 16;     // LDS row of V, padded so that a transpose load's rows fall on distinct banks
  static constexpr int LDS_BYTES = KT * VP * 2;
  struct Query {
    bf16x8 f[KS];
  };
  struct Step {
    bf16x8 k[SUBS][KS];
    u16x8 v[VG][4];
  };
  static __device__ __forceinline__ int dim(int t, int g, int r) { return t * 16 + 4 * g + r; }
  static __device__ __forceinline__ void zero(Query& x) {
#pragma unroll
    for (int j = 0; j < KS; ++j) x.f[j] = bf16x8{};
  }
  static __device__ __forceinline__ void load(Query& x, const uint16_t* row, int g) {
#pragma unroll
    for (int j = 0; j < KS; ++j) x.f[j] = *reinterpret_cast<const bf16x8*>(row + j * 32 + g * 8);
  }
  // the step's keys key0 .. key0 + 31; those past `last` repeat it
  template <bool NT = true>
  static __device__ __forceinline__ void load_k(Step& s, const uint16_t* k, int key0, int last, int l, int g) {
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      const uint16_t* row = k + (int64_t)min(key0 + sub * 16 + l, last) * DH + g * 8;
#pragma unroll
      for (int j = 0; j < KS; ++j) s.k[sub][j] = load16<NT>(reinterpret_cast<const bf16x8*>(row + j * 32));
    }
  }
  static __device__ __forceinline__ void load_v(Step& s, const uint16_t* v, int key0, int last, int l, int g) {
    const int lane = g * 16 + l;
#pragma unroll
    for (int j = 0; j < VG; ++j) {
      const int gi = lane + j * WAVE, c = gi % (DH / 8) * 8, r4 = gi / (DH / 8) * 4;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        s.v[j][u] = __builtin_nontemporal_load(reinterpret_cast<const u16x8*>(v + (int64_t)min(key0 + r4 + u, last) * DH + c));
    }
  }
  // V into the wave's LDS rows
  static __device__ __forceinline__ void stage(const Step& s, void* lds, int l, int g) {
    uint16_t(*rows)[VP] = reinterpret_cast<uint16_t(*)[VP]>(lds);
    const int lane = g * 16 + l;
#pragma unroll
    for (int j = 0; j < VG; ++j) {
      const int gi = lane + j * WAVE, c = gi % (DH / 8) * 8, r4 = gi / (DH / 8) * 4;
#pragma unroll
      for (int u = 0; u < 4; ++u) *reinterpret_cast<u16x8*>(&rows[r4 + u][c]) = s.v[j][u];
    }
    wave_lds_fence();
  }
  static __device__ __forceinline__ void scores(f32x4 (&st)[SUBS], const Step& s, const Query& x) {
#pragma unroll
    for (int sub = 0; sub < SUBS; ++sub) {
      st[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < KS; ++j) st[sub] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s.k[sub][j], x.f[j], st[sub], 0, 0, 0);
    }
  }
  // S[row][key] of 16 rows and the keys 16 sub + l
  static __device__ __forceinline__ void col_scores(f32x4& st, const Step& s, int sub, const Query& x) {
#pragma unroll
    for (int j = 0; j < KS; ++j) st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.f[j], s.k[sub][j], st, 0, 0, 0);
  }
  // O^T += V^T P^T; lane (l, g) of the transpose load that addresses row k0 + l / 4, dims
  // d0 + 4 (l % 4)..+3 gets V[k0 + s][d0 + l], s = 0..3
  template <bool SAFE>
  static __device__ __forceinline__ void add(f32x4 (&o)[OT], const f32x4 (&p)[SUBS], const Step&, void* lds, int l, int g) {
    uint16_t(*rows)[VP] = reinterpret_cast<uint16_t(*)[VP]>(lds);
    bf16x8 b;
#pragma unroll
    for (int r = 0; r < 8; ++r) b[r] = (__bf16)(p[r / 4][r % 4]);
    const int col = 4 * (l & 3), row = l >> 2;
#pragma unroll
    for (int t = 0; t < OT; ++t) {
      v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)&rows[4 * g + row][t * 16 + col]);
      v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)&rows[16 + 4 * g + row][t * 16 + col]);
      if (SAFE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if ((lo[e] & 0x7f80) == 0x7f80) lo[e] = 0;
          if ((hi[e] & 0x7f80) == 0x7f80) hi[e] = 0;
        }
      }
      const bf16x8 a = __builtin_bit_cast(bf16x8, v8i16{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
      o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, o[t], 0, 0, 0);
    }
  }
};

template <int DH>
struct Tile<float, DH> {
  static constexpr int DIM = DH, KT = 16, SUBS = 1, OT = DH / 16;
  static constexpr int LDS_BYTES = 0;
  struct Query {
    f32x4 f[DH / 16];
  };
  struct Step {
    f32x4 k[DH / 16];
    f32x4 v[4][DH / 64];     // v[r][c]: key 4 g + r, dims 64 c + 4 l .. + 3
  };
  // output tile 4 c + e takes the dims 64 c + 4 i + e of its rows i
  static __device__ __forceinline__ int dim(int t, int g, int r) { return t / 4 * 64 + 16 * g + 4 * r + t % 4; }
  static __device__ __forceinline__ void zero(Query& x) {
#pragma unroll
    for (int j = 0; j < DH / 16; ++j) x.f[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  static __device__ __forceinline__ void load(Query& x, const float* row, int g) {
#pragma unroll
    for (int j = 0; j < DH / 16; ++j) x.f[j] = *reinterpret_cast<const f32x4*>(row + j * 16 + g * 4);
  }
  template <bool NT = true>
  static __device__ __forceinline__ void load_k(Step& s, const float* k, int key0, int last, int l, int g) {
    const float* row = k + (int64_t)min(key0 + l, last) * DH + g * 4;
#pragma unroll
    for (int j = 0; j < DH / 16; ++j) s.k[j] = load16<NT>(reinterpret_cast<const f32x4*>(row + j * 16));
  }
  static __device__ __forceinline__ void load_v(Step& s, const float* v, int key0, int last, int l, int g) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float* row = v + (int64_t)min(key0 + 4 * g + r, last) * DH + 4 * l;
#pragma unroll
      for (int c = 0; c < DH / 64; ++c) s.v[r][c] = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(row + c * 64));
    }
  }
  static __device__ __forceinline__ void stage(const Step&, void*, int, int) {}
  static __device__ __forceinline__ void scores(f32x4 (&st)[SUBS], const Step& s, const Query& x) {
    st[0] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < DH / 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) st[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(s.k[j][e], x.f[j][e], st[0], 0, 0, 0);
  }
  static __device__ __forceinline__ void col_scores(f32x4& st, const Step& s, int, const Query& x) {
#pragma unroll
    for (int j = 0; j < DH / 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_16x16x4f32(x.f[j][e], s.k[j][e], st, 0, 0, 0);
  }
  template <bool SAFE>
  static __device__ __forceinline__ void add(f32x4 (&o)[OT], const f32x4 (&p)[SUBS], const Step& s, void*, int, int) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        float a = s.v[r][t / 4][t % 4];
        if (SAFE && not_finite(a)) a = 0.f;
        o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, p[0][r], o[t], 0, 0, 0);
      }
  }
};

// How the keys of one (sequence, key-value head, row group) are dealt out: `units` of them (steps, or
// stages of two) to `n` of the launch's splits, at least `per` each, so that a split is worth its
// start whatever the launch's bounds were, and short sequences and long ones take workgroups of much
// the same work.  Split 0 leaves n for the merge.
struct Deal {
  int splits, per;          // of the launch; units per split
  int32_t* live;            // [B][Hkv][groups] n, or null (one split)
  __device__ __forceinline__ int splits_of(int units) const { return max(1, min(splits, (units + per - 1) / per)); }
  __device__ __forceinline__ int live_splits(int64_t i) const { return max(0, min(live[i], splits)); }
};

// The chosen blocks of a pair into LDS; ends with a barrier.
__device__ __forceinline__ void copy_list(const uint16_t* blocks, int count, uint16_t* chosen) {
  for (int j = threadIdx.x; j < count; j += blockDim.x) chosen[j] = blocks[j];
  __syncthreads();
}

// Log-sum-exp merge of parts (m, l, o), eight at a time and in order.
struct RunningMerge {
  float m = -INFINITY, l = 0.f;
  f32x4 o{0.f, 0.f, 0.f, 0.f};
  // one part at the running maximum `top` (0 where that is -inf); one that saw nothing, (-inf, 0), adds nothing
  __device__ __forceinline__ void add_one(float pm, float pl, const f32x4& po, float top) {
    const float wt = pm == -INFINITY && pl == 0.f ? 0.f : exp2_hw(pm - top);
    if (wt == 0.f && pl == pl) return;
    l += wt * pl;
    o += wt * po;
  }
  __device__ __forceinline__ void add(const float2 (&ml)[8], const f32x4 (&x)[8], int n, int stride = 1) {
    float mn = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) mn = fmaxf(mn, ml[j].x);
    const float top = mn == -INFINITY ? 0.f : mn, down = m == -INFINITY ? 1.f : exp2_hw(m - top);
    m = mn;
    l *= down;
    o *= down;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j * stride < n) add_one(ml[j].x, ml[j].y, x[j], top);
  }
};

// What a step's values that are not finite add to the rows that see them: o[t][r] (dim(t, r) of row
// l) += p v over the keys of the step whose value v at that dim is one.  p: this lane's probabilities
// of row l, for keys 16 sub + 4 g + r; seen(key): whether row l sees key k0 + key.
template <class X, typename T, class F>
__device__ __forceinline__ void add_not_finite(f32x4 (&o)[X::OT], const f32x4 (&p)[X::SUBS], const T* v, int k0, int last,
                                               int l, int g, F seen) {
  for (int key = 0; key < X::KT; ++key) {
    float mine = 0.f;
#pragma unroll
    for (int sub = 0; sub < X::SUBS; ++sub)
#pragma unroll
      for (int r = 0; r < 4; ++r) mine = key / 16 == sub && key % 4 == r ? p[sub][r] : mine;
    const float pk = __shfl(mine, l + 16 * (key % 16 / 4), WAVE);
    const bool vis = seen(key);
    const T* row = v + (int64_t)min(k0 + key, last) * X::DIM;
#pragma unroll
    for (int t = 0; t < X::OT; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float x = Elem<T>::load(row, X::dim(t, g, r));
        if (vis && not_finite(x)) o[t][r] += pk * x;
      }
  }
}

// (registers: outputs 16 RT DH / 64 a lane, and a step's K and V: one wave per SIMD at RT = 4, where head size
// 128 over chosen blocks still spills 40 of them)
template <typename T, int DH, int RT, bool SPARSE>
__global__ __launch_bounds__(CA_THREADS, RT == 4 ? 1 : 2) void cache_attn_kernel(CacheAttn a, Deal deal,
                                                                                float* __restrict__ part_o,
                                                                                float* __restrict__ part_ml,
                                                                                float* __restrict__ kept) {
  typedef Tile<T, DH> X;
  constexpr int KT = X::KT, SUBS = X::SUBS, OT = X::OT;
  constexpr bool MERGE = SPARSE && RT == 1;
  constexpr int MP = DH + 4;                                       // row of a merged tile
  constexpr int STEP_BYTES = CA_WAVES * X::LDS_BYTES;
  constexpr int MERGE_BYTES = CA_WAVES * 16 * (MP + 2) * 4;
  __shared__ __attribute__((aligned(16))) unsigned char smem[STEP_BYTES > MERGE_BYTES ? STEP_BYTES : MERGE_BYTES];
  extern __shared__ uint16_t chosen[];                             // SPARSE: the blocks that any row chose
  const int h = blockIdx.x % a.Hkv, rg = blockIdx.x / a.Hkv, b = blockIdx.y, sp = blockIdx.z;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
  const int l = lane & 15, g = lane >> 4;
  const int rows = a.nq_max * a.G, live_rows = max(0, min(a.n_q[b], a.nq_max)) * a.G;
  const int r0 = rg * 16 * RT;
  if (r0 >= live_rows) return;
  const int L = max(0, min(a.kv_len[b], a.kv_cap));
  const int total = min((int64_t)L + max(0, min(a.n_tail[b], ADT_MAX_NODES)), (int64_t)a.kv_cap);
  if (threadIdx.x == 0 && (int64_t)a.kv_len[b] + a.n_tail[b] > a.kv_cap) dev_fail(DEVINV_KV_RANGE);
  const int64_t pair = (int64_t)b * a.Hkv + h;
  const int per_blk = SPARSE ? a.block / KT : 1;
  const int prefix_steps = SPARSE ? a.lists.count[pair] * per_blk : (L + KT - 1) / KT;
  const int steps = prefix_steps + (total - L + KT - 1) / KT;
  const int splits = deal.splits, n_live = deal.splits_of(steps);
  if (sp >= n_live) return;
  if (deal.live && sp == 0 && threadIdx.x == 0) deal.live[(int64_t)b * gridDim.x + blockIdx.x] = n_live;
  const uint64_t* marks = a.lists.marks + pair * a.n_blk * ADT_MASK_WORDS;
  const T* kb = (const T*)a.k + b * a.sb + h * a.sh;
  const T* vb = (const T*)a.v + b * a.sb + h * a.sh;

  typename X::Query q[RT];
  uint64_t aw0[RT], aw1[RT];
  int node[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    X::zero(q[t]);
    aw0[t] = aw1[t] = 0;
    node[t] = -1;
    const int row = r0 + t * 16 + l;
    if (row < live_rows) {
      const int i = row / a.G, u = row - i * a.G;
      node[t] = i;
      X::load(q[t], (const T*)a.q + (((int64_t)b * a.nq_max + i) * a.Hkv + h) * a.G * DH + (int64_t)u * DH, g);
      const uint64_t* mp = a.mask + ((int64_t)b * a.nq_max + i) * ADT_MASK_WORDS;
      aw0[t] = mp[0];
      aw1[t] = mp[1];
    }
  }
  if (SPARSE) copy_list(a.lists.blocks + pair * a.n_blk, a.lists.count[pair], chosen);
  const float scale_log2 = a.scale * LOG2E;
  void* lds = smem + wave * X::LDS_BYTES;

  f32x4 o[RT][OT];
  float m_run[RT], l_run[RT];      // running maximum (log2 domain), this lane's share of the sum
  typename X::Step step;
  // key0, the last key, and the rows that chose the step's block
  int key0 = 0, last = 0;
  uint64_t w0 = 0, w1 = 0;
  auto request = [&](int s, int& key0, int& last, uint64_t& w0, uint64_t& w1) {
    if (s < prefix_steps) {
      key0 = s * KT;
      last = L - 1;
      if (SPARSE) {
        const int at = s / per_blk, j = __builtin_amdgcn_readfirstlane((int)chosen[at]);
        key0 = j * a.block + s % per_blk * KT;
        last = min(L, (j + 1) * a.block) - 1;
        w0 = marks[2 * at];
        w1 = marks[2 * at + 1];
      }
    } else {
      key0 = L + (s - prefix_steps) * KT;
      last = total - 1;
    }
    X::load_k(step, kb, key0, last, l, g);
    X::load_v(step, vb, key0, last, l, g);
  };
  auto pass = [&](auto safe_tag) {
    constexpr bool SAFE = decltype(safe_tag)::value;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m_run[t] = -INFINITY;
      l_run[t] = 0.f;
#pragma unroll
      for (int d = 0; d < OT; ++d) o[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int stride = n_live * CA_WAVES;
    int s = sp * CA_WAVES + wave;
    if (s < steps) request(s, key0, last, w0, w1);
    for (; s < steps; s += stride) {
      const int k0 = key0, k_last = last;
      const uint64_t c0 = w0, c1 = w1;
      const bool tail = s >= prefix_steps;
      X::stage(step, lds, l, g);
      f32x4 st[RT][SUBS];
      bool sees[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const uint64_t w = node[t] < 64 ? c0 : c1;
        sees[t] = node[t] >= 0 && (tail || !SPARSE || (w >> (node[t] & 63) & 1));
        if (!SPARSE || __any(sees[t])) X::scores(st[t], step, q[t]);
      }
      if constexpr (X::LDS_BYTES > 0) {
        if (s + stride < steps) request(s + stride, key0, last, w0, w1);
      }
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        if (SPARSE && !__any(sees[t])) continue;
        float mx = -INFINITY;
        if (!tail && k0 + KT - 1 <= k_last) {
#pragma unroll
          for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              if (SPARSE) st[t][sub][r] = sees[t] ? st[t][sub][r] : -INFINITY;
              mx = fmaxf(mx, st[t][sub][r]);
            }
        } else {
#pragma unroll
          for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int key = k0 + sub * 16 + 4 * g + r, j = key - L;
              const uint64_t w = j < 64 ? aw0[t] : aw1[t];
              const bool vis = sees[t] & (key <= k_last) & (!tail | (bool)(w >> (j & 63) & 1));
              const float v = vis ? st[t][sub][r] : -INFINITY;
              st[t][sub][r] = v;
              mx = fmaxf(mx, v);
            }
        }
        if (RT == 1 && !SPARSE && kept && node[0] >= 0) {
          // the masked scores, for the weights of the slots
          float* to = kept + (pair * rows + l) * a.kv_cap + k0 + 4 * g;
#pragma unroll
          for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int r = 0; r < 4; ++r)
              if (k0 + sub * 16 + 4 * g + r <= k_last) to[sub * 16 + r] = st[0][sub][r];
        }
        mx = xor16_max(mx);
        mx = xor32_max(mx);
        const float m_new = fmaxf(m_run[t], mx * scale_log2);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;     // nothing seen yet: weights 0, not NaN
        const float alpha = m_new == m_run[t] ? 1.f : exp2_hw(m_run[t] - m_use);
        m_run[t] = m_new;
        float rs = 0.f;
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = exp2_hw(fmaf(st[t][sub][r], scale_log2, -m_use));
            st[t][sub][r] = p;
            rs += p;
          }
        l_run[t] = l_run[t] * alpha + rs;
        if (!__all(alpha == 1.f)) {
#pragma unroll
          for (int d = 0; d < OT; ++d) o[t][d] *= alpha;
        }
        X::template add<SAFE>(o[t], st[t], step, lds, l, g);
        if (SAFE)
          add_not_finite<X>(o[t], st[t], vb, k0, k_last, l, g, [&](int key) {
            const int j = k0 + key - L;
            return sees[t] & (k0 + key <= k_last) & (!tail | (bool)((j < 64 ? aw0[t] : aw1[t]) >> (j & 63) & 1));
          });
      }
      if (X::LDS_BYTES > 0) wave_lds_fence();
      if constexpr (X::LDS_BYTES == 0) {
        if (s + stride < steps) request(s + stride, key0, last, w0, w1);
      }
    }
  };
  pass(std::false_type{});
  float odd = 0.f;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) odd += o[t][d][r] * 0.f;
  if (__any(odd != odd)) pass(std::true_type{});

  // merge of the waves, tile by tile, in wave order
  float* mo = reinterpret_cast<float*>(smem);                      // [wave][16][MP]
  float* mml = mo + CA_WAVES * 16 * MP;                            // [wave][16][2]
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l_run[t] = xor16_add(l_run[t]);
    l_run[t] = xor32_add(l_run[t]);
    __syncthreads();
    float* row = mo + (wave * 16 + l) * MP;
#pragma unroll
    for (int d = 0; d < OT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) row[X::dim(d, g, r)] = o[t][d][r];
    if (g == 0) {
      mml[(wave * 16 + l) * 2] = m_run[t];
      mml[(wave * 16 + l) * 2 + 1] = l_run[t];
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < 16 * (DH / 4); idx += CA_THREADS) {
      const int i = idx / (DH / 4), d = idx % (DH / 4) * 4, rr = r0 + t * 16 + i;
      if (rr >= live_rows) continue;
      float M = -INFINITY;
#pragma unroll
      for (int w = 0; w < CA_WAVES; ++w) M = fmaxf(M, mml[(w * 16 + i) * 2]);
      float ls = 0.f;
      f32x4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < CA_WAVES; ++w) {
        const float mw = mml[(w * 16 + i) * 2], lw = mml[(w * 16 + i) * 2 + 1];
        const float wt = mw == -INFINITY && lw == 0.f ? 0.f : exp2_hw(mw - (M == -INFINITY ? 0.f : M));
        if (wt == 0.f && lw == lw) continue;
        ls += wt * lw;
        acc += wt * *reinterpret_cast<const f32x4*>(&mo[(w * 16 + i) * MP + d]);
      }
      const int64_t at = (pair * splits + sp) * rows + rr;
      if (n_live == 1) {
        const float inv = ls == 0.f ? 0.f : 1.f / ls;
        const int64_t at_o = (((int64_t)b * a.nq_max + rr / a.G) * a.Hkv + h) * a.G * DH + (int64_t)(rr % a.G) * DH + d;
        store4((T*)a.out + at_o, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      } else if (MERGE) {
        agent_store2(part_o + at * DH + d, acc[0], acc[1]);
        agent_store2(part_o + at * DH + d + 2, acc[2], acc[3]);
      } else {
        *reinterpret_cast<f32x4*>(part_o + at * DH + d) = acc;
      }
      if (part_ml && d == 0) {
        if (MERGE) {
          agent_store2(part_ml + at * 2, M, ls);
        } else {
          part_ml[at * 2] = M;
          part_ml[at * 2 + 1] = ls;
        }
      }
    }
  }
  // Few rows over chosen blocks: the last split of the pair to get here merges them all, in split order,
  // four dims of one row a thread.  The partials of a split are complete at the agent's coherence point
  // (write-through stores, waited for) before its arrival counts, and are read past the local caches.
  if constexpr (MERGE) {
    if (n_live == 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    uint32_t* last = reinterpret_cast<uint32_t*>(smem);
    if (threadIdx.x == 0)
      *last = __hip_atomic_fetch_add(a.lists.arrived + pair, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    __syncthreads();
    if (*last != (uint32_t)n_live) return;
    for (int idx = threadIdx.x; idx < live_rows * (DH / 4); idx += CA_THREADS) {
      const int rr = idx / (DH / 4), d = idx % (DH / 4) * 4;
      const int64_t base = pair * splits * rows + rr;
      RunningMerge acc;
      for (int s0 = 0; s0 < n_live; s0 += 8) {       // eight splits requested at a time
        float2 ml[8];
        f32x4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t at = base + (int64_t)min(s0 + j, n_live - 1) * rows;
          ml[j] = agent_load2(part_ml + at * 2);
          const float2 lo = agent_load2(part_o + at * DH + d), hi = agent_load2(part_o + at * DH + d + 2);
          x[j] = f32x4{lo.x, lo.y, hi.x, hi.y};
        }
        acc.add(ml, x, n_live - s0);
      }
      const float inv = acc.l == 0.f ? 0.f : 1.f / acc.l;
      const int64_t at_o = (((int64_t)b * a.nq_max + rr / a.G) * a.Hkv + h) * a.G * DH + (int64_t)(rr % a.G) * DH + d;
      store4((T*)a.out + at_o, acc.o[0] * inv, acc.o[1] * inv, acc.o[2] * inv, acc.o[3] * inv);
    }
  }
}

// Many rows (more than 16) in bf16: the waves of a workgroup share the keys instead.  A stage of two
// 32-key steps comes into LDS once, fetched by all threads into registers P stages (one or three) ahead;
// wave w computes row tile w % TILES, for step w / TILES of the stage (KH = 2) or both (KH = 1), so a
// wave holds one tile's outputs and the CU two or four waves per SIMD (the four at head size 128 have 128
// registers a lane: 6 are spilled over chosen blocks, with 65 and more rows 47, over all slots 7).  Rows of K and V lie in 16-byte
// chunks swizzled by row, so that the operand reads (16 rows of one chunk column; 8 rows of two in the
// transpose load) touch distinct banks.
template <int DH>
__device__ __forceinline__ int swz_k(int row) { return DH == 128 ? (row & 15) : ((row >> 1) & 7); }
template <int DH>
__device__ __forceinline__ int swz_v(int row) { return DH == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); }

template <int DH, int NW, int KH, int P, bool SPARSE>
__global__ __launch_bounds__(NW * WAVE, P > 1 ? 2 : NW / 2) void cache_attn_shared_kernel(CacheAttn a, Deal deal,
                                                                                   float* __restrict__ part_o,
                                                                                   float* __restrict__ part_ml) {
  typedef Tile<uint16_t, DH> X;
  constexpr int TILES = NW / KH, KT = X::KT, SK = 2 * KT;          // keys per stage
  constexpr int CH = DH / 8, OT = DH / 16, KS = DH / 32;
  constexpr int BYTES = SK * DH * 2;                               // a stage of K or of V
  constexpr int LOADS = BYTES / (NW * WAVE * 16);                  // 16-byte loads per thread, stage and operand
  constexpr int OWN = 2 / KH;                                      // steps of a stage per wave
  static_assert((KH - 1) * TILES * (OT * 4 + 2) * WAVE * 4 <= 4 * BYTES, "merge area");
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * BYTES];   // [buffer][K, V]
  extern __shared__ uint16_t chosen[];                             // SPARSE: the blocks that any row chose
  const int h = blockIdx.x % a.Hkv, rg = blockIdx.x / a.Hkv, b = blockIdx.y, sp = blockIdx.z;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  const int l = lane & 15, g = lane >> 4;
  const int tile = wave % TILES, kpart = wave / TILES;
  const int rows = a.nq_max * a.G, live_rows = max(0, min(a.n_q[b], a.nq_max)) * a.G;
  const int r0 = rg * 16 * TILES;
  if (r0 >= live_rows) return;
  const int L = max(0, min(a.kv_len[b], a.kv_cap));
  const int total = min((int64_t)L + max(0, min(a.n_tail[b], ADT_MAX_NODES)), (int64_t)a.kv_cap);
  if (tid == 0 && (int64_t)a.kv_len[b] + a.n_tail[b] > a.kv_cap) dev_fail(DEVINV_KV_RANGE);
  const int64_t pair = (int64_t)b * a.Hkv + h;
  const int per_blk = SPARSE ? a.block / KT : 1;
  const int prefix_steps = SPARSE ? a.lists.count[pair] * per_blk : (L + KT - 1) / KT;
  const int steps = prefix_steps + (total - L + KT - 1) / KT;
  const int splits = deal.splits, n_live = deal.splits_of((steps + 1) / 2);
  if (sp >= n_live) return;
  if (deal.live && sp == 0 && tid == 0) deal.live[(int64_t)b * gridDim.x + blockIdx.x] = n_live;
  const int stages = max(0, ((steps + 1) / 2 - sp + n_live - 1) / n_live);   // of this split: sp, sp + n_live, ...
  const uint32_t* marks = reinterpret_cast<const uint32_t*>(a.lists.marks + pair * a.n_blk * ADT_MASK_WORDS);
  const uint16_t* kb = (const uint16_t*)a.k + b * a.sb + h * a.sh;
  const uint16_t* vb = (const uint16_t*)a.v + b * a.sb + h * a.sh;

  typename X::Query q;
  X::zero(q);
  uint64_t aw0 = 0, aw1 = 0;
  int node = -1;
  const int row = r0 + tile * 16 + l;
  if (row < live_rows) {
    node = row / a.G;
    X::load(q, (const uint16_t*)a.q + (((int64_t)b * a.nq_max + node) * a.Hkv + h) * a.G * DH + (int64_t)(row - node * a.G) * DH, g);
    const uint64_t* mp = a.mask + ((int64_t)b * a.nq_max + node) * ADT_MASK_WORDS;
    aw0 = mp[0];
    aw1 = mp[1];
  }
  if (SPARSE) copy_list(a.lists.blocks + pair * a.n_blk, a.lists.count[pair], chosen);
  const bool tile_live = r0 + tile * 16 < live_rows;
  const float scale_log2 = a.scale * LOG2E;

  // Stage i's two steps: their blocks in the list (read a stage ahead of their use, as stages are
  // fetched in order), first keys and last ones (a step past the end has none: last < key0).
  int block_of[2] = {0, 0};
  auto look_up = [&](int i) {
    if (!SPARSE) return;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int s = 2 * (sp + n_live * i) + w;
      block_of[w] = s < prefix_steps ? (int)chosen[s / per_blk] : 0;
    }
  };
  struct Span {
    int key0, last;
  };
  auto span = [&](int s, int j) {
    if (s >= steps) return Span{0, -1};
    if (s >= prefix_steps) return Span{L + (s - prefix_steps) * KT, total - 1};
    if (SPARSE) {
      const int blk = __builtin_amdgcn_readfirstlane(j);
      return Span{blk * a.block + s % per_blk * KT, min(L, (blk + 1) * a.block) - 1};
    }
    return Span{s * KT, L - 1};
  };
  // Slot x (16 bytes) of a stage holds row x / CH, chunk (x % CH) ^ swizzle(row); thread t fills slots
  // r * NW * 64 + t.  Rows past a step's last key repeat it.  Requests are never skipped (a stage past
  // the range reads the head's first row), so the count of loads in flight is the same on every path.
  u16x8 kr[P][LOADS], vr[P][LOADS];
  Span sp0[P], sp1[P];
  uint32_t mk[P][OWN] = {};       // of the blocks' marks, the word with this lane's row
  auto fetch = [&](int u, int i) {
    const int s0 = 2 * (sp + n_live * i);
    sp0[u] = span(i < stages ? s0 : steps, block_of[0]);
    sp1[u] = span(i < stages ? s0 + 1 : steps, block_of[1]);
    look_up(i + 1);
#pragma unroll
    for (int r = 0; r < LOADS; ++r) {
      const int slot = r * NW * WAVE + tid, x = slot / CH, phys = slot % CH;
      const int half = x / KT;
      const int key = max(0, min((half ? sp1[u].key0 : sp0[u].key0) + x % KT, half ? sp1[u].last : sp0[u].last));
      kr[u][r] = load16<false>(      // (kept in the caches: the slots' weights take the keys once more)
          reinterpret_cast<const u16x8*>(kb + (int64_t)key * DH + (phys ^ swz_k<DH>(x)) * 8));
      vr[u][r] = __builtin_nontemporal_load(
          reinterpret_cast<const u16x8*>(vb + (int64_t)key * DH + (phys ^ swz_v<DH>(x)) * 8));
    }
    if (SPARSE) {
#pragma unroll
      for (int w = 0; w < OWN; ++w) {
        const int s = min(s0 + (KH == 2 ? kpart : w), max(prefix_steps - 1, 0));
        const int at = i < stages ? s / per_blk : 0;
        mk[u][w] = prefix_steps > 0 ? marks[4 * at + (max(node, 0) >> 5)] : 0;
      }
    }
  };
  auto store = [&](int u, int buf) {
    unsigned char* at = smem + buf * 2 * BYTES;
#pragma unroll
    for (int r = 0; r < LOADS; ++r) {
      const int slot = r * NW * WAVE + tid;
      *reinterpret_cast<u16x8*>(at + slot * 16) = kr[u][r];
      *reinterpret_cast<u16x8*>(at + BYTES + slot * 16) = vr[u][r];
    }
  };

  f32x4 o[OT];
  float m_run, l_run;             // running maximum (log2 domain), this lane's share of the sum
  // this wave's steps of stage i, whose blocks the rows of `m` chose
  auto compute = [&](auto safe_tag, int i, const Span& span0, const Span& span1, const uint32_t (&m)[OWN]) {
    constexpr bool SAFE = decltype(safe_tag)::value;
    const unsigned char* ks = smem + (i & 1) * 2 * BYTES;
    const unsigned char* vs = ks + BYTES;
#pragma unroll
    for (int w = 0; w < OWN; ++w) {
      const int half = KH == 2 ? kpart : w, s = 2 * (sp + n_live * i) + half;
      if (s >= steps) continue;
      const int k0 = half ? span1.key0 : span0.key0, k_last = half ? span1.last : span0.last;
      const bool tail = s >= prefix_steps;
      const bool sees = node >= 0 && (tail || !SPARSE || (m[w] >> (node & 31) & 1));
      if (SPARSE && !__any(sees)) continue;
      f32x4 st[2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        st[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int x = half * KT + sub * 16 + l;
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          const bf16x8 f = *reinterpret_cast<const bf16x8*>(ks + x * DH * 2 + ((j * 4 + g) ^ swz_k<DH>(x)) * 16);
          st[sub] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q.f[j], st[sub], 0, 0, 0);
        }
      }
      auto seen = [&](int key) {
        const int j = k0 + key - L;
        return sees & (k0 + key <= k_last) & (!tail | (bool)((j < 64 ? aw0 : aw1) >> (j & 63) & 1));
      };
      float mx = -INFINITY;
      if (!tail && k0 + KT - 1 <= k_last) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (SPARSE) st[e / 4][e % 4] = sees ? st[e / 4][e % 4] : -INFINITY;
          mx = fmaxf(mx, st[e / 4][e % 4]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = seen(e / 4 * 16 + 4 * g + e % 4) ? st[e / 4][e % 4] : -INFINITY;
          st[e / 4][e % 4] = v;
          mx = fmaxf(mx, v);
        }
      }
      mx = xor16_max(mx);
      mx = xor32_max(mx);
      const float m_new = fmaxf(m_run, mx * scale_log2);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;     // nothing seen yet: weights 0, not NaN
      const float alpha = m_new == m_run ? 1.f : exp2_hw(m_run - m_use);
      m_run = m_new;
      float rs = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = exp2_hw(fmaf(st[e / 4][e % 4], scale_log2, -m_use));
        st[e / 4][e % 4] = p;
        rs += p;
      }
      l_run = l_run * alpha + rs;
      if (!__all(alpha == 1.f)) {
#pragma unroll
        for (int d = 0; d < OT; ++d) o[d] *= alpha;
      }
      bf16x8 pb;
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[e] = (__bf16)st[e / 4][e % 4];
      const int lo_x = half * KT + 4 * g + (l >> 2), hi_x = lo_x + 16;
#pragma unroll
      for (int d = 0; d < OT; ++d) {
        const int c = 2 * d + ((l & 3) >> 1), part = l & 1;
        v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_v4i16*)(vs + lo_x * DH * 2 + ((c ^ swz_v<DH>(lo_x)) * 16) + part * 8));
        v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_v4i16*)(vs + hi_x * DH * 2 + ((c ^ swz_v<DH>(hi_x)) * 16) + part * 8));
        if (SAFE) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if ((lo[e] & 0x7f80) == 0x7f80) lo[e] = 0;
            if ((hi[e] & 0x7f80) == 0x7f80) hi[e] = 0;
          }
        }
        const bf16x8 f = __builtin_bit_cast(bf16x8, v8i16{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, pb, o[d], 0, 0, 0);
      }
      if (SAFE) add_not_finite<X>(o, st, vb, k0, k_last, l, g, seen);
    }
  };
  auto pass = [&](auto safe_tag) {
    m_run = -INFINITY;
    l_run = 0.f;
#pragma unroll
    for (int d = 0; d < OT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
    look_up(0);
    // (the stages are requested in order: the scheduler may not interleave them, or the first one
    // stored could be the last to arrive)
#pragma unroll
    for (int u = 0; u < P; ++u) {
      fetch(u, u);
      __builtin_amdgcn_sched_barrier(0);
    }
    for (int base = 0; base < stages; base += P) {
#pragma unroll
      for (int u = 0; u < P; ++u) {
        const int i = base + u;
        uint32_t m[OWN];
        const Span span0 = sp0[u], span1 = sp1[u];
#pragma unroll
        for (int w = 0; w < OWN; ++w) m[w] = mk[u][w];
        // the buffer written here was last read two stages ago, before the previous barrier
        store(u, i & 1);
        __syncthreads();
        fetch(u, i + P);
        if (tile_live && i < stages) compute(safe_tag, i, span0, span1, m);
      }
    }
  };
  pass(std::false_type{});
  float odd = 0.f;
#pragma unroll
  for (int d = 0; d < OT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r) odd += o[d][r] * 0.f;
  if (__syncthreads_or(odd != odd)) pass(std::true_type{});

  l_run = xor16_add(l_run);
  l_run = xor32_add(l_run);
  if constexpr (KH > 1) {
    // the second part of a tile passes its state through LDS to the first
    float* mo = reinterpret_cast<float*>(smem) + (size_t)tile * (OT * 4 + 2) * WAVE;
    __syncthreads();
    if (kpart == 1) {
#pragma unroll
      for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) mo[(d * 4 + r) * WAVE + lane] = o[d][r];
      mo[OT * 4 * WAVE + lane] = m_run;
      mo[(OT * 4 + 1) * WAVE + lane] = l_run;
    }
    __syncthreads();
    if (kpart == 0) {
      const float m1 = mo[OT * 4 * WAVE + lane], l1 = mo[(OT * 4 + 1) * WAVE + lane];
      const float M = fmaxf(m_run, m1), Mu = M == -INFINITY ? 0.f : M;
      const float w0 = m_run == -INFINITY && l_run == 0.f ? 0.f : exp2_hw(m_run - Mu);
      const float w1 = m1 == -INFINITY && l1 == 0.f ? 0.f : exp2_hw(m1 - Mu);
#pragma unroll
      for (int d = 0; d < OT; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = mo[(d * 4 + r) * WAVE + lane];
          o[d][r] = (w0 == 0.f ? 0.f : o[d][r] * w0) + (w1 == 0.f ? 0.f : x * w1);
        }
      l_run = (w0 == 0.f && l_run == l_run ? 0.f : l_run * w0) + (w1 == 0.f && l1 == l1 ? 0.f : l1 * w1);
      m_run = M;
    }
  }
  if (kpart == 0 && node >= 0) {
    const int64_t at = (pair * splits + sp) * rows + row;
    if (n_live == 1) {
      const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
      uint16_t* to = (uint16_t*)a.out + (((int64_t)b * a.nq_max + node) * a.Hkv + h) * a.G * DH + (int64_t)(row - node * a.G) * DH;
#pragma unroll
      for (int d = 0; d < OT; ++d) store4(to + d * 16 + 4 * g, o[d][0] * inv, o[d][1] * inv, o[d][2] * inv, o[d][3] * inv);
    } else {
#pragma unroll
      for (int d = 0; d < OT; ++d) *reinterpret_cast<f32x4*>(part_o + at * DH + d * 16 + 4 * g) = o[d];
    }
    if (part_ml && g == 0) {
      part_ml[at * 2] = m_run;
      part_ml[at * 2 + 1] = l_run;
    }
  }
}

// Log-sum-exp merge of the splits: DH / 4 threads take four dims each of one row, and `count` groups of
// them deal out the row's splits, up to eight requested at a time; the groups' sums meet in LDS, in
// their order.  A workgroup takes as many rows as fit it, from row r0 on.  row_ml (if given) gets the
// rows' maxima and sums.
struct MergeScratch {
  f32x4 acc[CA_THREADS];
  float2 ml[CA_THREADS];
};
__device__ __forceinline__ void merge_rows(const CacheAttn& a, const Deal& deal, int group_rows, bool bf16, int r0,
                                           int count, int h, int b, const float* part_o, const float* part_ml,
                                           float* row_ml, MergeScratch& sh) {
  const int per = a.Dh / 4, unit = threadIdx.x / per, grp = unit % count, d = threadIdx.x % per * 4;
  const int live = max(0, min(a.n_q[b], a.nq_max)) * a.G;
  if (r0 >= live) return;
  const int rr = r0 + unit / count;
  const int rows = a.nq_max * a.G, groups = (rows + group_rows - 1) / group_rows;
  const int64_t pair = (int64_t)b * a.Hkv + h, base = pair * deal.splits * rows + rr;
  const int splits = rr < live ? deal.live_splits(((int64_t)b * groups + rr / group_rows) * a.Hkv + h) : 0;
  // (one split has written the output; its maximum and sum are the only ones)
  if (splits == 1 && row_ml && grp == 0 && d == 0) {
    row_ml[(pair * rows + rr) * 2] = part_ml[base * 2];
    row_ml[(pair * rows + rr) * 2 + 1] = part_ml[base * 2 + 1];
  }
  RunningMerge acc;
  for (int s0 = splits > 1 ? grp : splits; s0 < splits; s0 += 8 * count) {
    float2 ml[8];
    f32x4 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t at = base + (int64_t)min(s0 + j * count, splits - 1) * rows;
      ml[j] = *reinterpret_cast<const float2*>(part_ml + at * 2);
      x[j] = *reinterpret_cast<const f32x4*>(part_o + at * a.Dh + d);
    }
    acc.add(ml, x, splits - s0, count);
  }
  if (count > 1) {
    sh.acc[threadIdx.x] = acc.o;
    sh.ml[threadIdx.x] = make_float2(acc.m, acc.l);
    __syncthreads();
    if (grp > 0) return;
    const int n = min(count, splits);
    for (int g = 1; g < n; ++g) acc.m = fmaxf(acc.m, sh.ml[threadIdx.x + g * per].x);
    const float top = acc.m == -INFINITY ? 0.f : acc.m;
    acc.l = 0.f;
    acc.o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int g = 0; g < n; ++g) {
      const float2 ml = sh.ml[threadIdx.x + g * per];
      acc.add_one(ml.x, ml.y, sh.acc[threadIdx.x + g * per], top);
    }
  }
  if (splits <= 1) return;
  const float inv = acc.l == 0.f ? 0.f : 1.f / acc.l;
  const int64_t at_o = (((int64_t)b * a.nq_max + rr / a.G) * a.Hkv + h) * a.G * a.Dh + (int64_t)(rr % a.G) * a.Dh + d;
  if (bf16) store4((uint16_t*)a.out + at_o, acc.o[0] * inv, acc.o[1] * inv, acc.o[2] * inv, acc.o[3] * inv);
  else store4((float*)a.out + at_o, acc.o[0] * inv, acc.o[1] * inv, acc.o[2] * inv, acc.o[3] * inv);
  if (row_ml && d == 0) {
    row_ml[(pair * rows + rr) * 2] = acc.m;
    row_ml[(pair * rows + rr) * 2 + 1] = acc.l;
  }
}

__global__ __launch_bounds__(CA_THREADS) void cache_merge_kernel(CacheAttn a, Deal deal, int group_rows, int count,
                                                                 int is_bf16,
                                                                 const float* __restrict__ part_o,
                                                                 const float* __restrict__ part_ml,
                                                                 float* __restrict__ row_ml) {
  __shared__ MergeScratch sh;
  merge_rows(a, deal, group_rows, is_bf16, blockIdx.x * (CA_THREADS / (a.Dh / 4) / count), count, blockIdx.y, blockIdx.z,
             part_o, part_ml, row_ml, sh);
}

// Where the weights of the slots go.
struct SlotWeights {
  const float* in;
  float* out;
  int64_t stride_b, stride_h;
  float decay;
  const float* row_weight;
  __device__ __forceinline__ float rating(int b, int nq_max, int node) const {
    return row_weight ? row_weight[(int64_t)b * nq_max + node] : 1.f;
  }
  // the earlier weight of a slot (0: none), and its new one
  __device__ __forceinline__ float before(int b, int h, int key, int L) const {
    return key < L && in ? in[b * stride_b + h * stride_h + key] : 0.f;
  }
  __device__ __forceinline__ void store(int b, int h, int key, int L, float was, float sum) const {
    out[b * stride_b + h * stride_h + key] = key < L && in ? decay * was + sum : sum;
  }
};

// A row's maximum and its weight over its sum, what a slot's weight takes of it; a row that saw
// nothing adds 2^(-inf - inf) * 0.
__device__ __forceinline__ float2 row_factor(float m, float sum, float rating) {
  if (sum == 0.f) return make_float2(INFINITY, 0.f);
  return make_float2(m == -INFINITY ? 0.f : m, rating / sum);
}

// The weight every slot received: S[row][key] once more, now with the rows' final maximum and sum,
// p = 2^(s - m) / l, added over the rows.  A wave takes CHUNK keys at a time, keeps them in registers,
// the next ones requested meanwhile, and goes through the query rows tile by tile (A = Q rows, B =
// K^T: lane (l, g) gets rows 4 g + r of key l, so a column adds up within its lanes).  The queries of
// up to QROWS rows lie in LDS; more are read from the L2 again for every chunk.  Few keys under many
// rows: the waves of a workgroup take the same 32 keys and deal the row tiles out.  Bound by the second
// read of K: sixteen trees of up to 61 rows of 32 heads 48 us, 4.1 TB/s.
constexpr int SW_CHUNK = 32;        // keys per wave and turn
template <typename T, int DH>
struct SlotTile {
  static constexpr int PITCH = DH + 16 / (int)sizeof(T);                              // a query row in LDS
  static constexpr int QROWS = 128 * 256 / (DH * (int)sizeof(T)) < 128 ? 64 : 128;
};

enum class Rows { LDS, L2, DEALT };

template <typename T, int DH, Rows HOW>
__global__ __launch_bounds__(CA_THREADS, sizeof(T) == 2 ? 4 : 2) void slot_weights_kernel(
    CacheAttn a, const float* __restrict__ row_ml, int turns, SlotWeights sw) {
  typedef Tile<T, DH> X;
  constexpr int STEPS = SW_CHUNK / X::KT, SUBS = SW_CHUNK / 16, PITCH = SlotTile<T, DH>::PITCH, V = 16 / sizeof(T);
  extern __shared__ __attribute__((aligned(16))) unsigned char rows_lds[];   // factors, then the queries
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  const int L = max(0, min(a.kv_len[b], a.kv_cap));
  const int total = min((int64_t)L + max(0, min(a.n_tail[b], ADT_MAX_NODES)), (int64_t)a.kv_cap);
  constexpr bool QLDS = HOW == Rows::LDS, DEALT = HOW == Rows::DEALT;
  const int first = blockIdx.x * (DEALT ? SW_CHUNK : turns * CA_WAVES * SW_CHUNK);
  if (first >= total) return;
  const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE), lane = tid % WAVE;
  const int l = lane & 15, g = lane >> 4;
  const int live_rows = max(0, min(a.n_q[b], a.nq_max)) * a.G, tiles = (live_rows + 15) / 16;
  const int64_t pair = (int64_t)b * a.Hkv + h;
  const T* kb = (const T*)a.k + b * a.sb + h * a.sh;
  typename X::Step step[2][STEPS];
  auto request = [&](int u, int k0) {
#pragma unroll
    for (int i = 0; i < STEPS; ++i) X::template load_k<false>(step[u][i], kb, min(k0, total - 1) + i * X::KT, total - 1, l, g);
  };
  request(0, DEALT ? first : first + wave * SW_CHUNK);
  float2* factor = reinterpret_cast<float2*>(rows_lds);
  T* qs = reinterpret_cast<T*>(factor + tiles * 16);
  auto q_row = [&](int r) {
    const int i = r / a.G;
    return (const T*)a.q + (((int64_t)b * a.nq_max + i) * a.Hkv + h) * a.G * DH + (int64_t)(r - i * a.G) * DH;
  };
  for (int r = tid; r < tiles * 16; r += CA_THREADS) {
    float2 f = make_float2(INFINITY, 0.f);
    if (r < live_rows) {
      const float* ml = row_ml + (pair * a.nq_max * a.G + r) * 2;
      f = row_factor(ml[0], ml[1], sw.rating(b, a.nq_max, r / a.G));
    }
    factor[r] = f;
  }
  if (QLDS) {
    for (int x = tid; x < tiles * 16 * (DH / V); x += CA_THREADS) {
      const int r = x / (DH / V), c = x % (DH / V) * V;
      *reinterpret_cast<u16x8*>(qs + r * PITCH + c) = *reinterpret_cast<const u16x8*>(q_row(min(r, live_rows - 1)) + c);
    }
  }
  __syncthreads();
  const float scale_log2 = a.scale * LOG2E;
  // (a turn's earlier weights are requested before the next turn's keys: loads return in order, and
  // asked for last they would have every turn wait for the keys of the next)
  auto sum = [&](float (&col)[SUBS], int u, int key0, int tile0, int tile_step) {
    const bool tail = key0 + SW_CHUNK > L;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) col[s] = 0.f;
    // masked: some row of the tile is none, or some key is the tree's
    auto tile = [&](auto masked_tag, int t) {
      constexpr bool MASKED = decltype(masked_tag)::value;
      typename X::Query q;
      X::load(q, QLDS ? qs + (t * 16 + l) * PITCH : q_row(min(t * 16 + l, live_rows - 1)), g);
      float2 f[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] = factor[t * 16 + 4 * g + r];
      f32x4 st[SUBS];
#pragma unroll
      for (int s = 0; s < SUBS; ++s) {
        st[s] = f32x4{0.f, 0.f, 0.f, 0.f};
        X::col_scores(st[s], step[u][s / X::SUBS], s % X::SUBS, q);
      }
#pragma unroll
      for (int s = 0; s < SUBS; ++s)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = exp2_hw(fmaf(st[s][r], scale_log2, -f[r].x)) * f[r].y;
          if (MASKED) {
            const int row = t * 16 + 4 * g + r, j = key0 + s * 16 + l - L;
            bool vis = row < live_rows;
            if (vis && j >= 0) {
              const uint64_t* mp = a.mask + ((int64_t)b * a.nq_max + row / a.G) * ADT_MASK_WORDS;
              vis = j < ADT_MAX_NODES && (mp[j >> 6] >> (j & 63) & 1);
            }
            col[s] += vis ? p : 0.f;
          } else {
            col[s] += p;
          }
        }
    };
    for (int t = tile0; t < tiles; t += tile_step) {
      if (tail || t * 16 + 16 > live_rows) tile(std::true_type{}, t);
      else tile(std::false_type{}, t);
    }
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      col[s] = xor16_add(col[s]);
      col[s] = xor32_add(col[s]);
    }
  };
  auto turn = [&](int u, int key0, const float (&was)[SUBS]) {
    float col[SUBS];
    sum(col, u, key0, 0, 1);
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      const int key = key0 + s * 16 + l;
      if (g == s && key < total) sw.store(b, h, key, L, was[s], col[s]);
    }
  };
  auto earlier = [&](float (&was)[SUBS], int key0) {
#pragma unroll
    for (int s = 0; s < SUBS; ++s) was[s] = sw.before(b, h, key0 + s * 16 + l, L);
  };
  if constexpr (DEALT) {
    __shared__ float part[CA_WAVES][SW_CHUNK];
    float col[SUBS];
    sum(col, 0, first, wave, CA_WAVES);
#pragma unroll
    for (int s = 0; s < SUBS; ++s)
      if (g == s) part[wave][s * 16 + l] = col[s];
    __syncthreads();
    const int key = first + tid;
    if (tid >= SW_CHUNK || key >= total) return;
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < CA_WAVES; ++w) all += part[w][tid];
    sw.store(b, h, key, L, sw.before(b, h, key, L), all);
  } else {
    const int stride = CA_WAVES * SW_CHUNK;
    int key0 = first + wave * SW_CHUNK;
    for (int c = 0; c < turns && key0 < total; c += 2, key0 += 2 * stride) {
      float was[SUBS];
      earlier(was, key0);
      if (c + 1 < turns) request(1, key0 + stride);
      turn(0, key0, was);
      if (c + 1 >= turns || key0 + stride >= total) break;
      earlier(was, key0 + stride);
      if (c + 2 < turns) request(0, key0 + 2 * stride);
      turn(1, key0 + stride, was);
    }
  }
}

// The same where the attention kept its masked scores (kept [B][Hkv][rows][kv_cap] fp32: few rows), and
// the merge of its splits in the same launch: the first `merges` workgroups of a pair merge a row each,
// the others take ST_KEYS keys, for which they merge the rows' maxima and sums themselves.
constexpr int ST_KEYS = 4 * CA_THREADS, ST_ROWS = 16;
__global__ __launch_bounds__(CA_THREADS) void slot_weights_kept_kernel(CacheAttn a, Deal deal, int is_bf16, int merges,
                                                                       const float* __restrict__ kept,
                                                                       const float* __restrict__ part_o,
                                                                       const float* __restrict__ part_ml,
                                                                       SlotWeights sw) {
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  __shared__ MergeScratch sh;
  if ((int)blockIdx.x < merges) {
    merge_rows(a, deal, ST_ROWS, is_bf16, blockIdx.x, CA_THREADS / (a.Dh / 4), h, b, part_o, part_ml, nullptr, sh);
    return;
  }
  const int L = max(0, min(a.kv_len[b], a.kv_cap));
  const int total = min((int64_t)L + max(0, min(a.n_tail[b], ADT_MAX_NODES)), (int64_t)a.kv_cap);
  const int key0 = (blockIdx.x - merges) * ST_KEYS + tid;
  if (key0 - tid >= total) return;
  __shared__ float2 factor[ST_ROWS];
  const int rows = a.nq_max * a.G, live_rows = max(0, min(a.n_q[b], a.nq_max)) * a.G;
  const int64_t pair = (int64_t)b * a.Hkv + h;
  {
    // row r's splits by the 16 lanes 16 r .. 16 r + 15
    const int r = tid / 16;
    float m = -INFINITY, ls = 0.f;
    if (r < live_rows) {
      const int splits = deal.live ? deal.live_splits((int64_t)b * a.Hkv + h) : 1;
      const float* ml = part_ml + (pair * deal.splits * rows + r) * 2;
      for (int s = tid % 16; s < splits; s += 16) m = fmaxf(m, ml[(int64_t)s * rows * 2]);
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, WAVE));
      for (int s = tid % 16; s < splits; s += 16) {
        const float ms = ml[(int64_t)s * rows * 2], l = ml[(int64_t)s * rows * 2 + 1];
        if (ms != -INFINITY || l != 0.f) ls += l * exp2_hw(ms - (m == -INFINITY ? 0.f : m));
      }
#pragma unroll
      for (int o = 1; o < 16; o <<= 1) ls += __shfl_xor(ls, o, WAVE);
    }
    if (tid % 16 == 0) factor[r] = r < live_rows ? row_factor(m, ls, sw.rating(b, a.nq_max, r / a.G)) : make_float2(INFINITY, 0.f);
  }
  __syncthreads();
  const float scale_log2 = a.scale * LOG2E;
  const float* s0 = kept + pair * rows * a.kv_cap;
  float sum[ST_KEYS / CA_THREADS] = {}, was[ST_KEYS / CA_THREADS];
#pragma unroll
  for (int j = 0; j < ST_KEYS / CA_THREADS; ++j) was[j] = sw.before(b, h, key0 + j * CA_THREADS, L);
  for (int r = 0; r < live_rows; r += 4) {
    float x[4][ST_KEYS / CA_THREADS];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < ST_KEYS / CA_THREADS; ++j)
        x[u][j] = s0[(int64_t)min(r + u, live_rows - 1) * a.kv_cap + min(key0 + j * CA_THREADS, total - 1)];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (r + u >= live_rows) continue;
      const float2 f = factor[r + u];
#pragma unroll
      for (int j = 0; j < ST_KEYS / CA_THREADS; ++j) {
        // (a masked score is -inf and stays 0 whatever the row's factor: not NaN for a row that is)
        const float p = exp2_hw(fmaf(x[u][j], scale_log2, -f.x)) * f.y;
        sum[j] += x[u][j] == -INFINITY ? 0.f : p;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < ST_KEYS / CA_THREADS; ++j)
    if (key0 + j * CA_THREADS < total) sw.store(b, h, key0 + j * CA_THREADS, L, was[j], sum[j]);
}

// ----------------------------------------------------------------------------- host
static size_t align_up16(size_t x) { return (x + 15) / 16 * 16; }

// How a launch covers its rows and keys.
struct CachePlan {
  bool shared;      // the waves of a workgroup share the keys (bf16, more than 16 rows)
  int tiles;        // row tiles per workgroup
  int groups;       // workgroups side by side for the rows of one key-value head
  int splits, per;  // most splits of the keys; steps (stages where shared) per split
  int likely;       // splits of the keys that the launch expects
  int deep;         // stages in flight (shared)
};
// Splits: as many as give the workgroups that the CUs hold at once (`slots`) equal shares of the keys
// the launch expects: the slots of the cache, or n_sel blocks, and for the rows of a tree half as many
// again.  That half is a number that measured well, no estimate of the union of the rows' blocks, which
// is larger and not known here (sixteen sequences of 16 rows taking 48 blocks each, 110 in all: 13 stages
// a split 108 us, 18 98, 24 107; once, twice, two and a half times n_sel instead, whole calls over 31 blocks
// of 64 slots of 8 key-value heads: sixteen sequences of 5 rows 82, 84, 68 us against 76, of 16 rows 126,
// 111, 114 against 120, four of 16 rows 52, 51, 59 against 52, of 61 rows 178, 153, 144 against 159; one
// sequence within 2.2 us).  Sequences that have more take more splits.  At
// least three stages, or two steps for each wave, pay for a split's start and its partial results; in
// fp32, whose products take longer and whose next step waits for them, one step does (17 rows over 300
// slots 8.7 -> 6.8 us, over 16 of 141 blocks 45 -> 39 in all; bf16, one row over 32 of 511 blocks, 10.3
// with two and 10.5 with one).  Where there is little work for workgroups that share their keys (under
// eight stages a CU), one to a CU is all they get, and those of 128 rows, whose waves take both steps of
// a stage, keep three stages in flight in place of one (244 rows of 8 heads over 16 of 141 blocks 55 us,
// 62 with one; 61 rows of 32 heads over 24 of 74 blocks 37.4 with one, 38.7 with three, in all).
static CachePlan cache_plan(const CacheAttn& a, int B, int dtype) {
  const int rows = a.nq_max * a.G;
  CachePlan p;
  p.shared = dtype == ADT_BF16 && rows > 16;
  p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 || !p.shared ? 4 : 8;
  p.groups = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
  const int unit = p.shared ? 64 : dtype == ADT_BF16 ? 32 : 16;
  const int least = p.shared ? 3 : dtype == ADT_BF16 ? 2 * CA_WAVES : CA_WAVES;
  int64_t most = a.kv_cap, expect = most;      // keys
  if (a.block) {
    most = std::min<int64_t>(most, (int64_t)a.n_sel * a.nq_max * a.block + ADT_MAX_NODES);
    expect = std::min<int64_t>(expect, (int64_t)a.n_sel * a.block * (a.nq_max > 1 ? 3 : 2) / 2 + a.nq_max);
  }
  most = (most + unit - 1) / unit + 1;
  expect = (expect + unit - 1) / unit;
  const int64_t pairs = (int64_t)B * a.Hkv * p.groups;
  const bool little = p.shared && pairs * expect < 8 * 256;
  p.deep = little && p.tiles == 8 ? 3 : 1;
  const int slots = p.shared ? (p.deep > 1 ? 256 : 512) : p.tiles == 1 ? 768 : p.tiles == 2 ? 512 : 256;
  p.per = (int)std::max<int64_t>(least, (pairs * expect + slots - 1) / slots);
  // (a few units more than one share are no reason for partial results and their merge)
  int64_t splits = most <= p.per + p.per / 4 ? 1 : (most + p.per - 1) / p.per;
  splits = std::min<int64_t>(splits, std::max<int64_t>(1, (little ? 256 : 4 * slots) / pairs));
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(splits, 64));
  p.likely = (int)std::min<int64_t>(p.splits, (expect + p.per - 1) / p.per);
  return p;
}

// Partial results of a plan with splits, in floats: outputs, maxima and sums, numbers of splits.
static size_t part_floats(const CacheAttn& a, int B, const CachePlan& p) {
  if (p.splits == 1) return 0;
  return (size_t)B * a.Hkv * ((size_t)p.splits * a.nq_max * a.G * (a.Dh + 2) + p.groups);
}

template <typename T, int DH, bool SPARSE>
static void attn_launch(const CacheAttn& a, int B, const CachePlan& p, const Deal& deal, float* part_o, float* part_ml,
                        float* kept, hipStream_t st) {
  const size_t list = SPARSE ? align_up16((size_t)a.n_blk * 2) : 0;
  const dim3 grid(a.Hkv * p.groups, B, p.splits);
#define ADT_CA(RT) cache_attn_kernel<T, DH, RT, SPARSE><<<grid, CA_THREADS, list, st>>>(a, deal, part_o, part_ml, kept)
#define ADT_CS(NW, KH, P) \
  cache_attn_shared_kernel<DH, NW, KH, P, SPARSE><<<grid, NW * WAVE, list, st>>>(a, deal, part_o, part_ml)
  if constexpr (sizeof(T) == 2) {
    if (p.shared) {
      if (p.tiles == 2) ADT_CS(4, 2, 1);
      else if (p.tiles == 4) ADT_CS(8, 2, 1);
      else if (p.deep > 1) ADT_CS(8, 1, 3);
      else ADT_CS(8, 1, 1);
    } else {
      ADT_CA(1);
    }
  } else {
    if (p.tiles == 1) ADT_CA(1);
    else if (p.tiles == 2) ADT_CA(2);
    else ADT_CA(4);
  }
#undef ADT_CS
#undef ADT_CA
}

// The attention's partial results in `part` (part_floats); one split leaves its rows' maxima and sums in
// row_ml ([B][Hkv][rows][2], may be null).
struct Partials {
  float *o, *ml;
  Deal deal;
};
static Partials partials(const CacheAttn& a, int B, const CachePlan& p, float* part, float* row_ml) {
  if (p.splits == 1) return Partials{nullptr, row_ml, Deal{1, p.per, nullptr}};
  const size_t rows = (size_t)B * a.Hkv * p.splits * a.nq_max * a.G;
  float* ml = part + rows * a.Dh;
  return Partials{part, ml, Deal{p.splits, p.per, (int32_t*)(ml + rows * 2)}};
}

static adt_status attn_launches(const CacheAttn& a, int B, const CachePlan& p, const Partials& w, float* kept, int dtype,
                                hipStream_t st) {
#define ADT_AL(TV, DHV)                                                                  \
  if (a.block) attn_launch<TV, DHV, true>(a, B, p, w.deal, w.o, w.ml, kept, st);         \
  else attn_launch<TV, DHV, false>(a, B, p, w.deal, w.o, w.ml, kept, st)
  if (dtype == ADT_BF16) {
    if (a.Dh == 128) { ADT_AL(uint16_t, 128); }
    else { ADT_AL(uint16_t, 64); }
  } else {
    if (a.Dh == 128) { ADT_AL(float, 128); }
    else { ADT_AL(float, 64); }
  }
#undef ADT_AL
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

static adt_status merge_launch(const CacheAttn& a, int B, const CachePlan& p, const Partials& w, float* row_ml, int dtype,
                               hipStream_t st) {
  if (p.splits == 1) return ADT_OK;
  // a thread for every four outputs, or for few outputs and many splits several (61 rows of 8 heads in
  // 14 splits, 64 at most: 8.8 us with eight threads, 4.4 with one)
  const int rows = a.nq_max * a.G, fit = CA_THREADS / (a.Dh / 4);
  const int count = p.likely > 16 && (int64_t)B * a.Hkv * rows * (a.Dh / 4) < 65536 ? fit : 1;
  cache_merge_kernel<<<dim3((rows * count + fit - 1) / fit, a.Hkv, B), CA_THREADS, 0, st>>>(
      a, w.deal, 16 * p.tiles, count, dtype == ADT_BF16, w.o, w.ml, row_ml);
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

// Workspace of attention over chosen blocks: the selection's scratch, the lists, partial results.
struct SparseWs {
  size_t marks, blocks, count, arrived, part, bytes;
};
static SparseWs sparse_ws(const CacheAttn& a, int B, const CachePlan& p) {
  const size_t pairs = (size_t)B * a.Hkv;
  SparseWs w;
  w.marks = align_up16(block_select_ws_bytes(B, a.Hkv, a.nq_max, a.n_blk));
  w.blocks = w.marks + pairs * a.n_blk * ADT_MASK_WORDS * sizeof(uint64_t);
  w.count = align_up16(w.blocks + pairs * a.n_blk * sizeof(uint16_t));
  w.arrived = w.count + pairs * sizeof(int32_t);
  w.part = align_up16(w.arrived + pairs * sizeof(uint32_t));
  w.bytes = w.part + part_floats(a, B, p) * sizeof(float);
  return w;
}

size_t sparse_attn_ws_bytes(const CacheAttn& a, int B, int dtype) {
  return sparse_ws(a, B, cache_plan(a, B, dtype)).bytes;
}

adt_status launch_sparse_attn(CacheAttn a, int B, const float* means, int64_t mb, int64_t mh, int n_first, int n_last,
                              int32_t* sel, int dtype, void* ws, hipStream_t st) {
  const CachePlan p = cache_plan(a, B, dtype);
  const SparseWs w = sparse_ws(a, B, p);
  char* base = (char*)ws;
  a.lists = BlockLists{(int32_t*)(base + w.count), (uint16_t*)(base + w.blocks), (uint64_t*)(base + w.marks),
                       (uint32_t*)(base + w.arrived)};
  adt_status e = launch_block_select(a.q, means, mb, mh, a.kv_len, a.n_q, B, a.Hkv, a.G, a.Dh, a.nq_max, a.kv_cap,
                                     a.block, a.n_sel, n_first, n_last, dtype, ws, a.lists, sel, st);
  if (e) return e;
  const Partials parts = partials(a, B, p, (float*)(base + w.part), nullptr);
  e = attn_launches(a, B, p, parts, nullptr, dtype, st);
  return e || p.tiles == 1 ? e : merge_launch(a, B, p, parts, nullptr, dtype, st);
}

// Workspace of attention that rates its slots: the rows' maxima and sums, the scores where they are
// kept, partial results.  Scores are kept, instead of computed again from the keys, where they take
// at most an eighth of the keys' bytes (written and read, a quarter of reading the keys again: one row
// of four heads over 65333 slots of 8 key-value heads, 32.7 us -> 6.7 for the slots' weights and the merge).
struct WeightsWs {
  bool keep;
  size_t kept, part, bytes;
};
static WeightsWs weights_ws(const CacheAttn& a, int B, const CachePlan& p, int dtype) {
  const int rows = a.nq_max * a.G, es = dtype == ADT_BF16 ? 2 : 4;
  const size_t pairs = (size_t)B * a.Hkv;
  WeightsWs w;
  w.keep = rows <= ST_ROWS && rows * 4 * 8 <= a.Dh * es;
  w.kept = align_up16(pairs * rows * 2 * sizeof(float));
  w.part = w.kept + (w.keep ? align_up16(pairs * rows * a.kv_cap * sizeof(float)) : 0);
  w.bytes = w.part + part_floats(a, B, p) * sizeof(float);
  return w;
}

size_t weights_attn_ws_bytes(const CacheAttn& a, int B, int dtype) {
  return weights_ws(a, B, cache_plan(a, B, dtype), dtype).bytes;
}

adt_status launch_weights_attn(const CacheAttn& a, int B, const float* w_in, float* w_out, int64_t stride_wb,
                               int64_t stride_wh, float decay, const float* row_weight, int dtype, void* ws,
                               hipStream_t st) {
  const CachePlan p = cache_plan(a, B, dtype);
  const WeightsWs w = weights_ws(a, B, p, dtype);
  const SlotWeights sw{w_in, w_out, stride_wb, stride_wh, decay, row_weight};
  float *row_ml = (float*)ws, *kept = w.keep ? (float*)((char*)ws + w.kept) : nullptr;
  const Partials parts = partials(a, B, p, (float*)((char*)ws + w.part), row_ml);
  adt_status e = attn_launches(a, B, p, parts, kept, dtype, st);
  if (e) return e;
  const int rows = a.nq_max * a.G;
  if (w.keep) {
    const int merges = p.splits > 1 ? rows : 0;
    slot_weights_kept_kernel<<<dim3(merges + (a.kv_cap + ST_KEYS - 1) / ST_KEYS, a.Hkv, B), CA_THREADS, 0, st>>>(
        a, parts.deal, dtype == ADT_BF16, merges, kept, parts.o, parts.ml, sw);
    ADT_LAUNCH_CHECK();
    return ADT_OK;
  }
  e = merge_launch(a, B, p, parts, row_ml, dtype, st);
  if (e) return e;
  // turns: four where that leaves two workgroups a CU or more, fewer for fewer keys; where there is not
  // one a CU, the waves deal out the rows instead (488 rows of 4 heads over 700 slots 53 -> 17 us)
  const int64_t units = ((int64_t)a.kv_cap + CA_WAVES * SW_CHUNK - 1) / (CA_WAVES * SW_CHUNK);
  const bool dealt = rows >= 16 * CA_WAVES && units * B * a.Hkv < 256;
  const int turns = dealt ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(4, units * B * a.Hkv / 512));
  const dim3 grid(dealt ? (a.kv_cap + SW_CHUNK - 1) / SW_CHUNK : (units + turns - 1) / turns, a.Hkv, B);
  const size_t padded = (rows + 15) / 16 * 16, factors = padded * sizeof(float2);
#define ADT_SW(TV, DHV)                                                                                                 \
  if (dealt) slot_weights_kernel<TV, DHV, Rows::DEALT><<<grid, CA_THREADS, factors, st>>>(a, row_ml, turns, sw);        \
  else if (rows <= SlotTile<TV, DHV>::QROWS)                                                                            \
    slot_weights_kernel<TV, DHV, Rows::LDS>                                                                             \
        <<<grid, CA_THREADS, factors + padded * SlotTile<TV, DHV>::PITCH * sizeof(TV), st>>>(a, row_ml, turns, sw);     \
  else slot_weights_kernel<TV, DHV, Rows::L2><<<grid, CA_THREADS, factors, st>>>(a, row_ml, turns, sw)
  if (dtype == ADT_BF16) {
    if (a.Dh == 128) { ADT_SW(uint16_t, 128); }
    else { ADT_SW(uint16_t, 64); }
  } else {
    if (a.Dh == 128) { ADT_SW(float, 128); }
    else { ADT_SW(float, 64); }
  }
#undef ADT_SW
  ADT_LAUNCH_CHECK();
  return ADT_OK;
}

}  // namespace adt
