// C ABI of the operators of a long or bounded cache: rotary append, block means, attention over
// chosen blocks, attention that rates its slots, eviction.  Argument checks only; the launches
// are in kernels/rope.hip, blocks.hip, cache_attn.hip and evict.hip.
#include <cmath>

#include "launch.h"

using namespace adt;

static bool known_dtype(int32_t dt) { return dt == ADT_F32 || dt == ADT_BF16; }
static int64_t elem_bytes(int32_t dt) { return dt == ADT_BF16 ? 2 : 4; }
static bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }
// a stride of `elems` elements of `bytes` each that keeps 16-byte alignment
static bool stride16(int64_t elems, int64_t bytes) { return elems >= 0 && elems * bytes % 16 == 0; }
constexpr int32_t MAX_GRID_YZ = 65535;
constexpr int32_t MAX_ROWS = 8192;      // query rows of one key-value head
// Slots of a cache that kernels loop over: an index past the last one by a round of a workgroup, or of
// a launch, still fits 32 bits.
constexpr int32_t MAX_SLOTS = 0x7f000000;

extern "C" adt_status adt_rope_freqs(const adt_rope_cfg* cfg, double* freq, float* gain) {
  ADT_CHECK_ARG(cfg && freq && gain, ADT_E_ARG, "rope_freqs: null pointer");
  const int rot = cfg->rot_dim;
  ADT_CHECK_ARG(rot >= 2 && rot <= 256 && rot % 2 == 0, ADT_E_SHAPE, "rope_freqs: rot_dim %d", rot);
  ADT_CHECK_ARG(cfg->scaling >= ADT_ROPE_PLAIN && cfg->scaling <= ADT_ROPE_RAMP, ADT_E_ARG, "rope_freqs: scaling %d",
                cfg->scaling);
  ADT_CHECK_ARG(std::isfinite(cfg->theta) && cfg->theta > 1.0, ADT_E_ARG, "rope_freqs: theta %g", cfg->theta);
  const bool plain = cfg->scaling == ADT_ROPE_PLAIN;
  ADT_CHECK_ARG(plain || (std::isfinite(cfg->factor) && cfg->factor >= 1.0), ADT_E_ARG, "rope_freqs: factor %g",
                cfg->factor);
  const bool ramp = cfg->scaling == ADT_ROPE_RAMP;
  ADT_CHECK_ARG(!ramp || (cfg->orig_len >= 1 && cfg->slow > 0.0 && cfg->fast > cfg->slow && std::isfinite(cfg->fast)),
                ADT_E_ARG, "rope_freqs: orig_len %d, turns %g and %g", cfg->orig_len, cfg->fast, cfg->slow);
  const double theta = cfg->scaling == ADT_ROPE_BASE && rot > 2
                           ? cfg->theta * std::pow(cfg->factor, (double)rot / (rot - 2))
                           : cfg->theta;
  double lo = 0.0, span = 1.0;
  if (ramp) {
    const double two_pi = 6.283185307179586476925;
    auto index = [&](double turns) { return rot * std::log(cfg->orig_len / (two_pi * turns)) / (2.0 * std::log(theta)); };
    lo = std::fmax(std::floor(index(cfg->fast)), 0.0);
    span = std::fmax(std::fmin(std::ceil(index(cfg->slow)), rot - 1.0) - lo, 0.001);
  }
  for (int i = 0; i < rot / 2; ++i) {
    const double f = std::pow(theta, -2.0 * i / rot);
    if (cfg->scaling == ADT_ROPE_LINEAR) {
      freq[i] = f / cfg->factor;
    } else if (ramp) {
      const double t = std::fmin(std::fmax((i - lo) / span, 0.0), 1.0);
      freq[i] = f * (1.0 - t) + f / cfg->factor * t;
    } else {
      freq[i] = f;
    }
  }
  *gain = ramp ? (float)(0.1 * std::log(cfg->factor) + 1.0) : 1.f;
  return ADT_OK;
}

extern "C" adt_status adt_rope_append(const void* q, const void* k, const void* v, int64_t ldq, int64_t ldk,
                                      int64_t ldv, const int32_t* pos, const int32_t* kv_len, const int32_t* n_rows,
                                      const double* freq, float gain, int32_t rot_dim, int32_t layout, int32_t B,
                                      int32_t n_max, int32_t H, int32_t Hkv, int32_t Dh, void* q_out, void* k_cache,
                                      void* v_cache, int64_t stride_b, int64_t stride_h, int32_t kv_cap, int32_t dtype,
                                      void* stream) {
  ADT_CHECK_ARG(q && k && v && pos && kv_len && n_rows && freq && q_out && k_cache && v_cache, ADT_E_ARG,
                "rope_append: null pointer");
  ADT_CHECK_ARG(known_dtype(dtype), ADT_E_ARG, "rope_append: bad dtype %d", dtype);
  ADT_CHECK_ARG(layout == ADT_ROPE_HALF || layout == ADT_ROPE_INTERLEAVED, ADT_E_ARG, "rope_append: layout %d", layout);
  ADT_CHECK_ARG(B >= 1 && B <= MAX_GRID_YZ && n_max >= 1 && H >= 1 && Hkv >= 1 && kv_cap >= 1, ADT_E_ARG,
                "rope_append: B=%d n_max=%d H=%d Hkv=%d kv_cap=%d", B, n_max, H, Hkv, kv_cap);
  ADT_CHECK_ARG(std::isfinite(gain), ADT_E_ARG, "rope_append: gain");
  ADT_CHECK_ARG(Dh >= 2 && Dh <= 256 && Dh % 2 == 0, ADT_E_SHAPE, "rope_append: head_dim %d", Dh);
  ADT_CHECK_ARG(rot_dim >= 2 && rot_dim <= Dh && rot_dim % 2 == 0, ADT_E_SHAPE, "rope_append: rot_dim %d of %d", rot_dim,
                Dh);
  ADT_CHECK_ARG((int64_t)H + 2 * (int64_t)Hkv <= (1 << 20), ADT_E_SHAPE, "rope_append: %d and %d heads", H, Hkv);
  ADT_CHECK_ARG(ldq >= (int64_t)H * Dh && ldk >= (int64_t)Hkv * Dh && ldv >= (int64_t)Hkv * Dh, ADT_E_SHAPE,
                "rope_append: rows %lld, %lld, %lld elements apart", (long long)ldq, (long long)ldk, (long long)ldv);
  ADT_CHECK_ARG(q_out != q || ldq == (int64_t)H * Dh, ADT_E_SHAPE, "rope_append: in place needs contiguous rows");
  ADT_CHECK_ARG(stride_h >= (int64_t)kv_cap * Dh, ADT_E_SHAPE, "rope_append: stride_h %lld < kv_cap*Dh",
                (long long)stride_h);
  ADT_CHECK_ARG(B == 1 || stride_b >= (int64_t)Hkv * stride_h, ADT_E_SHAPE, "rope_append: stride_b too small");
  const RopeRows a{q, k, v, ldq, ldk, ldv, pos, kv_len, n_rows, n_max, H, Hkv, Dh, rot_dim, q_out, k_cache, v_cache,
                   stride_b, stride_h, kv_cap};
  return launch_rope_append(a, B, freq, gain, layout == ADT_ROPE_INTERLEAVED, dtype, (hipStream_t)stream);
}

extern "C" adt_status adt_block_keys(const void* k_cache, int64_t stride_b, int64_t stride_h, const int32_t* start,
                                     const int32_t* kv_len, int32_t B, int32_t Hkv, int32_t Dh, int32_t block,
                                     int32_t kv_cap, float* means, int64_t stride_mb, int64_t stride_mh, int32_t dtype,
                                     void* stream) {
  ADT_CHECK_ARG(k_cache && kv_len && means, ADT_E_ARG, "block_keys: null pointer");
  ADT_CHECK_ARG(known_dtype(dtype), ADT_E_ARG, "block_keys: bad dtype %d", dtype);
  ADT_CHECK_ARG(B >= 1 && B <= MAX_GRID_YZ && Hkv >= 1 && Hkv <= MAX_GRID_YZ && kv_cap >= 1, ADT_E_ARG,
                "block_keys: B=%d Hkv=%d kv_cap=%d", B, Hkv, kv_cap);
  ADT_CHECK_ARG(Dh == 64 || Dh == 128, ADT_E_SHAPE, "block_keys: head_dim %d not in {64, 128}", Dh);
  ADT_CHECK_ARG(block == 32 || block == 64 || block == 128, ADT_E_SHAPE, "block_keys: block %d not in {32, 64, 128}",
                block);
  ADT_CHECK_ARG(kv_cap <= MAX_SLOTS, ADT_E_CAPACITY, "block_keys: kv_cap %d", kv_cap);
  ADT_CHECK_ARG(stride_h >= (int64_t)kv_cap * Dh && (B == 1 || stride_b >= (int64_t)Hkv * stride_h), ADT_E_SHAPE,
                "block_keys: cache strides too small");
  const int64_t n_blk = ((int64_t)kv_cap + block - 1) / block;
  ADT_CHECK_ARG(stride_mh >= n_blk * Dh && (B == 1 || stride_mb >= (int64_t)Hkv * stride_mh), ADT_E_SHAPE,
                "block_keys: strides of the means too small for %lld blocks", (long long)n_blk);
  const int64_t es = elem_bytes(dtype);
  ADT_CHECK_ARG(aligned16(k_cache) && aligned16(means) && stride16(stride_b, es) && stride16(stride_h, es) &&
                    stride16(stride_mb, 4) && stride16(stride_mh, 4),
                ADT_E_SHAPE, "block_keys: addresses and strides must be multiples of 16 bytes");
  return launch_block_keys(k_cache, stride_b, stride_h, start, kv_len, B, Hkv, Dh, block, kv_cap, means, stride_mb,
                           stride_mh, dtype, (hipStream_t)stream);
}

// What both attentions ask of their common arguments.
static adt_status check_cache_attn(const char* who, const CacheAttn& a, int32_t B, int32_t H, int32_t dtype) {
  ADT_CHECK_ARG(a.q && a.k && a.v && a.kv_len && a.n_q && a.n_tail && a.mask && a.out, ADT_E_ARG, "%s: null pointer",
                who);
  ADT_CHECK_ARG(known_dtype(dtype), ADT_E_ARG, "%s: bad dtype %d", who, dtype);
  ADT_CHECK_ARG(B >= 1 && B <= MAX_GRID_YZ && H >= 1 && a.Hkv >= 1 && a.kv_cap >= 1, ADT_E_ARG,
                "%s: B=%d H=%d Hkv=%d kv_cap=%d", who, B, H, a.Hkv, a.kv_cap);
  ADT_CHECK_ARG(a.Dh == 64 || a.Dh == 128, ADT_E_SHAPE, "%s: head_dim %d not in {64, 128}", who, a.Dh);
  ADT_CHECK_ARG(H % a.Hkv == 0 && a.Hkv <= MAX_GRID_YZ && (int64_t)B * a.Hkv <= MAX_GRID_YZ, ADT_E_SHAPE,
                "%s: %d query heads over %d key-value heads of %d sequences", who, H, a.Hkv, B);
  ADT_CHECK_ARG(a.nq_max >= 1 && a.nq_max <= ADT_MAX_NODES, ADT_E_CAPACITY, "%s: nq_max %d", who, a.nq_max);
  ADT_CHECK_ARG((int64_t)a.nq_max * (H / a.Hkv) <= MAX_ROWS, ADT_E_CAPACITY, "%s: %d rows of %d heads per key-value head",
                who, a.nq_max, H / a.Hkv);
  ADT_CHECK_ARG(a.kv_cap <= MAX_SLOTS, ADT_E_CAPACITY, "%s: kv_cap %d", who, a.kv_cap);
  ADT_CHECK_ARG(a.sh >= (int64_t)a.kv_cap * a.Dh && (B == 1 || a.sb >= (int64_t)a.Hkv * a.sh), ADT_E_SHAPE,
                "%s: cache strides too small", who);
  const int64_t es = elem_bytes(dtype);
  ADT_CHECK_ARG(aligned16(a.q) && aligned16(a.k) && aligned16(a.v) && aligned16(a.out) && stride16(a.sb, es) &&
                    stride16(a.sh, es),
                ADT_E_SHAPE, "%s: addresses and strides must be multiples of 16 bytes", who);
  ADT_CHECK_ARG(std::isfinite(a.scale) && a.scale > 0.f, ADT_E_ARG, "%s: scale", who);
  return ADT_OK;
}

// Sizes an attention's workspace depends on; false if the call would be refused anyway.
static bool sized(CacheAttn& a, int32_t B, int32_t H, int32_t Hkv, int32_t Dh, int32_t nq_max, int32_t kv_cap,
                  int32_t dtype) {
  if (B < 1 || H < 1 || Hkv < 1 || H % Hkv || (Dh != 64 && Dh != 128) || nq_max < 1 || nq_max > ADT_MAX_NODES ||
      kv_cap < 1 || !known_dtype(dtype))
    return false;
  // (past these the products of the sizes would leave 32 bits)
  if ((int64_t)B * Hkv > MAX_GRID_YZ || (int64_t)nq_max * (H / Hkv) > MAX_ROWS || kv_cap > MAX_SLOTS) return false;
  a.Hkv = Hkv;
  a.G = H / Hkv;
  a.Dh = Dh;
  a.nq_max = nq_max;
  a.kv_cap = kv_cap;
  return true;
}
// Whether the output rows share memory with the queries (both [B][nq_max][H][Dh], contiguous).
static bool out_overlaps_q(const CacheAttn& a, int32_t B, int32_t dtype) {
  const uintptr_t q = (uintptr_t)a.q, out = (uintptr_t)a.out;
  return (q < out ? out - q : q - out) < (size_t)B * a.nq_max * a.Hkv * a.G * a.Dh * elem_bytes(dtype);
}
constexpr int32_t MAX_BLOCKS = 16384;
static bool known_block(int32_t block) { return block == 32 || block == 64 || block == 128; }

extern "C" size_t adt_sparse_tree_attn_workspace_size(int32_t B, int32_t H, int32_t Hkv, int32_t Dh, int32_t nq_max,
                                                      int32_t kv_cap, int32_t block, int32_t n_sel, int32_t dtype) {
  CacheAttn a{};
  if (!sized(a, B, H, Hkv, Dh, nq_max, kv_cap, dtype) || !known_block(block) || n_sel < 1) return 0;
  a.block = block;
  a.n_blk = (int)(((int64_t)kv_cap + block - 1) / block);
  a.n_sel = n_sel;
  if (a.n_blk > MAX_BLOCKS) return 0;
  return sparse_attn_ws_bytes(a, B, dtype);
}

extern "C" adt_status adt_sparse_tree_attn(const void* q, const void* k_cache, const void* v_cache, int64_t stride_b,
                                           int64_t stride_h, const float* means, int64_t stride_mb, int64_t stride_mh,
                                           const int32_t* kv_len, const int32_t* n_q, const int32_t* n_tail,
                                           const uint64_t* anc_mask, int32_t B, int32_t H, int32_t Hkv, int32_t Dh,
                                           int32_t nq_max, int32_t kv_cap, int32_t block, int32_t n_sel,
                                           int32_t n_first, int32_t n_last, float scale, int32_t dtype, void* out,
                                           int32_t* sel, void* workspace, size_t workspace_bytes, void* stream) {
  CacheAttn a{q, k_cache, v_cache, stride_b, stride_h, kv_len, n_q, n_tail, anc_mask, Hkv, Hkv > 0 ? H / Hkv : 0, Dh,
              nq_max, kv_cap, scale, out};
  const adt_status e = check_cache_attn("sparse_tree_attn", a, B, H, dtype);
  if (e) return e;
  ADT_CHECK_ARG(means, ADT_E_ARG, "sparse_tree_attn: null pointer");
  ADT_CHECK_ARG(known_block(block), ADT_E_SHAPE, "sparse_tree_attn: block %d not in {32, 64, 128}", block);
  ADT_CHECK_ARG(n_sel >= 1 && n_first >= 0 && n_last >= 0 && (int64_t)n_first + n_last <= n_sel, ADT_E_ARG,
                "sparse_tree_attn: %d first and %d last of %d blocks", n_first, n_last, n_sel);
  const int64_t n_blk = ((int64_t)kv_cap + block - 1) / block;
  ADT_CHECK_ARG(n_blk <= MAX_BLOCKS, ADT_E_CAPACITY, "sparse_tree_attn: %lld blocks", (long long)n_blk);
  ADT_CHECK_ARG(stride_mh >= n_blk * Dh && (B == 1 || stride_mb >= (int64_t)Hkv * stride_mh), ADT_E_SHAPE,
                "sparse_tree_attn: strides of the means too small for %lld blocks", (long long)n_blk);
  ADT_CHECK_ARG(aligned16(means) && stride16(stride_mb, 4) && stride16(stride_mh, 4) && aligned16(workspace),
                ADT_E_SHAPE, "sparse_tree_attn: addresses and strides must be multiples of 16 bytes");
  a.block = block;
  a.n_blk = (int)n_blk;
  a.n_sel = n_sel;
  const size_t need = sparse_attn_ws_bytes(a, B, dtype);
  ADT_CHECK_ARG(workspace && workspace_bytes >= need, ADT_E_CAPACITY, "sparse_tree_attn: workspace %zu < %zu bytes",
                workspace_bytes, need);
  // (a workgroup has read its rows' queries before it writes them, so the queries themselves will do)
  ADT_CHECK_ARG(out == q || !out_overlaps_q(a, B, dtype), ADT_E_ARG, "sparse_tree_attn: out overlaps q");
  return launch_sparse_attn(a, B, means, stride_mb, stride_mh, n_first, n_last, sel, dtype, workspace,
                            (hipStream_t)stream);
}

extern "C" size_t adt_tree_attn_weights_workspace_size(int32_t B, int32_t H, int32_t Hkv, int32_t Dh, int32_t nq_max,
                                                       int32_t kv_cap, int32_t dtype) {
  CacheAttn a{};
  return sized(a, B, H, Hkv, Dh, nq_max, kv_cap, dtype) ? weights_attn_ws_bytes(a, B, dtype) : 0;
}

extern "C" adt_status adt_tree_attn_weights(const void* q, const void* k_cache, const void* v_cache, int64_t stride_b,
                                            int64_t stride_h, const int32_t* kv_len, const int32_t* n_q,
                                            const int32_t* n_tail, const uint64_t* anc_mask, int32_t B, int32_t H,
                                            int32_t Hkv, int32_t Dh, int32_t nq_max, int32_t kv_cap, float scale,
                                            int32_t dtype, void* out, const float* weights_in, float* weights_out,
                                            int64_t stride_wb, int64_t stride_wh, float decay, const float* row_weight,
                                            void* workspace, size_t workspace_bytes, void* stream) {
  const CacheAttn a{q, k_cache, v_cache, stride_b, stride_h, kv_len, n_q, n_tail, anc_mask, Hkv, Hkv > 0 ? H / Hkv : 0,
                    Dh, nq_max, kv_cap, scale, out};
  const adt_status e = check_cache_attn("tree_attn_weights", a, B, H, dtype);
  if (e) return e;
  ADT_CHECK_ARG(weights_out, ADT_E_ARG, "tree_attn_weights: null pointer");
  ADT_CHECK_ARG(std::isfinite(decay), ADT_E_ARG, "tree_attn_weights: decay");
  ADT_CHECK_ARG(stride_wh >= kv_cap && (B == 1 || stride_wb >= (int64_t)Hkv * stride_wh), ADT_E_SHAPE,
                "tree_attn_weights: strides of the weights too small");
  ADT_CHECK_ARG(aligned16(workspace), ADT_E_SHAPE, "tree_attn_weights: workspace not 16-byte aligned");
  const size_t need = weights_attn_ws_bytes(a, B, dtype);
  ADT_CHECK_ARG(workspace && workspace_bytes >= need, ADT_E_CAPACITY, "tree_attn_weights: workspace %zu < %zu bytes",
                workspace_bytes, need);
  // (the slots' weights take the queries again after the output was written)
  ADT_CHECK_ARG(!out_overlaps_q(a, B, dtype), ADT_E_ARG, "tree_attn_weights: out overlaps q");
  return launch_weights_attn(a, B, weights_in, weights_out, stride_wb, stride_wh, decay, row_weight, dtype, workspace,
                             (hipStream_t)stream);
}

extern "C" adt_status adt_kv_evict(const void* k_cache, const void* v_cache, const float* weights, int64_t stride_b,
                                   int64_t stride_slice, int64_t stride_wb, int64_t stride_ws, const int32_t* kv_len,
                                   int32_t B, int32_t slices, int32_t Dh, int32_t kv_cap, int32_t budget,
                                   int32_t n_first, int32_t n_last, void* k_out, void* v_out, float* weights_out,
                                   int64_t out_stride_b, int64_t out_stride_slice, int64_t out_stride_wb,
                                   int64_t out_stride_ws, int32_t* kept, int32_t* new_len, int32_t dtype,
                                   void* stream) {
  ADT_CHECK_ARG(k_cache && v_cache && weights && kv_len && k_out && v_out && weights_out && kept && new_len, ADT_E_ARG,
                "kv_evict: null pointer");
  ADT_CHECK_ARG(known_dtype(dtype), ADT_E_ARG, "kv_evict: bad dtype %d", dtype);
  ADT_CHECK_ARG(B >= 1 && B <= MAX_GRID_YZ && slices >= 1 && Dh >= 1 && kv_cap >= 1, ADT_E_ARG,
                "kv_evict: B=%d slices=%d Dh=%d kv_cap=%d", B, slices, Dh, kv_cap);
  ADT_CHECK_ARG(budget >= 1 && n_first >= 0 && n_last >= 0 && (int64_t)n_first + n_last <= budget, ADT_E_ARG,
                "kv_evict: %d first and %d last of %d slots", n_first, n_last, budget);
  ADT_CHECK_ARG(kv_cap <= MAX_SLOTS, ADT_E_CAPACITY, "kv_evict: kv_cap %d", kv_cap);
  const int64_t es = elem_bytes(dtype), row = Dh * es;
  ADT_CHECK_ARG(row % 16 == 0 && row <= 16384, ADT_E_SHAPE, "kv_evict: rows of %lld bytes", (long long)row);
  // in place: every part is its source, with the source's strides; else none of them is
  const bool place = k_out == k_cache;
  // (a launch of 2^32 threads or more in a dimension would wrap: 512 a slice in place, 256 into another
  // cache; the selection's 1024 only where 2^22 slices would be 2^38 bytes of keys)
  ADT_CHECK_ARG(slices < (place ? 1 << 23 : 1 << 24), ADT_E_SHAPE, "kv_evict: %d slices", slices);
  ADT_CHECK_ARG((v_out == v_cache) == place && (weights_out == weights) == place, ADT_E_ARG,
                "kv_evict: caches and weights in place or none of them");
  ADT_CHECK_ARG(!place || (out_stride_b == stride_b && out_stride_slice == stride_slice && out_stride_wb == stride_wb &&
                           out_stride_ws == stride_ws),
                ADT_E_SHAPE, "kv_evict: in place needs the source's strides");
  const int64_t most = kv_cap < budget ? kv_cap : budget;      // rows that a slice of the output takes
  ADT_CHECK_ARG(stride_slice >= (int64_t)kv_cap * Dh && stride_ws >= kv_cap && out_stride_slice >= most * Dh &&
                    out_stride_ws >= most,
                ADT_E_SHAPE, "kv_evict: slice strides too small");
  ADT_CHECK_ARG(B == 1 || (stride_b >= slices * stride_slice && stride_wb >= slices * stride_ws &&
                           out_stride_b >= slices * out_stride_slice && out_stride_wb >= slices * out_stride_ws),
                ADT_E_SHAPE, "kv_evict: sequence strides too small");
  ADT_CHECK_ARG(aligned16(k_cache) && aligned16(v_cache) && aligned16(k_out) && aligned16(v_out) &&
                    stride16(stride_b, es) && stride16(stride_slice, es) && stride16(out_stride_b, es) &&
                    stride16(out_stride_slice, es),
                ADT_E_SHAPE, "kv_evict: addresses and strides must be multiples of 16 bytes");
  // (one cache for both, into another one for both, is moved twice to the same result; in place it is not)
  ADT_CHECK_ARG(k_out != v_out || (!place && k_cache == v_cache), ADT_E_ARG, "kv_evict: one destination for keys and values");
  const EvictMove a{k_cache, v_cache, weights, stride_b * es, stride_slice * es, stride_wb, stride_ws, kv_len, kv_cap,
                    slices, budget, (int)row, k_out, v_out, weights_out, out_stride_b * es, out_stride_slice * es,
                    out_stride_wb, out_stride_ws, kept, new_len};
  return launch_kv_evict(a, B, n_first, n_last, (hipStream_t)stream);
}

extern "C" adt_status adt_weights_compact(float* weights, int32_t B, int32_t slices, int64_t stride_wb,
                                          int64_t stride_ws, const int32_t* kv_len, int32_t kv_cap, const int32_t* path,
                                          int32_t path_stride, const int32_t* n_acc, int32_t a_max, void* stream) {
  ADT_CHECK_ARG(weights && kv_len && path && n_acc, ADT_E_ARG, "weights_compact: null pointer");
  ADT_CHECK_ARG(B >= 1 && B <= MAX_GRID_YZ && slices >= 1 && kv_cap >= 1, ADT_E_ARG,
                "weights_compact: B=%d slices=%d kv_cap=%d", B, slices, kv_cap);
  ADT_CHECK_ARG(a_max >= 0 && a_max < ADT_MAX_NODES && path_stride >= a_max + 1, ADT_E_CAPACITY,
                "weights_compact: a_max %d path_stride %d", a_max, path_stride);
  ADT_CHECK_ARG(stride_ws >= kv_cap && (B == 1 || stride_wb >= slices * stride_ws), ADT_E_SHAPE,
                "weights_compact: strides too small");
  ADT_CHECK_ARG(slices < 1 << 25, ADT_E_SHAPE, "weights_compact: %d slices", slices);   // (as above, 128 a slice)
  if (a_max == 0) return ADT_OK;
  return launch_weights_compact(weights, B, slices, stride_wb, stride_ws, kv_len, kv_cap, path, path_stride, n_acc,
                                a_max, (hipStream_t)stream);
}
