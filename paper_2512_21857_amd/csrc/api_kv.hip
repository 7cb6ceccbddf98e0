// C ABI of the operators over caches of any type (adt_kv_cache): norms with rotation and append,
// conversion, accepted paths, tree attention with or without a shared prefix.  Argument checks only;
// the launches are in kernels/kv_rows.hip and kv_attn.hip.
#include <cmath>

#include "launch.h"

using namespace adt;

static bool plain_type(int32_t t) { return t == ADT_F32 || t == ADT_BF16; }
static bool eight_bit(int32_t t) { return t == ADT_E4M3 || t == ADT_I8; }
static int64_t elem_bytes(int32_t t) { return t == ADT_F32 ? 4 : t == ADT_BF16 ? 2 : 1; }
static bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }
constexpr int32_t MAX_GRID_YZ = 65535;
constexpr int32_t MAX_HEADS = 32767;    // keys and values of a head are two of a launch's second dimension
constexpr int32_t MAX_ROWS = 8192;      // query rows of one key-value head
constexpr int32_t MAX_GROUP = 4096;     // sequences behind one prefix
// Slots of a cache that kernels loop over: an index past the last one by a round of a launch still
// fits 32 bits.
constexpr int32_t MAX_SLOTS = 0x7f000000;

// A cache's own consistency.  written: the call stores to it.
static adt_status check_cache(const char* who, const char* which, const adt_kv_cache* c, bool written) {
  ADT_CHECK_ARG(c && c->k && c->v, ADT_E_ARG, "%s: %s: null pointer", who, which);
  ADT_CHECK_ARG(plain_type(c->type) || eight_bit(c->type), ADT_E_ARG, "%s: %s: type %d", who, which, c->type);
  ADT_CHECK_ARG(eight_bit(c->type) ? c->k_scale && c->v_scale : !c->k_scale && !c->v_scale, ADT_E_ARG,
                "%s: %s: scales go with eight-bit types only", who, which);
  ADT_CHECK_ARG(c->B >= 1 && c->heads >= 1 && c->cap >= 1 && c->Dh >= 1, ADT_E_ARG, "%s: %s: B=%d heads=%d cap=%d Dh=%d",
                who, which, c->B, c->heads, c->cap, c->Dh);
  ADT_CHECK_ARG(c->B <= MAX_GRID_YZ && c->heads <= MAX_HEADS && c->Dh <= 256 && c->Dh % 2 == 0, ADT_E_SHAPE,
                "%s: %s: B=%d heads=%d Dh=%d", who, which, c->B, c->heads, c->Dh);
  ADT_CHECK_ARG(c->cap <= MAX_SLOTS, ADT_E_CAPACITY, "%s: %s: %d slots", who, which, c->cap);
  ADT_CHECK_ARG(c->stride_h >= (int64_t)c->cap * c->Dh && (c->B == 1 || c->stride_b >= c->heads * c->stride_h), ADT_E_SHAPE,
                "%s: %s: strides too small", who, which);
  ADT_CHECK_ARG(plain_type(c->type) || (c->scale_h >= c->cap && (c->B == 1 || c->scale_b >= c->heads * c->scale_h)),
                ADT_E_SHAPE, "%s: %s: strides of the scales too small", who, which);
  ADT_CHECK_ARG(!written || (c->k != c->v && (plain_type(c->type) || c->k_scale != c->v_scale)), ADT_E_ARG,
                "%s: %s: keys and values need memory of their own", who, which);
  return ADT_OK;
}

// Whether two stretches of memory share bytes.
struct Stretch {
  uintptr_t at;
  uint64_t bytes;
};
static bool overlap(const Stretch& a, const Stretch& b) { return a.at < b.at + b.bytes && b.at < a.at + a.bytes; }
// From the first element of a cache's keys (values) to the last.
static Stretch extent(const adt_kv_cache& c, const void* p) {
  const uint64_t elems = (uint64_t)(c.B - 1) * c.stride_b + (uint64_t)(c.heads - 1) * c.stride_h + (uint64_t)c.cap * c.Dh;
  return {(uintptr_t)p, elems * elem_bytes(c.type)};
}
static Stretch scale_extent(const adt_kv_cache& c, const float* p) {
  const uint64_t n = (uint64_t)(c.B - 1) * c.scale_b + (uint64_t)(c.heads - 1) * c.scale_h + (uint64_t)c.cap;
  return {(uintptr_t)p, n * sizeof(float)};
}

extern "C" adt_status adt_norm_rope_append(const void* q, const void* k, const void* v, int64_t ldq, int64_t ldk,
                                           int64_t ldv, const float* q_norm, const float* k_norm,
                                           int32_t norm_per_head, float eps, const int32_t* pos, const int32_t* kv_len,
                                           const int32_t* n_rows, const double* freq, float gain, int32_t rot_dim,
                                           int32_t layout, int32_t n_max, int32_t H, int32_t dtype, void* q_out,
                                           const adt_kv_cache* cache, void* stream) {
  const adt_status e = check_cache("norm_rope_append", "cache", cache, true);
  if (e) return e;
  const int32_t Dh = cache->Dh, heads = cache->heads, B = cache->B;
  ADT_CHECK_ARG(q && k && v && pos && kv_len && n_rows && freq && q_out, ADT_E_ARG, "norm_rope_append: null pointer");
  ADT_CHECK_ARG(plain_type(dtype), ADT_E_ARG, "norm_rope_append: bad dtype %d", dtype);
  ADT_CHECK_ARG(cache->type == dtype || eight_bit(cache->type), ADT_E_UNSUPPORTED,
                "norm_rope_append: rows of type %d into a cache of type %d", dtype, cache->type);
  ADT_CHECK_ARG(layout == ADT_ROPE_HALF || layout == ADT_ROPE_INTERLEAVED, ADT_E_ARG, "norm_rope_append: layout %d", layout);
  ADT_CHECK_ARG(n_max >= 1 && H >= 1 && (norm_per_head == 0 || norm_per_head == 1), ADT_E_ARG,
                "norm_rope_append: n_max=%d H=%d norm_per_head=%d", n_max, H, norm_per_head);
  ADT_CHECK_ARG(std::isfinite(gain), ADT_E_ARG, "norm_rope_append: gain");
  ADT_CHECK_ARG((!q_norm && !k_norm) || (std::isfinite(eps) && eps >= 1.17549435e-38f), ADT_E_ARG,
                "norm_rope_append: eps");
  ADT_CHECK_ARG(rot_dim >= 2 && rot_dim <= Dh && rot_dim % 2 == 0, ADT_E_SHAPE, "norm_rope_append: rot_dim %d of %d",
                rot_dim, Dh);
  ADT_CHECK_ARG((int64_t)H + 2 * (int64_t)heads <= (1 << 20), ADT_E_SHAPE, "norm_rope_append: %d and %d heads", H, heads);
  ADT_CHECK_ARG(ldq >= (int64_t)H * Dh && ldk >= (int64_t)heads * Dh && ldv >= (int64_t)heads * Dh, ADT_E_SHAPE,
                "norm_rope_append: rows %lld, %lld, %lld elements apart", (long long)ldq, (long long)ldk, (long long)ldv);
  ADT_CHECK_ARG(q_out != q || ldq == (int64_t)H * Dh, ADT_E_SHAPE, "norm_rope_append: in place needs contiguous rows");
  const int64_t rows = (int64_t)B * n_max;
  auto span = [&](const void* p, int64_t ld, int64_t h) {
    return Stretch{(uintptr_t)p, (uint64_t)((rows - 1) * ld + h * Dh) * (uint64_t)elem_bytes(dtype)};
  };
  const Stretch out = span(q_out, (int64_t)H * Dh, H);
  ADT_CHECK_ARG((q_out == q || !overlap(out, span(q, ldq, H))) && !overlap(out, span(k, ldk, heads)) &&
                    !overlap(out, span(v, ldv, heads)),
                ADT_E_ARG, "norm_rope_append: q_out overlaps the rows");
  const NormRopeRows a{q,   k,      v,      ldq,  ldk,  ldv,   q_norm, k_norm, norm_per_head ? Dh : 0, eps,
                       pos, kv_len, n_rows, freq, gain, n_max, H,      rot_dim, q_out, *cache};
  return launch_norm_rope_append(a, layout == ADT_ROPE_INTERLEAVED, dtype, (hipStream_t)stream);
}

extern "C" adt_status adt_cache_convert(const adt_kv_cache* src, const adt_kv_cache* dst, const int32_t* length,
                                        int32_t n_max, const int32_t* src_start, const int32_t* dst_start,
                                        void* stream) {
  adt_status e = check_cache("cache_convert", "source", src, false);
  if (!e) e = check_cache("cache_convert", "destination", dst, true);
  if (e) return e;
  ADT_CHECK_ARG(length, ADT_E_ARG, "cache_convert: null pointer");
  ADT_CHECK_ARG(n_max >= 1, ADT_E_ARG, "cache_convert: n_max %d", n_max);
  ADT_CHECK_ARG(n_max <= MAX_SLOTS, ADT_E_CAPACITY, "cache_convert: n_max %d", n_max);
  ADT_CHECK_ARG(eight_bit(src->type) != eight_bit(dst->type), ADT_E_UNSUPPORTED, "cache_convert: from type %d to type %d",
                src->type, dst->type);
  ADT_CHECK_ARG(src->B == dst->B && src->heads == dst->heads && src->Dh == dst->Dh, ADT_E_SHAPE,
                "cache_convert: caches of %d x %d x %d and %d x %d x %d", src->B, src->heads, src->Dh, dst->B, dst->heads,
                dst->Dh);
  for (const void* s : {src->k, src->v})
    for (const void* d : {dst->k, dst->v})
      ADT_CHECK_ARG(!overlap(extent(*src, s), extent(*dst, d)), ADT_E_ARG, "cache_convert: the caches overlap");
  // (the scales are the eight-bit side's, beside the other side's keys and values)
  const adt_kv_cache &codes = eight_bit(src->type) ? *src : *dst, &plain = eight_bit(src->type) ? *dst : *src;
  for (const float* s : {codes.k_scale, codes.v_scale})
    for (const void* x : {plain.k, plain.v})
      ADT_CHECK_ARG(!overlap(scale_extent(codes, s), extent(plain, x)), ADT_E_ARG, "cache_convert: the caches overlap");
  return launch_cache_convert(*src, *dst, length, n_max, src_start, dst_start, (hipStream_t)stream);
}

extern "C" adt_status adt_cache_compact(const adt_kv_cache* cache, const int32_t* kv_len, const int32_t* path,
                                        int32_t path_stride, const int32_t* n_acc, int32_t a_max, void* stream) {
  const adt_status e = check_cache("cache_compact", "cache", cache, true);
  if (e) return e;
  ADT_CHECK_ARG(kv_len && path && n_acc, ADT_E_ARG, "cache_compact: null pointer");
  ADT_CHECK_ARG(a_max >= 0 && a_max < ADT_MAX_NODES && path_stride >= a_max + 1, ADT_E_CAPACITY,
                "cache_compact: a_max %d path_stride %d", a_max, path_stride);
  const int64_t es = elem_bytes(cache->type);
  ADT_CHECK_ARG(cache->Dh * es % 16 == 0 && aligned16(cache->k) && aligned16(cache->v) &&
                    cache->stride_b * es % 16 == 0 && cache->stride_h * es % 16 == 0,
                ADT_E_SHAPE, "cache_compact: rows, addresses and strides must be multiples of 16 bytes");
  if (a_max == 0) return ADT_OK;
  return launch_cache_compact(*cache, kv_len, path, path_stride, n_acc, a_max, (hipStream_t)stream);
}

// Sizes of an attention; false if the call would be refused for them.
static bool sized(KvAttn& a, int32_t B, int32_t H, int32_t heads, int32_t Dh, int32_t nq_max, int32_t kv_cap,
                  int32_t groups, int32_t prefix_cap, int32_t type) {
  if (B < 1 || H < 1 || heads < 1 || H % heads || (Dh != 64 && Dh != 128) || nq_max < 1 || nq_max > ADT_MAX_NODES ||
      kv_cap < 1 || kv_cap > MAX_SLOTS || (!plain_type(type) && !eight_bit(type)))
    return false;
  if (heads > MAX_HEADS || (int64_t)B * heads > MAX_GRID_YZ || (int64_t)nq_max * (H / heads) > MAX_ROWS) return false;
  if (groups < 0 || (groups && (B % groups || B / groups > MAX_GROUP || prefix_cap < 1 || prefix_cap > MAX_SLOTS)))
    return false;
  a.B = B;
  a.Hkv = heads;
  a.G = H / heads;
  a.Dh = Dh;
  a.nq_max = nq_max;
  a.own.cap = kv_cap;
  a.groups = groups;
  a.group = groups ? B / groups : 1;
  a.pre.cap = groups ? prefix_cap : 0;
  a.type = type;
  return true;
}

extern "C" size_t adt_cache_tree_attn_workspace_size(int32_t B, int32_t H, int32_t heads, int32_t Dh, int32_t nq_max,
                                                     int32_t kv_cap, int32_t groups, int32_t prefix_cap, int32_t type) {
  KvAttn a{};
  return sized(a, B, H, heads, Dh, nq_max, kv_cap, groups, prefix_cap, type) ? kv_attn_ws_bytes(a) : 0;
}

extern "C" adt_status adt_cache_tree_attn(const void* q, const adt_kv_cache* cache, const int32_t* kv_len,
                                          const int32_t* n_q, const int32_t* n_tail, const uint64_t* anc_mask,
                                          int32_t H, int32_t nq_max, int32_t kv_cap, const adt_kv_cache* prefix,
                                          const int32_t* prefix_len, int32_t prefix_cap, float scale, int32_t dtype,
                                          void* out, void* workspace, size_t workspace_bytes, void* stream) {
  adt_status e = check_cache("cache_tree_attn", "cache", cache, false);
  if (!e && prefix) e = check_cache("cache_tree_attn", "prefix", prefix, false);
  if (e) return e;
  const adt_kv_cache& c = *cache;
  ADT_CHECK_ARG(q && kv_len && n_q && n_tail && anc_mask && out && (!prefix || prefix_len), ADT_E_ARG,
                "cache_tree_attn: null pointer");
  ADT_CHECK_ARG(plain_type(dtype), ADT_E_ARG, "cache_tree_attn: bad dtype %d", dtype);
  ADT_CHECK_ARG(c.type == dtype || (dtype == ADT_BF16 && eight_bit(c.type)), ADT_E_UNSUPPORTED,
                "cache_tree_attn: rows of type %d over a cache of type %d", dtype, c.type);
  ADT_CHECK_ARG(H >= 1 && kv_cap >= 1 && (!prefix || prefix_cap >= 1), ADT_E_ARG, "cache_tree_attn: H=%d kv_cap=%d prefix_cap=%d",
                H, kv_cap, prefix_cap);
  ADT_CHECK_ARG(kv_cap <= c.cap && (!prefix || prefix_cap <= prefix->cap), ADT_E_CAPACITY,
                "cache_tree_attn: bounds %d and %d past the caches", kv_cap, prefix_cap);
  ADT_CHECK_ARG(std::isfinite(scale) && scale > 0.f, ADT_E_ARG, "cache_tree_attn: scale");
  ADT_CHECK_ARG(c.Dh == 64 || c.Dh == 128, ADT_E_SHAPE, "cache_tree_attn: head_dim %d not in {64, 128}", c.Dh);
  ADT_CHECK_ARG(H % c.heads == 0 && (int64_t)c.B * c.heads <= MAX_GRID_YZ, ADT_E_SHAPE,
                "cache_tree_attn: %d query heads over %d key-value heads of %d sequences", H, c.heads, c.B);
  ADT_CHECK_ARG(nq_max >= 1 && nq_max <= ADT_MAX_NODES && (int64_t)nq_max * (H / c.heads) <= MAX_ROWS, ADT_E_CAPACITY,
                "cache_tree_attn: %d rows of %d heads per key-value head", nq_max, H / c.heads);
  if (prefix) {
    ADT_CHECK_ARG(prefix->type == c.type, ADT_E_UNSUPPORTED, "cache_tree_attn: a prefix of type %d with a cache of type %d",
                  prefix->type, c.type);
    ADT_CHECK_ARG(prefix->heads == c.heads && prefix->Dh == c.Dh && c.B % prefix->B == 0, ADT_E_SHAPE,
                  "cache_tree_attn: a prefix of %d x %d x %d with a cache of %d x %d x %d", prefix->B, prefix->heads,
                  prefix->Dh, c.B, c.heads, c.Dh);
    ADT_CHECK_ARG(c.B / prefix->B <= MAX_GROUP, ADT_E_CAPACITY, "cache_tree_attn: %d sequences a group", c.B / prefix->B);
  }
  const int64_t es = elem_bytes(c.type);
  bool fit = aligned16(q) && aligned16(out) && aligned16(workspace);
  for (const adt_kv_cache* x : {cache, prefix})
    if (x) fit = fit && aligned16(x->k) && aligned16(x->v) && x->stride_b * es % 16 == 0 && x->stride_h * es % 16 == 0;
  ADT_CHECK_ARG(fit, ADT_E_SHAPE, "cache_tree_attn: addresses and strides must be multiples of 16 bytes");
  KvAttn a{};
  if (!sized(a, c.B, H, c.heads, c.Dh, nq_max, kv_cap, prefix ? prefix->B : 0, prefix_cap, c.type)) return ADT_E_SHAPE;
  a.q = q;
  a.own = KvPart{c.k, c.v, c.k_scale, c.v_scale, c.stride_b, c.stride_h, c.scale_b, c.scale_h, kv_len, kv_cap};
  if (prefix)
    a.pre = KvPart{prefix->k,        prefix->v,       prefix->k_scale, prefix->v_scale, prefix->stride_b,
                   prefix->stride_h, prefix->scale_b, prefix->scale_h, prefix_len,      prefix_cap};
  a.n_q = n_q;
  a.n_tail = n_tail;
  a.mask = anc_mask;
  a.scale = scale;
  a.out = out;
  const size_t need = kv_attn_ws_need(a);
  ADT_CHECK_ARG(need == 0 || (workspace && workspace_bytes >= need), ADT_E_CAPACITY,
                "cache_tree_attn: workspace %zu < %zu bytes", workspace_bytes, need);
  // (a workgroup has read its rows' queries before any row is written, so the queries themselves will do)
  const Stretch rows{(uintptr_t)q, (uint64_t)c.B * nq_max * H * c.Dh * (uint64_t)elem_bytes(dtype)};
  ADT_CHECK_ARG(out == q || !overlap(rows, Stretch{(uintptr_t)out, rows.bytes}), ADT_E_ARG, "cache_tree_attn: out overlaps q");
  return launch_kv_attn(a, workspace, (hipStream_t)stream);
}
