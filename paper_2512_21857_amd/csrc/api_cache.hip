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
  const int64_t es = elem_bytes(dtype), row = Dh * es;
  ADT_CHECK_ARG(row % 16 == 0 && row <= 16384, ADT_E_SHAPE, "kv_evict: rows of %lld bytes", (long long)row);
  // in place: every part is its source, with the source's strides; else none of them is
  const bool place = k_out == k_cache;
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
  if (a_max == 0) return ADT_OK;
  return launch_weights_compact(weights, B, slices, stride_wb, stride_ws, kv_len, kv_cap, path, path_stride, n_acc,
                                a_max, (hipStream_t)stream);
}
