// Host side of the rotary and 8-bit cache entry points: argument checks and launches.
#include <string.h>

#include "fnpu_internal.h"

namespace fnpu {
namespace {

bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// The kernel's form of a descriptor, for rows of head_dim columns.
int rope_args(const fnpu_rope_desc *d, const float *inv_freq, const int32_t *positions, int32_t head_dim, int32_t n, RopeArgs *r) {
    if (!d || !inv_freq || !positions) return FNPU_EINVAL;
    if (d->rotary_dim <= 0 || d->rotary_dim % 2 || d->rotary_offset < 0) return FNPU_EINVAL;
    if (static_cast<int64_t>(d->rotary_offset) + d->rotary_dim > head_dim) return FNPU_EINVAL;
    if (d->num_axes < 1 || d->num_axes > kRopeMaxAxes) return FNPU_EINVAL;
    if (d->num_axes > 1 && !d->pair_axis) return FNPU_EINVAL;
    if (d->interleaved != 0 && d->interleaved != 1) return FNPU_EINVAL;
    if (d->inverse != 0 && d->inverse != 1) return FNPU_EINVAL;
    if (misaligned(inv_freq, 16) || misaligned(positions, 4)) return FNPU_EINVAL;
    if (d->rotary_dim / 2 > kRopeMaxPairs) return FNPU_EUNSUPPORTED;
    *r = RopeArgs{};
    r->inv_freq = inv_freq;
    r->positions = positions;
    r->n = n;
    r->pairs = d->rotary_dim / 2;
    r->offset = d->rotary_offset;
    r->interleaved = d->interleaved;
    r->axes = d->num_axes;
    r->sign = d->inverse ? -1.f : 1.f;
    if (d->num_axes > 1) {
        for (int i = 0; i < r->pairs; ++i)
            if (d->pair_axis[i] >= d->num_axes) return FNPU_EINVAL;
        memcpy(r->axis, d->pair_axis, static_cast<size_t>(r->pairs));
    }
    return FNPU_OK;
}

bool attn_shape_ok(const fnpu_attn_desc *d) {
    if (!d || d->num_q_heads <= 0 || d->num_kv_heads <= 0 || d->num_q_heads % d->num_kv_heads) return false;
    if (d->head_dim_qk <= 0 || d->head_dim_v <= 0 || d->block_size <= 0 || d->num_blocks <= 0) return false;
    if (d->head_dim_qk % 8 || d->head_dim_v % 8 || (d->kv_fp8 != 0 && d->kv_fp8 != 1)) return false;
    return !d->v_in_k_latent || (d->num_kv_heads == 1 && d->head_dim_v <= d->head_dim_qk);
}

// The cache a call works on: EINVAL for a format that there is none of or a bad
// shape, EUNSUPPORTED where the format has no such cache.
int cache_ok(const fnpu_attn_desc *d, int32_t format) {
    if (!attn_shape_ok(d) || format < FNPU_KV_BF16 || format > FNPU_KV_E4M3_BLOCK) return FNPU_EINVAL;
    if (format != FNPU_KV_BF16) return kv8_supported(d) ? FNPU_OK : FNPU_EUNSUPPORTED;
    return d->kv_fp8 ? FNPU_EUNSUPPORTED : FNPU_OK;
}

}  // namespace
}  // namespace fnpu

using namespace fnpu;

extern "C" {

int fnpu_rope(const fnpu_rope_desc *rope, const float *inv_freq, const int32_t *positions, const void *x, int64_t x_stride,
              int32_t num_heads, int32_t head_dim, int32_t num_tokens, void *out, int64_t out_stride, void *stream) {
    if (num_heads < 1 || head_dim < 1 || num_tokens < 0) return FNPU_EINVAL;
    if (num_tokens == 0) return FNPU_OK;
    RopeArgs r;
    const int rc = rope_args(rope, inv_freq, positions, head_dim, num_tokens, &r);
    if (rc != FNPU_OK) return rc;
    const int64_t row = static_cast<int64_t>(num_heads) * head_dim;
    if (!x || !out || misaligned(x, 2) || misaligned(out, 2) || x_stride < row || out_stride < row) return FNPU_EINVAL;
    if (x == out && x_stride != out_stride) return FNPU_EINVAL;
    auto fits = [&](int w) {  // everything a multiple of w columns, and of its bytes
        const uintptr_t at = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out);
        return r.pairs % w == 0 && r.offset % w == 0 && head_dim % w == 0 && x_stride % w == 0 && out_stride % w == 0 && at % (2 * w) == 0;
    };
    return launch_rope(r, x, x_stride, num_heads, head_dim, out, out_stride, fits(8) ? 8 : fits(4) ? 4 : 1, stream);
}

int fnpu_rope_append(const fnpu_attn_desc *desc, int32_t kv_format, const fnpu_rope_desc *rope, const float *inv_freq,
                     const int32_t *positions, const void *q, int64_t q_stride, const void *k_new, int64_t k_stride,
                     const void *v_new, int64_t v_stride, const int64_t *slot_mapping, int32_t num_tokens, void *q_out,
                     void *k_cache, void *v_cache, void *stream) {
    int rc = cache_ok(desc, kv_format);
    if (rc != FNPU_OK) return rc;
    if (num_tokens < 0) return FNPU_EINVAL;
    if (num_tokens == 0) return FNPU_OK;
    const bool latent = desc->v_in_k_latent != 0;
    const int64_t d = desc->head_dim_qk, k_row = desc->num_kv_heads * d, q_row = desc->num_q_heads * d;
    const int64_t v_row = latent ? 0 : static_cast<int64_t>(desc->num_kv_heads) * desc->head_dim_v;
    if (!k_new || !slot_mapping || !k_cache || (!latent && (!v_new || !v_cache))) return FNPU_EINVAL;
    if (misaligned(k_new, 16) || misaligned(k_cache, 16) || misaligned(slot_mapping, 8) || k_stride < k_row || k_stride % 8)
        return FNPU_EINVAL;
    if (!latent && (misaligned(v_new, 16) || misaligned(v_cache, 16) || v_stride < v_row || v_stride % 8)) return FNPU_EINVAL;
    if (q && (!rope || !q_out || misaligned(q, 16) || misaligned(q_out, 16) || q_stride < q_row || q_stride % 8)) return FNPU_EINVAL;
    if (q && q == q_out && q_stride != q_row) return FNPU_EINVAL;
    RopeArgs r = {};
    r.n = num_tokens;
    if (rope) {
        rc = rope_args(rope, inv_freq, positions, desc->head_dim_qk, num_tokens, &r);
        if (rc != FNPU_OK) return rc;
        if (r.pairs % 8 || r.offset % (kv_format == FNPU_KV_BF16 ? 8 : 16)) return FNPU_EUNSUPPORTED;
    } else if (kv_format == FNPU_KV_BF16) {  // rows as they are, one after the other: the plain append
        if (k_stride != k_row || (!latent && v_stride != v_row)) return FNPU_EUNSUPPORTED;
        return fnpu_kv_append(desc, k_new, v_new, slot_mapping, num_tokens, k_cache, v_cache, stream);
    }
    RopeAppendArgs p = {};
    p.q = static_cast<const __nv_bfloat16 *>(q);
    p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = latent ? nullptr : static_cast<const __nv_bfloat16 *>(v_new);
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.slots = slot_mapping;
    p.q_out = static_cast<__nv_bfloat16 *>(q_out);
    p.k_cache = k_cache;
    p.v_cache = latent ? nullptr : v_cache;
    p.num_slots = static_cast<int64_t>(desc->num_blocks) * desc->block_size;
    p.q_heads = q ? desc->num_q_heads : 0;
    p.kv_heads = desc->num_kv_heads;
    p.d = desc->head_dim_qk;
    p.d_v = desc->head_dim_v;
    p.block_size = desc->block_size;
    rc = global_error_address(&p.err);
    if (rc != FNPU_OK) return rc;
    return kv_format == FNPU_KV_BF16 ? launch_rope_append(r, p, stream) : launch_kv8_append(kv_format, r, p, stream);
}

int fnpu_kv_read(const fnpu_attn_desc *desc, int32_t kv_format, const int64_t *slots, int32_t n, const void *k_cache,
                 const void *v_cache, void *k_out, void *v_out, void *stream) {
    int rc = cache_ok(desc, kv_format);
    if (rc != FNPU_OK) return rc;
    if (n < 0) return FNPU_EINVAL;
    if (n == 0) return FNPU_OK;
    const bool latent = desc->v_in_k_latent != 0;
    if (!slots || !k_cache || !k_out || (!latent && (!v_cache || !v_out))) return FNPU_EINVAL;
    if (misaligned(slots, 8) || misaligned(k_cache, 16) || misaligned(k_out, 16)) return FNPU_EINVAL;
    if (!latent && (misaligned(v_cache, 16) || misaligned(v_out, 16))) return FNPU_EINVAL;
    int *err = nullptr;
    rc = global_error_address(&err);
    if (rc != FNPU_OK) return rc;
    if (kv_format == FNPU_KV_BF16) return launch_kv_read_bf16(desc, slots, n, k_cache, v_cache, k_out, v_out, err, stream);
    return launch_kv8_read(kv_format, desc, slots, n, k_cache, v_cache, k_out, v_out, err, stream);
}

int fnpu_kv8_block_bytes(const fnpu_attn_desc *desc, int32_t kv_format, int64_t *bytes) {
    if (!bytes || (kv_format != FNPU_KV_INT8_BLOCK && kv_format != FNPU_KV_E4M3_BLOCK)) return FNPU_EINVAL;
    const int rc = cache_ok(desc, kv_format);
    if (rc != FNPU_OK) return rc;
    *bytes = kv8_block_bytes(desc->num_kv_heads, desc->block_size, desc->head_dim_qk);
    return FNPU_OK;
}

}  // extern "C"
