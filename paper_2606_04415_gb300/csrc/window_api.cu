// Host side of windowed attention without a plan: argument checks, the split of
// the keys, the workspace.
#include <math.h>

#include <algorithm>
#include <mutex>

#include "fnpu_internal.h"

namespace fnpu {
namespace {

constexpr int kMaxDevices = 64;
std::mutex g_setup_mu;
bool g_ready[kMaxDevices];

// Loads the code of every kernel that a call may come to, once a device.
int prepare(int *sms) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return FNPU_ECUDA;
    if (dev < 0 || dev >= kMaxDevices) return FNPU_EUNSUPPORTED;
    std::lock_guard<std::mutex> lk(g_setup_mu);
    if (!g_ready[dev]) {
        const int rc = prepare_decode_tma_noplan(true);
        if (rc != FNPU_OK) return rc;
        g_ready[dev] = true;
    }
    return FNPU_OK;
}

struct Split {
    int64_t items, parts;  // of the bound; partial results
    int32_t keys, most;    // keys a split, splits a sequence
    int64_t lse_floats(int32_t hq) const { return (parts * hq + 63) / 64 * 64; }
    int64_t bytes(const fnpu_attn_desc *d) const {
        return most > 1 ? 4 * (lse_floats(d->num_q_heads) + parts * d->num_q_heads * d->head_dim_v) : 0;
    }
};

// Checks what both calls are given, and cuts the keys that a sequence may see (the
// window, the sinks and what whole stages add to them) into splits: without a
// plan the grid is sized by the host's bound, so lengths that the caller leaves
// open follow the number of items, like the plan-free decode of all keys.
int window_split(const fnpu_attn_desc *d, int32_t window, int32_t sinks, int32_t num_seqs, int32_t max_context_len,
                 int32_t split_keys, Split *out) {
    if (!d || num_seqs < 0 || window < 1 || sinks < 0 || max_context_len < 0) return FNPU_EINVAL;
    const int32_t Hq = d->num_q_heads, Hkv = d->num_kv_heads, D = d->head_dim_qk;
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv || D <= 0 || d->head_dim_v <= 0 || d->block_size <= 0 || d->num_blocks <= 0) return FNPU_EINVAL;
    if ((d->kv_fp8 != 0 && d->kv_fp8 != 1) || split_keys < 0 || split_keys % 64 != 0) return FNPU_EINVAL;
    if (d->v_in_k_latent || d->kv_fp8 || !decode_tma_supported(D, d->head_dim_v, Hq / Hkv, d->block_size)) return FNPU_EUNSUPPORTED;
    const Window w = make_window(window, sinks);
    const int64_t seen = static_cast<int64_t>(w.sink_keys(kDecodeStageKeys)) + window + kDecodeStageKeys - 1;
    const int64_t keys = std::max<int64_t>(1, std::min<int64_t>(max_context_len, seen));
    const int32_t hpi = decode_tma_heads_per_item(), hgroups = (Hkv + hpi - 1) / hpi;
    auto items = [&](int64_t sk) { return static_cast<int64_t>(num_seqs) * hgroups * ((keys + sk - 1) / sk); };
    int64_t sk = split_keys;
    constexpr int64_t kSms = 152;
    if (sk == 0) {
        // the shortest whose items fit the device at once (three CTAs an SM); where none does, by
        // a model if the bound lies well past the window (rows of one length then), else 256.
        // us a call, kv heads x rows, window: 4 x 4, 1024: 64 keys 11.1, 128 13.2; 4 x 64, 1024:
        // 128 keys 36.5, 192 29.8, 256 31.2; 8 x 16, 1024: 64 18.3, 128 14.9; 8 x 24, 4096: 256
        // 71.1, 512 67.8; 4 x 64, 4096 (none fits): 256 101.9, 512 110.7, 768 87.3
        sk = 0;
        for (int64_t k : {64, 128, 192, 256, 512})
            if (items(k) <= 3 * kSms) {
                sk = k;
                break;
            }
        if (sk == 0 && max_context_len < 2 * keys) sk = 256;
        if (sk == 0)
            sk = window_heavy_split(static_cast<int64_t>(std::min(hpi, Hkv)) * D * 4, 3 * kSms, [&](int32_t split, auto f) {
                const int64_t rows = static_cast<int64_t>(num_seqs) * hgroups, whole = keys / split, rest = keys % split;
                f(rows * whole, split);
                if (rest > 0) f(rows, static_cast<double>(rest));
            });
    }
    sk = std::max<int64_t>(sk, (keys + 256 * 64 - 1) / (256 * 64) * 64);  // at most 256 splits of a sequence
    out->keys = static_cast<int32_t>(std::min<int64_t>(sk, 1 << 30));
    out->most = static_cast<int32_t>((keys + out->keys - 1) / out->keys);
    out->items = items(out->keys);
    out->parts = static_cast<int64_t>(num_seqs) * out->most;
    if (out->items > INT32_MAX / 2 || out->parts > INT32_MAX / 2) return FNPU_EINVAL;
    return FNPU_OK;
}

}  // namespace
}  // namespace fnpu

using namespace fnpu;

extern "C" {

int fnpu_window_decode_workspace(const fnpu_attn_desc *desc, int32_t window, int32_t sinks, int32_t num_seqs,
                                 int32_t max_context_len, int32_t split_keys, int64_t *bytes) {
    if (!bytes) return FNPU_EINVAL;
    Split s;
    const int rc = window_split(desc, window, sinks, num_seqs, max_context_len, split_keys, &s);
    if (rc == FNPU_OK) *bytes = s.bytes(desc);
    return rc;
}

int fnpu_window_decode(const fnpu_attn_desc *desc, int32_t window, int32_t sinks, int32_t num_seqs, const int32_t *context_len,
                       const int32_t *block_table, int32_t block_table_stride, int32_t max_context_len, int32_t split_keys,
                       const void *q, const void *k_cache, const void *v_cache, void *out, float *lse, void *workspace,
                       int64_t workspace_bytes, void *stream) {
    Split s;
    int rc = window_split(desc, window, sinks, num_seqs, max_context_len, split_keys, &s);
    if (rc != FNPU_OK) return rc;
    if (num_seqs == 0) return FNPU_OK;
    if (static_cast<int64_t>(block_table_stride) * desc->block_size < max_context_len) return FNPU_EINVAL;
    if (!context_len || !block_table || !q || !k_cache || !v_cache || !out || !lse) return FNPU_EINVAL;
    const uintptr_t mis = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache) |
                          reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(workspace);
    if ((mis & 15u) || ((reinterpret_cast<uintptr_t>(context_len) | reinterpret_cast<uintptr_t>(block_table)) & 3u)) return FNPU_EINVAL;
    if (s.bytes(desc) > 0 && (!workspace || workspace_bytes < s.bytes(desc))) return FNPU_EINVAL;
    int sms = 0;
    rc = prepare(&sms);
    if (rc != FNPU_OK) return rc;
    AttnParams a = {};
    rc = global_error_address(&a.err);
    if (rc != FNPU_OK) return rc;
    a.q = q;
    a.k_cache = k_cache;
    a.v_cache = v_cache;
    a.out = out;
    a.lse = lse;
    a.block_table = block_table;
    a.bt_stride = block_table_stride;
    a.num_q_heads = desc->num_q_heads;
    a.num_kv_heads = desc->num_kv_heads;
    a.group = desc->num_q_heads / desc->num_kv_heads;
    a.block_size = desc->block_size;
    a.num_blocks = desc->num_blocks;
    a.num_tokens = num_seqs;
    a.head_dim_qk = a.head_dim_v = desc->head_dim_qk;
    const float scale = desc->softmax_scale > 0.f ? desc->softmax_scale
                                                  : static_cast<float>(1.0 / sqrt(static_cast<double>(desc->head_dim_qk)));
    a.scale_log2 = scale * 1.4426950408889634f;
    a.part_lse = static_cast<float *>(workspace);
    a.part_o = a.part_lse + s.lse_floats(desc->num_q_heads);
    a.na_ctx = context_len;
    a.na_num_seqs = num_seqs;
    a.na_max_ctx = max_context_len;
    a.na_split = s.keys;
    a.na_max_splits = s.most;
    a.num_ditems = static_cast<int32_t>(s.items);
    a.num_mgroups = num_seqs;
    const Window w = make_window(window, sinks);
    a.window = w.size;
    a.sinks = w.sinks;
    a.sink_keys = w.sink_keys(kDecodeStageKeys);
    return launch_decode_tma_noplan(a, stream, 3 * sms);
}

}  // extern "C"
