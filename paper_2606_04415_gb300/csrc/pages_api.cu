// Host side of the page operations: argument checks, workspaces and launches.
#include "fnpu_internal.h"

namespace fnpu {
namespace {

bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// (ids, positions and what is added to them stay within 32 bits)
int pages_ok(const fnpu_pages_desc *d, int64_t rows, int64_t width) {
    if (!d || d->block_size < 1 || d->num_blocks < 1 || rows < 0 || width < 0) return FNPU_EINVAL;
    if (d->block_size > (1 << 16) || d->num_blocks > (1 << 30) || rows > kPagesMaxRows) return FNPU_EUNSUPPORTED;
    return width * d->block_size > INT32_MAX - (1 << 17) ? FNPU_EUNSUPPORTED : FNPU_OK;
}

// Blocks of a CTA's chunk: kPagesChunk, or as many of them as leave kPagesMostChunks chunks
// (each CTA adds up all chunks' counts).
int32_t chunk_of(const fnpu_pages_desc *d) {
    constexpr int32_t kAll = kPagesChunk * kPagesMostChunks;
    return kPagesChunk * ((d->num_blocks - 1) / kAll + 1);
}
int32_t chunks_of(const fnpu_pages_desc *d) { return (d->num_blocks - 1) / chunk_of(d) + 1; }

// Workspace, in int32: chunk counts, three values a row (two at least), two a block.
int64_t words(const fnpu_pages_desc *d, int32_t rows) {
    return static_cast<int64_t>(chunks_of(d)) + 3ll * (rows + 2) + 2ll * d->num_blocks;
}

void place(const fnpu_pages_desc *d, int32_t rows, void *workspace, PagesArgs *a) {
    a->chunks = chunks_of(d);
    a->chunk = chunk_of(d);
    a->block_size = d->block_size;
    a->num_blocks = d->num_blocks;
    a->chunk_count = static_cast<int32_t *>(workspace);
    a->row_length = a->chunk_count + a->chunks;
    a->row_tail = a->row_length + rows + 2;
    a->row_refs = a->row_tail + rows + 2;
    a->block_a = a->row_refs + rows + 2;
    a->block_b = a->block_a + d->num_blocks;
}

bool workspace_ok(const fnpu_pages_desc *d, int32_t rows, const void *workspace, int64_t bytes) {
    return workspace && !misaligned(workspace, 16) && bytes >= 4 * words(d, rows);
}

}  // namespace
}  // namespace fnpu

using namespace fnpu;

extern "C" {

int fnpu_pages_workspace(const fnpu_pages_desc *desc, int32_t rows, int64_t *bytes) {
    if (!bytes) return FNPU_EINVAL;
    const int rc = pages_ok(desc, rows, 0);
    if (rc == FNPU_OK) *bytes = (4 * words(desc, rows) + 15) / 16 * 16;
    return rc;
}

int fnpu_pages_free(const fnpu_pages_desc *desc, int32_t *table, int32_t *length, int32_t rows, int32_t width, const uint8_t *ends,
                    int32_t window, int32_t sinks, int32_t *refs, void *stream) {
    int rc = pages_ok(desc, rows, width);
    if (rc != FNPU_OK) return rc;
    if (window < 0 || sinks < 0) return FNPU_EINVAL;
    if (rows == 0 || (window == 0 && !ends)) return FNPU_OK;
    if (!table || !length || !refs || misaligned(table, 4) || misaligned(length, 4) || misaligned(refs, 4)) return FNPU_EINVAL;
    PagesArgs a = {};
    rc = global_error_address(&a.err);
    if (rc != FNPU_OK) return rc;
    a.table = table;
    a.length = length;
    a.refs = refs;
    a.block_size = desc->block_size;
    a.num_blocks = desc->num_blocks;
    a.rows = rows;
    a.width = width;
    return launch_pages_free(a, length, ends, window, sinks, stream);
}

int fnpu_pages_fork(const fnpu_pages_desc *desc, const int32_t *table, const int32_t *length, int32_t rows, int32_t width,
                    const int32_t *parents, int32_t new_rows, int32_t grow, int32_t *refs, int32_t *new_table, int32_t *new_length,
                    int64_t *slots, int32_t *copies, int32_t *stats, void *workspace, int64_t workspace_bytes, void *stream) {
    int rc = pages_ok(desc, rows > new_rows ? rows : new_rows, width);
    if (rc != FNPU_OK) return rc;
    if (rows < 0 || new_rows < 0 || grow < 0 || (!parents && new_rows > 0 && rows != new_rows)) return FNPU_EINVAL;
    if (grow > (1 << 16)) return FNPU_EUNSUPPORTED;
    if (!stats || !refs || misaligned(stats, 4) || misaligned(refs, 4)) return FNPU_EINVAL;
    if (rows > 0 && (!table || !length || misaligned(table, 4) || misaligned(length, 4))) return FNPU_EINVAL;
    if (new_rows > 0 && (!new_table || !new_length || !copies || (grow > 0 && !slots) || misaligned(new_table, 4) ||
                         misaligned(new_length, 4) || misaligned(copies, 4) || misaligned(slots, 8) || misaligned(parents, 4)))
        return FNPU_EINVAL;
    if (parents && rows > 0 && new_rows > 0 && (new_table == table || new_length == length)) return FNPU_EINVAL;
    if (!workspace_ok(desc, new_rows, workspace, workspace_bytes)) return FNPU_EINVAL;
    PagesArgs a = {};
    place(desc, new_rows, workspace, &a);
    rc = global_error_address(&a.err);
    if (rc != FNPU_OK) return rc;
    a.table = const_cast<int32_t *>(table);
    a.length = length;
    a.parents = parents;
    a.refs = refs;
    a.new_table = new_table;
    a.new_length = new_length;
    a.copies = copies;
    a.stats = stats;
    a.slots = slots;
    a.rows = rows;
    a.width = width;
    a.new_rows = new_rows;
    a.grow = grow;
    return launch_pages_fork(a, stream);
}

int fnpu_pages_compact(const fnpu_pages_desc *desc, int32_t *table, const int32_t *length, int32_t rows, int32_t width, int32_t *refs,
                       int32_t *copies, int32_t max_copies, int32_t *remap, int32_t *stats, void *workspace, int64_t workspace_bytes,
                       void *stream) {
    int rc = pages_ok(desc, rows, width);
    if (rc != FNPU_OK) return rc;
    if (max_copies < 0 || !refs || !remap || !stats || (max_copies > 0 && !copies)) return FNPU_EINVAL;
    if (rows > 0 && (!table || !length)) return FNPU_EINVAL;
    if (misaligned(table, 4) || misaligned(length, 4) || misaligned(refs, 4) || misaligned(copies, 4) || misaligned(remap, 4) ||
        misaligned(stats, 4) || !workspace_ok(desc, rows, workspace, workspace_bytes))
        return FNPU_EINVAL;
    PagesArgs a = {};
    place(desc, rows, workspace, &a);
    rc = global_error_address(&a.err);
    if (rc != FNPU_OK) return rc;
    a.table = table;
    a.length = length;
    a.refs = refs;
    a.copies = copies;
    a.stats = stats;
    a.remap = remap;
    a.rows = rows;
    a.width = width;
    a.max_copies = max_copies;
    return launch_pages_compact(a, stream);
}

int fnpu_kv_copy_blocks(const fnpu_attn_desc *desc, int32_t kv_format, const int32_t *copies, int32_t num_copies, void *const *k_pools,
                        void *const *v_pools, int32_t num_pools, void *stream) {
    if (!desc || desc->num_q_heads <= 0 || desc->num_kv_heads <= 0 || desc->num_q_heads % desc->num_kv_heads || desc->head_dim_qk <= 0 ||
        desc->head_dim_v <= 0 || desc->head_dim_qk % 8 || desc->head_dim_v % 8 || desc->block_size <= 0 || desc->num_blocks <= 0 ||
        (desc->kv_fp8 != 0 && desc->kv_fp8 != 1) || (desc->v_in_k_latent && desc->num_kv_heads != 1) || kv_format < FNPU_KV_BF16 ||
        kv_format > FNPU_KV_E4M3_BLOCK || num_copies < 0 || num_pools < 0)
        return FNPU_EINVAL;
    const bool latent = desc->v_in_k_latent != 0;
    int64_t k_bytes, v_bytes;
    if (kv_format != FNPU_KV_BF16) {
        if (!kv8_supported(desc)) return FNPU_EUNSUPPORTED;
        k_bytes = v_bytes = kv8_block_bytes(desc->num_kv_heads, desc->block_size, desc->head_dim_qk);
    } else if (desc->kv_fp8) {
        if (latent || !decode_fp8_supported(desc->head_dim_qk, desc->head_dim_v, desc->num_kv_heads, desc->num_q_heads / desc->num_kv_heads,
                                            desc->block_size))
            return FNPU_EUNSUPPORTED;
        k_bytes = v_bytes = static_cast<int64_t>(desc->block_size) * desc->num_kv_heads * (desc->head_dim_qk + 4);  // codes, fp32 scales
    } else {
        const int64_t slots = static_cast<int64_t>(desc->block_size) * desc->num_kv_heads;
        k_bytes = 2 * slots * desc->head_dim_qk;
        v_bytes = latent ? 0 : 2 * slots * desc->head_dim_v;
    }
    if (num_copies == 0 || num_pools == 0) return FNPU_OK;
    if (!copies || misaligned(copies, 4) || !k_pools || (!latent && !v_pools)) return FNPU_EINVAL;
    for (int32_t i = 0; i < num_pools; ++i)
        if (!k_pools[i] || misaligned(k_pools[i], 16) || (!latent && (!v_pools[i] || misaligned(v_pools[i], 16)))) return FNPU_EINVAL;
    CopyArgs a = {};
    const int rc = global_error_address(&a.err);
    if (rc != FNPU_OK) return rc;
    a.copies = copies;
    a.num_copies = num_copies;
    a.num_blocks = desc->num_blocks;
    // one list of pools a size of blocks (K and V differ only where their widths do)
    auto copy = [&](int64_t bytes, bool k, bool v) -> int {
        a.block_bytes = bytes;
        a.pools = 0;
        for (int32_t i = 0; i < num_pools; ++i) {
            if (k) a.pool[a.pools++] = k_pools[i];
            if (v) a.pool[a.pools++] = v_pools[i];
            if (a.pools > kCopyPools - 2 || i == num_pools - 1) {
                const int st = launch_copy_blocks(a, stream);
                if (st != FNPU_OK) return st;
                a.pools = 0;
            }
        }
        return FNPU_OK;
    };
    if (k_bytes == v_bytes || latent) return copy(k_bytes, true, !latent);
    const int st = copy(k_bytes, true, false);
    return st != FNPU_OK ? st : copy(v_bytes, false, true);
}

}  // extern "C"
