// Internal structures shared between the host planner and the kernels.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/fnpu.h"

namespace fnpu {

// One decode split item: keys [key_begin, key_end) of sequence `seq` at the
// sequence's single query position, for kv head `kvh` and its G query heads
// (per-head kernel) or for the kv heads [kvh, kvh + 4) below Hkv (TMA kernel). Splits
// of one group share `group` (their merge counter) and write partial results
// to scratch rows part_base + split. The item also carries its sequence's
// query token and block-table row and the ids of its first four blocks, so
// that a kernel can issue its first copies after one load.
// 8-bit block kernel: the item is rows [row_begin, row_begin + the rows that the
// kernel takes) of the q_len x G rows (token, query head of the kv head) of the
// sequence, at most kKv8MaxItemKeys keys; blk[0] is the sequence's context length.
// With a window (TMA kernel): the keys are virtual, row_begin is the number of
// 16-key stages left out behind the sinks, q_len the first key of the window and
// blk[i] the block of the item's stage i.
struct DecodeItem {
    int32_t seq, kvh, key_begin, key_end;
    int32_t split, num_splits, part_base, group;
    int32_t q_start, bt_row, row_begin, q_len;  // (the last two: 8-bit block kernel, see below)
    int32_t blk[4];  // block_table[bt_row][key_begin / bs + i], 0 past the item
};
static_assert(sizeof(DecodeItem) == 64, "DecodeItem layout");

// One prefill tile: query rows [row_begin, row_begin + rows) of sequence
// `seq`'s chunk for query head `head` (the mma.sync path) or for kv head
// `head` with all its query heads packed (the tcgen05 path). The tcgen05 path
// may split the keys of a tile: the item then covers 64-key tiles
// [kt_begin, kt_end) only, writes its partial result to scratch row
// part_base + split and the last split of the tile to finish (merge counter
// `group`) combines all num_splits of them. Unsplit items have
// num_splits == 1 and cover every key their rows can see.
struct PrefillItem {
    int32_t seq, head, row_begin, rows;
    int32_t kt_begin, kt_end, split, num_splits;
    int32_t part_base, group;
    int32_t q_start, prefix, ctx_len, bt_row;  // the sequence's SeqInfo, so one load decodes an item
    int32_t dual;  // tcgen05 path: at most one Q tile of rows, its key tiles alternate between the two softmax paths
    int32_t pad0;
};
static_assert(sizeof(PrefillItem) == 64, "PrefillItem layout");

// One latent-attention (MLA) work item: query heads [64 hb, 64 hb + 64) of
// query row `row` of sequence `seq` (a prefill or a decode row alike) over
// keys [key_begin, key_end); splits of one (token, head block) share `group`
// and write partials to scratch rows part_base + split. On the tcgen05 path hb
// is the half of d_v (all 128 heads). The query token and the sequence's
// context length and block-table row come along, so one load decodes an item.
struct MlaItem {
    int32_t seq, row, hb, key_begin;
    int32_t key_end, split, num_splits, part_base;
    int32_t group, token, ctx_len, bt_row;
};
static_assert(sizeof(MlaItem) == 48, "MlaItem layout");

// The key splits of one decode token, merged by a separate kernel (TMA
// decode path): partial rows part_base .. part_base + num_splits - 1.
struct MergeGroup {
    int32_t token, num_splits, part_base, pad;
};
static_assert(sizeof(MergeGroup) == 16, "MergeGroup layout");

// Per-sequence metadata on the device.
struct SeqInfo {
    int32_t q_start;  // first query token of the sequence in q/out/lse
    int32_t q_len;
    int32_t ctx_len;  // includes this step's q_len new tokens
    int32_t bt_row;   // row of the sequence in the device block table
};
static_assert(sizeof(SeqInfo) == 16, "SeqInfo layout");

struct AttnParams {
    const void *q;        // bf16 [T, Hq, dqk]
    const void *k_cache;  // bf16 [nb, bs, Hkv, dqk] (latent: [nb, bs, dqk])
    const void *v_cache;  // bf16 [nb, bs, Hkv, dv]  (latent: == k_cache)
    void *out;            // bf16 [T, Hq, dv]
    float *lse;           // fp32 [T, Hq]
    const SeqInfo *seqs;
    const int32_t *block_table;  // [num_seqs, bt_stride]
    int32_t bt_stride;
    int32_t num_q_heads, num_kv_heads, group, block_size, num_blocks;
    int64_t num_tokens;
    int32_t head_dim_qk, head_dim_v;
    int64_t k_slot_stride;  // elements between consecutive slots of k_cache
    int64_t v_slot_stride;
    float scale_log2;       // softmax scale * log2(e)
    // decode split-KV
    const DecodeItem *ditems;
    int32_t num_ditems;
    float *part_o;          // fp32 [num_parts, group, dv]
    float *part_lse;        // fp32 [num_parts, group] (log2 domain)
    int32_t *counters;      // [num_groups], zero between runs (per-head decode kernel)
    const MergeGroup *mgroups;  // TMA decode path: split tokens to merge after the decode kernel
    int32_t num_mgroups;
    // prefill
    const PrefillItem *pitems;
    int32_t num_pitems;
    int32_t pitems_dual;    // some of them have `dual` set
    float *ppart_o;         // fp32 split-prefill partials, per partial: [2 tiles][dv / 4][128 rows] float4
    float *ppart_lse;       // fp32 [num_pparts, 2, 128] (log2 domain)
    int32_t *pcounters;     // [num_pgroups, 8] one per softmax warp, zero between runs
    // latent attention (MLA): one work list for both phases
    const MlaItem *mitems;
    int32_t num_mitems;
    int32_t *err;           // device error flag of the plan
    int32_t *sched;         // persistent work queues: [0..1] prefill, [2..3] decode (next item, finished CTAs)
    // the step's append of the prefill-path rows inside the tcgen05 prefill
    // (fnpu_mixed_step): fa_count null = none. Tokens fa_tokens[0 .. n) of
    // k_new / v_new go to their slots; a grid-wide count (zero between runs)
    // says when every CTA has written its share.
    const uint4 *fa_k_new;
    const uint4 *fa_v_new;
    const int64_t *fa_slots;
    const int32_t *fa_tokens;
    uint4 *fa_k_cache;
    uint4 *fa_v_cache;
    int32_t *fa_count;
    int *fa_range_err;      // the library-wide error flag (bit 0: a slot past the pool)
    int32_t fa_num_tokens, fa_k_chunks, fa_v_chunks;
    int64_t fa_num_slots;
    // decode without a plan (one query row per sequence): context lengths on
    // the device, the host's bound on them, keys per split and the splits that
    // bound allows; err is the library-wide flag (bit 1: out of range, bit 2:
    // a wait that gave up)
    const int32_t *na_ctx;
    int32_t na_num_seqs, na_max_ctx, na_split, na_max_splits;
    // sliding window (0: none): a query at position p sees keys p - window + 1 .. p
    // and those below `sinks`; sink_keys: sinks up to a whole stage or key tile
    int32_t window, sinks, sink_keys;
};

// Rotation of column pairs: pair i of a row turns by positions[axis[i]][t] *
// inv_freq[i]; sign -1 turns back.
constexpr int kRopeMaxAxes = 4;
constexpr int kRopeMaxPairs = 128;
struct RopeArgs {
    const float *inv_freq;     // [pairs]
    const int32_t *positions;  // [axes, n]
    int64_t n;                 // tokens
    int32_t pairs, offset, interleaved, axes;
    float sign;
    uint8_t axis[kRopeMaxPairs];
};

// Rows of an append: queries and keys may turn (RopeArgs), keys and values go to
// their slots. Strides in elements between tokens; q null: no queries.
struct RopeAppendArgs {
    const __nv_bfloat16 *q, *k_new, *v_new;
    int64_t q_stride, k_stride, v_stride;
    const int64_t *slots;
    __nv_bfloat16 *q_out;
    void *k_cache, *v_cache;  // v_new, v_cache null: a latent cache
    int64_t num_slots;
    int32_t q_heads, kv_heads, d, d_v, block_size;
    int *err;                 // the library-wide error flag
};

// Selection of a beam search: rows of logits (groups x beams), each in `slices`
// pieces; parts: (maximum, sum of exp(x - maximum)) of each, keys: its best `select`.
struct BeamArgs {
    const void *logits;
    int64_t stride;  // values between rows
    const float *scores;
    const uint8_t *finished;  // may be null
    float2 *parts;
    uint64_t *keys;
    float *out_scores;
    int32_t *out_parents, *out_tokens;
    int32_t groups, beams, vocab, select, end_token, slices;
};
int beam_slices(const fnpu_beam_desc *d);
int launch_beam_select(const BeamArgs &a, bool fp32, void *stream);

// Page operations (pages.cu); see fnpu.h. Workspace pieces are laid out by the host.
constexpr int32_t kPagesChunk = 2048;    // counts that a CTA looks through at a time
constexpr int32_t kPagesMostChunks = 2048;
constexpr int32_t kPagesMaxRows = 8192;
struct PagesArgs {
    int32_t *table;             // rows x width (fork: the old one, read only)
    const int32_t *length;
    const int32_t *parents;     // may be null: row r continues row r
    int32_t *refs;
    int32_t *new_table, *new_length, *copies, *stats, *remap;
    int64_t *slots;
    // workspace: live blocks of each chunk; of each new row: length, last page if
    // partly filled (-1: none, -2: the row cannot grow), its count; of each block: rows
    // whose last page it is, the lowest of them (fork) or the free and moving blocks' places (compact)
    int32_t *chunk_count, *row_length, *row_tail, *row_refs, *block_a, *block_b;
    int *err;                   // the library-wide error flag
    int32_t block_size, num_blocks, rows, width, new_rows, grow, max_copies, chunks, chunk;
};
int launch_pages_free(const PagesArgs &a, int32_t *length, const uint8_t *ends, int32_t window, int32_t sinks, void *stream);
int launch_pages_fork(const PagesArgs &a, void *stream);
int launch_pages_compact(const PagesArgs &a, void *stream);
constexpr int kCopyPools = 128;  // pools of one launch: K and V of 64 layers
struct CopyArgs {
    const int32_t *copies;
    int *err;
    int64_t block_bytes;
    int32_t num_copies, num_blocks, pools;
    void *pool[kCopyPools];
};
int launch_copy_blocks(const CopyArgs &a, void *stream);

// A sliding window (size 0: none): a query at position p sees keys p - size + 1 .. p
// and the first `sinks` of its sequence.
struct Window {
    int32_t size = 0, sinks = 0;
    // the first key of the window of a query at the end of `keys` keys
    int32_t first_key(int32_t keys) const { return size > 0 && keys > size ? keys - size : 0; }
    // the sinks up to a whole tile of `tile` keys
    int32_t sink_keys(int32_t tile) const { return (sinks + tile - 1) / tile * tile; }
};
// The window of a call. Larger windows and sinks see as much, no context being longer; the
// room left is for rounding sinks up and for a tile's distances from its rows, which lie up
// to a tile below zero (2^31 - 1 taken from those would not fit).
constexpr int32_t kMostSeen = INT32_MAX - 1024;
inline Window make_window(int32_t size, int32_t sinks) {
    return Window{size < kMostSeen ? size : kMostSeen, sinks < kMostSeen ? sinks : kMostSeen};
}
// Keys a split for windowed decodes whose items are more than fit the device at once
// (window_api.cu). add(split, f) calls f(items, keys) for all items of `split` keys, then
// for the shorter ones with their mean.
template <typename Add>
int32_t window_heavy_split(int64_t key_bytes, int32_t slots, Add add) {
    // The CTAs of a round start together and share 7 TB/s, one by itself takes 30 GB/s, and a
    // round's start and end are 2 us. A last round with few CTAs is what costs most, and rows
    // under a window all have its length. Over 30 steps of 64 to 300 rows the choice was 1.3% (10% at
    // most) longer than the best of 192 to 1024 keys, where 256 always is 7.8% (23%), and 512 6.2%.
    constexpr double kAll = 7.0e6, kOne = 30e3, kRound = 2.0;  // bytes a us; us
    double least = 0.0;
    int32_t best = 0;
    for (int32_t split : {256, 320, 384, 448, 512, 768, 1024}) {
        double t = 0.0, longest = 0.0, open = 0.0;  // of the round that fills: its longest item, bytes
        int64_t in_round = 0;
        auto close = [&](double rounds) {
            const double all = open / kAll, one = in_round < slots ? longest / kOne : 0.0;
            t += rounds * (kRound + (all > one ? all : one));
            open = longest = 0.0;
            in_round = 0;
        };
        add(split, [&](int64_t items, double keys) {
            const double bytes = keys * static_cast<double>(key_bytes);
            while (items > 0) {
                const bool whole = in_round == 0 && items >= slots;
                const int64_t n = whole ? slots : items < slots - in_round ? items : slots - in_round;
                in_round += n;
                open += static_cast<double>(n) * bytes;
                if (bytes > longest) longest = bytes;
                const int64_t rounds = whole ? items / slots : 1;
                items -= whole ? rounds * slots : n;
                if (in_round == slots) close(static_cast<double>(rounds));
            }
        });
        if (in_round > 0) close(1.0);
        if (best == 0 || t < least) {
            least = t;
            best = split;
        }
    }
    return best;
}
constexpr int kDecodeStageKeys = 16;              // keys of a stage of the TMA decode kernel

// cuTensorMapEncodeTiled, looked up once through the runtime's driver entry
// point (the library does not link the driver library); null if unavailable.
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn tensor_map_encoder();

// Record a failed CUDA call for fnpu_last_cuda_error(); returns FNPU_ECUDA.
int cuda_fail(cudaError_t e, const char *where);
#define FNPU_CUDA_TRY(call)                                   \
    do {                                                      \
        cudaError_t e_ = (call);                              \
        if (e_ != cudaSuccess) return ::fnpu::cuda_fail(e_, #call); \
    } while (0)

// Launchers (defined in the .cu files).
int launch_kv_append(const fnpu_attn_desc *d, const void *k_new, const void *v_new,
                     const int64_t *slots, int32_t num_tokens, void *k_cache, void *v_cache,
                     void *stream);
// the same append for the tokens tokens[0 .. n) of k_new / v_new only
int launch_kv_append_list(const fnpu_attn_desc *d, const void *k_new, const void *v_new, const int64_t *slots,
                          const int32_t *tokens, int32_t n, void *k_cache, void *v_cache, void *stream);
int read_and_clear_global_error(void *stream, int *flag);
// Device address of the library-wide error flag on the current device (looked
// up once per device), for kernels of other translation units that raise it.
int global_error_address(int **out);
// MLA expansion: gather the c parts of latent rows (512 + 64 columns) into ws
// [n, 512] and broadcast their r parts into columns 128..191 of k_out [n, heads, 192]
int launch_mla_gather(const void *latent, const int64_t *slots, int32_t n, int64_t num_slots, int32_t heads,
                      void *ws, void *k_out, void *stream);
// FP8 (e4m3) cache: append (quantising) and decode (split-KV, TMA-fed)
int launch_kv_append_fp8(const fnpu_attn_desc *d, const void *k_new, const void *v_new,
                         const int64_t *slots, int32_t num_tokens, void *k_cache, void *v_cache,
                         void *stream);
// alone: the decode has the device to itself, as a programmatic dependent
// launch of the kernel before it (else it follows events on its own stream)
int launch_decode_fp8(const AttnParams &p, void *stream, int max_ctas, bool alone);
int launch_prefill_fp8(const AttnParams &p, void *stream);
// Staging of the FP8 cache for the tcgen05 prefill: job j dequantises source
// block `src` (valid slots) into f16 block `dst` of k_f16 / v_f16 (plain
// layout [16 slots][4 heads][128]); the queries are converted bf16 -> f16.
struct Fp8StageJob {
    int32_t dst, src, valid, pad;
};
int launch_fp8_stage(const void *k_pool, const void *v_pool, const Fp8StageJob *jobs, int32_t num_jobs, void *k_f16,
                     void *v_f16, const void *q_bf16, void *q_f16, int64_t q_values, void *stream, bool pdl);
// Rotary positions. width: the pairs that may be read together, in chunks of as many
// columns (8: 16 bytes, 4: 8 bytes), or 1: one by one.
int launch_rope(const RopeArgs &r, const void *x, int64_t x_stride, int heads, int d, void *out, int64_t out_stride,
                int width, void *stream);
// The heads and tokens that one warp turns, in a launch of warps_per_sm resident warps.
struct RopeSplit {
    int heads, tokens;
};
RopeSplit rope_split(int64_t n, int heads, int width, int pairs, int d, int warps_per_sm, int most_passes, bool many);
int launch_rope_append(const RopeArgs &r, const RopeAppendArgs &p, void *stream);
// 8-bit cache with a scale for each (block, kv head), format FNPU_KV_INT8_BLOCK or
// FNPU_KV_E4M3_BLOCK: append (turning rows where r.pairs > 0), rows read back as
// bf16, staging of listed blocks as bf16 blocks for the tcgen05 prefill, and the
// split-KV attention of few rows a sequence
bool kv8_supported(const fnpu_attn_desc *d);
int64_t kv8_block_bytes(int hkv, int block_size, int d);
int launch_kv8_append(int format, const RopeArgs &r, const RopeAppendArgs &p, void *stream);
int launch_kv8_read(int format, const fnpu_attn_desc *d, const int64_t *slots, int32_t n, const void *k_pool,
                    const void *v_pool, void *k_out, void *v_out, int *err, void *stream);
int launch_kv_read_bf16(const fnpu_attn_desc *d, const int64_t *slots, int32_t n, const void *k_cache, const void *v_cache,
                        void *k_out, void *v_out, int *err, void *stream);
int launch_kv8_stage(int format, const fnpu_attn_desc *d, const void *k_pool, const void *v_pool, const Fp8StageJob *jobs,
                     int32_t num_jobs, void *k_bf16, void *v_bf16, void *stream, bool pdl);
// (rows: of an item, from kv8_rows_per_item of the largest sequence's)
int launch_decode_kv8(int format, const AttnParams &p, int rows, void *stream, bool alone);
int kv8_rows_per_item(int64_t rows);
constexpr int kKv8MaxItemKeys = 4096;
// Ranges of a sequence that one CTA merges; more are merged in groups first, which
// have a counter each behind the sequence's and a partial result each behind its ranges'.
constexpr int kKv8MergeAtOnce = 12, kKv8MergeGroup = 8;
bool decode_fp8_supported(int d_qk, int d_v, int hkv, int group, int block_size);
int launch_decode_mma(const AttnParams &p, void *stream);
int launch_decode_tma(const AttnParams &p, void *stream, int max_ctas, bool alone);
bool decode_tma_supported(int d_qk, int d_v, int group, int block_size);
int decode_tma_heads_per_item();
// without a plan: p.na_*, num_ditems = sequences x head groups x na_max_splits,
// num_mgroups = sequences, partial rows sequence x na_max_splits + split
int launch_decode_tma_noplan(const AttnParams &p, void *stream, int max_ctas);
// Loads every kernel that launch_decode_tma_noplan may launch on the current
// device: which one follows from the batch, and a first use later could load
// code under a stream capture or where no device memory may be taken.
int prepare_decode_tma_noplan(bool window);
int launch_prefill_mma(const AttnParams &p, void *stream);
int launch_mla(const AttnParams &p, void *stream);
// tcgen05 latent attention: items are (token, d_v half, key range) of 128 heads
int launch_mla_tc(const AttnParams &p, void *stream, int max_ctas);
bool mla_tc_supported(int d_qk, int d_v, int hq, int hkv, int block_size);
int mla_tc_keys_per_tile();
// log-sum-exp merge of the split tokens listed in p.mgroups (partials [part, Hq, dv])
int launch_split_merge(const AttnParams &p, void *stream);
bool mla_supported(int d_qk, int d_v, int hq, int hkv);
int mla_heads_per_item();
// started (a cudaEvent_t, may be null): recorded once every CTA has begun;
// f16: Q, K and V are f16 (d = 128 only), else bf16; pdl: a programmatic
// dependent launch of the kernel before it on `stream`. With p.fa_count set
// the CTAs first write the prefill-path rows of the step (a cooperative
// launch: they wait for one another before reading the cache).
int launch_prefill_tc(const AttnParams &p, void *stream, int max_ctas, void *started = nullptr, bool f16 = false,
                      bool pdl = false);
bool prefill_tc_supported(int d_qk, int d_v, int block_size, int group);
int prefill_tc_rows_per_item(int group);
int prefill_tc_keys_per_tile();

}  // namespace fnpu
