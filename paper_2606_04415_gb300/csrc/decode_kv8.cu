// Split-KV attention of few query rows a sequence (one-token decodes, short
// multi-token decodes) over the 8-bit cache with a scale per block and kv head;
// d = 64 or 128, blocks of 16, 32 or 64 slots, any number of query heads a kv head.
//
// Bound by the cache bytes: two operations a byte and query row. An item is a key
// range of one sequence, up to four kv heads and up to 8 (wide: 16) of the q_len x
// G rows of each. The kernel has the structure of the library's other TMA-fed
// decode kernels: persistent CTAs on an atomic queue, one item ahead; a producer
// warp that fills a ring of stages; four compute warps; partial results for the
// merge kernel. What is its own:
//   * A stage is 8 (d = 64: 16) tiles of 16 keys x one kv head, two (four) for each
//     warp, K and V. With four kv heads an item a warp has a head; with two or one,
//     two or four warps share a head and take its tiles in turn, as key parts that
//     write partial results of their own, so that no warp idles on a narrow cache.
//   * Tiles lie in shared memory as rows of d codes, 16-byte chunks swizzled by
//     TMA, and ldmatrix moves them as pairs of codes: read as they are, a lane has
//     four consecutive columns of a key, two f16 operands of S^T = K Q^T (the order
//     of the columns is the query's to follow); read transposed, it has two
//     neighbouring columns of two consecutive keys, two operands of O^T += V^T P^T.
//     So one 32-bit register of codes becomes two f16x2 operands, without a shuffle
//     and whatever the layout: an 8-bit cache needs no transposed copy of V.
//   * Codes are exact in f16. The query is scaled by a power of two per row to the
//     top of the f16 range, so bf16 queries lose nothing of consequence.
//   * The K scale of a tile multiplies its scores. The V scale 2^e goes into the
//     exponent: w = 2^(s + e - m) with m the running maximum of s + e enters P V,
//     and the row sum takes w 2^-e. So w is at most 2^kSlack whatever the scales.
//   * m moves only when a score passes it by more than kSlack: no shuffles for a
//     maximum, and no rescaling of O, in most stages.
// Keys that a row may not see are masked to -inf in S; the V operands of keys
// past the item are set to zero in the tail (stale codes may be NaN).
// Every mbarrier wait is bounded; a timeout raises the plan's error flag, and the
// CTA lets its copies land and exits.
#include <math.h>

#include "kv8.cuh"
#include "tc.cuh"

namespace fnpu {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * (kWarps + 1);  // + the producer warp
constexpr int kKeys = 16;                    // keys of a tile
constexpr int kRing = 8;                     // item ring: more than stages + 1 entries
constexpr int kMaxStages = 6;
constexpr float kSlack = 8.f;                // weights up to 2^8 before the maximum moves
constexpr float kNoMax = -1e30f;             // below any score; finite, so that a fully masked row is 0, not NaN

template <int D>
struct Cfg {
    static constexpr int kTiles = 256 / D;               // tiles a warp takes from a stage
    static constexpr int kTileBytes = kKeys * D;         // K or V codes of a tile
    static constexpr int kHalf = kWarps * kTiles * kTileBytes;  // K or V of a stage (16 KB)
    static constexpr int kScaleOff = 2 * kHalf;          // 16 bytes of K and of V scales a box
    static constexpr int kStageStride = 2 * kHalf + 1024;
    static_assert(kWarps * kTiles * 32 <= 1024, "a box per tile when an item has one kv head");
};

struct Kv8Maps {
    CUtensorMap k, v;
};


// rows of a query in f16 times 2^shift: columns 16 kk + 4 t .. + 3 of row `row`
template <int D>
__device__ __forceinline__ float load_q(const AttnParams &p, int token, int head, bool valid, int t4, uint32_t (&qb)[D / 16][2]) {
    const __nv_bfloat16 *row = static_cast<const __nv_bfloat16 *>(p.q) + (static_cast<int64_t>(token) * p.num_q_heads + head) * D;
    uint2 raw[D / 16];
    uint32_t top = 0;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        raw[kk] = valid ? __ldg(reinterpret_cast<const uint2 *>(row + 16 * kk + 4 * t4)) : make_uint2(0u, 0u);
        const uint32_t a = raw[kk].x & 0x7FFF7FFFu, b = raw[kk].y & 0x7FFF7FFFu;
        top = max(max(top, max(a >> 16, a & 0xFFFFu)), max(b >> 16, b & 0xFFFFu));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // magnitude in [2^x, 2^(x + 1)) -> [2^14, 2^15); zero, subnormal and non-finite rows as they are
    const int x = static_cast<int>(top >> 7) - 127;
    const int shift = (top >= 0x7F80u || top < 0x80u) ? 0 : min(14 - x, 126);
    const float up = __uint_as_float(static_cast<uint32_t>(shift + 127) << 23);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        qb[kk][0] = pack_f16x2(__uint_as_float(raw[kk].x << 16) * up, __uint_as_float(raw[kk].x & 0xFFFF0000u) * up);
        qb[kk][1] = pack_f16x2(__uint_as_float(raw[kk].y << 16) * up, __uint_as_float(raw[kk].y & 0xFFFF0000u) * up);
    }
    return __uint_as_float(static_cast<uint32_t>(127 - shift) << 23);
}

// kN: tiles of 8 query rows
template <int D, int kFormat, int kN>
__global__ void __launch_bounds__(kThreads, kN == 1 ? 3 : 2)
    decode_kv8_kernel(const AttnParams p, const __grid_constant__ Kv8Maps maps, const int stages, const int heads_per_item) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t s_base = smem_u32(smem);
    const uint32_t bar_off = stages * C::kStageStride;
    const uint32_t s_bars = s_base + bar_off;
    auto FULL = [&](int s) { return s_bars + 8 * s; };
    auto EMPTY = [&](int s) { return s_bars + 8 * (kMaxStages + s); };
    auto ITEM = [&](int k) { return s_bars + 8 * (2 * kMaxStages + (k & (kRing - 1))); };
    volatile int *ring = reinterpret_cast<int *>(smem + bar_off + 8 * (2 * kMaxStages + kRing));  // [kRing]
    volatile int *abort_flag = ring + kRing;
    int *sched = p.sched + 2;  // the decode work queue: next item, finished CTAs

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int n_items = p.num_ditems;
    pdl_trigger();  // the merge grid may be placed once these CTAs are; it waits for them to finish
    if ((s_base & 1023u) != 0) {  // the swizzled tiles need 1024-byte alignment
        pdl_wait();
        if (tid == 0) atomicOr(p.err, 2);
        return;
    }
    if (tid == 0) {
        for (int s = 0; s < stages; ++s) {
            tc::mbar_init(FULL(s), 1);
            tc::mbar_init(EMPTY(s), kWarps);
        }
        for (int k = 0; k < kRing; ++k) tc::mbar_init(ITEM(k), 1);
        *abort_flag = 0;
        tc::fence_mbar_init();
    }
    if (warp == kWarps && lane == 0) {
        tc::prefetch_tmap(&maps.k);
        tc::prefetch_tmap(&maps.v);
    }
    __syncthreads();
    pdl_wait();  // the kernel before: the step's append, a writer of q, the last run's merge

    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        if (tc::mbar_try_wait(bar, parity)) return true;
        if (*abort_flag) return false;
        if (tc::mbar_wait(bar, parity)) return true;
        *abort_flag = 1;
        atomicOr(p.err, 1);
        return false;
    };
    const int bs = p.block_size, hkv = p.num_kv_heads, G = p.group, Hq = p.num_q_heads;
    const int boxes = kWarps * C::kTiles / heads_per_item;  // 16-key boxes of a full stage
    const int box_keys = boxes * kKeys;
    const int box_heads = min(heads_per_item, hkv);  // (three kv heads leave the fourth warp idle)

    if (warp == kWarps) {
        // ---------------------------------------------------- TMA producer
        const int64_t bytes = kv8::block_bytes(hkv, bs, D);
        const uint8_t *k_pool = static_cast<const uint8_t *>(p.k_cache), *v_pool = static_cast<const uint8_t *>(p.v_cache);
        const int box_bytes = box_heads * C::kTileBytes;
        int st = 0, turn = 0;
        bool ok = true;
        int idx = blockIdx.x;  // the first item without the queue (grid <= items)
        DecodeItem it = p.ditems[idx];
        for (int k = 0; ok; ++k) {
            if (lane == 0) {
                ring[k & (kRing - 1)] = idx < n_items ? idx : -1;
                tc::mbar_arrive(ITEM(k));
            }
            __syncwarp();
            if (idx >= n_items) break;
            int next = 0;
            if (lane == 0) next = static_cast<int>(gridDim.x) + atomicAdd(sched, 1);
            const int32_t *table = p.block_table + static_cast<int64_t>(it.bt_row) * p.bt_stride;
            const int b0 = it.key_begin / bs, blast = (it.key_end - 1) / bs;
            int ids = b0 + lane <= blast ? __ldg(table + b0 + lane) : 0;  // of blocks base .. base + 31
            int base = b0;
            DecodeItem nit{};
            bool have_next = false;
            for (int key = it.key_begin; ok && key < it.key_end; key += box_keys) {
                if (turn > 0 && !wait(EMPTY(st), (turn - 1) & 1)) { ok = false; break; }
                const uint32_t sK = s_base + st * C::kStageStride, sV = sK + C::kHalf, sS = sK + C::kScaleOff;
                const int nb = min(boxes, (it.key_end - key + kKeys - 1) / kKeys);
                tc::mbar_arrive_expect_tx_warp(FULL(st), nb * (2 * box_bytes + 32));
                for (int b = 0; b < nb; ++b) {
                    const int key0 = key + b * kKeys, j = key0 / bs;
                    int blk;
                    if (j - b0 < 4) {  // from the item itself: the lanes' loads may still be in flight
                        blk = j == b0 ? it.blk[0] : j == b0 + 1 ? it.blk[1] : j == b0 + 2 ? it.blk[2] : it.blk[3];
                    } else {
                        if (j >= base + 32) {
                            base = j;
                            ids = base + lane <= blast ? __ldg(table + base + lane) : 0;
                        }
                        blk = __shfl_sync(0xffffffffu, ids, j - base);
                    }
                    const int64_t scales = blk * bytes + static_cast<int64_t>(hkv) * bs * D + 4 * it.kvh;
                    tc::tma_load_4d_warp(sK + b * box_bytes, &maps.k, FULL(st), 0, key0 - j * bs, it.kvh, blk);
                    tc::tma_load_4d_warp(sV + b * box_bytes, &maps.v, FULL(st), 0, key0 - j * bs, it.kvh, blk);
                    tc::bulk_load_warp(sS + 32 * b, k_pool + scales, 16, FULL(st));
                    tc::bulk_load_warp(sS + 32 * b + 16, v_pool + scales, 16, FULL(st));
                }
                if (!have_next) {  // the next item's descriptor, while this item's stages go out
                    have_next = true;
                    next = __shfl_sync(0xffffffffu, next, 0);
                    if (next < n_items) nit = p.ditems[next];
                }
                if (++st == stages) { st = 0; ++turn; }
            }
            idx = next;
            it = nit;
        }
    } else {
        // ------------------------------------------------------- compute warps
        const int g8 = lane >> 2, t4 = lane & 3;
        const int parts = kWarps / heads_per_item, hl = warp % heads_per_item, part = warp / heads_per_item;
        // ldmatrix: lane l gives row l mod 16 (keys 0-7, then 8-15), chunk l / 16 of a pair
        const int lrow = lane & 15;
        const int swz = D == 128 ? lrow & 7 : (lrow >> 1) & 3;
        const uint32_t lofs = lrow * D + (((lane >> 4) ^ swz) << 4);  // chunk 2 i of it: lofs ^ 32 i
        int st = 0, turn = 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            if (!wait(ITEM(k), (k / kRing) & 1)) break;
            const int idx = ring[k & (kRing - 1)];
            if (idx < 0) break;
            const DecodeItem it = p.ditems[idx];
            const int kvh = it.kvh + hl;
            const bool has_head = kvh < hkv;
            const int rows = it.q_len * G;
            float o[kN][D / 16][4], m[kN][2], l[kN][2], qs[kN][2];
            int lim[kN][2];  // keys that the row may see
            uint32_t qb[kN][D / 16][2];
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                const int row = it.row_begin + 8 * n + g8;
                const float down = load_q<D>(p, it.q_start + row / G, kvh * G + row % G, has_head && row < rows, t4, qb[n]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    qs[n][e] = __shfl_sync(0xffffffffu, down, 4 * (2 * t4 + e)) * p.scale_log2;
                    const int col = min(it.row_begin + 8 * n + 2 * t4 + e, rows - 1);
                    lim[n][e] = min(it.key_end, it.group - it.q_len + col / G + 1);
                    m[n][e] = kNoMax;
                    l[n][e] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
            }
            const int all_see = min(it.key_end, it.group - it.q_len + 1);  // keys below it every row sees
            const bool two = kN > 1 && it.row_begin + 8 < rows;            // the second row tile is not empty
            for (int key = it.key_begin; key < it.key_end; key += box_keys) {
                if (!wait(FULL(st), turn & 1)) { ok = false; break; }
                const uint32_t sK = s_base + st * C::kStageStride;
                const float *scales = reinterpret_cast<const float *>(smem + st * C::kStageStride + C::kScaleOff) + hl;
                if (has_head) {
#pragma unroll
                    for (int i = 0; i < C::kTiles; ++i) {
                        const int box = part + i * parts, key0 = key + box * kKeys;
                        if (key0 >= it.key_end) break;
                        const uint32_t tK = sK + (box * box_heads + hl) * C::kTileBytes, tV = tK + C::kHalf;
                        const float ks = kv8::pow2(kv8::scale_exp(scales[8 * box]));
                        const int ve = kv8::scale_exp(scales[8 * box + 4]);
                        float s[kN][4];
#pragma unroll
                        for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t r0, r1, r2, r3;  // keys 0-7 and 8-15 of chunk 2 c, then of chunk 2 c + 1
                            ldmatrix_x4(r0, r1, r2, r3, tK + (lofs ^ 32 * c));
                            const uint32_t a0 = kv8::codes_f16x2<kFormat, 0, 1>(r0), a1 = kv8::codes_f16x2<kFormat, 0, 1>(r1);
                            const uint32_t a2 = kv8::codes_f16x2<kFormat, 2, 3>(r0), a3 = kv8::codes_f16x2<kFormat, 2, 3>(r1);
                            const uint32_t b0 = kv8::codes_f16x2<kFormat, 0, 1>(r2), b1 = kv8::codes_f16x2<kFormat, 0, 1>(r3);
                            const uint32_t b2 = kv8::codes_f16x2<kFormat, 2, 3>(r2), b3 = kv8::codes_f16x2<kFormat, 2, 3>(r3);
#pragma unroll
                            for (int n = 0; n < kN; ++n) {
                                if (n > 0 && !two) continue;
                                mma_f16_16816(s[n], a0, a1, a2, a3, qb[n][2 * c][0], qb[n][2 * c][1]);
                                mma_f16_16816(s[n], b0, b1, b2, b3, qb[n][2 * c + 1][0], qb[n][2 * c + 1][1]);
                            }
                        }
                        const bool tail = key0 + kKeys > all_see;
                        const float vef = static_cast<float>(ve), vinv = kv8::pow2(-ve);
                        uint32_t pb[kN][2];
#pragma unroll
                        for (int n = 0; n < kN; ++n) {
                            if (n > 0 && !two) continue;
                            float x[4];
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const float f = ks * qs[n][e];
                                x[e] = __fmaf_rn(s[n][e], f, vef);
                                x[e + 2] = __fmaf_rn(s[n][e + 2], f, vef);
                                if (tail) {
                                    if (key0 + g8 >= lim[n][e]) x[e] = -INFINITY;
                                    if (key0 + g8 + 8 >= lim[n][e]) x[e + 2] = -INFINITY;
                                }
                            }
                            float t0 = fmaxf(x[0], x[2]), t1 = fmaxf(x[1], x[3]);
                            if (__any_sync(0xffffffffu, t0 > m[n][0] + kSlack || t1 > m[n][1] + kSlack)) {
#pragma unroll
                                for (int d = 4; d < 32; d *= 2) {
                                    t0 = warp_max_xor(t0, d);
                                    t1 = warp_max_xor(t1, d);
                                }
                                const float m0 = fmaxf(m[n][0], t0), m1 = fmaxf(m[n][1], t1);
                                const float al0 = fast_exp2(m[n][0] - m0), al1 = fast_exp2(m[n][1] - m1);
                                m[n][0] = m0;
                                m[n][1] = m1;
                                l[n][0] *= al0;
                                l[n][1] *= al1;
#pragma unroll
                                for (int j = 0; j < D / 16; ++j) {
                                    o[n][j][0] *= al0; o[n][j][1] *= al1; o[n][j][2] *= al0; o[n][j][3] *= al1;
                                }
                            }
                            const float p0 = fast_exp2(x[0] - m[n][0]), p1 = fast_exp2(x[1] - m[n][1]);
                            const float p2 = fast_exp2(x[2] - m[n][0]), p3 = fast_exp2(x[3] - m[n][1]);
                            l[n][0] = __fmaf_rn(p0 + p2, vinv, l[n][0]);
                            l[n][1] = __fmaf_rn(p1 + p3, vinv, l[n][1]);
                            pb[n][0] = movmatrix_trans(pack_f16x2(p0, p1));
                            pb[n][1] = movmatrix_trans(pack_f16x2(p2, p3));
                        }
                        const int nv = it.key_end - key0;  // V of keys past the item is zero
                        const bool cut = nv < kKeys;
                        const uint32_t lo = (2 * t4 < nv ? 0xFFFFu : 0u) | (2 * t4 + 1 < nv ? 0xFFFF0000u : 0u);
                        const uint32_t hi = (2 * t4 + 8 < nv ? 0xFFFFu : 0u) | (2 * t4 + 9 < nv ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t r[4];
                            ldmatrix_x4_trans(r[0], r[1], r[2], r[3], tV + (lofs ^ 32 * c));
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                uint32_t a0 = kv8::codes_f16x2<kFormat, 0, 2>(r[2 * h]), a1 = kv8::codes_f16x2<kFormat, 1, 3>(r[2 * h]);
                                uint32_t a2 = kv8::codes_f16x2<kFormat, 0, 2>(r[2 * h + 1]),
                                         a3 = kv8::codes_f16x2<kFormat, 1, 3>(r[2 * h + 1]);
                                if (cut) { a0 &= lo; a1 &= lo; a2 &= hi; a3 &= hi; }
#pragma unroll
                                for (int n = 0; n < kN; ++n) {
                                    if (n > 0 && !two) continue;
                                    mma_f16_16816(o[n][2 * c + h], a0, a1, a2, a3, pb[n][0], pb[n][1]);
                                }
                            }
                        }
                    }
                }
                __syncwarp();
                tc::mbar_arrive_warp(EMPTY(st));
                if (++st == stages) { st = 0; ++turn; }
            }
            if (!ok) break;
            if (!has_head) continue;
            // O^T: rows g8, g8 + 8 of tile i are columns 16 i + 2 g8, + 1; columns of it are query rows
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                if (n > 0 && !two) continue;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float sum = l[n][e];
                    sum += __shfl_xor_sync(0xffffffffu, sum, 4);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
                    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
                    const int row = it.row_begin + 8 * n + 2 * t4 + e;
                    if (row >= rows) continue;
                    // (a part that saw no key of the row: weight zero in the merge)
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    const float lse = m[n][e] + log2f(sum);
                    const int tok = row / G, head = kvh * G + row % G;
                    if (it.num_splits == 1) {
                        const int64_t at = static_cast<int64_t>(it.q_start + tok) * Hq + head;
                        __nv_bfloat16 *r = static_cast<__nv_bfloat16 *>(p.out) + at * D + 2 * g8;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i)
                            *reinterpret_cast<uint32_t *>(r + 16 * i) = pack_bf16x2(o[n][i][e] * inv, o[n][i][e + 2] * inv);
                        if (g8 == 0) p.lse[at] = lse * kLn2;
                    } else {
                        const int64_t at = static_cast<int64_t>(it.part_base + tok * it.num_splits + it.split + part) * Hq + head;
                        float *r = p.part_o + at * D + 2 * g8;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i)
                            *reinterpret_cast<float2 *>(r + 16 * i) = make_float2(o[n][i][e] * inv, o[n][i][e + 2] * inv);
                        if (g8 == 0) p.part_lse[at] = lse;
                    }
                }
            }
        }
    }

    __syncthreads();
    if (*abort_flag && warp == kWarps) tc::drain_copies(FULL(0), stages);
    if (tid == 0) {  // the last CTA out resets the work queue for the next run
        __threadfence();
        if (atomicAdd(sched + 1, 1) == static_cast<int>(gridDim.x) - 1) {
            sched[0] = 0;
            sched[1] = 0;
            __threadfence();
        }
    }
}

// codes [blocks][kv heads][slots][d]: a box is d columns, 16 slots, the item's kv
// heads (past the last: zeros), one block
bool encode_map(CUtensorMap *m, const void *base, int d, int hkv, int bs, int nblocks, int heads) {
    EncodeTiledFn enc = tensor_map_encoder();
    if (!enc) return false;
    cuuint64_t dims[4] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(bs), static_cast<cuuint64_t>(hkv),
                          static_cast<cuuint64_t>(nblocks)};
    cuuint64_t strides[3] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(bs) * d,
                             static_cast<cuuint64_t>(kv8::block_bytes(hkv, bs, d))};
    cuuint32_t box[4] = {static_cast<cuuint32_t>(d), kKeys, static_cast<cuuint32_t>(heads), 1};
    cuuint32_t es[4] = {1, 1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int kFormat, int kN>
int launch(const AttnParams &p, cudaStream_t st, int max_ctas, bool alone) {
    auto kernel = decode_kv8_kernel<D, kFormat, kN>;
    const int heads = kv8_heads_per_item(p.num_kv_heads);
    const int box_heads = heads < p.num_kv_heads ? heads : p.num_kv_heads;
    Kv8Maps maps;
    if (!encode_map(&maps.k, p.k_cache, D, p.num_kv_heads, p.block_size, p.num_blocks, box_heads) ||
        !encode_map(&maps.v, p.v_cache, D, p.num_kv_heads, p.block_size, p.num_blocks, box_heads))
        return cuda_fail(cudaErrorInvalidValue, "cuTensorMapEncodeTiled (8-bit decode)");
    // An SM's shared memory holds six stages: all of them in flight however many
    // CTAs it has.
    const int sms = max_ctas / 3;
    const int ctas = kN == 1 ? max_ctas : 2 * sms;
    const int grid = p.num_ditems < ctas ? p.num_ditems : ctas;
    const int stages = !alone ? 2 : grid <= sms ? 6 : (kN > 1 || grid <= 2 * sms) ? 3 : 2;
    const size_t bytes = static_cast<size_t>(stages) * Cfg<D>::kStageStride + 8 * (2 * kMaxStages + kRing) + 4 * (kRing + 1);
    FNPU_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       6 * Cfg<D>::kStageStride + 8 * (2 * kMaxStages + kRing) + 4 * (kRing + 1)));
    FNPU_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    FNPU_CUDA_TRY(launch_ex(kernel, grid, kThreads, bytes, st, alone, nullptr, p, maps, stages, heads));
    return launch_split_merge(p, st);
}

template <int D, int kFormat>
int launch(const AttnParams &p, bool wide, cudaStream_t st, int max_ctas, bool alone) {
    return wide ? launch<D, kFormat, 2>(p, st, max_ctas, alone) : launch<D, kFormat, 1>(p, st, max_ctas, alone);
}

}  // namespace

int kv8_heads_per_item(int hkv) { return hkv == 1 ? 1 : hkv == 2 ? 2 : kWarps; }
int kv8_rows_per_item(bool wide) { return wide ? 16 : 8; }

int launch_decode_kv8(int format, const AttnParams &p, bool wide, void *stream, int max_ctas, bool alone) {
    if (p.num_ditems == 0) return FNPU_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (format == FNPU_KV_INT8_BLOCK)
        return p.head_dim_qk == 64 ? launch<64, FNPU_KV_INT8_BLOCK>(p, wide, st, max_ctas, alone)
                                   : launch<128, FNPU_KV_INT8_BLOCK>(p, wide, st, max_ctas, alone);
    return p.head_dim_qk == 64 ? launch<64, FNPU_KV_E4M3_BLOCK>(p, wide, st, max_ctas, alone)
                               : launch<128, FNPU_KV_E4M3_BLOCK>(p, wide, st, max_ctas, alone);
}

}  // namespace fnpu
