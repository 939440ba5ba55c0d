// Split-KV attention of few query rows a sequence (one-token decodes, short
// multi-token decodes) over the 8-bit cache with a scale per block and kv head;
// d = 64 or 128, blocks of 16, 32 or 64 slots, any number of query heads a kv head.
//
// Bound by the cache bytes: two operations a byte and query row. 256 decodes of
// 500..8000 keys, 8 kv heads: 323 us for 2.2 GB, the copy rate; 64 of 512..4096, 4 kv
// heads: 33 us for 150 MB (22 at the copy rate; a launch's start, its first loads and
// the merge are 8 of them, and SMs end up to 4 apart); with 32 rows an item the chain
// of a tile binds: 75 us where the bytes are 43. A CTA of four warps takes one item: a
// key range of one sequence and kv head, up to 4096 keys, and up to 8, 16 or 32 of
// its q_len x G query rows.
//   * The warps take the range's 16-key tiles in turn, each with a ring of its own
//     that it fills itself by cp.async, and meet at the end of the item only. (The
//     codes of a block and kv head are contiguous, so a tile is a plain copy. Fed by
//     TMA through a producer warp, an SM took 50 GB/s however much was in flight: a
//     bulk copy costs its issuer some 80 ns, and tiles are 2 KB; cp.async reaches 190
//     GB/s an SM, so that few SMs, or the last ones at work, are not slowed down.)
//   * ldmatrix moves codes as pairs: read as they are, a lane has four consecutive
//     columns of a key, two f16 operands of S^T = K Q^T (the order of the columns is
//     the query's to follow); read transposed, it has two neighbouring columns of two
//     consecutive keys, two operands of O^T += V^T P^T. So one 32-bit register of
//     codes becomes two f16x2 operands without a shuffle, and an 8-bit cache needs no
//     transposed copy of V. Codes are exact in f16; the query is scaled by a power
//     of two a row to the top of the f16 range, so bf16 queries lose nothing of
//     consequence.
//   * The K scale of a tile multiplies its scores. The V scale 2^e goes into the
//     exponent: w = 2^(s + e - m) with m the running maximum of s + e enters P V,
//     and the row sum takes w 2^-e. So w is at most 2^kSlack whatever the scales.
//   * m moves only when a score passes it by more than kSlack: no shuffles for a
//     maximum, and no rescaling of O, in most tiles.
//   * The last CTA of a sequence's kv head to finish merges the ranges' partial
//     results, in the order of the ranges: a step is one launch, and its result does
//     not depend on which CTA that was.
// Keys that a row may not see are masked to -inf in S; the V operands of keys
// past the item are set to zero in the tail (stale codes may be NaN).
#include <math.h>

#include "kv8.cuh"

namespace fnpu {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kKeys = 16;                    // keys of a tile
constexpr int kMaxBlocks = kKv8MaxItemKeys / 16;
constexpr float kSlack = 8.f;                // weights up to 2^8 before the maximum moves
constexpr float kNoMax = -1e30f;             // below any score; finite, so that a fully masked row is 0, not NaN

// kN: tiles of 8 query rows that a CTA can take. CTAs on an SM: 4, 3 or 2, by
// registers; the rings share its shared memory.
template <int D, int kN>
struct Cfg {
    static constexpr int kCtas = kN == 1 ? 4 : kN == 2 ? 3 : 2;
    static constexpr int kTileBytes = 2 * kKeys * D;                                   // K, then V
    static constexpr int kSlots = (kN == 1 ? 3 : kN == 2 ? 4 : 6) * (128 / D);         // of a warp's ring
    static constexpr int kRing = kWarps * kSlots * kTileBytes;
    static constexpr int kOStride = D + 8;                                             // floats; staggers the banks
    static constexpr int kOBytes = kWarps * 8 * kN * kOStride * 4;                     // the warps' O, over the ring
    static_assert(kOBytes <= kRing, "the merge buffer lies over the ring");
    static constexpr int kQBytes = kN == 4 ? 32 * D * 2 : 0;                           // (four row tiles: Q in shared memory)
    static constexpr int kQOff = kRing;
    static constexpr int kMetaOff = kQOff + kQBytes;
    static constexpr int kMetaBytes = 3 * 4 * kMaxBlocks + 4 * (2 * kWarps + 1) * 8 * kN + 16;
    static constexpr int kSmem = kMetaOff + kMetaBytes;
};

// Query row in f16 times 2^shift: columns 16 kk + 4 t .. + 3; returns 2^-shift.
template <int D>
__device__ __forceinline__ float load_q(const __nv_bfloat16 *row, bool valid, int t4, uint32_t (&qb)[D / 16][2]) {
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

// A CTA, an item, up to 8 kN rows.
template <int D, int kFormat, int kN>
__global__ void __launch_bounds__(kThreads, Cfg<D, kN>::kCtas) decode_kv8_kernel(const AttnParams p) {
    using C = Cfg<D, kN>;
    extern __shared__ __align__(128) uint8_t smem[];
    const DecodeItem it = p.ditems[blockIdx.x];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3;
    const int bs = p.block_size, sh = 31 - __clz(bs), hkv = p.num_kv_heads, G = p.group, Hq = p.num_q_heads;
    const int rows = it.q_len * G, ctx = it.blk[0];
    int *ids = reinterpret_cast<int *>(smem + C::kMetaOff);
    float *k_scale = reinterpret_cast<float *>(ids + kMaxBlocks), *v_exp = k_scale + kMaxBlocks;
    float *m_sh = v_exp + kMaxBlocks, *l_sh = m_sh + kWarps * 8 * kN;  // [warp][row]
    int *lim_sh = reinterpret_cast<int *>(l_sh + kWarps * 8 * kN);  // [row]: keys that it may see
    int *last_sh = lim_sh + 8 * kN;

    // the item's blocks: metadata of the plan, which the kernel before does not write
    const int b0 = it.key_begin >> sh, nblk = ((it.key_end - 1) >> sh) - b0 + 1;
    for (int j = tid; j < nblk; j += kThreads) ids[j] = __ldg(p.block_table + static_cast<int64_t>(it.bt_row) * p.bt_stride + b0 + j);
    if (tid < 8 * kN) lim_sh[tid] = min(it.key_end, ctx - it.q_len + min(it.row_begin + tid, rows - 1) / G + 1);
    __syncthreads();
    pdl_wait();  // the kernel before: the step's append, a writer of q, this plan's last run

    // ---- the warp's ring
    const int64_t block_bytes = kv8::block_bytes(hkv, bs, D);
    const uint8_t *k_pool = static_cast<const uint8_t *>(p.k_cache), *v_pool = static_cast<const uint8_t *>(p.v_cache);
    const int ntiles = (it.key_end - it.key_begin + kKeys - 1) / kKeys;
    const int mine = (ntiles - warp + kWarps - 1) / kWarps;  // tiles warp, warp + 4, ...
    const uint32_t ring = smem_u32(smem) + warp * C::kSlots * C::kTileBytes;
    // 16-byte chunks of a row are swizzled: by the row for 128-byte rows, by pairs of
    // rows for 64-byte ones, so that eight rows' chunks lie in different banks
    constexpr int kChunks = D / 16, kPerLane = kKeys * kChunks / 32;
    const int crow = lane / kChunks, cc = lane % kChunks;  // this lane copies rows crow + k 32 / kChunks
    const uint32_t cdst = crow * D + ((cc ^ (D == 128 ? crow & 7 : (crow >> 1) & 3)) << 4);
    auto load_tile = [&](int i, uint32_t slot) {
        if (i < mine) {
            const int key = it.key_begin + (warp + kWarps * i) * kKeys, j = key >> sh;
            const int64_t at = ids[j - b0] * block_bytes + (static_cast<int64_t>(it.kvh) * bs + (key & (bs - 1))) * D + 16 * lane;
#pragma unroll
            for (int k = 0; k < kPerLane; ++k) {
                // (d = 128: rows four apart, whose swizzles differ in chunk bit 2)
                const uint32_t dst = slot + (D == 128 ? cdst ^ (64 * (k & 1)) : cdst) + 512 * k;
                cp_async_16(dst, k_pool + at + 512 * k, true);
                cp_async_16(dst + kKeys * D, v_pool + at + 512 * k, true);
            }
        }
        cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < C::kSlots - 1; ++i) load_tile(i, ring + i * C::kTileBytes);

    // ---- scales and the query, while the first tiles come
    for (int j = tid; j < nblk; j += kThreads) {
        const int64_t at = ids[j] * block_bytes + static_cast<int64_t>(hkv) * bs * D + 4 * it.kvh;
        const float ks = __ldg(reinterpret_cast<const float *>(k_pool + at)), vs = __ldg(reinterpret_cast<const float *>(v_pool + at));
        k_scale[j] = kv8::pow2(kv8::scale_exp(ks));
        v_exp[j] = static_cast<float>(kv8::scale_exp(vs));
    }
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p.q);
    uint32_t qb[kN == 4 ? 1 : kN][D / 16][2];
    uint8_t *q_sh = smem + C::kQOff;  // [row tile][column pair c][lane]: 16 bytes, columns 32 c + 4 t4 .. + 3 and + 16
    float o[kN][D / 16][4], m[kN][2], l[kN][2], qs[kN][2];
    auto query = [&](int n, uint32_t(&to)[D / 16][2]) -> float {  // row tile n: operands, and the scale of this lane's row
        const int row = it.row_begin + 8 * n + g8;
        const __nv_bfloat16 *src = q + (static_cast<int64_t>(it.q_start + row / G) * Hq + it.kvh * G + row % G) * D;
        return load_q<D>(src, row < rows, t4, to) * p.scale_log2;
    };
    if constexpr (kN == 4) {  // a row tile each for the four warps, through shared memory
        const float down = query(warp, qb[0]);
        if (t4 == 0) m_sh[8 * warp + g8] = down;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
            *reinterpret_cast<uint4 *>(q_sh + ((warp * (D / 32) + c) * 32 + lane) * 16) =
                make_uint4(qb[0][2 * c][0], qb[0][2 * c][1], qb[0][2 * c + 1][0], qb[0][2 * c + 1][1]);
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < kN; ++n) {
        const float down = kN == 4 ? 0.f : query(n, qb[kN == 4 ? 0 : n]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            qs[n][e] = kN == 4 ? m_sh[8 * n + 2 * t4 + e] : __shfl_sync(0xffffffffu, down, 4 * (2 * t4 + e));
            m[n][e] = mine > 0 ? 0.f : kNoMax;  // (a warp without a tile: nothing)
            l[n][e] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
    }
    __syncthreads();

    // ---- the tiles
    const int all_see = min(it.key_end, ctx - it.q_len + 1);  // keys below it every row sees
    const int lrow = lane & 15;  // ldmatrix: lane l gives row l mod 16 (keys 0-7, then 8-15), chunk l / 16 of a pair
    const uint32_t lofs = lrow * D + (((lane >> 4) ^ (D == 128 ? lrow & 7 : (lrow >> 1) & 3)) << 4);
    int slot = 0, fill = C::kSlots - 1;
    for (int i = 0; i < mine; ++i) {
        cp_async_wait<C::kSlots - 2>();
        __syncwarp();  // every lane's copies of tile i are there, and every lane is done with tile i - 1
        load_tile(i + C::kSlots - 1, ring + fill * C::kTileBytes);
        fill = slot;
        const uint32_t tK = ring + slot * C::kTileBytes, tV = tK + kKeys * D;
        slot = slot + 1 == C::kSlots ? 0 : slot + 1;
        float s[kN][4];
        const int key = it.key_begin + (warp + kWarps * i) * kKeys, j = (key >> sh) - b0;
        const float ks = k_scale[j], vef = v_exp[j];
#pragma unroll
        for (int n = 0; n < kN; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t r[4], a[8];  // keys 0-7 and 8-15 of chunk 2 c, then of chunk 2 c + 1
            ldmatrix_x4(r[0], r[1], r[2], r[3], tK + (lofs ^ 32 * c));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                kv8::codes_to_f16<kFormat, false>(r[2 * h], a[4 * h], a[4 * h + 2]);
                kv8::codes_to_f16<kFormat, false>(r[2 * h + 1], a[4 * h + 1], a[4 * h + 3]);
            }
#pragma unroll
            for (int n = 0; n < kN; ++n) {
                uint4 b;
                if constexpr (kN == 4) b = *reinterpret_cast<const uint4 *>(q_sh + ((n * (D / 32) + c) * 32 + lane) * 16);
                else b = make_uint4(qb[n][2 * c][0], qb[n][2 * c][1], qb[n][2 * c + 1][0], qb[n][2 * c + 1][1]);
                mma_f16_16816(s[n], a[0], a[1], a[2], a[3], b.x, b.y);
                mma_f16_16816(s[n], a[4], a[5], a[6], a[7], b.z, b.w);
            }
        }
        const bool tail = key + kKeys > all_see;
        const float vinv = kv8::pow2(static_cast<int>(-vef));
        // s becomes s + e - m; the first tile sets m (of 0 until then)
        bool moves = i == 0;
#pragma unroll
        for (int n = 0; n < kN; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float f = ks * qs[n][e], c = vef - m[n][e];
                s[n][e] = __fmaf_rn(s[n][e], f, c);
                s[n][e + 2] = __fmaf_rn(s[n][e + 2], f, c);
                if (__builtin_expect(tail, 0)) {  // keys that the row may see
                    const int lim = lim_sh[8 * n + 2 * t4 + e] - key;
                    if (g8 >= lim) s[n][e] = -INFINITY;
                    if (g8 + 8 >= lim) s[n][e + 2] = -INFINITY;
                }
                moves |= fmaxf(s[n][e], s[n][e + 2]) > kSlack;
            }
        if (__builtin_expect(__any_sync(0xffffffffu, moves), 0)) {
#pragma unroll
            for (int n = 0; n < kN; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = fmaxf(s[n][e], s[n][e + 2]);
                    t = warp_max_xor(t, 4);
                    t = warp_max_xor(t, 8);
                    t = fmaxf(i == 0 ? kNoMax : 0.f, warp_max_xor(t, 16));
                    const float al = i == 0 ? 0.f : fast_exp2(-t);
                    m[n][e] += t;
                    s[n][e] -= t;
                    s[n][e + 2] -= t;
                    l[n][e] *= al;
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        o[n][d][e] *= al;
                        o[n][d][e + 2] *= al;
                    }
                }
        }
        uint32_t pb[kN][2];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
            const float p0 = fast_exp2(s[n][0]), p1 = fast_exp2(s[n][1]), p2 = fast_exp2(s[n][2]), p3 = fast_exp2(s[n][3]);
            l[n][0] = __fmaf_rn(p0 + p2, vinv, l[n][0]);
            l[n][1] = __fmaf_rn(p1 + p3, vinv, l[n][1]);
            pb[n][0] = movmatrix_trans(pack_f16x2(p0, p1));
            pb[n][1] = movmatrix_trans(pack_f16x2(p2, p3));
        }
        const int nv = it.key_end - key;  // V of keys past the item is zero
        const bool cut = nv < kKeys;
        const uint32_t lo = (2 * t4 < nv ? 0xFFFFu : 0u) | (2 * t4 + 1 < nv ? 0xFFFF0000u : 0u);
        const uint32_t hi = (2 * t4 + 8 < nv ? 0xFFFFu : 0u) | (2 * t4 + 9 < nv ? 0xFFFF0000u : 0u);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t r[4];
            ldmatrix_x4_trans(r[0], r[1], r[2], r[3], tV + (lofs ^ 32 * c));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t a0, a1, a2, a3;
                kv8::codes_to_f16<kFormat, true>(r[2 * h], a0, a1);
                kv8::codes_to_f16<kFormat, true>(r[2 * h + 1], a2, a3);
                if (__builtin_expect(cut, 0)) { a0 &= lo; a1 &= lo; a2 &= hi; a3 &= hi; }
#pragma unroll
                for (int n = 0; n < kN; ++n) mma_f16_16816(o[n][2 * c + h], a0, a1, a2, a3, pb[n][0], pb[n][1]);
            }
        }
    }

    // ---- the warps' results together, through shared memory
    cp_async_wait<0>();
    pdl_trigger();  // the next kernel's CTAs may be placed and read the plan
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float sum = l[n][e];
            sum += __shfl_xor_sync(0xffffffffu, sum, 4);
            sum += __shfl_xor_sync(0xffffffffu, sum, 8);
            sum += __shfl_xor_sync(0xffffffffu, sum, 16);
            if (g8 == 0) {
                m_sh[warp * 8 * kN + 8 * n + 2 * t4 + e] = m[n][e];
                l_sh[warp * 8 * kN + 8 * n + 2 * t4 + e] = sum;
            }
        }
    __syncthreads();  // (also: every warp is done with its ring)
    float *o_sh = reinterpret_cast<float *>(smem);  // [warp][row][column]
#pragma unroll
    for (int n = 0; n < kN; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * t4 + e;
            float top = m_sh[r];
#pragma unroll
            for (int w = 1; w < kWarps; ++w) top = fmaxf(top, m_sh[w * 8 * kN + r]);
            const float al = fast_exp2(m[n][e] - top);
            // O^T: rows g8, g8 + 8 of tile i are columns 16 i + 2 g8, + 1
            float *dst = o_sh + (warp * 8 * kN + r) * C::kOStride + 2 * g8;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) *reinterpret_cast<float2 *>(dst + 16 * i) = make_float2(o[n][i][e] * al, o[n][i][e + 2] * al);
        }
    __syncthreads();
    constexpr int kCol = D / 8, kPass = kThreads / kCol;  // a thread has 8 columns of a row
    const int col = tid % kCol * 8;
    auto store_part = [&](int64_t part, int r, const float (&f)[8], float lse) {
        float4 *dst = reinterpret_cast<float4 *>(p.part_o + (part * 8 * kN + r) * D + col);
        __stcg(dst, make_float4(f[0], f[1], f[2], f[3]));
        __stcg(dst + 1, make_float4(f[4], f[5], f[6], f[7]));
        if (col == 0) __stcg(p.part_lse + part * 8 * kN + r, lse);
    };
    auto store_row = [&](int r, const float (&f)[8], float lse) {
        const int row = it.row_begin + r;
        const int64_t at = static_cast<int64_t>(it.q_start + row / G) * Hq + it.kvh * G + row % G;
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.out) + at * D + col) =
            make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
        if (col == 0) p.lse[at] = lse * kLn2;
    };
    for (int r = tid / kCol; r < 8 * kN && it.row_begin + r < rows; r += kPass) {
        float top = m_sh[r], sum = 0.f, f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 1; w < kWarps; ++w) top = fmaxf(top, m_sh[w * 8 * kN + r]);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            sum += l_sh[w * 8 * kN + r] * fast_exp2(m_sh[w * 8 * kN + r] - top);
            const float4 *src = reinterpret_cast<const float4 *>(o_sh + (w * 8 * kN + r) * C::kOStride + col);
            const float4 a = src[0], b = src[1];
            f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w;
            f[4] += b.x; f[5] += b.y; f[6] += b.z; f[7] += b.w;
        }
        // (no key of the range is visible to the row: weight zero in the merge)
        const float inv = sum == 0.f ? 0.f : 1.f / sum, lse = top + log2f(sum);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= inv;
        if (it.num_splits == 1) {
            store_row(r, f, lse);
        } else {
            store_part(it.part_base + it.split, r, f, lse);
        }
    }
    if (it.num_splits == 1) return;

    // ---- the last CTA of the sequence's kv head and rows merges all ranges; with many
    // of them, the last of each kKv8MergeGroup merges those first. (A row's partial
    // results are 32-byte loads of each thread, eight in flight: one CTA that merged all
    // 76 ranges of a 100000-key sequence took some 10 us.)
    auto is_last = [&](int counter, int count) -> bool {
        // the barrier orders every thread's partial results before thread 0's count, and
        // its acquire-release those of other CTAs before what this one reads next
        __syncthreads();
        if (tid == 0) {
            int n;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;\n" : "=r"(n) : "l"(p.counters + counter) : "memory");
            *last_sh = n == count - 1;
            if (n == count - 1) p.counters[counter] = 0;  // zero for the next run
        }
        __syncthreads();
        return *last_sh != 0;
    };
    auto merge = [&](int64_t first, int count, int r, float (&f)[8]) -> float {
        const float *lse = p.part_lse + first * 8 * kN + r;
        const float *src = p.part_o + (first * 8 * kN + r) * D + col;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int c = 0; c < 8; ++c) f[c] = 0.f;
        for (int s0 = 0; s0 < count; s0 += kKv8MergeGroup) {
            float x[kKv8MergeGroup], t = top;
            float4 a[kKv8MergeGroup], b[kKv8MergeGroup];
#pragma unroll
            for (int u = 0; u < kKv8MergeGroup; ++u) {
                const bool in = s0 + u < count;
                x[u] = in ? __ldcg(lse + (s0 + u) * 8 * kN) : -INFINITY;
                const float4 *at = reinterpret_cast<const float4 *>(src + static_cast<int64_t>(in ? s0 + u : s0) * 8 * kN * D);
                a[u] = __ldcg(at);
                b[u] = __ldcg(at + 1);
            }
#pragma unroll
            for (int u = 0; u < kKv8MergeGroup; ++u) t = fmaxf(t, x[u]);
            // (the first range of any group has a key that every row sees, but not of the
            // last group where the rows are of several tokens: no weight, no NaN)
            const float base = t == -INFINITY ? 0.f : t, al = fast_exp2(top - base);
            top = t;
            sum *= al;
#pragma unroll
            for (int c = 0; c < 8; ++c) f[c] *= al;
#pragma unroll
            for (int u = 0; u < kKv8MergeGroup; ++u) {
                const float w = fast_exp2(x[u] - base);
                sum += w;
                f[0] = __fmaf_rn(w, a[u].x, f[0]); f[1] = __fmaf_rn(w, a[u].y, f[1]);
                f[2] = __fmaf_rn(w, a[u].z, f[2]); f[3] = __fmaf_rn(w, a[u].w, f[3]);
                f[4] = __fmaf_rn(w, b[u].x, f[4]); f[5] = __fmaf_rn(w, b[u].y, f[5]);
                f[6] = __fmaf_rn(w, b[u].z, f[6]); f[7] = __fmaf_rn(w, b[u].w, f[7]);
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
        for (int c = 0; c < 8; ++c) f[c] *= inv;
        return top + log2f(sum);
    };
    int64_t first = it.part_base;
    int count = it.num_splits;
    if (count > kKv8MergeAtOnce) {
        const int g = it.split / kKv8MergeGroup, at = g * kKv8MergeGroup;
        const int size = min(kKv8MergeGroup, count - at);
        if (!is_last(it.group + 1 + g, size)) return;
        for (int r = tid / kCol; r < 8 * kN && it.row_begin + r < rows; r += kPass) {
            float f[8];
            const float lse = merge(first + at, size, r, f);
            store_part(first + count + g, r, f, lse);
        }
        first += count;  // the groups' results lie behind the ranges'
        count = (count + kKv8MergeGroup - 1) / kKv8MergeGroup;
    }
    if (!is_last(it.group, count)) return;
    for (int r = tid / kCol; r < 8 * kN && it.row_begin + r < rows; r += kPass) {
        float f[8];
        const float lse = merge(first, count, r, f);
        store_row(r, f, lse);
    }
}

template <int D, int kFormat, int kN>
int launch(const AttnParams &p, cudaStream_t st, bool alone) {
    auto kernel = decode_kv8_kernel<D, kFormat, kN>;
    FNPU_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D, kN>::kSmem));
    FNPU_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    FNPU_CUDA_TRY(launch_ex(kernel, p.num_ditems, kThreads, Cfg<D, kN>::kSmem, st, alone, nullptr, p));
    return FNPU_OK;
}

template <int D, int kFormat>
int launch(const AttnParams &p, int rows, cudaStream_t st, bool alone) {
    return rows == 8 ? launch<D, kFormat, 1>(p, st, alone) : rows == 16 ? launch<D, kFormat, 2>(p, st, alone) : launch<D, kFormat, 4>(p, st, alone);
}

}  // namespace

int kv8_rows_per_item(int64_t rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : 32; }

int launch_decode_kv8(int format, const AttnParams &p, int rows, void *stream, bool alone) {
    if (p.num_ditems == 0) return FNPU_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (format == FNPU_KV_INT8_BLOCK)
        return p.head_dim_qk == 64 ? launch<64, FNPU_KV_INT8_BLOCK>(p, rows, st, alone) : launch<128, FNPU_KV_INT8_BLOCK>(p, rows, st, alone);
    return p.head_dim_qk == 64 ? launch<64, FNPU_KV_E4M3_BLOCK>(p, rows, st, alone) : launch<128, FNPU_KV_E4M3_BLOCK>(p, rows, st, alone);
}

}  // namespace fnpu
