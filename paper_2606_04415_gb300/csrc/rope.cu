// Rotary positions on one to four axes, by themselves and on the way into a
// bf16 paged cache.
//
// y1 = x1 cos - x2 sin, y2 = x2 cos + x1 sin for each pair of columns, with the
// angle position[axis(pair)] * inv_freq[pair]; the inverse turns back, which
// is also the gradient (the rotation is orthogonal). Bound by HBM: 4 bytes a
// value against some 5 operations, and an angle costs about 20 instructions but
// serves every head of its token. 24000 tokens of 28 heads of 128: 54 us for 344 MB
// (51 at the copy rate). The append beside it moves 201 MB for 8192 tokens of 32/8
// heads in 37.6 us (30): a warp's chain of loads, angles and stores, at 28 warps an SM.
#include "rope.cuh"

namespace fnpu {
namespace {

// Latency is hidden by warps: 32 an SM for the rotation (64 registers), 28 for the append
// (72, and still 32 bytes of spills a thread, 48 where a warp has several tokens).
constexpr int kWarpsPerCta = 4, kCtasPerSm = 8, kAppendCtasPerSm = 7;
// Passes over the heads of one warp, at most. The rotation by itself is best at 4 for
// some waves (5000 tokens, 28 heads: 13.8 us, 15.4 with 7) and at 8 for many, where the
// angles' work counts (24000 tokens on three axes: 53.7 us, 56.6 with 4); the append,
// whose warps hold value rows too, at 8 (8000 tokens: 27.4 us, 28.9 with 4).
constexpr int kFewPasses = 4, kMostPasses = 8, kManyWaves = 4;
constexpr int kValues = 2;  // chunks of value rows that a lane of the append holds

// A warp per token (kMany: per `tokens` tokens) and group of heads_per_warp heads.
template <int W, bool kMany>
__global__ void __launch_bounds__(32 * kWarpsPerCta, kCtasPerSm)
    rope_kernel(const __grid_constant__ RopeArgs r, const __nv_bfloat16 *x, int64_t x_stride, int heads, int d,
                __nv_bfloat16 *out, int64_t out_stride, int groups, int heads_per_warp, int tokens) {
    pdl_trigger();
    pdl_wait();  // writers of x, earlier readers of out
    const int lane = threadIdx.x & 31;
    const int64_t w = blockIdx.x * static_cast<int64_t>(kWarpsPerCta) + (threadIdx.x >> 5), wt = w / groups;
    const int64_t t0 = kMany ? wt * tokens : wt;
    if (t0 >= r.n) return;
    RopeLane my = rope_lane<kMany>(lane, rope_lanes(W, r.pairs, d), tokens);
    const int64_t t = kMany ? t0 + my.token : t0;
    if (kMany) my.on = my.on && t < r.n;
    const int h0 = static_cast<int>(w - wt * groups) * heads_per_warp;
    rope_heads<W>(r, t, h0, min(heads, h0 + heads_per_warp), d, lane, my,
                  [&](int h) { return x + t * x_stride + static_cast<int64_t>(h) * d; },
                  [&](int h) { return out + t * out_stride + static_cast<int64_t>(h) * d; });
}

// Any even rotary width, offset, stride and alignment: a thread per pair of a
// row, then per column that does not turn. For rows that are off 8 bytes; an angle a pair
// and 2-byte accesses: 24000 tokens of 28 heads of 128 one column off take 310 us (54
// aligned, 51 at the copy rate), 20000 of 8 x 80 49 us.
__global__ void __launch_bounds__(256)
    rope_any_kernel(const __grid_constant__ RopeArgs r, const __nv_bfloat16 *x, int64_t x_stride, int heads, int d,
                    __nv_bfloat16 *out, int64_t out_stride) {
    pdl_trigger();
    pdl_wait();
    const int per = d - r.pairs;  // pairs, then plain columns
    const int64_t total = r.n * heads * per;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
        const int64_t row = i / per, t = row / heads;
        const int j = static_cast<int>(i - row * per), h = static_cast<int>(row - t * heads);
        const __nv_bfloat16 *from = x + t * x_stride + static_cast<int64_t>(h) * d;
        __nv_bfloat16 *to = out + t * out_stride + static_cast<int64_t>(h) * d;
        if (j < r.pairs) {
            float s, c;
            rope_cos_sin(rope_turns_any(r.positions[r.axis[j] * r.n + t], r.inv_freq[j]), c, s);
            s *= r.sign;
            const int a = r.offset + (r.interleaved ? 2 * j : j), b = r.interleaved ? a + 1 : a + r.pairs;
            const float u = __bfloat162float(from[a]), v = __bfloat162float(from[b]);
            to[a] = __float2bfloat16_rn(u * c - v * s);
            to[b] = __float2bfloat16_rn(v * c + u * s);
        } else {
            const int col = j - r.pairs < r.offset ? j - r.pairs : j + r.pairs;
            if (to != from) to[col] = from[col];
        }
    }
}

// The append: the query heads and then the key heads of a token are the heads
// that turn, into q_out and into the token's cache slot; value rows are copied,
// shared out among the warps of the token (kMany: of the `tokens` tokens).
template <bool kMany>
__global__ void __launch_bounds__(32 * kWarpsPerCta, kAppendCtasPerSm)
    rope_append_kernel(const __grid_constant__ RopeArgs r, const __grid_constant__ RopeAppendArgs p, int groups,
                       int heads_per_warp, int tokens) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int64_t w = blockIdx.x * static_cast<int64_t>(kWarpsPerCta) + (threadIdx.x >> 5), wt = w / groups;
    const int64_t t0 = kMany ? wt * tokens : wt;
    if (t0 >= r.n) return;
    const int g = static_cast<int>(w - wt * groups);
    RopeLane my = rope_lane<kMany>(lane, rope_lanes(8, r.pairs, p.d), tokens);
    const int64_t t = kMany ? t0 + my.token : t0;
    if (kMany) my.on = my.on && t < r.n;
    const int64_t slot = !kMany || t < r.n ? __ldg(p.slots + t) : -1;
    const bool stored = slot >= 0 && slot < p.num_slots;
    if (slot >= p.num_slots && g == 0 && (kMany || lane == 0)) atomicOr(p.err, 1);
    // value rows, this warp's share: the first loads are in flight while heads turn
    const int v_row = p.v_new ? p.kv_heads * p.d_v / 8 : 0, v_step = 32 * groups;
    const int v_chunks = kMany ? v_row * static_cast<int>(min(static_cast<int64_t>(tokens), r.n - t0)) : v_row;
    auto v_from = [&](int i) {
        return reinterpret_cast<const uint4 *>(p.v_new + (kMany ? t0 + i / v_row : t) * p.v_stride) + (kMany ? i % v_row : i);
    };
    uint4 v[kValues];
#pragma unroll
    for (int u = 0; u < kValues; ++u) {
        const int i = g * 32 + lane + u * v_step;
        if (i < v_chunks) v[u] = __ldg(v_from(i));
    }
    const int h0 = g * heads_per_warp;
    rope_heads<8>(r, t, h0, min(p.q_heads + p.kv_heads, h0 + heads_per_warp), p.d, lane, my,
               [&](int h) -> const __nv_bfloat16 * {
                   return h < p.q_heads ? p.q + t * p.q_stride + static_cast<int64_t>(h) * p.d
                                        : p.k_new + t * p.k_stride + static_cast<int64_t>(h - p.q_heads) * p.d;
               },
               [&](int h) -> __nv_bfloat16 * {
                   if (h < p.q_heads) return p.q_out + (t * p.q_heads + h) * p.d;
                   return stored ? static_cast<__nv_bfloat16 *>(p.k_cache) + (slot * p.kv_heads + h - p.q_heads) * p.d : nullptr;
               });
    if (!kMany && !stored) return;
    auto v_store = [&](int i, const uint4 &x) {
        const int64_t s = kMany ? __ldg(p.slots + t0 + i / v_row) : slot;
        if (!kMany || (s >= 0 && s < p.num_slots)) reinterpret_cast<uint4 *>(p.v_cache)[s * v_row + (kMany ? i % v_row : i)] = x;
    };
#pragma unroll
    for (int u = 0; u < kValues; ++u) {
        const int i = g * 32 + lane + u * v_step;
        if (i < v_chunks) v_store(i, v[u]);
    }
    for (int i = g * 32 + lane + kValues * v_step; i < v_chunks; i += v_step) v_store(i, __ldg(v_from(i)));
}

int sm_count() {
    int dev = 0, sms = 152;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms;
}

}  // namespace

RopeSplit rope_split(int64_t n, int heads, int width, int pairs, int d, int warps_per_sm, int most_passes, bool many) {
    const int per = rope_lanes(width, pairs, d), hp = 32 / per;
    const int64_t resident = static_cast<int64_t>(warps_per_sm) * sm_count();
    // Few heads: a warp takes several tokens beside each other, so that the angles of
    // a token serve kFewPasses of its heads and no lane is idle, once a warp for each
    // token is more than one and a half waves (4 heads of 80, 100000 tokens: 24.8 us,
    // 64.7 with a token a warp; 9000: 5.0 and 5.8; but 5000 of 4 x 128 4.6 and 4.0).
    int step = hp;
    if (many && 2 * n > 3 * resident && (heads + kFewPasses - 1) / kFewPasses <= hp / 2 &&
        per >= pairs / width + ((d - 2 * pairs) / width + 1) / 2)  // (not where unturned columns have no lane)
        step = (heads + kFewPasses - 1) / kFewPasses;
    const int tokens = hp / step, passes = (heads + step - 1) / step, least = (passes + most_passes - 1) / most_passes;
    // Angles are worked out once per warp, so a warp should have many heads; but a
    // call of few tokens is its longest chain, and there each warp has one pass. In
    // between a token has as many warps as all tokens can have at once: a second
    // wave for the last few costs more than longer warps (28 heads of 128 and their
    // keys into a cache, 2000 tokens: 8.7 us with 2 groups, 10.3 with 3; 1200 tokens:
    // 5.5 with 3, 6.7 with 4). Beyond one wave a warp has most_passes at most; the
    // passes are shared out evenly.
    int64_t groups = resident * tokens / n;
    groups = groups < least ? least : groups > passes ? passes : groups;
    return {step * static_cast<int>((passes + groups - 1) / groups), tokens};
}

int launch_rope(const RopeArgs &r, const void *x, int64_t x_stride, int heads, int d, void *out, int64_t out_stride,
                int width, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const __nv_bfloat16 *xp = static_cast<const __nv_bfloat16 *>(x);
    __nv_bfloat16 *op = static_cast<__nv_bfloat16 *>(out);
    if (width == 1) {
        const int64_t want = (r.n * heads * (d - r.pairs) + 255) / 256;
        const int grid = static_cast<int>(want < 64ll * sm_count() ? want : 64ll * sm_count());
        FNPU_CUDA_TRY(launch_ex(rope_any_kernel, grid, 256, 0, st, true, nullptr, r, xp, x_stride, heads, d, op, out_stride));
        return FNPU_OK;
    }
    constexpr int kWarps = kWarpsPerCta * kCtasPerSm;  // resident on an SM
    const int most = r.n < static_cast<int64_t>(kManyWaves) * kWarps * sm_count() ? kFewPasses : kMostPasses;
    const RopeSplit by = rope_split(r.n, heads, width, r.pairs, d, kWarps, most, true);
    const int groups = (heads + by.heads - 1) / by.heads;
    const int64_t ctas = ((r.n + by.tokens - 1) / by.tokens * groups + kWarpsPerCta - 1) / kWarpsPerCta;
    if (ctas > INT32_MAX) return FNPU_EUNSUPPORTED;
    auto kernel = by.tokens > 1 ? (width == 8 ? rope_kernel<8, true> : rope_kernel<4, true>)
                                : (width == 8 ? rope_kernel<8, false> : rope_kernel<4, false>);
    FNPU_CUDA_TRY(launch_ex(kernel, static_cast<int>(ctas), 32 * kWarpsPerCta, 0, st, true, nullptr, r, xp, x_stride, heads, d, op,
                            out_stride, groups, by.heads, by.tokens));
    return FNPU_OK;
}

int launch_rope_append(const RopeArgs &r, const RopeAppendArgs &p, void *stream) {
    const int heads = p.q_heads + p.kv_heads;
    const RopeSplit by = rope_split(r.n, heads, 8, r.pairs, p.d, kWarpsPerCta * kAppendCtasPerSm, kMostPasses, true);
    const int groups = (heads + by.heads - 1) / by.heads;
    const int64_t ctas = ((r.n + by.tokens - 1) / by.tokens * groups + kWarpsPerCta - 1) / kWarpsPerCta;
    if (ctas > INT32_MAX) return FNPU_EUNSUPPORTED;
    FNPU_CUDA_TRY(launch_ex(by.tokens > 1 ? rope_append_kernel<true> : rope_append_kernel<false>, static_cast<int>(ctas), 32 * kWarpsPerCta,
                            0, static_cast<cudaStream_t>(stream), true, nullptr, r, p, groups, by.heads, by.tokens));
    return FNPU_OK;
}

}  // namespace fnpu
