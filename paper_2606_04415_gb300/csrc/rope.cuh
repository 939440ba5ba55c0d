// Rotary positions: angles, and the rotation of eight column pairs of a bf16
// row held in two 16-byte chunks.
#pragma once

#include "common.cuh"

namespace fnpu {

// Angles. angle = position * inv_freq wants more than 32 bits: at position
// 100000 the rounded product alone is up to 0.004 rad off. In turns (angle / 2 pi)
// only the fraction counts, so inv_freq / 2 pi is kept as a sum of two fp32 values
// (48 bits) and the product's whole turns are dropped before anything small is
// added. What is left is good to 2^-24 turns for positions below 2^20, and is 0.52
// turns at most there (0.71 up to 2^24). A position beyond 2^24 is cut into two parts
// that fp32 holds exactly; the product's rounding error and the low half's product are
// whole turns themselves there (up to 16 and 14 at 2^31), dropped likewise, so that the
// hardware functions get half a turn. The angle is good to 2^-47 of itself.
struct RopeFreq {
    float f, g;  // inv_freq / 2 pi = f + g
    __device__ __forceinline__ explicit RopeFreq(float inv_freq) {
        constexpr float kHi = 0.15915494f, kLo = 6.4206382e-09f;  // kHi + kLo = 1 / (2 pi) to 2^-53
        f = inv_freq * kHi;
        g = __fmaf_rn(inv_freq, kHi, -f) + inv_freq * kLo;
    }
};
__device__ __forceinline__ bool rope_is_far(int32_t position) {  // beyond +-2^24
    return static_cast<uint32_t>(position) + (1u << 24) > 2u << 24;
}
__device__ __forceinline__ float rope_turns(int32_t position, float inv_freq) {
    const RopeFreq q(inv_freq);
    const float p = static_cast<float>(position), t = p * q.f;
    return (t - rintf(t)) + (__fmaf_rn(p, q.f, -t) + p * q.g);
}
__device__ __forceinline__ float rope_turns_any(int32_t position, float inv_freq) {
    if (!rope_is_far(position)) return rope_turns(position, inv_freq);
    const RopeFreq q(inv_freq);
    auto part = [&](float p) {
        const float t = p * q.f, r = __fmaf_rn(p, q.f, -t), u = p * q.g;
        return (t - rintf(t)) + ((r - rintf(r)) + ((u - rintf(u)) + __fmaf_rn(p, q.g, -u)));
    };
    const float s = part(static_cast<float>(position & ~4095)) + part(static_cast<float>(position & 4095));
    return s - rintf(s);
}
// cosine and sine of a turn's fraction (0.71 at most, 0.52 below position 2^20): the
// hardware functions, whose error of some 2^-20 is far below a bf16 result's
__device__ __forceinline__ void rope_cos_sin(float turns, float &c, float &s) {
    const float a = turns * 6.2831853f;
    c = __cosf(a);
    s = __sinf(a);
}

// cosine and sine of pairs W c .. W c + W - 1 at token t (inv_freq is 16-byte aligned)
template <int W>
__device__ __forceinline__ void rope_angles(const RopeArgs &r, int64_t t, int c, float (&cs)[W], float (&sn)[W]) {
    int32_t pos[kRopeMaxAxes];
    bool far = false;
#pragma unroll
    for (int a = 0; a < kRopeMaxAxes; ++a) {
        pos[a] = a < r.axes ? __ldg(r.positions + a * r.n + t) : 0;
        far |= rope_is_far(pos[a]);
    }
    float f[W];
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
        const float4 v = __ldg(reinterpret_cast<const float4 *>(r.inv_freq) + W / 4 * c + i);
        f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
    }
    auto each = [&](auto turns) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            int32_t p = pos[0];
            if (r.axes > 1) {
                const int a = r.axis[W * c + i];
                p = a == 0 ? pos[0] : a == 1 ? pos[1] : a == 2 ? pos[2] : pos[3];
            }
            f[i] = turns(p, f[i]);
        }
    };
    // (one test for all pairs: with one for each, 24000 tokens of 28 heads took 54.4 us in
    // place of 53.8, 3001 tokens on half a head 11.1 and 10.7)
    if (__builtin_expect(far, 0)) each([](int32_t p, float q) { return rope_turns_any(p, q); });
    else each([](int32_t p, float q) { return rope_turns(p, q); });
#pragma unroll
    for (int i = 0; i < W; ++i) {
        rope_cos_sin(f[i], cs[i], sn[i]);
        sn[i] *= r.sign;
    }
}

// W columns of a bf16 row: 16 bytes for eight, 8 for four.
template <int W>
struct RopeChunk;
template <>
struct RopeChunk<8> {
    using Type = uint4;
};
template <>
struct RopeChunk<4> {
    using Type = uint2;
};
template <int W>
__device__ __forceinline__ void bf16_to_f32(const typename RopeChunk<W>::Type &v, float (&f)[W]) {
    const uint32_t *w = reinterpret_cast<const uint32_t *>(&v);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
template <int W>
__device__ __forceinline__ typename RopeChunk<W>::Type f32_to_bf16(const float (&f)[W]) {
    typename RopeChunk<W>::Type v;
    uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
    for (int i = 0; i < W / 2; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    return v;
}

// Where pairs W c .. W c + W - 1 lie: columns col_a .. + W - 1 and col_b .. + W - 1.
template <int W>
__device__ __forceinline__ void rope_columns(const RopeArgs &r, int c, int &col_a, int &col_b) {
    col_a = r.offset + (r.interleaved ? 2 * W * c : W * c);
    col_b = r.interleaved ? col_a + W : col_a + r.pairs;
}

// The two chunks rotated: y1 = x1 cos - x2 sin, y2 = x2 cos + x1 sin in fp32.
// Half-split pairs have x1 in a and x2 in b; interleaved pairs are neighbours.
template <int W>
__device__ __forceinline__ void rope_rotate(bool interleaved, const float (&cs)[W], const float (&sn)[W], float (&a)[W],
                                            float (&b)[W]) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
            a[2 * i] = x * cs[i] - y * sn[i];
            a[2 * i + 1] = y * cs[i] + x * sn[i];
            b[2 * i] = z * cs[i + W / 2] - w * sn[i + W / 2];
            b[2 * i + 1] = w * cs[i + W / 2] + z * sn[i + W / 2];
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * cs[i] - y * sn[i];
            b[i] = y * cs[i] + x * sn[i];
        }
    }
}

// One warp rotates heads [h0, h1) of one or more tokens: src(h) and dst(h) give the rows
// of the calling lane's token (dst null: the head is left out). A lane owns W pairs,
// whose angles it works out once for all its heads, or two chunks that do not turn; the
// lanes of a head lie side by side, and kRopeUnroll passes over the heads are in flight
// per lane. (Rows with more chunks than a warp has lanes, a latent cache's, have those
// that do not turn copied afterwards; such a warp has one token.)
constexpr int kRopeUnroll = 3;
__host__ __device__ __forceinline__ int rope_lanes(int width, int pairs, int d) {  // lanes of a head
    const int turn = pairs / width, rest = ((d - 2 * pairs) / width + 1) >> 1;
    return turn + rest <= 32 ? turn + rest : turn;
}
// A lane's part: its chunk, token and first head, and the heads from pass to pass.
struct RopeLane {
    int chunk, token, head, step;
    bool on;
};
template <bool kMany>
__device__ __forceinline__ RopeLane rope_lane(int lane, int per, int tokens) {
    const int g = lane / per, hp = 32 / per;
    if (!kMany) return {lane - g * per, 0, g, hp, g < hp};
    const int step = hp / tokens, token = g / step;
    return {lane - g * per, token, g - token * step, step, token < tokens};
}
template <int W, class Src, class Dst>
__device__ __forceinline__ void rope_heads(const RopeArgs &r, int64_t t, int h0, int h1, int d, int lane, const RopeLane &my, Src src, Dst dst) {
    using Chunk = typename RopeChunk<W>::Type;
    const int turn = r.pairs / W, chunks = (d - 2 * r.pairs) / W, per = rope_lanes(W, r.pairs, d), hp = my.step, c = my.chunk;
    const bool turns = c < turn;
    auto plain = [&](int j) { return W * j < r.offset ? W * j : W * j + 2 * r.pairs; };
    int ca, cb;
    if (turns) {
        rope_columns<W>(r, c, ca, cb);
    } else {
        ca = plain(2 * (c - turn));
        cb = 2 * (c - turn) + 1 < chunks ? plain(2 * (c - turn) + 1) : ca;
    }
    Chunk a[kRopeUnroll], b[kRopeUnroll];
    auto load = [&](int u, int h) {
        if (h >= h1) return;
        const __nv_bfloat16 *row = src(h);
        a[u] = *reinterpret_cast<const Chunk *>(row + ca);
        b[u] = *reinterpret_cast<const Chunk *>(row + cb);
    };
    if (my.on) {
#pragma unroll
        for (int u = 0; u < kRopeUnroll; ++u) load(u, h0 + my.head + u * hp);
        float cs[W], sn[W];
        if (turns) rope_angles<W>(r, t, c, cs, sn);
        for (int h = h0 + my.head; h < h1; h += kRopeUnroll * hp) {
#pragma unroll
            for (int u = 0; u < kRopeUnroll; ++u) {
                if (h + u * hp >= h1) break;
                __nv_bfloat16 *row = dst(h + u * hp);
                if (turns) {
                    float x[W], y[W];
                    bf16_to_f32<W>(a[u], x);
                    bf16_to_f32<W>(b[u], y);
                    rope_rotate<W>(r.interleaved != 0, cs, sn, x, y);
                    a[u] = f32_to_bf16<W>(x);
                    b[u] = f32_to_bf16<W>(y);
                }
                if (row && (turns || row != src(h + u * hp))) {
                    *reinterpret_cast<Chunk *>(row + ca) = a[u];
                    *reinterpret_cast<Chunk *>(row + cb) = b[u];
                }
                load(u, h + (u + kRopeUnroll) * hp);  // in flight over the next ones
            }
        }
    }
    if (per > turn || chunks == 0) return;
#pragma unroll 4
    for (int i = lane; i < (h1 - h0) * chunks; i += 32) {
        const int h = h0 + i / chunks, col = plain(i % chunks);
        const __nv_bfloat16 *from = src(h);
        __nv_bfloat16 *to = dst(h);
        if (to && to != from) *reinterpret_cast<Chunk *>(to + col) = *reinterpret_cast<const Chunk *>(from + col);
    }
}

}  // namespace fnpu
