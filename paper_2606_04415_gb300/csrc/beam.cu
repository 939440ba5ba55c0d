// Selection of a beam search: the best continuations (beam, token) of every
// group of beams, by score[b] + log softmax(logits[b])[v].
//
// What bounds it is the one read of the logits. Two kernels, the second a
// dependent launch of the first:
//   * A CTA of the first takes a slice of a row and leaves its maximum, the sum of
//     exp(x - max) and its best num_select values in order. Within a row the order
//     of the totals is the order of the logits, ties to the lower token, so candidates
//     need no normalisation. A value costs a conversion, half a paired multiply-add,
//     an exponential and half a paired addition, and bf16 maxima go in pairs; a
//     reference that all of a warp's sums share moves only when a tile has a value 2^8
//     above it. Each thread keeps its tiles' maxima in shared memory. Once the slice is
//     read, the K-th largest of the maxima of 64 subsets of it is a bound that K
//     values reach; only the tiles that reach it, some K of them, are read again (from
//     L2) for their values. (A bound that follows the reading, with a list of chunks
//     that reach it, costs more: 512 rows of 151936, 43 us against 37 of this form then, 34 by now.)
//     Slices, chunks and the order of the sums go by token numbers, wherever a row
//     starts in memory: beams with equal logits have equal sums to the last bit.
//   * A CTA of the second takes a group: the rows' log-sum-exps from their slices',
//     then the best of all slices' lists by the total. Totals of different beams
//     may lie closer than an fp32 score of some hundred resolves (3e-5), and fp64 is slow
//     on this device (a warp's instruction takes some 60 cycles), so totals are
//     unevaluated sums of two floats (Dekker 1971), compared as order-preserving integers.
// 512 rows of 151936 in bf16 (140 MB of open beams): 34 us, 4.1 TB/s. Some 8 us of it are what
// the smallest call takes (4 rows of 32000 8.5 us: first loads, the bound, the merge); the
// reading by itself runs at 6 TB/s (rows of 151936 against rows of 32000). Both steps in one kernel,
// a cluster a group with the lists in its first CTA's shared memory, took as long.
#include <float.h>

#include "common.cuh"

namespace fnpu {
namespace {

constexpr int kThreads = 256;       // of the first kernel
constexpr int kWarps = kThreads / 32;
constexpr int kLoads = 8;           // 16-byte loads of a lane in a tile, all in flight
constexpr int kGroup = 4;           // of them that are taken together
constexpr int kMergeThreads = 256;  // of the second
constexpr int kSubsets = 64;        // (num_select is at most as many)
constexpr int kMergeSubsets = 128;  // (two threads count for each)
constexpr int kTops = 32;           // tiles' maxima that a thread keeps (of several tiles each where there are more)
constexpr int kHits = 256;          // of them that reach the bound
constexpr int kList = 512;          // candidates of a CTA

// Order-preserving bits of a float, and back.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t o) {
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// A candidate of a row: larger is better, ties to the lower token; 0 is none. (x + 0
// makes a negative zero a positive one: they are equal, and their bits are not.)
__device__ __forceinline__ uint64_t row_key(float x, int token) {
    return (static_cast<uint64_t>(order_bits(x + 0.f)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(token));
}
__device__ __forceinline__ float key_value(uint64_t key) { return from_order(static_cast<uint32_t>(key >> 32)); }
__device__ __forceinline__ uint64_t warp_max(uint64_t k) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        k = max(k, static_cast<uint64_t>(__shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(k), o)));
    return k;
}

// A beam without continuations of its own: finished, or without a score.
__device__ __forceinline__ bool row_closed(const BeamArgs &a, int row) {
    const float s = a.scores[row];
    return !(s > -INFINITY) || (a.finished != nullptr && a.finished[row] != 0);
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t x, uint32_t y) {  // (NaN gives way)
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;\n" : "=r"(r) : "r"(x), "r"(y));
    return r;
}

// 16 bytes of a row: values, and maxima of two subsets of them.
template <typename T>
struct Pack;
template <>
struct Pack<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xFF80FF80u;  // -inf twice
    typedef uint32_t Max;
    static __device__ __forceinline__ float get(const uint4 &v, int j) {
        const uint32_t w = j < 2 ? v.x : j < 4 ? v.y : j < 6 ? v.z : v.w;
        return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ Max none() { return kNone; }
    static __device__ __forceinline__ Max max_of(const uint4 &v) {
        return max_bf16x2(max_bf16x2(v.x, v.y), max_bf16x2(v.z, v.w));
    }
    static __device__ __forceinline__ Max join(Max a, Max b) { return max_bf16x2(a, b); }
    static __device__ __forceinline__ float lo(Max m) { return __uint_as_float(m << 16); }
    static __device__ __forceinline__ float hi(Max m) { return __uint_as_float(m & 0xFFFF0000u); }
};
template <>
struct Pack<float> {
    static constexpr int kN = 4;
    static constexpr uint32_t kNone = 0xFF800000u;
    typedef float2 Max;
    static __device__ __forceinline__ float get(const uint4 &v, int j) {
        return __uint_as_float(j == 0 ? v.x : j == 1 ? v.y : j == 2 ? v.z : v.w);
    }
    static __device__ __forceinline__ Max none() { return make_float2(-INFINITY, -INFINITY); }
    static __device__ __forceinline__ Max max_of(const uint4 &v) {
        return make_float2(fmaxf(fmaxf(get(v, 0), get(v, 2)), -INFINITY), fmaxf(fmaxf(get(v, 1), get(v, 3)), -INFINITY));
    }
    static __device__ __forceinline__ Max join(Max a, Max b) { return make_float2(fmaxf(a.x, b.x), fmaxf(a.y, b.y)); }
    static __device__ __forceinline__ float lo(Max m) { return m.x; }
    static __device__ __forceinline__ float hi(Max m) { return m.y; }
};

// NaN counts as -inf, +inf as the largest finite value.
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, -INFINITY), FLT_MAX); }

// The K-th largest of a warp's 64 values, two a lane (order bits, of which the
// `kBits` highest differ).
template <int kBits>
__device__ __forceinline__ uint32_t kth_of_64(uint32_t a, uint32_t b, int K) {
    uint32_t top = 0u;
#pragma unroll
    for (int i = 30; i >= 32 - kBits; i -= 2) {  // two bits a step: the three thresholds' votes are independent
        uint32_t next = top;
#pragma unroll
        for (uint32_t j = 1; j < 4; ++j) {
            const uint32_t t = top | j << i;
            if (__popc(__ballot_sync(0xffffffffu, a >= t)) + __popc(__ballot_sync(0xffffffffu, b >= t)) >= K) next = t;
        }
        top = next;
    }
    // (of a negative value the bits below are ones)
    return kBits < 32 && !(top >> 31) ? top | 0xFFFFu : top;
}

// A row as chunks of 16 bytes from its first token on; past its end there is -inf.
// Where its rows do not start on 16 bytes a chunk is cut from two neighbouring ones.
template <typename T, bool kAligned>
struct Row {
    static constexpr int kV = Pack<T>::kN;
    const T *src;
    const uint4 *base;  // 16-byte boundary at or before the row
    int vocab, head;    // values between `base` and the row

    __device__ __forceinline__ Row(const void *logits, int64_t at, int n) : src(static_cast<const T *>(logits) + at), vocab(n) {
        head = kAligned ? 0 : static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
        base = reinterpret_cast<const uint4 *>(src - head);
    }
    __device__ __forceinline__ uint4 chunk(int c) const {
        const int first = c * kV;
        if (kAligned || head == 0) {
            if (first + kV <= vocab) return __ldcs(base + c);
        } else if (first >= head && first + 2 * kV - head <= vocab) {  // (both boundaries' chunks are the row's)
            uint4 l = __ldcs(base + c), h = __ldcs(base + c + 1);
            const int s = head * static_cast<int>(sizeof(T));  // bytes to leave out
            if (s & 8) {
                l = make_uint4(l.z, l.w, h.x, h.y);
                h.x = h.z;
                h.y = h.w;
            }
            if (s & 4) {
                l = make_uint4(l.y, l.z, l.w, h.x);
                h.x = h.y;
            }
            if (sizeof(T) == 2 && (s & 2))
                l = make_uint4(__funnelshift_r(l.x, l.y, 16), __funnelshift_r(l.y, l.z, 16), __funnelshift_r(l.z, l.w, 16),
                               __funnelshift_r(l.w, h.x, 16));
            return l;
        }
        uint4 v = make_uint4(Pack<T>::kNone, Pack<T>::kNone, Pack<T>::kNone, Pack<T>::kNone);
        T *t = reinterpret_cast<T *>(&v);
#pragma unroll
        for (int j = 0; j < kV; ++j)
            if (first + j < vocab) t[j] = src[first + j];
        return v;
    }
    // f(key) of every value of a chunk that may be a candidate
    template <typename F>
    __device__ __forceinline__ void keys(int c, F f) const {
        const uint4 v = chunk(c);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float x = clean(Pack<T>::get(v, j));
            if (x > -INFINITY) f(row_key(x, c * kV + j));
        }
    }
};

// The maximum and sum of a slice again, value by value.
template <typename T>
__device__ __noinline__ float2 clean_sum(const T *src, int e0, int e1, float *s_part) {
    const int tid = threadIdx.x;
    auto block = [&](float v, bool sum) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float x = __shfl_xor_sync(0xffffffffu, v, o);
            v = sum ? v + x : fmaxf(v, x);
        }
        __syncthreads();
        if ((tid & 31) == 0) s_part[tid >> 5] = v;
        __syncthreads();
        v = s_part[0];
        for (int i = 1; i < kWarps; ++i) v = sum ? v + s_part[i] : fmaxf(v, s_part[i]);
        return v;
    };
    float m = -INFINITY, z = 0.f;
    for (int e = e0 + tid; e < e1; e += kThreads) m = fmaxf(m, clean(static_cast<float>(src[e])));
    m = block(m, false);
    if (m > -INFINITY)
        for (int e = e0 + tid; e < e1; e += kThreads) z += fast_exp2((clean(static_cast<float>(src[e])) - m) * kLog2e);
    return make_float2(m, block(z, true));
}

template <typename T, bool kAligned>
__global__ void __launch_bounds__(kThreads, 4) beam_slice_kernel(const BeamArgs a) {
    typedef Pack<T> P;
    constexpr int kV = P::kN, kBits = 8 * sizeof(T);
    constexpr int kMore = kSubsets + kThreads * kV;  // candidates kept, and those of a chunk a thread
    __shared__ union {
        float tops[kTops][kThreads];
        struct {
            uint64_t list[kList];
            int hits[kHits];
        } few;  // (tops are read before)
        uint64_t more[kMore];
    } u;
    __shared__ uint32_t s_seen[kWarps][kSubsets];
    __shared__ float s_ref[kWarps], s_sum[kWarps], s_part[kWarps];
    __shared__ uint64_t s_best[kWarps];
    __shared__ float s_bound;
    __shared__ int s_hits, s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = blockIdx.x / a.slices, slice = blockIdx.x - r * a.slices;
    const int K = a.select;
    pdl_trigger();
    pdl_wait();  // the logits and scores of the kernel before, and the last call's reads of the workspace
    if (tid == 0) s_hits = s_count = 0;

    const Row<T, kAligned> row(a.logits, static_cast<int64_t>(r) * a.stride, a.vocab);
    const int chunks = (a.vocab + kV - 1) / kV, per = (chunks + a.slices - 1) / a.slices;
    const int c0 = min(chunks, slice * per), c1 = min(chunks, c0 + per);
    const int tiles = (c1 - c0 + kThreads * kLoads - 1) / (kThreads * kLoads), run = (tiles + kTops - 1) / kTops;
    const uint4 none = make_uint4(P::kNone, P::kNone, P::kNone, P::kNone);
    auto load = [&](int c) { return c < c1 ? row.chunk(c) : none; };

    uint64_t *keys = a.keys + static_cast<int64_t>(blockIdx.x) * K;
    typename P::Max seen = P::none();  // maxima of the thread's two subsets
    float ref = -INFINITY, c = 0.f;    // the sums' reference, and ref log2(e) as fp32 has it
    uint64_t z = f2_pack(0.f, 0.f);    // (a group's values are added up first: rounding errors grow with the groups alone)
    uint4 v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) v[i] = load(c0 + i * kThreads + tid);
    if (row_closed(a, r)) return;  // (known while the first values are on their way)
    float run_top = -INFINITY;
    for (int t = 0, in_run = 0, at = c0; t < tiles; ++t, at += kLoads * kThreads) {
#pragma unroll
        for (int g = 0; g < kLoads; g += kGroup) {
            if (at + g * kThreads >= c1) break;
            typename P::Max all = P::max_of(v[g]);
#pragma unroll
            for (int i = 1; i < kGroup; ++i) all = P::join(all, P::max_of(v[g + i]));
            seen = P::join(seen, all);
            const float top = fmaxf(P::lo(all), P::hi(all));
            run_top = fmaxf(run_top, top);
            if (__any_sync(0xffffffffu, top > ref + 5.5f)) {  // (e^5.5 < 2^8)
                const float m = fminf(from_order(__reduce_max_sync(0xffffffffu, order_bits(fmaxf(top, ref)))), FLT_MAX);
                const float cn = __fmul_rn(m, kLog2e);  // (rounded wherever it is used, never part of a multiply-add)
                const float f = ref > -INFINITY ? fast_exp2(c - cn) : 0.f;
                z = f2_fma(z, f2_pack(f, f), f2_pack(0.f, 0.f));
                ref = m;
                c = cn;
            }
            if (ref > -INFINITY) {
                const uint64_t l2 = f2_pack(kLog2e, kLog2e), c2 = f2_pack(-c, -c);
                uint64_t z0 = f2_pack(0.f, 0.f), z1 = z0;
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
#pragma unroll
                    for (int j = 0; j < kV; j += 2) {
                        float x, y;
                        f2_unpack(f2_fma(f2_pack(P::get(v[g + i], j), P::get(v[g + i], j + 1)), l2, c2), x, y);
                        const uint64_t e = f2_pack(fast_exp2(x), fast_exp2(y));
                        if (j & 2) z1 = f2_add(z1, e);
                        else z0 = f2_add(z0, e);
                    }
                z = f2_add(z, f2_add(z0, z1));
            }
#pragma unroll
            for (int i = g; i < g + kGroup; ++i) v[i] = load(at + (kLoads + i) * kThreads + tid);
        }
        if (++in_run == run || t + 1 == tiles) {
            u.tops[t / run][tid] = run_top;
            run_top = -INFINITY;
            in_run = 0;
        }
    }
    {
        float x, y;
        f2_unpack(z, x, y);
        x += y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane == 0) {
            s_ref[warp] = ref;
            s_sum[warp] = x;
        }
        s_seen[warp][lane] = order_bits(P::lo(seen));
        s_seen[warp][lane + 32] = order_bits(P::hi(seen));
    }
    __syncthreads();
    if (warp == 0) {  // the bound: by one warp, the issue slots go to the SM's other CTAs
        uint32_t x = s_seen[0][lane], y = s_seen[0][lane + 32];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) {
            x = max(x, s_seen[w][lane]);
            y = max(y, s_seen[w][lane + 32]);
        }
        x = kth_of_64<kBits>(x, y, K);
        if (lane == 0) s_bound = fmaxf(clean(from_order(max(x, order_bits(-INFINITY)))), -FLT_MAX);
    }
    // The slice's sum over 2^c, c = max log2(e) rounded, then over e^max: the rounding of c, d = max
    // log2(e) - c (exact), is taken out as 2^-d = 1 + expm1(-d ln 2), which costs an ordinary row, whose
    // d is next to nothing, no accuracy. From maxima of 1.5 10^6 on d may be 1/8 and more (0.5 at
    // 10^7): the rounding of d ln 2 would count, and such slices are summed again.
    float m = s_ref[0], sum = 0.f;
#pragma unroll
    for (int i = 1; i < kWarps; ++i) m = fmaxf(m, s_ref[i]);
    c = __fmul_rn(m, kLog2e);
    for (int i = 0; i < kWarps; ++i)
        if (s_ref[i] > -INFINITY) sum += s_sum[i] * fast_exp2(__fmul_rn(s_ref[i], kLog2e) - c);
    const float d = fmaf(m, kLog2e, -c);
    sum = fmaf(sum, expm1f(-d * kLn2), sum);
    float2 part = make_float2(m, sum);
    // (and those with NaN or an infinity among them, or a maximum whose product with log2(e) overflows;
    // of others the reference, which some value was, gives 1)
    if (m > -INFINITY && !(fabsf(d) < 0.125f && sum > 0.5f && sum < INFINITY))
        part = clean_sum(row.src, c0 * kV, min(a.vocab, c1 * kV), s_part);
    if (tid == 0) a.parts[blockIdx.x] = part;
    __syncthreads();
    const float bound = s_bound;
    auto note = [&](uint64_t key) {
        if (key_value(key) < bound) return;
        const int n = atomicAdd(&s_count, 1);
        if (n < kList) u.few.list[n] = key;
    };
    auto rank = [&](int n) {
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t key = u.few.list[i];
            int better = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) better += u.few.list[j] > key;
            if (better < K) keys[better] = key;
        }
        for (int i = n + tid; i < K; i += kThreads) keys[i] = 0ull;
    };
    uint32_t reach = 0u;  // the thread's runs of tiles that reach the bound
    for (int i = 0; i * run < tiles; ++i) reach |= (u.tops[i][tid] >= bound ? 1u : 0u) << i;
    __syncthreads();
    while (reach) {
        const int i = __ffs(reach) - 1, n = atomicAdd(&s_hits, 1);
        reach &= reach - 1;
        if (n < kHits) u.few.hits[n] = i * kThreads + tid;
    }
    __syncthreads();
    const int hits = s_hits;
    if (hits <= kHits) {
        const int loads = run * kLoads;  // of a hit
        for (int i = tid; i < hits * loads; i += kThreads) {
            const int hit = u.few.hits[i / loads], at = c0 + (hit / kThreads * loads + i % loads) * kThreads + hit % kThreads;
            if (at < c1) row.keys(at, note);
        }
        __syncthreads();
        if (s_count <= kList) return rank(s_count);
    }
    // Many values reach the bound (equals of it, or large values in few subsets): the
    // slice again, a chunk a thread, whose candidates are cut to the best K each time.
    __syncthreads();
    if (tid == 0) s_count = 0;
    __syncthreads();
    uint64_t worst = 0ull;  // of K kept ones; the later tokens of equals are worse
    for (int at = c0; at < c1; at += kThreads) {
        if (at + tid < c1)
            row.keys(at + tid, [&](uint64_t key) {
                if (key > worst && key_value(key) >= bound) u.more[atomicAdd(&s_count, 1)] = key;
            });
        __syncthreads();
        const int n = s_count;
        if (n > K) {
            uint64_t last = ~0ull, mine = 0ull;
            for (int i = 0; i < K; ++i) {
                uint64_t k = 0ull;
                for (int j = tid; j < n; j += kThreads)
                    if (u.more[j] < last) k = max(k, u.more[j]);
                k = warp_max(k);
                if (lane == 0) s_best[warp] = k;
                __syncthreads();
                last = s_best[0];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) last = max(last, s_best[w]);
                if (tid == i) mine = last;
                __syncthreads();
            }
            if (tid < K) u.more[tid] = mine;
            if (tid == 0) s_count = K;
            worst = last;
        }
        __syncthreads();
    }
    for (int i = tid; i < K; i += kThreads) {
        // (cut lists are in order; one that never was is ranked)
        const int n = s_count;
        int rank = i;
        uint64_t key = i < n ? u.more[i] : 0ull;
        if (i < n) {
            rank = 0;
            for (int j = 0; j < n; ++j) rank += u.more[j] > key;
        }
        keys[rank] = key;
    }
}

// Unevaluated sums of two floats, the second at most half a step of the first.
struct Two {
    float hi, lo;
};
__device__ __forceinline__ Two two_sum(float a, float b) {  // exact
    const float s = a + b, t = s - a;
    return Two{s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ Two two_norm(float hi, float lo) {
    if (!(fabsf(hi) < INFINITY)) return Two{hi, 0.f};  // (`lo` is NaN then)
    const float s = hi + lo;
    return Two{s + 0.f, (lo - (s - hi)) + 0.f};  // (no zero is negative)
}
// ln z, z of 1 or more (but for rounding): z = 2^e f, ln f = 2 atanh((f - 1) / (f + 1))
// by its series. Off by some 1e-9.
__device__ Two two_log(float z) {
    const int bits = __float_as_int(z), e = (bits - __float_as_int(0.70710678f)) >> 23;
    const float f = __int_as_float(bits - (e << 23)), n = f - 1.f;  // (exact: f is 0.7 .. 1.42)
    const Two d = two_sum(f, 1.f);
    const float q = __fdividef(n, d.hi), q1 = __fdividef(fmaf(-q, d.hi, n) - q * d.lo, d.hi), s = q * q;  // (q1 takes q's error out)
    const float p = s * fmaf(s, fmaf(s, fmaf(s, fmaf(s, 1.f / 11, 1.f / 9), 1.f / 7), 1.f / 5), 1.f / 3);
    constexpr float kHi = 45426.f / 65536.f;  // (16 bits of ln 2: e kHi is exact)
    constexpr float kLo = static_cast<float>(0.69314718055994530942 - 45426.0 / 65536.0);
    const Two t = two_sum(e * kHi, 2.f * q);
    return two_norm(t.hi, t.lo + fmaf(static_cast<float>(e), kLo, 2.f * fmaf(q, p, q1)));
}

// A candidate of a group: a larger total (order-preserving bits of its two floats) is
// better, ties to the lower beam and token.
struct Cand {
    uint64_t total;
    int64_t tie;  // beam * 2^32 + token
};
__device__ __forceinline__ Cand no_cand() { return Cand{0ull, INT64_MAX}; }
__device__ __forceinline__ bool better(const Cand &a, const Cand &b) {
    return a.total > b.total || (a.total == b.total && a.tie < b.tie);
}
__device__ __forceinline__ uint64_t order_bits2(Two x) { return static_cast<uint64_t>(order_bits(x.hi)) << 32 | order_bits(x.lo); }

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const BeamArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    // of the group's beams: maximum logit, and score - log sum exp(x - maximum)
    Two *s_off = reinterpret_cast<Two *>(smem);
    float *s_max = reinterpret_cast<float *>(s_off + a.beams);
    int *s_open = reinterpret_cast<int *>(s_max + a.beams);
    __shared__ Cand s_best[kMergeThreads];
    __shared__ Cand s_list[kList];
    __shared__ uint32_t s_top[kMergeSubsets];
    __shared__ __align__(16) uint32_t s_sub[kMergeSubsets];
    __shared__ uint32_t s_bound;
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = blockIdx.x, W = a.beams, S = a.slices, K = a.select;
    pdl_trigger();
    pdl_wait();
    if (tid == 0) {
        s_count = 0;
        s_bound = ~0u;
    }
    // what a thread looks at below, on its way before the sums are known (a closed
    // beam's lists are not written; they are not looked at either)
    const uint64_t *keys = a.keys + static_cast<int64_t>(g) * W * S * K;
    // (the lists' heads, and where there are few lists what is next in them)
    const int deep = min(K, (kMergeSubsets + W * S - 1) / (W * S));
    const uint64_t head0 = tid < W * S * deep ? keys[tid % (W * S) * K + tid / (W * S)] : 0ull;
    const uint64_t key0 = tid < W * S * K ? keys[tid] : 0ull;
    const uint64_t key1 = tid + kMergeThreads < W * S * K ? keys[tid + kMergeThreads] : 0ull;
    for (int w = warp; w < W; w += kMergeThreads / 32) {
        const int row = g * W + w;
        const float2 *part = a.parts + static_cast<int64_t>(row) * S;
        const float2 first = lane < S ? part[lane] : make_float2(-INFINITY, 0.f);  // (with the score's load; not used of a closed row)
        const bool open = !row_closed(a, row);
        float m = -INFINITY, z = 0.f;
        if (open) {
            m = first.x;
            for (int s = lane + 32; s < S; s += 32) m = fmaxf(m, part[s].x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            for (int s = lane; s < S; s += 32) {
                const float2 p = s == lane ? first : part[s];
                if (p.x > -INFINITY) z += p.y * expf(p.x - m);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        }
        if (lane == 0) {
            s_max[w] = m;
            s_open[w] = open && m > -INFINITY;
            if (s_open[w]) {
                const Two l = two_log(z), o = two_sum(a.scores[row], -l.hi);
                s_off[w] = two_norm(o.hi, o.lo - l.lo);
            }
        }
    }
    __syncthreads();
    auto cand = [&](int w, uint64_t key) {
        const Two d = two_sum(key_value(key), -s_max[w]), off = s_off[w], t = two_sum(d.hi, off.hi);
        return Cand{order_bits2(two_norm(t.hi, t.lo + (d.lo + off.lo))),
                    static_cast<int64_t>(w) << 32 | (0xFFFFFFFFu - static_cast<uint32_t>(key))};
    };
    auto end_of = [&](int w) {  // the one continuation of a finished beam
        const int row = g * W + w;
        const float s = a.scores[row];
        if (a.finished == nullptr || a.finished[row] == 0 || a.end_token < 0 || !(s > -INFINITY)) return no_cand();
        return Cand{order_bits2(two_norm(s, 0.f)), static_cast<int64_t>(w) << 32 | a.end_token};
    };
    auto put = [&](int r, const Cand &c) {
        const int64_t o = static_cast<int64_t>(g) * K + r;
        const bool none = c.total == 0ull;
        a.out_scores[o] = none ? -INFINITY : from_order(static_cast<uint32_t>(c.total >> 32));
        a.out_parents[o] = none ? -1 : g * W + static_cast<int>(c.tie >> 32);
        a.out_tokens[o] = none ? -1 : static_cast<int32_t>(c.tie);
    };
    if (W * S * K <= kMergeThreads / 4) {
        // few: all are ranked, four threads each (4 rows of 4000, 16 chosen: 8.6 us with the bound
        // below, 7.7 so; with 128 candidates, two threads each, it takes 0.9 us longer)
        Cand c = no_cand();
        if (tid < W * S * K) {
            const int w = tid / (S * K);
            if (s_open[w]) {
                if (key0 != 0ull) c = cand(w, key0);
            } else if (tid == w * S * K) {
                c = end_of(w);
            }
            s_list[tid] = c;
        }
        const int n = __syncthreads_count(c.total != 0ull);
        int r = 0;
        c = tid / 4 < W * S * K ? s_list[tid / 4] : no_cand();
        if (c.total != 0ull) {
#pragma unroll 4
            for (int i = tid % 4; i < W * S * K; i += 4) r += better(s_list[i], c);
        }
        r += __shfl_xor_sync(0xffffffffu, r, 1);
        r += __shfl_xor_sync(0xffffffffu, r, 2);
        if (tid % 4 == 0 && c.total != 0ull && r < K) put(r, c);
        for (int i = n + tid; i < K; i += kMergeThreads) put(i, no_cand());
        return;
    }
    // the K-th best of the subsets' bests (threads t and t + kMergeSubsets; by the first of the
    // two floats), which K candidates reach: the least of those that fewer than K are above
    uint32_t best = 0u;
    for (int i = tid; i < W * S * deep; i += kMergeThreads) {
        const int l = i % (W * S), w = l / S;
        const uint64_t key = !s_open[w] ? 0ull : i == tid ? head0 : keys[l * K + i / (W * S)];
        if (key != 0ull) best = max(best, static_cast<uint32_t>(cand(w, key).total >> 32));
    }
    for (int w = tid; w < W; w += kMergeThreads) best = max(best, static_cast<uint32_t>(end_of(w).total >> 32));
    if (tid >= kMergeSubsets) s_top[tid - kMergeSubsets] = best;
    __syncthreads();
    if (tid < kMergeSubsets) s_sub[tid] = max(best, s_top[tid]);
    __syncthreads();
    {
        const uint32_t mine = s_sub[tid / 2];
        int above = 0;
#pragma unroll
        for (int i = 0; i < kMergeSubsets / 8; ++i) {
            const uint4 o = reinterpret_cast<const uint4 *>(s_sub)[2 * i + tid % 2];
            above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
        above += __shfl_xor_sync(0xffffffffu, above, 1);
        const uint32_t least = __reduce_min_sync(0xffffffffu, above < K ? mine : ~0u);
        if (lane == 0) atomicMin(&s_bound, least);
    }
    __syncthreads();
    const uint32_t bound = s_bound;  // (0: there are fewer)
    auto take = [&](const Cand &c) {
        if (c.total == 0ull || static_cast<uint32_t>(c.total >> 32) < bound) return;
        const int n = atomicAdd(&s_count, 1);
        if (n < kList) s_list[n] = c;
    };
    // Visits every candidate of the thread.
    auto visit = [&](auto f) {
        for (int i = tid; i < W * S * K; i += kMergeThreads) {
            const int w = i / (S * K);
            if (!s_open[w]) continue;
            const uint64_t key = i == tid ? key0 : i == tid + kMergeThreads ? key1 : keys[i];
            if (key != 0ull) f(cand(w, key));
        }
        for (int w = tid; w < W; w += kMergeThreads) f(end_of(w));
    };
    visit(take);
    __syncthreads();
    const int n = s_count;
    if (n <= kList) {
        for (int i = tid; i < n; i += kMergeThreads) {
            const Cand c = s_list[i];
            int r = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) r += better(s_list[j], c);
            if (r < K) put(r, c);
        }
        for (int i = n + tid; i < K; i += kMergeThreads) put(i, no_cand());
        return;
    }
    Cand last = no_cand();  // K rounds of a maximum below the last one
    for (int r = 0; r < K; ++r) {
        Cand c = no_cand();
        visit([&](const Cand &o) {
            if ((r == 0 || better(last, o)) && better(o, c)) c = o;
        });
        __syncthreads();
        s_best[tid] = c;
        __syncthreads();
        for (int h = kMergeThreads / 2; h > 0; h >>= 1) {
            if (tid < h && better(s_best[tid + h], s_best[tid])) s_best[tid] = s_best[tid + h];
            __syncthreads();
        }
        last = s_best[0];
        if (tid == 0) put(r, last);
        if (last.total == 0ull) {  // none left
            for (int i = r + 1 + tid; i < K; i += kMergeThreads) put(i, last);
            return;
        }
    }
}

}  // namespace

// Slices a row: what the SMs hold at once (4 CTAs each), but no more than balances a
// slice's time with what each adds to the merge (s slices of n / s chunks: s^2 = n / 185).
// us a call, rows x vocabulary in bf16: 152 x 151936 19.6 with 4, 20.6 with 3, 23.4 with 6;
// 512 x 151936 35.6 with 1, 40.1 with 2; 4 x 151936 10.7 with 8, 11.4 with 4, 17.2 with 1;
// 8 x 32000 9.9 with 4, 10.6 with 1, 12.4 with 16.
int beam_slices(const fnpu_beam_desc *d) {
    const int64_t rows = static_cast<int64_t>(d->num_groups) * d->num_beams;
    const int64_t chunks = d->dtype == FNPU_LOGITS_FP32 ? (static_cast<int64_t>(d->vocab) + 3) / 4 : (static_cast<int64_t>(d->vocab) + 7) / 8;
    int64_t s = 1;
    while ((s + 1) * rows <= 4 * 152 && (s + 1) * (s + 1) * 185 <= chunks) ++s;
    return static_cast<int>(s);
}

int launch_beam_select(const BeamArgs &a, bool fp32, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t grid = static_cast<int64_t>(a.groups) * a.beams * a.slices;
    const bool aligned = (reinterpret_cast<uintptr_t>(a.logits) & 15u) == 0 &&
                         (a.groups * a.beams == 1 || a.stride % (fp32 ? 4 : 8) == 0);
    auto kernel = fp32 ? (aligned ? beam_slice_kernel<float, true> : beam_slice_kernel<float, false>)
                       : (aligned ? beam_slice_kernel<__nv_bfloat16, true> : beam_slice_kernel<__nv_bfloat16, false>);
    FNPU_CUDA_TRY(launch_ex(kernel, static_cast<unsigned>(grid), kThreads, 0, st, true, nullptr, a));
    const size_t smem = static_cast<size_t>(a.beams) * (sizeof(Two) + sizeof(float) + sizeof(int));
    FNPU_CUDA_TRY(launch_ex(beam_merge_kernel, static_cast<unsigned>(a.groups), kMergeThreads, smem, st, true, nullptr, a));
    return FNPU_OK;
}

}  // namespace fnpu
