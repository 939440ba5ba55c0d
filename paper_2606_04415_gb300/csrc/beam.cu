// Selection of a beam search: the best continuations (beam, token) of every
// group of beams, by score[b] + log softmax(logits[b])[v].
//
// What bounds it is the one read of the logits. Two kernels, the second a
// dependent launch of the first:
//   * A CTA of the first takes a slice of a row and leaves its maximum, the sum of
//     exp(x - max) and its best num_select values in order. Within a row the order
//     of the totals is the order of the logits, ties to the lower token, so candidates
//     need no normalisation. Each warp streams a part of the slice by itself: a value
//     costs a conversion, half a paired multiply-add, an exponential and half a paired
//     addition, and bf16 maxima go in pairs; a reference that all of a warp's sums share moves only when
//     a tile has a value 2^8 above it. Candidates are what reaches a bound: the
//     K-th largest of the maxima of 64 subsets of what the warp has seen, which at least
//     K values reach. It is formed anew after 1, 2, 4, .. tiles, so that some K log n
//     values become candidates; a list that fills up is cut to its best K.
//   * A CTA of the second takes a group: the rows' log-sum-exps from their slices',
//     then the best of all slices' lists by the total in 64 bits. Totals of
//     different beams may lie closer than an fp32 score of some hundred resolves
//     (3e-5); fp64 is slow on this device, so only what an fp32 total with its error
//     cannot rule out is added in 64 bits, and order-preserving integers are compared.
#include <float.h>

#include "common.cuh"

namespace fnpu {
namespace {

constexpr int kThreads = 256;       // of the first kernel
constexpr int kWarps = kThreads / 32;
constexpr int kLoads = 4;           // 16-byte loads of a lane in a tile
constexpr int kMergeThreads = 256;  // of the second
constexpr int kSubsets = 64;        // (num_select is at most as many)
constexpr int kWarpList = 384;      // candidates of a warp: 64, and 256 of one load
constexpr int kList = 512;          // candidates of a CTA

// Order-preserving bits of a float, and back.
__device__ __forceinline__ uint32_t order_bits(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float from_order(uint32_t o) {
    return __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
// A candidate of a row: larger is better, ties to the lower token; 0 is none.
__device__ __forceinline__ uint64_t row_key(float x, int token) {
    return (static_cast<uint64_t>(order_bits(x)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(token));
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

// The K-th largest of a warp's 64 values, two a lane (order bits).
__device__ __forceinline__ uint32_t kth_of_64(uint32_t a, uint32_t b, int K, int lane) {
    const bool low = K > 32;  // from the other end: the (65 - K)-th smallest
    const int n = low ? 65 - K : K;
    if (low) {
        a = ~a;
        b = ~b;
    }
    uint32_t top = 0u;
    for (int r = 0; r < n; ++r) {
        top = __reduce_max_sync(0xffffffffu, max(a, b));
        const uint32_t who = __ballot_sync(0xffffffffu, a == top || b == top);
        if (lane == __ffs(who) - 1) {  // one of them goes (0 is below every value's bits, and above none's)
            if (a == top) a = 0u;
            else b = 0u;
        }
    }
    return low ? ~top : top;
}

// The best K of a warp's list, in its first K places; returns the K-th.
__device__ __noinline__ uint64_t cut_list(uint64_t *list, int n, int K) {
    const int lane = threadIdx.x & 31;
    uint64_t keep0 = 0, keep1 = 0, last = ~0ull;
    __syncwarp();
    for (int r = 0; r < K; ++r) {
        uint64_t k = 0;
        for (int i = lane; i < n; i += 32) {
            const uint64_t e = list[i];
            if (e < last) k = max(k, e);
        }
        last = warp_max(k);
        if (lane == (r & 31)) {
            if (r < 32) keep0 = last;
            else keep1 = last;
        }
    }
    __syncwarp();
    if (lane < K) list[lane] = keep0;
    if (lane + 32 < K) list[lane + 32] = keep1;
    __syncwarp();
    return last;
}

// The maximum and sum of a slice again, value by value, where NaN or an infinity is among them.
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

template <typename T>
__global__ void __launch_bounds__(kThreads, 6) beam_slice_kernel(const BeamArgs a) {
    typedef Pack<T> P;
    constexpr int kV = P::kN;
    __shared__ uint64_t s_lists[kWarps][kWarpList];
    __shared__ uint64_t s_list[kList];
    __shared__ float s_ref[kWarps], s_sum[kWarps], s_bound[kWarps], s_part[kWarps];
    __shared__ uint64_t s_best[kWarps];
    __shared__ int s_len[kWarps], s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices;
    const int K = a.select;
    pdl_trigger();
    pdl_wait();  // the logits and scores of the kernel before, and the last call's reads of the workspace
    if (row_closed(a, row)) return;
    if (tid == 0) s_count = 0;

    // 16-byte chunks of memory; the row's first and last may hold neighbours' values
    const T *src = static_cast<const T *>(a.logits) + static_cast<int64_t>(row) * a.stride;
    const int head = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
    const uint4 *base = reinterpret_cast<const uint4 *>(src - head);
    const int chunks = (head + a.vocab + kV - 1) / kV;
    const int per = (chunks + a.slices - 1) / a.slices;
    const int c0 = min(chunks, slice * per), c1 = min(chunks, c0 + per);
    // (whole loads of a warp to each warp)
    const int wper = ((c1 - c0 + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int w0 = min(c1, c0 + warp * wper), w1 = min(c1, w0 + wper);
    auto load = [&](int c) -> uint4 {
        const int first = c * kV - head;
        if (c < w1 && first >= 0 && first + kV <= a.vocab) return __ldcs(base + c);
        uint4 v = make_uint4(P::kNone, P::kNone, P::kNone, P::kNone);
        if (c < w1) {  // the row's first or last chunk
            T *t = reinterpret_cast<T *>(&v);
#pragma unroll
            for (int j = 0; j < kV; ++j)
                if (first + j >= 0 && first + j < a.vocab) t[j] = src[first + j];
        }
        return v;
    };

    uint64_t *list = s_lists[warp];
    int len = 0;
    typename P::Max seen = P::none();           // maxima of the lane's two subsets
    float bound = -INFINITY, reach = -FLT_MAX;  // K values of the list reach `bound`; candidates reach `reach`
    float ref = -INFINITY, c = 0.f;             // the sums' reference, and ref log2(e) as fp32 has it
    uint64_t z0 = f2_pack(0.f, 0.f), z1 = z0;
    for (int t = 0, at = w0; at < w1; ++t, at += 32 * kLoads) {
        uint4 v[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) v[i] = load(at + 32 * i + lane);
        typename P::Max mx[kLoads], all = P::none();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            mx[i] = P::max_of(v[i]);
            all = P::join(all, mx[i]);
        }
        seen = P::join(seen, all);
        const float top = fmaxf(P::lo(all), P::hi(all));
        if (__any_sync(0xffffffffu, top > ref + 5.5f)) {  // (e^5.5 < 2^8)
            const float m = fminf(from_order(__reduce_max_sync(0xffffffffu, order_bits(fmaxf(top, ref)))), FLT_MAX);
            const float cn = m * kLog2e;
            const float f = ref > -INFINITY ? fast_exp2(c - cn) : 0.f;
            const uint64_t f2 = f2_pack(f, f), o2 = f2_pack(0.f, 0.f);
            z0 = f2_fma(z0, f2, o2);
            z1 = f2_fma(z1, f2, o2);
            ref = m;
            c = cn;
        }
        if (ref > -INFINITY) {
            const uint64_t l2 = f2_pack(kLog2e, kLog2e), c2 = f2_pack(-c, -c);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int j = 0; j < kV; j += 2) {
                    float x, y;
                    f2_unpack(f2_fma(f2_pack(P::get(v[i], j), P::get(v[i], j + 1)), l2, c2), x, y);
                    const uint64_t e = f2_pack(fast_exp2(x), fast_exp2(y));
                    if (j & 2) z1 = f2_add(z1, e);
                    else z0 = f2_add(z0, e);
                }
        }
        const bool renew = (t & (t + 1)) == 0;
        if (renew) {
            const uint32_t k = kth_of_64(order_bits(P::lo(seen)), order_bits(P::hi(seen)), K, lane);
            const float b = fminf(from_order(k), FLT_MAX);
            if (b > bound) {
                bound = b;
                reach = fmaxf(reach, b);
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (!__any_sync(0xffffffffu, fmaxf(P::lo(mx[i]), P::hi(mx[i])) >= reach)) continue;
            if (len > kWarpList - 32 * kV) {
                const float b = key_value(cut_list(list, len, K));
                len = K;
                bound = fmaxf(bound, b);
                reach = fmaxf(reach, from_order(order_bits(b) + 1));  // (later equals are higher tokens)
            }
#pragma unroll
            for (int j = 0; j < kV; ++j) {
                const float x = P::get(v[i], j);
                const bool in = x >= reach;
                const uint32_t who = __ballot_sync(0xffffffffu, in);
                if (in) list[len + __popc(who & ((1u << lane) - 1))] = row_key(fminf(x, FLT_MAX), (at + 32 * i + lane) * kV - head + j);
                len += __popc(who);
            }
        }
        // from the next tile on, equals of the bound are higher tokens than K that are in the list
        if (renew && bound > -INFINITY) reach = fmaxf(reach, from_order(order_bits(bound) + 1));
    }
    {
        float x, y;
        f2_unpack(f2_add(z0, z1), x, y);
        float z = x + y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        if (lane == 0) {
            s_ref[warp] = ref;
            s_sum[warp] = z;
            s_bound[warp] = bound;
            s_len[warp] = len;
        }
    }
    __syncthreads();
    // the slice's sum over 2^c, c = max log2(e) rounded, then over e^max: the rounding of c is taken out
    float m = s_ref[0], floor = s_bound[0], z = 0.f;
#pragma unroll
    for (int i = 1; i < kWarps; ++i) {
        m = fmaxf(m, s_ref[i]);
        floor = fmaxf(floor, s_bound[i]);
    }
    c = m * kLog2e;
    for (int i = 0; i < kWarps; ++i)
        if (s_ref[i] > -INFINITY) z += s_sum[i] * fast_exp2(s_ref[i] * kLog2e - c);
    z -= z * fmaf(m, kLog2e, -c) * kLn2;
    float2 part = make_float2(m, z);
    if (m > -INFINITY && !(z < INFINITY)) {  // NaN or +inf among the values
        const int e0 = max(0, c0 * kV - head), e1 = min(a.vocab, c1 * kV - head);
        part = clean_sum(src, e0, e1, s_part);
    }
    if (tid == 0) a.parts[blockIdx.x] = part;
    // what reaches the best of the warps' bounds (K values of that warp do)
    for (int i0 = 0; i0 < len; i0 += 32) {
        const uint64_t key = i0 + lane < len ? list[i0 + lane] : 0ull;
        const bool in = key != 0ull && key_value(key) >= floor;
        const uint32_t who = __ballot_sync(0xffffffffu, in);
        int n = 0;
        if (lane == 0 && who) n = atomicAdd(&s_count, __popc(who));
        n = __shfl_sync(0xffffffffu, n, 0) + __popc(who & ((1u << lane) - 1));
        if (in && n < kList) s_list[n] = key;
    }
    __syncthreads();
    const int n = s_count;
    uint64_t *keys = a.keys + static_cast<int64_t>(blockIdx.x) * K;
    if (n <= kList) {
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t key = s_list[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += s_list[j] > key;
            if (r < K) keys[r] = key;
        }
        for (int i = n + tid; i < K; i += kThreads) keys[i] = 0ull;
        return;
    }
    uint64_t last = ~0ull;  // K rounds of a maximum over the warps' lists
    for (int r = 0; r < K; ++r) {
        uint64_t k = 0ull;
        for (int i = lane; i < len; i += 32)
            if (list[i] < last) k = max(k, list[i]);
        k = warp_max(k);
        __syncthreads();
        if (lane == 0) s_best[warp] = k;
        __syncthreads();
        last = s_best[0];
#pragma unroll
        for (int i = 1; i < kWarps; ++i) last = max(last, s_best[i]);
        if (tid == 0) keys[r] = last;  // (0 once there are none left)
    }
}

// A candidate of a group: a larger total (order-preserving bits of a double) is
// better, ties to the lower beam and token.
struct Cand {
    uint64_t total;
    int64_t tie;  // beam * vocab + token
};
__device__ __forceinline__ Cand no_cand() { return Cand{0ull, INT64_MAX}; }
__device__ __forceinline__ bool better(const Cand &a, const Cand &b) {
    return a.total > b.total || (a.total == b.total && a.tie < b.tie);
}
__device__ __forceinline__ uint64_t order_bits64(double x) {
    const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x));
    return b ^ ((b >> 63) ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ double from_order64(uint64_t o) {
    return __longlong_as_double(static_cast<long long>(o ^ ((o >> 63) ? 1ull << 63 : ~0ull)));
}

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const BeamArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    // of the group's beams: maximum logit, score - log sum exp(x - maximum), and both in fp32
    double *s_max = reinterpret_cast<double *>(smem), *s_off = s_max + a.beams;
    float *s_maxf = reinterpret_cast<float *>(s_off + a.beams), *s_offf = s_maxf + a.beams;
    int *s_open = reinterpret_cast<int *>(s_offf + a.beams);
    __shared__ Cand s_best[kMergeThreads];
    __shared__ Cand s_sub[kSubsets];
    __shared__ Cand s_list[kList];
    __shared__ Cand s_bound;
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = blockIdx.x, W = a.beams, S = a.slices, K = a.select;
    pdl_trigger();
    pdl_wait();
    if (tid == 0) s_count = 0;
    for (int w = warp; w < W; w += kMergeThreads / 32) {
        const int row = g * W + w;
        const bool open = !row_closed(a, row);
        float m = -INFINITY;
        double z = 0.0;
        if (open) {
            const float2 *part = a.parts + static_cast<int64_t>(row) * S;
            for (int s = lane; s < S; s += 32) m = fmaxf(m, part[s].x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            for (int s = lane; s < S; s += 32) {
                const float2 p = part[s];
                if (p.x > -INFINITY) z += static_cast<double>(p.y * expf(p.x - m));
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        }
        if (lane == 0) {
            s_max[w] = s_maxf[w] = m;
            s_off[w] = z;
            s_open[w] = open && m > -INFINITY;
        }
    }
    __syncthreads();
    for (int w = tid; w < W; w += kMergeThreads) {  // (one warp's logarithms cost as much as one lane's)
        s_off[w] = s_open[w] ? static_cast<double>(a.scores[g * W + w]) - log(s_off[w]) : 0.0;
        s_offf[w] = static_cast<float>(s_off[w]);
    }
    __syncthreads();
    const uint64_t *keys = a.keys + static_cast<int64_t>(g) * W * S * K;
    auto cand = [&](int w, uint64_t key) {
        return Cand{order_bits64((static_cast<double>(key_value(key)) - s_max[w]) + s_off[w]),
                    static_cast<int64_t>(w) * a.vocab + static_cast<int64_t>(0xFFFFFFFFu - static_cast<uint32_t>(key))};
    };
    auto end_of = [&](int w) {  // the one continuation of a finished beam
        const int row = g * W + w;
        const float s = a.scores[row];
        if (a.finished == nullptr || a.finished[row] == 0 || a.end_token < 0 || !(s > -INFINITY)) return no_cand();
        return Cand{order_bits64(static_cast<double>(s)), static_cast<int64_t>(w) * a.vocab + a.end_token};
    };
    // each thread's best of the lists' heads, and the K-th best of the subsets of threads
    Cand best = no_cand();
    for (int l = tid; l < W * S; l += kMergeThreads) {
        const int w = l / S;
        const uint64_t key = s_open[w] ? keys[static_cast<int64_t>(l) * K] : 0ull;
        if (key != 0ull) {
            const Cand c = cand(w, key);
            if (better(c, best)) best = c;
        }
    }
    for (int w = tid; w < W; w += kMergeThreads) {
        const Cand c = end_of(w);
        if (better(c, best)) best = c;
    }
    s_best[tid] = best;
    __syncthreads();
    if (tid < kSubsets) {
#pragma unroll
        for (int i = 1; i < kMergeThreads / kSubsets; ++i)
            if (better(s_best[tid + kSubsets * i], best)) best = s_best[tid + kSubsets * i];
        s_sub[tid] = best;
    }
    __syncthreads();
    {  // four threads a subset count the better ones (of equal ones, which are none, those before)
        const int s = tid / 4;
        const Cand mine = s_sub[s];
        int r = 0;
#pragma unroll 4
        for (int i = tid % 4; i < kSubsets; i += 4) {
            const Cand o = s_sub[i];
            r += better(o, mine) || (o.total == mine.total && o.tie == mine.tie && i < s);
        }
        r += __shfl_xor_sync(0xffffffffu, r, 1);
        r += __shfl_xor_sync(0xffffffffu, r, 2);
        if (r == K - 1 && tid % 4 == 0) s_bound = mine;
    }
    __syncthreads();
    const Cand bound = s_bound;
    const bool all = bound.total == 0ull;
    const float bound_f = all ? -INFINITY : __double2float_rd(from_order64(bound.total));
    auto take = [&](const Cand &c) {
        if (c.total == 0ull || (!all && better(bound, c))) return;
        const int n = atomicAdd(&s_count, 1);
        if (n < kList) s_list[n] = c;
    };
    // Visits every candidate of the thread that may reach the bound.
    auto visit = [&](auto f) {
        for (int i = tid; i < W * S * K; i += kMergeThreads) {
            const int w = i / (S * K);
            if (!s_open[w]) continue;
            const uint64_t key = keys[i];
            if (key == 0ull) continue;
            if (!all) {  // ruled out in fp32: the sums round twice, the offset once
                const float d = key_value(key) - s_maxf[w], o = s_offf[w];
                if (d + o + 4e-7f * (fabsf(d) + fabsf(o)) < bound_f) continue;
            }
            f(cand(w, key));
        }
        for (int w = tid; w < W; w += kMergeThreads) f(end_of(w));
    };
    visit(take);
    __syncthreads();
    const int n = s_count;
    auto put = [&](int r, const Cand &c) {
        const int64_t o = static_cast<int64_t>(g) * K + r;
        const bool none = c.total == 0ull;
        const int w = none ? 0 : static_cast<int>(c.tie / a.vocab);
        a.out_scores[o] = none ? -INFINITY : static_cast<float>(from_order64(c.total));
        a.out_parents[o] = none ? -1 : g * W + w;
        a.out_tokens[o] = none ? -1 : static_cast<int32_t>(c.tie - static_cast<int64_t>(w) * a.vocab);
    };
    if (n <= kList) {
        for (int i = tid; i < n; i += kMergeThreads) {
            const Cand c = s_list[i];
            int r = 0;
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

// 16-byte chunks of a row that starts anywhere (one more than its bytes fill)
int64_t most_chunks(int64_t vocab, bool fp32) { return fp32 ? (vocab + 3) / 4 + 1 : (vocab + 7) / 8 + 1; }

}  // namespace

// Slices a row: as many CTAs as fit the SMs at once, of a load for each lane at least.
int beam_slices(const fnpu_beam_desc *d) {
    const int64_t rows = static_cast<int64_t>(d->num_groups) * d->num_beams;
    const int64_t chunks = most_chunks(d->vocab, d->dtype == FNPU_LOGITS_FP32);
    const int64_t fit = rows > 0 ? 6 * 152 / rows : 1, most = (chunks + kThreads - 1) / kThreads;
    return static_cast<int>(fit < 1 ? 1 : fit < most ? fit : most);
}

int launch_beam_select(const BeamArgs &a, bool fp32, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int64_t grid = static_cast<int64_t>(a.groups) * a.beams * a.slices;
    auto kernel = fp32 ? beam_slice_kernel<float> : beam_slice_kernel<__nv_bfloat16>;
    FNPU_CUDA_TRY(launch_ex(kernel, static_cast<unsigned>(grid), kThreads, 0, st, true, nullptr, a));
    const size_t smem = static_cast<size_t>(a.beams) * (2 * sizeof(double) + 2 * sizeof(float) + sizeof(int));
    FNPU_CUDA_TRY(launch_ex(beam_merge_kernel, static_cast<unsigned>(a.groups), kMergeThreads, smem, st, true, nullptr, a));
    return FNPU_OK;
}

}  // namespace fnpu
