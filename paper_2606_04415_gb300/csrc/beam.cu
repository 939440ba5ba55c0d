// Selection of a beam search: the best continuations (beam, token) of every
// group of beams, by score[b] + log softmax(logits[b])[v].
//
// What bounds it is the one read of the logits. Two kernels, the second a
// dependent launch of the first:
//   * A CTA of the first holds a slice of one row in registers (up to 32
//     values a thread, all loads in flight at once) and leaves its maximum, the sum
//     of exp(x - max) and its best num_select values in order. Within a row the
//     order of the totals is the order of the logits, ties to the lower token, so a
//     slice's candidates need no normalisation.
//   * A CTA of the second takes a group: the rows' log-sum-exps from their slices'
//     (log-sum-exp combination), then the best of all slices' lists by the total in
//     64 bits. Totals of different beams may lie closer than an fp32 score of some
//     hundred resolves (3e-5); fp64 is slow on this device, so only what an fp32
//     total with its error cannot rule out is added in 64 bits.
// Both choose the best K of many in the same way: the K-th best of 64 subsets'
// bests is a lower bound of the K-th best of all (K values are at least as good), so
// what reaches it is a superset of the best K, seldom much larger; those few are
// ordered by counting the better ones. Where more reach it than the list holds
// (all of a row's large values in few threads), K rounds of a maximum take its place.
#include <float.h>

#include "common.cuh"

namespace fnpu {
namespace {

constexpr int kThreads = 256;       // of the first kernel
constexpr int kMergeThreads = 512;  // of the second
constexpr int kSubsets = 64;        // (threads t mod 64; num_select is at most as many)
constexpr int kList = 512;          // candidates that a list holds

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

template <typename T>
__device__ __forceinline__ float widen(T v);
template <>
__device__ __forceinline__ float widen<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float widen<float>(float v) { return v; }

// A beam without continuations of its own: finished, or without a score.
__device__ __forceinline__ bool row_closed(const BeamArgs &a, int row) {
    const float s = a.scores[row];
    return !(s > -INFINITY) || (a.finished != nullptr && a.finished[row] != 0);
}

template <typename T, int E>
__global__ void __launch_bounds__(kThreads, E == 32 ? 4 : E == 16 ? 5 : 6) beam_slice_kernel(const BeamArgs a) {
    constexpr int kV = 16 / sizeof(T);  // values of a 16-byte load
    constexpr int kN = E / kV;          // loads a thread
    __shared__ uint64_t s_best[kThreads];
    __shared__ uint64_t s_sub[kSubsets];
    __shared__ uint64_t s_list[kList];
    __shared__ float s_part[kThreads / 32];
    __shared__ uint64_t s_bound;
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x - row * a.slices;
    const int K = a.select;
    pdl_trigger();
    pdl_wait();  // the logits and scores of the kernel before, and the last call's reads of the workspace
    if (row_closed(a, row)) return;

    // 16-byte chunks of memory; the row's first and last may hold neighbours' values
    const T *src = static_cast<const T *>(a.logits) + static_cast<int64_t>(row) * a.stride;
    const int head = static_cast<int>((reinterpret_cast<uintptr_t>(src) & 15u) / sizeof(T));
    const T *base = src - head;
    const int chunks = (head + a.vocab + kV - 1) / kV;
    const int per = (chunks + a.slices - 1) / a.slices;
    const int c0 = slice * per, c1 = min(chunks, c0 + per);
    uint4 raw[kN];
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int c = c0 + tid + kThreads * i;
        const int first = c * kV - head;
        if (c < c1 && first >= 0 && first + kV <= a.vocab) raw[i] = __ldcs(reinterpret_cast<const uint4 *>(base) + c);
    }
    float x[E];
    float best = -INFINITY;
    int at = 0;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
        const int c = c0 + tid + kThreads * i;
        const int first = c * kV - head;
        const bool whole = c < c1 && first >= 0 && first + kV <= a.vocab;
        const T *v = reinterpret_cast<const T *>(&raw[i]);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const int e = first + j;
            float y = -INFINITY;
            if (whole) y = widen<T>(v[j]);
            else if (c < c1 && e >= 0 && e < a.vocab) y = widen<T>(src[e]);
            // NaN counts as -inf, +inf as the largest finite value
            y = fminf(fmaxf(y, -INFINITY), FLT_MAX);
            x[i * kV + j] = y;
            if (y > best) {
                best = y;
                at = e;
            }
        }
    }
    // the slice's maximum and its sum of exponentials
    float m = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (lane == 0) s_part[warp] = m;
    s_best[tid] = best > -INFINITY ? row_key(best, at) : 0ull;
    if (tid == 0) s_count = 0;
    __syncthreads();
    m = s_part[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) m = fmaxf(m, s_part[i]);
    __syncthreads();  // (s_part is used again)
    float z = 0.f;
    if (m > -INFINITY) {
#pragma unroll
        for (int j = 0; j < E; ++j) z += fast_exp2((x[j] - m) * kLog2e);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    if (lane == 0) s_part[warp] = z;
    // the K-th best of the subsets' bests
    if (warp == 0) {
        uint64_t k[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int s = lane + 32 * h;
            k[h] = s_best[s];
#pragma unroll
            for (int i = 1; i < kThreads / kSubsets; ++i) k[h] = max(k[h], s_best[s + kSubsets * i]);
            s_sub[s] = k[h];
        }
        __syncwarp();
        int r0 = 0, r1 = 0;  // better ones (of equal ones, which are all 0, those before)
#pragma unroll 8
        for (int s = 0; s < kSubsets; ++s) {
            const uint64_t o = s_sub[s];
            r0 += o > k[0] || (o == k[0] && s < lane);
            r1 += o > k[1] || (o == k[1] && s < lane + 32);
        }
        if (r0 == K - 1) s_bound = k[0];
        if (r1 == K - 1) s_bound = k[1];
    }
    __syncthreads();
    const uint64_t bound = s_bound;
    const float bound_x = bound ? from_order(static_cast<uint32_t>(bound >> 32)) : -INFINITY;
    if (best >= bound_x && best > -INFINITY) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (x[j] >= bound_x && x[j] > -INFINITY) {
                const uint64_t key = row_key(x[j], (c0 + tid + kThreads * (j / kV)) * kV - head + j % kV);
                if (key >= bound) {
                    const int n = atomicAdd(&s_count, 1);
                    if (n < kList) s_list[n] = key;
                }
            }
        }
    }
    __syncthreads();
    const int n = s_count;
    uint64_t *keys = a.keys + static_cast<int64_t>(blockIdx.x) * K;
    if (tid == 0) {
        float sum = s_part[0];
#pragma unroll
        for (int i = 1; i < kThreads / 32; ++i) sum += s_part[i];
        a.parts[blockIdx.x] = make_float2(m, sum);
    }
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
    // K rounds of a maximum
    uint64_t last = ~0ull;
    for (int r = 0; r < K; ++r) {
        uint64_t k = 0ull;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (x[j] > -INFINITY) {
                const uint64_t key = row_key(x[j], (c0 + tid + kThreads * (j / kV)) * kV - head + j % kV);
                if (key < last) k = max(k, key);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) k = max(k, static_cast<uint64_t>(__shfl_xor_sync(0xffffffffu, static_cast<unsigned long long>(k), o)));
        __syncthreads();
        if (lane == 0) s_best[warp] = k;
        __syncthreads();
        k = s_best[0];
#pragma unroll
        for (int i = 1; i < kThreads / 32; ++i) k = max(k, s_best[i]);
        if (tid == 0) keys[r] = k;
        last = k;
        if (k == 0ull) last = 0ull;
    }
}

// A candidate of a group: a larger total is better, ties to the lower beam and token.
struct Cand {
    double total;
    int64_t tie;  // beam * vocab + token; -1: none
};
__device__ __forceinline__ bool better(const Cand &a, const Cand &b) {
    if (a.tie < 0 || b.tie < 0) return a.tie >= 0 && b.tie < 0;
    return a.total > b.total || (a.total == b.total && a.tie < b.tie);
}

__global__ void __launch_bounds__(kMergeThreads) beam_merge_kernel(const BeamArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    // of the group's beams: maximum logit, score - log sum exp(x - maximum), and both in fp32
    double *s_max = reinterpret_cast<double *>(smem), *s_off = s_max + a.beams;
    float *s_offf = reinterpret_cast<float *>(s_off + a.beams);
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
            s_max[w] = m;
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
        return Cand{(static_cast<double>(from_order(static_cast<uint32_t>(key >> 32))) - s_max[w]) + s_off[w],
                    static_cast<int64_t>(w) * a.vocab + static_cast<int64_t>(0xFFFFFFFFu - static_cast<uint32_t>(key))};
    };
    auto end_of = [&](int w) {  // the one continuation of a finished beam
        const int row = g * W + w;
        const float s = a.scores[row];
        if (a.finished == nullptr || a.finished[row] == 0 || a.end_token < 0 || !(s > -INFINITY)) return Cand{0.0, -1};
        return Cand{static_cast<double>(s), static_cast<int64_t>(w) * a.vocab + a.end_token};
    };
    // each thread's best of the lists' heads, and the K-th best of the subsets of threads
    Cand best{0.0, -1};
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
    if (warp == 0) {
        Cand k[2];
        for (int h = 0; h < 2; ++h) {
            const int s = lane + 32 * h;
            k[h] = s_best[s];
            for (int i = 1; i < kMergeThreads / kSubsets; ++i)
                if (better(s_best[s + kSubsets * i], k[h])) k[h] = s_best[s + kSubsets * i];
            s_sub[s] = k[h];
        }
        __syncwarp();
        int r0 = 0, r1 = 0;
        for (int s = 0; s < kSubsets; ++s) {
            const Cand o = s_sub[s];
            r0 += better(o, k[0]) || (!better(k[0], o) && s < lane);
            r1 += better(o, k[1]) || (!better(k[1], o) && s < lane + 32);
        }
        if (r0 == K - 1) s_bound = k[0];
        if (r1 == K - 1) s_bound = k[1];
    }
    __syncthreads();
    const Cand bound = s_bound;
    const bool all = bound.tie < 0;
    const float bound_f = __double2float_rd(bound.total);
    auto take = [&](const Cand &c) {
        if (c.tie < 0 || (!all && better(bound, c))) return;
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
                const float d = from_order(static_cast<uint32_t>(key >> 32)) - static_cast<float>(s_max[w]), o = s_offf[w];
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
        const int w = c.tie < 0 ? 0 : static_cast<int>(c.tie / a.vocab);
        a.out_scores[o] = c.tie < 0 ? -INFINITY : static_cast<float>(c.total);
        a.out_parents[o] = c.tie < 0 ? -1 : g * W + w;
        a.out_tokens[o] = c.tie < 0 ? -1 : static_cast<int32_t>(c.tie - static_cast<int64_t>(w) * a.vocab);
    };
    if (n <= kList) {
        for (int i = tid; i < n; i += kMergeThreads) {
            const Cand c = s_list[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += better(s_list[j], c);
            if (r < K) put(r, c);
        }
        for (int i = n + tid; i < K; i += kMergeThreads) put(i, Cand{0.0, -1});
        return;
    }
    Cand last{0.0, -1};  // K rounds of a maximum below the last one
    for (int r = 0; r < K; ++r) {
        Cand c{0.0, -1};
        visit([&](const Cand &o) {
            if (o.tie >= 0 && (r == 0 || better(last, o)) && better(o, c)) c = o;
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
        if (last.tie < 0) {  // none left
            for (int i = r + 1 + tid; i < K; i += kMergeThreads) put(i, last);
            return;
        }
    }
}

template <typename T>
int launch_slices(const BeamArgs &a, int values, cudaStream_t st) {
    const int64_t grid = static_cast<int64_t>(a.groups) * a.beams * a.slices;
    auto kernel = values == 8 ? beam_slice_kernel<T, 8> : values == 16 ? beam_slice_kernel<T, 16> : beam_slice_kernel<T, 32>;
    FNPU_CUDA_TRY(launch_ex(kernel, static_cast<unsigned>(grid), kThreads, 0, st, true, nullptr, a));
    return FNPU_OK;
}

// 16-byte chunks of a row that starts anywhere (one more than its bytes fill)
int64_t most_chunks(int64_t vocab, bool fp32) { return fp32 ? (vocab + 3) / 4 + 1 : (vocab + 7) / 8 + 1; }

}  // namespace

// Values a thread of a slice and slices a row: the longest slices that leave every
// SM its CTAs (few rows: shorter ones, so that more SMs share a row).
void beam_split(const fnpu_beam_desc *d, int *values, int *slices) {
    const bool fp32 = d->dtype == FNPU_LOGITS_FP32;
    const int64_t rows = static_cast<int64_t>(d->num_groups) * d->num_beams, chunks = most_chunks(d->vocab, fp32);
    for (int v = 32;; v /= 2) {
        const int64_t per = kThreads * (v / (fp32 ? 4 : 8));
        *values = v;
        *slices = static_cast<int>((chunks + per - 1) / per);
        if (v == 8 || rows * *slices >= 4 * 152) return;
    }
}

int launch_beam_select(const BeamArgs &a, int values, bool fp32, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int rc = fp32 ? launch_slices<float>(a, values, st) : launch_slices<__nv_bfloat16>(a, values, st);
    if (rc != FNPU_OK) return rc;
    const size_t smem = static_cast<size_t>(a.beams) * (2 * sizeof(double) + sizeof(float) + sizeof(int));
    FNPU_CUDA_TRY(launch_ex(beam_merge_kernel, static_cast<unsigned>(a.groups), kMergeThreads, smem, st, true, nullptr, a));
    return FNPU_OK;
}

}  // namespace fnpu
