// Writing to and reading from the 8-bit cache with a scale per block and kv head.
#include "kv8.cuh"
#include "rope.cuh"

namespace fnpu {
namespace {

// ------------------------------------------------------------------ append
//
// The rows that a call stores in one block are a run: consecutive tokens at
// consecutive slots of it. They and the rows before them share one scale per kv
// head, so a run is one piece of work per kv head and side (K or V): take the
// largest magnitude of its rows, and where that asks for a larger exponent than the
// block has, store the rows before the run anew. A block whose slot 0 is in the
// run is a fresh one; what it held and its scale are dead.
//
// A CTA has a warp for each 512 values of a block and kv head, 16 columns a lane (the
// eight pairs that a lane turns among them), so that rows are loaded, turned and
// stored in one pass through few registers. It looks for runs that begin in a window
// of tokens, one token while the grid is one wave: no list of runs to build. A run of
// no more rows than a warp has at once (a decode step's have one) is one warp's, and
// the warps take such runs in turn; a longer one is the CTA's, whose warps meet for the
// largest magnitude. (One run after the other by the whole CTA, 86 rows of 8 kv heads
// into blocks of 32: 16.1 us with their reading back, 9.7 so.) The queries are
// turned by further CTAs of the same launch.
template <int kFormat, int kD>
struct RunRows {
    static constexpr int kLanesPerRow = kD / 16, kRows = 32 / kLanesPerRow;  // rows that a warp has at once
};

// whole: by all warps of the CTA, each its rows of the block; else by this warp alone.
template <int kFormat, int kD>
__device__ __forceinline__ void append_run(const RopeArgs &r, const RopeAppendArgs &p, int64_t t, int64_t slot, int n, int head,
                                           bool is_v, bool whole, uint32_t *amax_sh) {
    constexpr int kLanesPerRow = RunRows<kFormat, kD>::kLanesPerRow, kRows = RunRows<kFormat, kD>::kRows;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int bs = p.block_size;
    const int off = static_cast<int>(slot & (bs - 1));
    uint8_t *blk = static_cast<uint8_t *>(is_v ? p.v_cache : p.k_cache) + (slot >> (__ffs(bs) - 1)) * kv8::block_bytes(p.kv_heads, bs, kD);
    uint8_t *rows = blk + static_cast<int64_t>(head) * bs * kD;
    float *scale = reinterpret_cast<float *>(blk + static_cast<int64_t>(p.kv_heads) * bs * kD) + head;
    const int e_old = off > 0 ? kv8::scale_exp(*scale) : kv8::kMinExp;
    const int o = (whole ? warp * kRows : off) + lane / kLanesPerRow, c = lane % kLanesPerRow;  // this lane's row and columns
    const int cp = is_v ? 0 : r.pairs >> 3;
    int ca, cb;
    if (c < cp) {
        rope_columns<8>(r, c, ca, cb);
    } else {  // 16 columns that do not turn
        ca = 16 * (c - cp);
        if (cp > 0 && ca >= r.offset) ca += 2 * r.pairs;
        cb = ca + 8;
    }
    const bool fresh = o >= off && o < off + n;
    float a[8], b[8];
    {
        uint4 ra = make_uint4(0u, 0u, 0u, 0u), rb = ra;
        if (fresh) {
            const __nv_bfloat16 *src = (is_v ? p.v_new : p.k_new) + (t + o - off) * (is_v ? p.v_stride : p.k_stride) +
                                       static_cast<int64_t>(head) * kD;
            ra = __ldg(reinterpret_cast<const uint4 *>(src + ca));
            rb = __ldg(reinterpret_cast<const uint4 *>(src + cb));
        }
        float cs[8], sn[8];
        if (fresh && c < cp) rope_angles<8>(r, t + o - off, c, cs, sn);  // while the row comes
        bf16_to_f32<8>(ra, a);
        bf16_to_f32<8>(rb, b);
        if (fresh && c < cp) rope_rotate<8>(r.interleaved != 0, cs, sn, a, b);
    }
    float amax = 0.f, zero = 0.f;  // (zero: NaN if a value is not finite)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        zero = __fmaf_rn(a[j], 0.f, zero);
        zero = __fmaf_rn(b[j], 0.f, zero);
        amax = fmax3(amax, fabsf(a[j]), fabsf(b[j]));
    }
    const bool odd = zero != 0.f;
    if (odd) {  // NaN is stored as zero, an infinity as the largest magnitude that the others allow
        amax = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (a[j] != a[j]) a[j] = 0.f;
            if (b[j] != b[j]) b[j] = 0.f;
            if (fabsf(a[j]) < INFINITY) amax = fmaxf(amax, fabsf(a[j]));
            if (fabsf(b[j]) < INFINITY) amax = fmaxf(amax, fabsf(b[j]));
        }
        atomicOr(p.err, 8);
    }
    // (non-negative floats order as integers)
    uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(amax));
    if (whole) {
        if (lane == 0) amax_sh[warp] = top;
        __syncthreads();  // (also: every warp has the old scale)
        for (int i = 0; i < warps; ++i) top = max(top, amax_sh[i]);
        __syncthreads();  // before another run's magnitudes
    }
    int e = max(e_old, kv8::required_exp<kFormat>(__uint_as_float(top)));
    const bool over = e > kv8::kMaxExp;
    if (over) {
        e = kv8::kMaxExp;
        if (lane == 0) atomicOr(p.err, 8);
    }
    if (over || odd) {
        const float most = kv8::kLargest<kFormat> * kv8::pow2(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            a[j] = fminf(fmaxf(a[j], -most), most);
            b[j] = fminf(fmaxf(b[j], -most), most);
        }
    }
    if (fresh) {
        const float inv = kv8::pow2(-e);
        *reinterpret_cast<uint2 *>(rows + o * kD + ca) = kv8::encode8<kFormat>(a, inv);
        *reinterpret_cast<uint2 *>(rows + o * kD + cb) = kv8::encode8<kFormat>(b, inv);
    }
    if (e > e_old) {  // the rows that the block held before, over the grown scale
        const float down = kv8::pow2(e_old - e);
        for (int i = (whole ? warp * kRows : 0) + lane / kLanesPerRow; i < off; i += whole ? bs : kRows)
            for (int s = 0; s < 2; ++s) {
                uint2 *at = reinterpret_cast<uint2 *>(rows + i * kD + (s ? cb : ca));
                const uint2 w = *at;
                float x[4], y[4];
                kv8::decode4<kFormat>(w.x, x);
                kv8::decode4<kFormat>(w.y, y);
                const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                *at = kv8::encode8<kFormat>(f, down);
            }
    }
    if (lane == 0 && (!whole || warp == 0) && (off == 0 || e > e_old)) *scale = kv8::pow2(e);
}

template <int kFormat, int kD>
__global__ void __launch_bounds__(512, 2)
    kv8_append_kernel(const __grid_constant__ RopeArgs r, const __grid_constant__ RopeAppendArgs p, int kv_ctas, int window,
                      int q_groups, int q_heads_per_warp) {
    constexpr int kRows = RunRows<kFormat, kD>::kRows;
    __shared__ uint32_t amax_sh[16];
    pdl_trigger();
    pdl_wait();  // writers of the rows, earlier readers of the blocks
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (static_cast<int>(blockIdx.x) >= kv_ctas) {
        const int64_t w = static_cast<int64_t>(blockIdx.x - kv_ctas) * warps + warp, t = w / q_groups;
        if (t >= r.n) return;
        const int h0 = static_cast<int>(w - t * q_groups) * q_heads_per_warp;
        rope_heads<8>(r, t, h0, min(p.q_heads, h0 + q_heads_per_warp), kD, lane, rope_lane<false>(lane, rope_lanes(8, r.pairs, kD), 1),
                      [&](int h) { return p.q + t * p.q_stride + static_cast<int64_t>(h) * kD; },
                      [&](int h) { return p.q_out + (t * p.q_heads + h) * kD; });
        return;
    }
    // tokens t0 .. t0 + window - 1 of one kv head and side; every warp finds the same runs
    const int per = 2 * p.kv_heads, w = blockIdx.x / per, j = blockIdx.x - w * per;
    const bool is_v = j >= p.kv_heads;
    const int head = is_v ? j - p.kv_heads : j;
    const int64_t t0 = static_cast<int64_t>(w) * window;
    int64_t slot = -1;
    bool begins = false;
    if (lane < window && t0 + lane < r.n) {
        const int64_t t = t0 + lane, before = t > 0 ? __ldg(p.slots + t - 1) : -1;
        slot = __ldg(p.slots + t);
        if (slot >= p.num_slots) {
            if (j == 0) atomicOr(p.err, 1);
            slot = -1;
        }
        begins = slot >= 0 && ((slot & (p.block_size - 1)) == 0 || before != slot - 1);
    }
    const uint32_t goes_on = __ballot_sync(0xffffffffu, slot >= 0 && !begins);
    int turn = 0;  // of the short runs
    for (uint32_t todo = __ballot_sync(0xffffffffu, begins); todo; todo &= todo - 1) {
        const int at = __ffs(todo) - 1;
        const int64_t t = t0 + at, s = __shfl_sync(0xffffffffu, slot, at);
        const int room = p.block_size - static_cast<int>(s & (p.block_size - 1));
        // rows of the run: tokens t + i at slot s + i, within the block; past the window, look
        int n = at == 31 ? 1 : __ffs(~(goes_on >> (at + 1)));
        if (at + n == window)
            for (int i0 = n; i0 < room; i0 += 32) {
                const int i = i0 + lane;
                const bool more = i < room && t + i < r.n && __ldg(p.slots + t + i) == s + i;
                const uint32_t miss = ~__ballot_sync(0xffffffffu, more);
                n += miss ? __ffs(miss) - 1 : 32;
                if (miss) break;
            }
        const bool whole = n > kRows;  // the CTA's, else the warp's whose turn it is
        if (!whole) {
            const bool mine = turn == warp;
            turn = turn + 1 == warps ? 0 : turn + 1;
            if (!mine) continue;
        }
        append_run<kFormat, kD>(r, p, t, s, n, head, is_v, whole, amax_sh);
    }
}

// -------------------------------------------------------------------- read

// 16 codes, scaled, as two 16-byte chunks of bf16 (exact)
template <int kFormat>
__device__ __forceinline__ void codes_to_bf16(const uint4 &w, float scale, uint4 &lo, uint4 &hi) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t out[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[4];
        kv8::decode4<kFormat>(in[i], f);
        out[2 * i] = pack_bf16x2(f[0] * scale, f[1] * scale);
        out[2 * i + 1] = pack_bf16x2(f[2] * scale, f[3] * scale);
    }
    lo = make_uint4(out[0], out[1], out[2], out[3]);
    hi = make_uint4(out[4], out[5], out[6], out[7]);
}

// A warp per row and side, 16 values a lane.
template <int kFormat>
__global__ void __launch_bounds__(256)
    kv8_read_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool, const int64_t *__restrict__ slots,
                    int64_t n, int64_t num_slots, int hkv, int bs, int d, uint4 *__restrict__ k_out, uint4 *__restrict__ v_out,
                    int *err) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x & 31, sh = d == 64 ? 2 : 3, per = hkv << sh;  // chunks of a row: 4 or 8 a kv head
    const int64_t bytes = kv8::block_bytes(hkv, bs, d), step = gridDim.x * 8ll;
    for (int64_t w = blockIdx.x * 8ll + (threadIdx.x >> 5); w < 2 * n; w += step) {
        const int64_t row = w >> 1;
        const bool v = (w & 1) != 0;
        const int64_t slot = __ldg(slots + row);
        const bool in = slot >= 0 && slot < num_slots;
        if (slot >= num_slots && !v && lane == 0) atomicOr(err, 1);
        const uint8_t *blk = (v ? v_pool : k_pool) + (in ? slot >> (__ffs(bs) - 1) : 0) * bytes;
        const int o = static_cast<int>(slot & (bs - 1));
        uint4 *to = (v ? v_out : k_out) + 2 * row * per;
        for (int i = lane; i < per; i += 32) {
            const int h = i >> sh, c = i & ((1 << sh) - 1);
            uint4 lo = make_uint4(0u, 0u, 0u, 0u), hi = lo;
            if (in) {
                const uint4 x = __ldg(reinterpret_cast<const uint4 *>(blk + (static_cast<int64_t>(h) * bs + o) * d) + c);
                const float scale = __ldg(reinterpret_cast<const float *>(blk + static_cast<int64_t>(hkv) * bs * d) + h);
                codes_to_bf16<kFormat>(x, scale, lo, hi);
            }
            to[2 * i] = lo;
            to[2 * i + 1] = hi;
        }
    }
}

__global__ void __launch_bounds__(256)
    kv_read_bf16_kernel(const uint4 *__restrict__ k_cache, const uint4 *__restrict__ v_cache, const int64_t *__restrict__ slots,
                        int64_t n, int64_t num_slots, int k_chunks, int v_chunks, uint4 *__restrict__ k_out,
                        uint4 *__restrict__ v_out, int *err) {
    pdl_trigger();
    pdl_wait();
    const int per = k_chunks + v_chunks;
    for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < n * per; i += gridDim.x * 256ll) {
        const int64_t row = i / per;
        const int c = static_cast<int>(i - row * per);
        const int64_t slot = __ldg(slots + row);
        uint4 w = make_uint4(0u, 0u, 0u, 0u);
        if (slot >= num_slots) {
            if (c == 0) atomicOr(err, 1);
        } else if (slot >= 0) {
            w = c < k_chunks ? __ldg(k_cache + slot * k_chunks + c) : __ldg(v_cache + slot * v_chunks + c - k_chunks);
        }
        if (c < k_chunks) k_out[row * k_chunks + c] = w;
        else v_out[row * v_chunks + c - k_chunks] = w;
    }
}

// ----------------------------------------------------------------- staging
//
// The tcgen05 prefill takes bf16 operands, which hold the stored values exactly; f16
// would not hold their range. Its weights are then bf16 too, 2^-9 off at most each where the
// decode kernel's are f16 and 2^-11: whether a middle chunk is staged depends on the step.
// A CTA writes one kv head of a source block, K and V, as bf16 rows [slots][kv
// heads][d] of block `dst`; rows past `valid` are zero.
template <int kFormat>
__global__ void __launch_bounds__(128)
    kv8_stage_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool, const Fp8StageJob *__restrict__ jobs,
                     int hkv, int bs, int d, uint4 *__restrict__ k_out, uint4 *__restrict__ v_out) {
    pdl_trigger();
    pdl_wait();  // the codes of the kernel before (the step's append)
    const Fp8StageJob jb = jobs[blockIdx.x / hkv];
    const int h = blockIdx.x % hkv;
    const int per_row = d >> 4, sh = d == 64 ? 2 : 3, per = bs * per_row;
    const int64_t src = jb.src * kv8::block_bytes(hkv, bs, d), codes = static_cast<int64_t>(hkv) * bs * d;
    const float ks = __ldg(reinterpret_cast<const float *>(k_pool + src + codes) + h);
    const float vs = __ldg(reinterpret_cast<const float *>(v_pool + src + codes) + h);
    for (int i = threadIdx.x; i < per; i += 128) {
        const int o = i >> sh, c = i & (per_row - 1);
        const int64_t from = src + (static_cast<int64_t>(h) * bs + o) * d;
        const uint4 kw = __ldg(reinterpret_cast<const uint4 *>(k_pool + from) + c);
        const uint4 vw = __ldg(reinterpret_cast<const uint4 *>(v_pool + from) + c);
        const int64_t to = (((static_cast<int64_t>(jb.dst) * bs + o) * hkv + h) * per_row + c) * 2;
        uint4 z = make_uint4(0u, 0u, 0u, 0u), klo = z, khi = z, vlo = z, vhi = z;
        if (o < jb.valid) {
            codes_to_bf16<kFormat>(kw, ks, klo, khi);
            codes_to_bf16<kFormat>(vw, vs, vlo, vhi);
        }
        k_out[to] = klo;
        k_out[to + 1] = khi;
        v_out[to] = vlo;
        v_out[to + 1] = vhi;
    }
}

int sm_count() {
    int dev = 0, sms = 152;
    cudaGetDevice(&dev);
    cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms;
}

template <int kFormat, int kD>
int launch_append(const RopeArgs &r, const RopeAppendArgs &p, cudaStream_t st) {
    const int warps = p.block_size * kD / 512, per = 2 * p.kv_heads;
    // one token a CTA in one wave of 32 warps an SM
    const int64_t wave = 32ll * sm_count() / warps, all = r.n * per;
    const int window = static_cast<int>(all <= wave ? 1 : all >= 32 * wave ? 32 : (all + wave - 1) / wave);
    const int64_t kv_ctas = (r.n + window - 1) / window * per;
    int groups = 1, hpw = 1;
    int64_t q_ctas = 0;
    if (p.q && p.q_heads > 0) {
        hpw = rope_split(r.n, p.q_heads, 8, r.pairs, p.d, 32, 4, false).heads;
        groups = (p.q_heads + hpw - 1) / hpw;
        q_ctas = (r.n * groups + warps - 1) / warps;
    }
    if (kv_ctas + q_ctas > INT32_MAX) return FNPU_EUNSUPPORTED;
    FNPU_CUDA_TRY(launch_ex(kv8_append_kernel<kFormat, kD>, static_cast<int>(kv_ctas + q_ctas), 32 * warps, 0, st, true, nullptr, r, p,
                            static_cast<int>(kv_ctas), window, groups, hpw));
    return FNPU_OK;
}

}  // namespace

bool kv8_supported(const fnpu_attn_desc *d) {
    return !d->v_in_k_latent && d->kv_fp8 == 0 && d->head_dim_qk == d->head_dim_v && (d->head_dim_qk == 64 || d->head_dim_qk == 128) &&
           (d->block_size == 16 || d->block_size == 32 || d->block_size == 64);
}

int64_t kv8_block_bytes(int hkv, int block_size, int d) { return kv8::block_bytes(hkv, block_size, d); }

int launch_kv8_append(int format, const RopeArgs &r, const RopeAppendArgs &p, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (format == FNPU_KV_INT8_BLOCK)
        return p.d == 64 ? launch_append<FNPU_KV_INT8_BLOCK, 64>(r, p, st) : launch_append<FNPU_KV_INT8_BLOCK, 128>(r, p, st);
    return p.d == 64 ? launch_append<FNPU_KV_E4M3_BLOCK, 64>(r, p, st) : launch_append<FNPU_KV_E4M3_BLOCK, 128>(r, p, st);
}

int launch_kv8_read(int format, const fnpu_attn_desc *d, const int64_t *slots, int32_t n, const void *k_pool, const void *v_pool,
                    void *k_out, void *v_out, int *err, void *stream) {
    const int64_t want = (2ll * n + 7) / 8, cap = 32ll * sm_count();
    const int grid = static_cast<int>(want < cap ? want : cap);
    auto kernel = format == FNPU_KV_INT8_BLOCK ? kv8_read_kernel<FNPU_KV_INT8_BLOCK> : kv8_read_kernel<FNPU_KV_E4M3_BLOCK>;
    FNPU_CUDA_TRY(launch_ex(kernel, grid, 256, 0, static_cast<cudaStream_t>(stream), true, nullptr,
                            static_cast<const uint8_t *>(k_pool), static_cast<const uint8_t *>(v_pool), slots, static_cast<int64_t>(n),
                            static_cast<int64_t>(d->num_blocks) * d->block_size, static_cast<int>(d->num_kv_heads),
                            static_cast<int>(d->block_size), static_cast<int>(d->head_dim_qk), static_cast<uint4 *>(k_out),
                            static_cast<uint4 *>(v_out), err));
    return FNPU_OK;
}

int launch_kv_read_bf16(const fnpu_attn_desc *d, const int64_t *slots, int32_t n, const void *k_cache, const void *v_cache,
                        void *k_out, void *v_out, int *err, void *stream) {
    const int kc = d->num_kv_heads * d->head_dim_qk / 8, vc = d->v_in_k_latent ? 0 : d->num_kv_heads * d->head_dim_v / 8;
    const int64_t want = (static_cast<int64_t>(n) * (kc + vc) + 255) / 256, cap = 32ll * sm_count();
    const int grid = static_cast<int>(want < cap ? want : cap);
    FNPU_CUDA_TRY(launch_ex(kv_read_bf16_kernel, grid, 256, 0, static_cast<cudaStream_t>(stream), true, nullptr,
                            static_cast<const uint4 *>(k_cache), static_cast<const uint4 *>(v_cache), slots, static_cast<int64_t>(n),
                            static_cast<int64_t>(d->num_blocks) * d->block_size, kc, vc, static_cast<uint4 *>(k_out),
                            static_cast<uint4 *>(v_out), err));
    return FNPU_OK;
}

int launch_kv8_stage(int format, const fnpu_attn_desc *d, const void *k_pool, const void *v_pool, const Fp8StageJob *jobs,
                     int32_t num_jobs, void *k_bf16, void *v_bf16, void *stream, bool pdl) {
    if (num_jobs == 0) return FNPU_OK;
    auto kernel = format == FNPU_KV_INT8_BLOCK ? kv8_stage_kernel<FNPU_KV_INT8_BLOCK> : kv8_stage_kernel<FNPU_KV_E4M3_BLOCK>;
    FNPU_CUDA_TRY(launch_ex(kernel, num_jobs * d->num_kv_heads, 128, 0, static_cast<cudaStream_t>(stream), pdl, nullptr,
                            static_cast<const uint8_t *>(k_pool), static_cast<const uint8_t *>(v_pool), jobs,
                            static_cast<int>(d->num_kv_heads), static_cast<int>(d->block_size), static_cast<int>(d->head_dim_qk),
                            static_cast<uint4 *>(k_bf16), static_cast<uint4 *>(v_bf16)));
    return FNPU_OK;
}

}  // namespace fnpu
