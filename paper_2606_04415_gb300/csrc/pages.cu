// The pages of a cache on the device: rows of a block table that share, fork, give
// up and move blocks, with a count of holders for each block, and the copies
// that go with it.
//
// The tables are small (some MB at most), so what bounds these calls is the chain
// of dependent steps: counts before free blocks, free blocks before their rows. Each
// step is a kernel over all SMs and a dependent launch of the one before. Every
// result is independent of the order of the atomics: counts are sums, the lowest row
// of a page a minimum, and the k-th block that is taken is the k-th free one by id, by a
// prefix sum over chunks of counts that each CTA forms for itself.
#include <limits.h>

#include "common.cuh"

namespace fnpu {
namespace {

constexpr int kRowThreads = 256;    // kernels over rows
constexpr int kScanThreads = 512;   // kernels over chunks of counts
constexpr int kPer = kPagesChunk / kScanThreads;

// States of a new row, where its last page is full or there is none to write to.
constexpr int kRowFull = -1;   // goes on with new blocks
constexpr int kRowStuck = -2;  // cannot grow: past the table, or its last page is gone
constexpr int kRowEmpty = -3;  // continues nothing

__device__ __forceinline__ int entries(int length, int bs) { return (length + bs - 1) / bs; }
__device__ __forceinline__ bool length_ok(const PagesArgs &a, int n) {
    return n >= 0 && n <= static_cast<int64_t>(a.width) * a.block_size;
}
// One holder less; a count that is not there is left at what it is.
__device__ __forceinline__ void drop(const PagesArgs &a, int page) {
    if (atomicSub(a.refs + page, 1) < 1) {
        atomicAdd(a.refs + page, 1);
        atomicOr(a.err, 1);
    }
}

template <int kThreads>
__device__ __forceinline__ int block_sum(int v, int *s) {  // s: [kThreads / 32]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();
    if (lane == 0) s[warp] = v;
    __syncthreads();
    v = 0;
    for (int i = 0; i < kThreads / 32; ++i) v += s[i];
    return v;
}
// The sum over the threads before this one; *total: of all.
template <int kThreads>
__device__ __forceinline__ int block_before(int v, int *s, int *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int up = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += x;
    }
    __syncthreads();
    if (lane == 31) s[warp] = up;
    __syncthreads();
    int before = up - v, all = 0;
    for (int i = 0; i < kThreads / 32; ++i) {
        if (i < warp) before += s[i];
        all += s[i];
    }
    *total = all;
    return before;
}

// Rows give pages up: a CTA a row.
__global__ void __launch_bounds__(kRowThreads) pages_free_kernel(const PagesArgs a, int32_t *length, const uint8_t *ends, int window, int sinks) {
    pdl_trigger();
    pdl_wait();
    const int r = blockIdx.x, bs = a.block_size;
    const int n = length[r];
    const bool end = ends != nullptr && ends[r] != 0;
    if (!length_ok(a, n)) {
        if (threadIdx.x == 0) atomicOr(a.err, 1);
        return;
    }
    int c0 = 0, c1 = entries(n, bs);
    if (!end) {
        if (window < 1 || n + 1 <= window) return;
        c1 = min(c1, (n + 1 - window) / bs);
        if (sinks > (c1 - 1) * bs) return;  // (and the entries of more sinks than that do not fit 32 bits)
        c0 = (sinks + bs - 1) / bs;
    }
    int32_t *row = a.table + static_cast<int64_t>(r) * a.width;
    for (int c = c0 + static_cast<int>(threadIdx.x); c < c1; c += kRowThreads) {
        const int e = row[c];
        if (e < 0) continue;
        if (e < a.num_blocks) drop(a, e);
        else atomicOr(a.err, 1);
        row[c] = -1;
    }
    if (end) {
        __syncthreads();  // (every thread has read the length)
        if (threadIdx.x == 0) length[r] = 0;
    }
}

// Fork, first step. CTAs 0 .. new_rows - 1: a new row's entries. The others: an old
// row's pages get as many holders more as rows continue it, less the one that it was
// (nothing to do where one row does, the usual case late in a search).
__global__ void __launch_bounds__(kRowThreads) fork_rows_kernel(const PagesArgs a) {
    __shared__ int s_sum[kRowThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, bs = a.block_size;
    if (static_cast<int>(blockIdx.x) < a.new_rows) {
        const int r = blockIdx.x;
        const int p = a.parents ? a.parents[r] : r;
        bool ok = p >= 0 && p < a.rows;
        if (p >= a.rows && tid == 0) atomicOr(a.err, 1);
        const int n = ok ? a.length[p] : 0;
        ok = ok && length_ok(a, n);
        const int held = ok ? entries(n, bs) : 0;
        const int32_t *from = a.table + static_cast<int64_t>(ok ? p : 0) * a.width;
        int32_t *to = a.new_table + static_cast<int64_t>(r) * a.width;
        for (int c = tid; c < a.width; c += kRowThreads) {
            int e = c < held ? from[c] : -1;
            if (e >= a.num_blocks) atomicOr(a.err, 1);
            if (e < 0 || e >= a.num_blocks) e = -1;
            to[c] = e;
        }
        if (tid == 0) {
            int tail = kRowFull;
            if (!ok) tail = kRowEmpty;
            else if (a.grow > 0 && static_cast<int64_t>(n) + a.grow > static_cast<int64_t>(a.width) * bs) tail = kRowStuck;
            else if (a.grow > 0 && n % bs != 0) {
                const int e = from[n / bs];
                tail = e >= 0 && e < a.num_blocks ? e : kRowStuck;
            }
            a.row_length[r] = ok ? n : 0;
            a.row_tail[r] = tail;
            if (tail >= 0) {  // (the same for every row with this page)
                a.block_a[tail] = 0;
                a.block_b[tail] = INT_MAX;
            }
        }
        return;
    }
    const int p = static_cast<int>(blockIdx.x) - a.new_rows;
    const int n = a.length[p];
    if (!length_ok(a, n)) {
        if (tid == 0) atomicOr(a.err, 1);
        return;
    }
    int next = a.new_rows > 0 ? 1 : 0;  // (no new rows: nobody continues any)
    if (a.parents) {
        int mine = 0;
        for (int r = tid; r < a.new_rows; r += kRowThreads) mine += a.parents[r] == p;
        next = block_sum<kRowThreads>(mine, s_sum);
    }
    const int32_t *row = a.table + static_cast<int64_t>(p) * a.width;
    for (int c = tid; c < entries(n, bs); c += kRowThreads) {
        const int e = row[c];
        if (e >= a.num_blocks) atomicOr(a.err, 1);
        if (e < 0 || e >= a.num_blocks || next == 1) continue;
        if (next > 1) atomicAdd(a.refs + e, next - 1);
        else drop(a, e);
    }
}

// Second step: the free blocks of each chunk, and the rows of each last page.
__global__ void __launch_bounds__(kScanThreads) fork_count_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x;
    if (static_cast<int>(blockIdx.x) < a.chunks) {
        int n = 0;
        const int c0 = blockIdx.x * kPagesChunk;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = c0 + i * kScanThreads + tid;
            n += id < a.num_blocks && a.refs[id] <= 0;
        }
        n = block_sum<kScanThreads>(n, s_sum);
        if (tid == 0) a.chunk_count[blockIdx.x] = n;
        return;
    }
    const int r = (static_cast<int>(blockIdx.x) - a.chunks) * kScanThreads + tid;
    if (r >= a.new_rows) return;
    const int tail = a.row_tail[r];
    if (tail < 0) return;
    atomicAdd(a.block_a + tail, 1);
    atomicMin(a.block_b + tail, r);
    a.row_refs[r] = a.refs[tail];
}

// Third step: a CTA a chunk. Each forms the rows' needs and their prefix sums, and
// hands its own free blocks to the rows whose turn they are; CTA 0 does what is
// left of every row.
__global__ void __launch_bounds__(kScanThreads) fork_take_kernel(const PagesArgs a) {
    extern __shared__ int s_off[];  // [new_rows + 1]: blocks that the rows before need * 2 + (it copies)
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, bs = a.block_size, R = a.new_rows;
    int before = 0, all = 0;
    for (int c = tid; c < a.chunks; c += kScanThreads) {
        const int n = a.chunk_count[c];
        all += n;
        if (c < static_cast<int>(blockIdx.x)) before += n;
    }
    before = block_sum<kScanThreads>(before, s_sum);
    const int free_blocks = block_sum<kScanThreads>(all, s_sum);
    auto need_of = [&](int r, bool *copy) {
        const int tail = a.row_tail[r], n = a.row_length[r];
        *copy = tail >= 0 && (a.block_b[tail] != r || a.row_refs[r] > a.block_a[tail]);
        return tail < kRowFull ? 0 : (*copy ? 1 : 0) + entries(n + a.grow, bs) - entries(n, bs);
    };
    const int per = (R + kScanThreads - 1) / kScanThreads;
    int mine = 0;
    bool copy;
    for (int r = tid * per; r < min(R, (tid + 1) * per); ++r) mine += need_of(r, &copy);
    int needed;
    int off = block_before<kScanThreads>(mine, s_sum, &needed);
    for (int r = tid * per; r < min(R, (tid + 1) * per); ++r) {
        const int n = need_of(r, &copy);
        s_off[r] = 2 * off + (copy ? 1 : 0);
        off += n;
    }
    if (tid == 0) s_off[R] = 2 * needed;
    __syncthreads();
    auto served = [&](int r) {
        const int o = s_off[r] >> 1, e = s_off[r + 1] >> 1;
        return e == o || e <= free_blocks;
    };
    if (before < needed) {
        // the chunk's free blocks in order, `kPer` neighbours a thread
        const int id0 = blockIdx.x * kPagesChunk + tid * kPer;
        uint32_t is_free = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (id0 + i < a.num_blocks && a.refs[id0 + i] <= 0) is_free |= 1u << i;
        int unused;
        int f = before + block_before<kScanThreads>(__popc(is_free), s_sum, &unused);  // (and all have read before any writes)
        for (int i = 0; i < kPer && f < needed; ++i) {
            if (!(is_free >> i & 1u)) continue;
            const int id = id0 + i, turn = f++;
            int lo = 0, hi = R - 1;  // the last row whose blocks begin at `turn` or before
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if ((s_off[mid] >> 1) <= turn) lo = mid;
                else hi = mid - 1;
            }
            const int r = lo;
            if (!served(r)) continue;
            const bool copies = s_off[r] & 1;
            const int k = turn - (s_off[r] >> 1), n = a.row_length[r];
            const int col = copies && k == 0 ? n / bs : entries(n, bs) + k - (copies ? 1 : 0);
            a.new_table[static_cast<int64_t>(r) * a.width + col] = id;
            a.refs[id] = 1;
            if (copies && k == 0) {
                const int tail = a.row_tail[r];
                atomicSub(a.refs + tail, 1);  // (another row or holder keeps it)
                a.copies[2 * r] = tail;
                a.copies[2 * r + 1] = id;
            }
            const int g1 = min(a.grow, (col + 1) * bs - n);
            for (int g = max(0, col * bs - n); g < g1; ++g)
                a.slots[static_cast<int64_t>(r) * a.grow + g] = static_cast<int64_t>(id) * bs + (n + g) % bs;
        }
    }
    if (blockIdx.x != 0) return;
    int taken = 0, unserved = 0, copied = 0;
    for (int r = tid; r < R; r += kScanThreads) {
        const int tail = a.row_tail[r], n = a.row_length[r];
        const bool copies = s_off[r] & 1, ok = tail >= kRowFull && served(r);
        a.new_length[r] = n + (ok ? a.grow : 0);
        if (!ok || !copies) a.copies[2 * r] = a.copies[2 * r + 1] = -1;
        if (!ok) {
            for (int g = 0; g < a.grow; ++g) a.slots[static_cast<int64_t>(r) * a.grow + g] = -1;
        } else {
            taken += (s_off[r + 1] >> 1) - (s_off[r] >> 1);
            if (tail >= 0 && !copies) {  // the first tokens go to the page that it keeps
                const int g1 = min(a.grow, bs - n % bs);
                for (int g = 0; g < g1; ++g) a.slots[static_cast<int64_t>(r) * a.grow + g] = static_cast<int64_t>(tail) * bs + (n + g) % bs;
            }
        }
        unserved += !ok && tail != kRowEmpty;
        copied += ok && copies;
    }
    taken = block_sum<kScanThreads>(taken, s_sum);
    unserved = block_sum<kScanThreads>(unserved, s_sum);
    copied = block_sum<kScanThreads>(copied, s_sum);
    if (tid == 0) {
        a.stats[0] = free_blocks - taken;
        a.stats[1] = taken;
        a.stats[2] = unserved;
        a.stats[3] = copied;
    }
}

// Compaction, first step: the live blocks of each chunk.
__global__ void __launch_bounds__(kScanThreads) compact_count_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    int n = 0;
    const int c0 = blockIdx.x * kPagesChunk;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int id = c0 + i * kScanThreads + static_cast<int>(threadIdx.x);
        n += id < a.num_blocks && a.refs[id] > 0;
    }
    n = block_sum<kScanThreads>(n, s_sum);
    if (threadIdx.x == 0) a.chunk_count[blockIdx.x] = n;
}

// Second step: with `live` live blocks, the i-th free id below it (block_a[i]) and, of
// each live id from there on, how many are above it (block_b[id]: its turn).
__global__ void __launch_bounds__(kScanThreads) compact_rank_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x;
    int before = 0, live = 0;
    for (int c = tid; c < a.chunks; c += kScanThreads) {
        const int n = a.chunk_count[c];
        live += n;
        if (c < static_cast<int>(blockIdx.x)) before += n;
    }
    before = block_sum<kScanThreads>(before, s_sum);
    live = block_sum<kScanThreads>(live, s_sum);
    const int id0 = blockIdx.x * kPagesChunk + tid * kPer;
    uint32_t is_live = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (id0 + i < a.num_blocks && a.refs[id0 + i] > 0) is_live |= 1u << i;
    int unused;
    before += block_before<kScanThreads>(__popc(is_live), s_sum, &unused);
    for (int i = 0; i < kPer && id0 + i < a.num_blocks; ++i) {
        const int id = id0 + i;
        const bool is = is_live >> i & 1u;
        if (id == live) a.row_length[1] = live - before;  // as many are free below it as are live from it on
        if (id < live) {
            a.remap[id] = is ? id : -1;
            if (!is) a.block_a[id - before] = id;
        } else {  // (INT_MAX: no page; an entry that names it has no count)
            a.block_b[id] = is ? live - 1 - before : INT_MAX;
        }
        before += is;
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.row_length[0] = live;
        if (live >= a.num_blocks) a.row_length[1] = 0;
    }
}

// Third step. CTAs 0 .. chunks - 1: the moving blocks' pairs, counts and new places, and
// the unused end of the list; the others: rows of the table.
__global__ void __launch_bounds__(kScanThreads) compact_move_kernel(const PagesArgs a) {
    pdl_trigger();
    pdl_wait();
    const int tid = threadIdx.x, live = a.row_length[0], moves = min(a.row_length[1], a.max_copies);
    if (static_cast<int>(blockIdx.x) < a.chunks) {
        for (int i = 0; i < kPer; ++i) {
            const int id = blockIdx.x * kPagesChunk + i * kScanThreads + tid;
            if (id >= a.num_blocks) break;
            if (id < live) continue;
            const int64_t turn = a.block_b[id];
            if (turn < moves) {
                const int to = a.block_a[turn];
                a.remap[id] = to;
                a.refs[to] = a.refs[id];
                a.refs[id] = 0;
                a.copies[2 * turn] = id;
                a.copies[2 * turn + 1] = to;
            } else {
                a.remap[id] = turn == INT_MAX ? -1 : id;
            }
        }
        for (int64_t i = moves + static_cast<int64_t>(blockIdx.x) * kScanThreads + tid; i < a.max_copies;
             i += static_cast<int64_t>(a.chunks) * kScanThreads)
            a.copies[2 * i] = a.copies[2 * i + 1] = -1;
        if (blockIdx.x == 0 && tid == 0) {
            a.stats[0] = live;
            a.stats[1] = moves;
        }
        return;
    }
    const int r = static_cast<int>(blockIdx.x) - a.chunks;
    const int n = a.length[r];
    if (!length_ok(a, n)) {
        if (tid == 0) atomicOr(a.err, 1);
        return;
    }
    int32_t *row = a.table + static_cast<int64_t>(r) * a.width;
    for (int c = tid; c < entries(n, a.block_size); c += kScanThreads) {
        const int e = row[c];
        if (e < live) continue;
        const int turn = e < a.num_blocks ? a.block_b[e] : INT_MAX;
        if (turn == INT_MAX) atomicOr(a.err, 1);
        else if (turn < moves) row[c] = a.block_a[turn];
    }
}

// Copies of blocks in every pool. A unit is one pool's part of a pair, up to 16 KB; the
// units of all pairs go round the CTAs, a warp's lanes looking at 32 of a CTA's at
// once, as most pairs of a fork's list are none.
constexpr int kCopyThreads = 256, kCopyLoads = 4;
constexpr int64_t kCopyPart = 16 * kCopyThreads * kCopyLoads;
__global__ void __launch_bounds__(kCopyThreads) copy_blocks_kernel(const __grid_constant__ CopyArgs a) {
    pdl_trigger();
    pdl_wait();
    const int parts = static_cast<int>((a.block_bytes + kCopyPart - 1) / kCopyPart);
    const int units = a.pools * parts;
    const int64_t total = static_cast<int64_t>(a.num_copies) * units;
    const int lane = threadIdx.x & 31;
    for (int64_t u0 = blockIdx.x; u0 < total; u0 += 32ll * gridDim.x) {
        const int64_t mine = u0 + static_cast<int64_t>(lane) * gridDim.x;
        int2 pair = make_int2(-1, -1);
        int unit = 0;
        if (mine < total) {
            const int64_t i = mine / units;
            unit = static_cast<int>(mine - i * units);
            pair = make_int2(a.copies[2 * i], a.copies[2 * i + 1]);
            if (pair.x >= a.num_blocks || pair.y >= a.num_blocks) {
                if (pair.x >= 0 && pair.y >= 0 && threadIdx.x < 32) atomicOr(a.err, 1);
                pair.x = -1;
            }
        }
        uint32_t have = __ballot_sync(0xffffffffu, pair.x >= 0 && pair.y >= 0);
        while (have) {
            const int l = __ffs(have) - 1;
            have &= have - 1;
            const int src = __shfl_sync(0xffffffffu, pair.x, l), dst = __shfl_sync(0xffffffffu, pair.y, l);
            const int w = __shfl_sync(0xffffffffu, unit, l);
            const int pool = w / parts;
            const int64_t at = static_cast<int64_t>(w - pool * parts) * kCopyPart;
            const int n = static_cast<int>(min(kCopyPart, a.block_bytes - at) / 16);
            uint8_t *base = static_cast<uint8_t *>(a.pool[pool]) + at;
            const uint4 *from = reinterpret_cast<const uint4 *>(base + src * a.block_bytes);
            uint4 *to = reinterpret_cast<uint4 *>(base + dst * a.block_bytes);
            uint4 v[kCopyLoads];
#pragma unroll
            for (int i = 0; i < kCopyLoads; ++i)
                if (i * kCopyThreads + static_cast<int>(threadIdx.x) < n) v[i] = __ldcs(from + i * kCopyThreads + threadIdx.x);
#pragma unroll
            for (int i = 0; i < kCopyLoads; ++i)
                if (i * kCopyThreads + static_cast<int>(threadIdx.x) < n) to[i * kCopyThreads + threadIdx.x] = v[i];
        }
    }
}

}  // namespace

int launch_pages_free(const PagesArgs &a, int32_t *length, const uint8_t *ends, int32_t window, int32_t sinks, void *stream) {
    FNPU_CUDA_TRY(launch_ex(pages_free_kernel, static_cast<unsigned>(a.rows), kRowThreads, 0, static_cast<cudaStream_t>(stream), true,
                            nullptr, a, length, ends, static_cast<int>(window), static_cast<int>(sinks)));
    return FNPU_OK;
}

int launch_pages_fork(const PagesArgs &a, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.new_rows + a.rows > 0)
        FNPU_CUDA_TRY(launch_ex(fork_rows_kernel, static_cast<unsigned>(a.new_rows + a.rows), kRowThreads, 0, st, true, nullptr, a));
    const int row_ctas = (a.new_rows + kScanThreads - 1) / kScanThreads;
    FNPU_CUDA_TRY(launch_ex(fork_count_kernel, static_cast<unsigned>(a.chunks + row_ctas), kScanThreads, 0, st, true, nullptr, a));
    FNPU_CUDA_TRY(launch_ex(fork_take_kernel, static_cast<unsigned>(a.chunks), kScanThreads, sizeof(int) * (a.new_rows + 1), st, true,
                            nullptr, a));
    return FNPU_OK;
}

int launch_pages_compact(const PagesArgs &a, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    FNPU_CUDA_TRY(launch_ex(compact_count_kernel, static_cast<unsigned>(a.chunks), kScanThreads, 0, st, true, nullptr, a));
    FNPU_CUDA_TRY(launch_ex(compact_rank_kernel, static_cast<unsigned>(a.chunks), kScanThreads, 0, st, true, nullptr, a));
    FNPU_CUDA_TRY(launch_ex(compact_move_kernel, static_cast<unsigned>(a.chunks + a.rows), kScanThreads, 0, st, true, nullptr, a));
    return FNPU_OK;
}

int launch_copy_blocks(const CopyArgs &a, void *stream) {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return FNPU_ECUDA;
    const int64_t units = static_cast<int64_t>(a.num_copies) * a.pools * ((a.block_bytes + kCopyPart - 1) / kCopyPart);
    const int64_t grid = units < 8ll * sms ? units : 8ll * sms;
    FNPU_CUDA_TRY(launch_ex(copy_blocks_kernel, static_cast<unsigned>(grid), kCopyThreads, 0, static_cast<cudaStream_t>(stream), true,
                            nullptr, a));
    return FNPU_OK;
}

}  // namespace fnpu
