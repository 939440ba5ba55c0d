// The pages of a cache on the device: rows of a block table that share, fork, give
// up and move blocks, with a count of holders for each block, and the copies
// that go with it.
//
// The tables are small (some MB at most), so what bounds these calls is the chain
// of dependent steps: counts before free blocks, free blocks before their rows. Each
// step is a kernel over all SMs and a dependent launch of the one before; where a step is a
// matter of some rows and one chunk of counts, all steps are one kernel of one CTA, a
// warp a row, with what passes between them in shared memory (a turn of 8 rows
// with its copies: 14.2 us in three kernels, 12.1 so, 10.8 since copies take many CTAs). Every
// result is independent of the order of the atomics: counts are sums, the lowest row
// of a page a minimum, and the k-th block that is taken is the k-th free one by id, by a
// prefix sum over chunks of counts that each CTA forms for itself.
#include <limits.h>

#include "common.cuh"

namespace fnpu {
namespace {

constexpr int kRowThreads = 256;    // kernels over rows
constexpr int kScanThreads = 512;   // kernels over chunks of counts, and those of one CTA
constexpr int kPer = kPagesChunk / kScanThreads;
constexpr int64_t kSmallEntries = 16384;  // of the tables that one CTA goes through
constexpr int kSmallRows = 64;            // and their rows (four a warp)

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

// The sum over a row's threads: a warp or the CTA.
template <int kGroup>
__device__ __forceinline__ int group_sum(int v, int *s) {
    if constexpr (kGroup == 32) return __reduce_add_sync(0xffffffffu, v);
    else return block_sum<kGroup>(v, s);
}
// The counts of a thread's kPer neighbours from `id0` on that are above zero, as bits.
__device__ __forceinline__ uint32_t live_bits(const PagesArgs &a, int id0) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        if (id0 + i < a.num_blocks && a.refs[id0 + i] > 0) bits |= 1u << i;
    return bits;
}
// How many of a chunk's counts are above zero. kFix: those below it, of more holders
// given up than were counted, are flagged and become 0.
template <bool kFix>
__device__ __forceinline__ int live_in_chunk(const PagesArgs &a, int chunk, int *s) {
    int n = 0;
    for (int i = 0; i < a.chunk; i += kScanThreads) {
        const int id = chunk * a.chunk + i + static_cast<int>(threadIdx.x);
        const int count = id < a.num_blocks ? a.refs[id] : 0;
        n += count > 0;
        if (kFix && count < 0) {
            a.refs[id] = 0;
            atomicOr(a.err, 1);
        }
    }
    return block_sum<kScanThreads>(n, s);
}
// Of all chunks' live counts: the sum, and that of the chunks before `chunk`.
__device__ __forceinline__ int live_before(const PagesArgs &a, int chunk, int *s, int *all) {
    int before = 0, sum = 0;
    for (int c = threadIdx.x; c < a.chunks; c += kScanThreads) {
        const int n = a.chunk_count[c];
        sum += n;
        if (c < chunk) before += n;
    }
    *all = block_sum<kScanThreads>(sum, s);
    return block_sum<kScanThreads>(before, s);
}

// Fork, first step. Units 0 .. new_rows - 1: a new row's entries. The others: an old
// row's pages get as many holders more as rows continue it, less the one that it was
// (nothing to do where one row does, the usual case late in a search). Sums alone: whether a count
// is below zero shows when all are in, whatever their order.
template <int kGroup>
__device__ __forceinline__ void fork_row(const PagesArgs &a, int unit, int *s_sum) {
    constexpr int kLoads = 4;  // entries in flight
    const int tid = threadIdx.x % kGroup, bs = a.block_size;
    if (unit < a.new_rows) {
        const int r = unit;
        const int p = a.parents ? a.parents[r] : r;
        bool ok = p >= 0 && p < a.rows;
        if (p >= a.rows && tid == 0) atomicOr(a.err, 1);
        const int n = ok ? a.length[p] : 0;
        ok = ok && length_ok(a, n);
        const int held = ok ? entries(n, bs) : 0;
        const int32_t *from = a.table + static_cast<int64_t>(ok ? p : 0) * a.width;
        int32_t *to = a.new_table + static_cast<int64_t>(r) * a.width;
        int tail = kRowFull;
        if (!ok) tail = kRowEmpty;
        else if (a.grow > 0 && static_cast<int64_t>(n) + a.grow > static_cast<int64_t>(a.width) * bs) tail = kRowStuck;
        else if (a.grow > 0 && n % bs != 0) {
            const int e = from[n / bs];
            tail = e >= 0 && e < a.num_blocks ? e : kRowStuck;
        }
        for (int c0 = tid; c0 < a.width; c0 += kLoads * kGroup) {
            int e[kLoads];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) e[i] = c0 + i * kGroup < held ? from[c0 + i * kGroup] : -1;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                if (c0 + i * kGroup >= a.width) break;
                if (e[i] >= a.num_blocks) atomicOr(a.err, 1);
                to[c0 + i * kGroup] = e[i] < 0 || e[i] >= a.num_blocks ? -1 : e[i];
            }
        }
        if (tid == 0) {
            a.row_length[r] = ok ? n : 0;
            a.row_tail[r] = tail;
            if (tail >= 0) {  // (the same for every row with this page)
                a.block_a[tail] = 0;
                a.block_b[tail] = INT_MAX;
            }
        }
        return;
    }
    const int p = unit - a.new_rows;
    const int n = a.length[p];
    if (!length_ok(a, n)) {
        if (tid == 0) atomicOr(a.err, 1);
        return;
    }
    int next = a.new_rows > 0 ? 1 : 0;  // (no new rows: nobody continues any)
    if (a.parents) {
        int mine = 0;
        for (int r = tid; r < a.new_rows; r += kGroup) mine += a.parents[r] == p;
        next = group_sum<kGroup>(mine, s_sum);
    }
    const int32_t *row = a.table + static_cast<int64_t>(p) * a.width;
    const int held = entries(n, bs);
    for (int c0 = tid; c0 < held; c0 += kLoads * kGroup) {
        int e[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) e[i] = c0 + i * kGroup < held ? row[c0 + i * kGroup] : -1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            if (e[i] >= a.num_blocks) atomicOr(a.err, 1);
            if (e[i] < 0 || e[i] >= a.num_blocks || next == 1) continue;
            atomicAdd(a.refs + e[i], next - 1);
        }
    }
}

// Second step: the rows of each last page (and the live blocks of each chunk).
__device__ __forceinline__ void fork_tail(const PagesArgs &a, int r) {
    const int tail = a.row_tail[r];
    if (tail < 0) return;
    atomicAdd(a.block_a + tail, 1);
    atomicMin(a.block_b + tail, r);
    a.row_refs[r] = max(0, a.refs[tail]);  // (one below zero may become 0 meanwhile)
}

// Third step, a chunk each CTA. All form the rows' needs and their prefix sums; a CTA
// hands its own free blocks to the rows whose turn they are, and that of chunk 0 does what
// is left of every row.
struct ForkShared {
    int sum[kScanThreads / 32];
    int free[kPagesChunk];
};
__device__ __forceinline__ void fork_take(const PagesArgs &a, int chunk, ForkShared *s, int *s_off) {
    const int tid = threadIdx.x, bs = a.block_size, R = a.new_rows;
    const int first = chunk * a.chunk;
    uint32_t live = live_bits(a, first + tid * kPer);
    // s_off[r]: blocks that row r needs, then that the rows before it do, * 2 + (it copies)
    for (int r = tid; r < R; r += kScanThreads) {
        const int tail = a.row_tail[r], n = a.row_length[r];
        const bool copy = tail >= 0 && (a.block_b[tail] != r || a.row_refs[r] > a.block_a[tail]);
        s_off[r] = tail < kRowFull ? 0 : 2 * ((copy ? 1 : 0) + entries(n + a.grow, bs) - entries(n, bs)) + (copy ? 1 : 0);
    }
    int live_blocks;
    const int live_chunks = live_before(a, chunk, s->sum, &live_blocks);  // (and s_off is written)
    const int free_blocks = a.num_blocks - live_blocks;
    int before = first - live_chunks;  // free ones of the chunks before
    const int per = (R + kScanThreads - 1) / kScanThreads;
    int mine = 0;
    for (int r = tid * per; r < min(R, (tid + 1) * per); ++r) mine += s_off[r] >> 1;
    int needed;
    int off = block_before<kScanThreads>(mine, s->sum, &needed);
    for (int r = tid * per; r < min(R, (tid + 1) * per); ++r) {
        const int v = s_off[r];
        s_off[r] = 2 * off + (v & 1);
        off += v >> 1;
    }
    if (tid == 0) s_off[R] = 2 * needed;
    __syncthreads();
    auto served = [&](int r) {
        const int o = s_off[r] >> 1, e = s_off[r + 1] >> 1;
        return e == o || e <= free_blocks;
    };
    for (int c = 0; c < a.chunk && before < needed; c += kPagesChunk) {
        // free blocks in order, kPer neighbours a thread
        const int id0 = first + c + tid * kPer;
        if (c > 0) live = live_bits(a, id0);
        uint32_t is_free = ~live & ((1u << kPer) - 1);
        if (id0 + kPer > a.num_blocks) is_free &= id0 < a.num_blocks ? (1u << (a.num_blocks - id0)) - 1 : 0u;
        int here;
        int f = block_before<kScanThreads>(__popc(is_free), s->sum, &here);  // (and the last round's ids are read)
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (is_free >> i & 1u) s->free[f++] = id0 + i;
        __syncthreads();
        for (int j = tid; j < min(here, needed - before); j += kScanThreads) {
            const int id = s->free[j], turn = before + j;
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
                if (a.row_refs[r] >= a.block_a[tail]) atomicSub(a.refs + tail, 1);  // (another row or holder keeps it: 1 at least is left)
                a.copies[2 * r] = tail;
                a.copies[2 * r + 1] = id;
            }
            const int g1 = min(a.grow, (col + 1) * bs - n);
            for (int g = max(0, col * bs - n); g < g1; ++g)
                a.slots[static_cast<int64_t>(r) * a.grow + g] = static_cast<int64_t>(id) * bs + (n + g) % bs;
        }
        before += here;
    }
    if (chunk != 0) return;
    int taken = 0, unserved = 0, copied = 0;
    for (int r = tid; r < R; r += kScanThreads) {
        const int tail = a.row_tail[r], n = a.row_length[r];
        const bool copies = s_off[r] & 1, ok = tail >= kRowFull && served(r);
        // (fewer holders counted than rows that have it last: its count would end at 0 or below, or pass
        // there while other CTAs look for free blocks; it stays)
        if (tail >= 0 && a.row_refs[r] < a.block_a[tail]) atomicOr(a.err, 1);
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
    taken = block_sum<kScanThreads>(taken, s->sum);
    unserved = block_sum<kScanThreads>(unserved, s->sum);
    copied = block_sum<kScanThreads>(copied, s->sum);
    if (tid == 0) {
        a.stats[0] = free_blocks - taken;
        a.stats[1] = taken;
        a.stats[2] = unserved;
        a.stats[3] = copied;
    }
}

__global__ void __launch_bounds__(kRowThreads) fork_rows_kernel(const PagesArgs a) {
    __shared__ int s_sum[kRowThreads / 32];
    pdl_trigger();
    pdl_wait();
    fork_row<kRowThreads>(a, blockIdx.x, s_sum);
}
__global__ void __launch_bounds__(kScanThreads) fork_count_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    if (static_cast<int>(blockIdx.x) < a.chunks) {
        const int n = live_in_chunk<true>(a, blockIdx.x, s_sum);
        if (threadIdx.x == 0) a.chunk_count[blockIdx.x] = n;
        return;
    }
    const int r = (static_cast<int>(blockIdx.x) - a.chunks) * kScanThreads + static_cast<int>(threadIdx.x);
    if (r < a.new_rows) fork_tail(a, r);
}
__global__ void __launch_bounds__(kScanThreads) fork_take_kernel(const PagesArgs a) {
    extern __shared__ int s_off[];  // [new_rows + 1]
    __shared__ ForkShared s;
    pdl_trigger();
    pdl_wait();
    fork_take(a, blockIdx.x, &s, s_off);
}
// What the workspace holds otherwise, where one CTA does all steps.
struct SmallShared {
    int rows[3][kSmallRows + 2];
    int blocks[2][kPagesChunk];
    int count;
};
__device__ __forceinline__ PagesArgs with_shared(PagesArgs a, SmallShared *s) {
    a.chunk_count = &s->count;
    a.row_length = s->rows[0];
    a.row_tail = s->rows[1];
    a.row_refs = s->rows[2];
    a.block_a = s->blocks[0];
    a.block_b = s->blocks[1];
    return a;
}
// All three steps, of one chunk.
__global__ void __launch_bounds__(kScanThreads) fork_small_kernel(const PagesArgs args) {
    extern __shared__ int s_off[];
    __shared__ ForkShared s;
    __shared__ SmallShared small;
    const PagesArgs a = with_shared(args, &small);
    pdl_trigger();
    pdl_wait();
    for (int u = threadIdx.x / 32; u < a.new_rows + a.rows; u += kScanThreads / 32) fork_row<32>(a, u, nullptr);
    __syncthreads();
    for (int r = threadIdx.x; r < a.new_rows; r += kScanThreads) fork_tail(a, r);
    const int n = live_in_chunk<true>(a, 0, s.sum);
    if (threadIdx.x == 0) a.chunk_count[0] = n;
    __syncthreads();
    fork_take(a, 0, &s, s_off);
}

// Compaction, second step (after the live blocks of each chunk): with `live` live
// blocks, the i-th free id below it (block_a[i]) and, of each live id from there on, how
// many are above it (block_b[id]: its turn).
__device__ __forceinline__ void compact_rank(const PagesArgs &a, int chunk, int *s_sum) {
    const int tid = threadIdx.x;
    int live;
    int base = live_before(a, chunk, s_sum, &live);
    for (int c = 0; c < a.chunk; c += kPagesChunk) {
        const int id0 = chunk * a.chunk + c + tid * kPer;
        const uint32_t is_live = live_bits(a, id0);
        int here;
        int before = base + block_before<kScanThreads>(__popc(is_live), s_sum, &here);
        base += here;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = id0 + i;
            if (id >= a.num_blocks) break;
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
    }
    if (chunk == 0 && tid == 0) {
        a.row_length[0] = live;
        if (live >= a.num_blocks) a.row_length[1] = 0;
    }
}

// Third step: the moving blocks' pairs, counts and new places, and the unused end of
// the list;
__device__ __forceinline__ void compact_move(const PagesArgs &a, int chunk, int live, int moves) {
    const int tid = threadIdx.x;
    for (int c = 0; c < a.chunk; c += kPagesChunk) {
        int id[kPer];
        int turn[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            id[i] = chunk * a.chunk + c + i * kScanThreads + tid;
            turn[i] = id[i] >= live && id[i] < a.num_blocks ? a.block_b[id[i]] : -1;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (turn[i] < 0) continue;
            if (turn[i] < moves) {
                const int to = a.block_a[turn[i]];
                a.remap[id[i]] = to;
                a.refs[to] = a.refs[id[i]];
                a.refs[id[i]] = 0;
                a.copies[2ll * turn[i]] = id[i];
                a.copies[2ll * turn[i] + 1] = to;
            } else {
                a.remap[id[i]] = turn[i] == INT_MAX ? -1 : id[i];
            }
        }
    }
    for (int64_t i = moves + static_cast<int64_t>(chunk) * kScanThreads + tid; i < a.max_copies;
         i += static_cast<int64_t>(a.chunks) * kScanThreads)
        a.copies[2 * i] = a.copies[2 * i + 1] = -1;
    if (chunk == 0 && tid == 0) {
        a.stats[0] = live;
        a.stats[1] = moves;
    }
}
// and a row of the table.
template <int kGroup>
__device__ __forceinline__ void compact_row(const PagesArgs &a, int r, int live, int moves) {
    const int tid = threadIdx.x % kGroup;
    const int n = a.length[r];
    if (!length_ok(a, n)) {
        if (tid == 0) atomicOr(a.err, 1);
        return;
    }
    int32_t *row = a.table + static_cast<int64_t>(r) * a.width;
    for (int c = tid; c < entries(n, a.block_size); c += kGroup) {
        const int e = row[c];
        if (e < live) continue;
        const int turn = e < a.num_blocks ? a.block_b[e] : INT_MAX;
        if (turn == INT_MAX) atomicOr(a.err, 1);
        else if (turn < moves) row[c] = a.block_a[turn];
    }
}

__global__ void __launch_bounds__(kScanThreads) compact_count_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int n = live_in_chunk<false>(a, blockIdx.x, s_sum);
    if (threadIdx.x == 0) a.chunk_count[blockIdx.x] = n;
}
__global__ void __launch_bounds__(kScanThreads) compact_rank_kernel(const PagesArgs a) {
    __shared__ int s_sum[kScanThreads / 32];
    pdl_trigger();
    pdl_wait();
    compact_rank(a, blockIdx.x, s_sum);
}
__global__ void __launch_bounds__(kScanThreads) compact_move_kernel(const PagesArgs a) {
    pdl_trigger();
    pdl_wait();
    const int live = a.row_length[0], moves = min(a.row_length[1], a.max_copies);
    if (static_cast<int>(blockIdx.x) < a.chunks) compact_move(a, blockIdx.x, live, moves);
    else compact_row<kScanThreads>(a, static_cast<int>(blockIdx.x) - a.chunks, live, moves);
}
// All three steps, of one chunk.
__global__ void __launch_bounds__(kScanThreads) compact_small_kernel(const PagesArgs args) {
    __shared__ int s_sum[kScanThreads / 32];
    __shared__ SmallShared small;
    const PagesArgs a = with_shared(args, &small);
    pdl_trigger();
    pdl_wait();
    const int n = live_in_chunk<false>(a, 0, s_sum);
    if (threadIdx.x == 0) a.chunk_count[0] = n;
    __syncthreads();
    compact_rank(a, 0, s_sum);
    __syncthreads();
    const int live = a.row_length[0], moves = min(a.row_length[1], a.max_copies);
    compact_move(a, 0, live, moves);
    for (int r = threadIdx.x / 32; r < a.rows; r += kScanThreads / 32) compact_row<32>(a, r, live, moves);
}

// Copies of blocks in every pool. A unit is one pool's part of a pair, up to 16 KB; the
// units of all pairs go round the CTAs, a warp's lanes looking at 32 of a CTA's at
// once, as most pairs of a fork's list are none. Many CTAs, each of a unit or two: which
// of them take long is left to the hardware (1.33 GB read and written: with 8 CTAs of 256 threads
// an SM 213 us, with up to 256 of 128 threads, 8 loads in flight each, 191: 7.0 TB/s).
constexpr int kCopyThreads = 128, kCopyLoads = 8;
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
    const size_t smem = sizeof(int) * (a.new_rows + 1);
    const int64_t rows = static_cast<int64_t>(a.new_rows) + a.rows;
    if (a.chunks == 1 && a.chunk == kPagesChunk && rows <= kSmallRows && rows * a.width <= kSmallEntries) {
        FNPU_CUDA_TRY(launch_ex(fork_small_kernel, 1u, kScanThreads, smem, st, true, nullptr, a));
        return FNPU_OK;
    }
    if (rows > 0) FNPU_CUDA_TRY(launch_ex(fork_rows_kernel, static_cast<unsigned>(rows), kRowThreads, 0, st, true, nullptr, a));
    const int row_ctas = (a.new_rows + kScanThreads - 1) / kScanThreads;
    FNPU_CUDA_TRY(launch_ex(fork_count_kernel, static_cast<unsigned>(a.chunks + row_ctas), kScanThreads, 0, st, true, nullptr, a));
    FNPU_CUDA_TRY(launch_ex(fork_take_kernel, static_cast<unsigned>(a.chunks), kScanThreads, smem, st, true, nullptr, a));
    return FNPU_OK;
}

int launch_pages_compact(const PagesArgs &a, void *stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.chunks == 1 && a.chunk == kPagesChunk && a.rows <= kSmallRows &&
        static_cast<int64_t>(a.rows) * a.width <= kSmallEntries) {
        FNPU_CUDA_TRY(launch_ex(compact_small_kernel, 1u, kScanThreads, 0, st, true, nullptr, a));
        return FNPU_OK;
    }
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
    const int64_t grid = units < 256ll * sms ? units : 256ll * sms;
    FNPU_CUDA_TRY(launch_ex(copy_blocks_kernel, static_cast<unsigned>(grid), kCopyThreads, 0, static_cast<cudaStream_t>(stream), true,
                            nullptr, a));
    return FNPU_OK;
}

}  // namespace fnpu
