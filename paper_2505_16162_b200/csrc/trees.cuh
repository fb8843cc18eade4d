// Drafts that branch: positions and masks of a tree's rows, which of its rows are kept, and their K and V moved together.
//
// A request's new rows are a tree of tokens: row 0 is the pending token, row i > 0 follows row parent[i] < i.  Siblings are tested in row order.
#pragma once

#include "device_common.cuh"

namespace knnssd {
namespace trees {

constexpr int WORD = 64;                  // bits of a row's mask: rows of tree behind a request's first chain

// A request's rows [row0, row0 + n), whatever row_start holds.
__device__ __forceinline__ void rows_of(const int *row_start, int R, int b, int &row0, int &n) {
    row0 = min(max(row_start[b], 0), R);
    n = max(min(max(row_start[b + 1], 0), R) - row0, 0);
}
// Rows before the first request's and behind the last one's, use(row) by the threads of the grid.
template <typename F> __device__ __forceinline__ void each_other_row(const int *row_start, int B, int R, F use) {
    const int first = min(max(row_start[0], 0), R), used = max(first, min(row_start[B], R)), others = first + R - used;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < others; i += (long long)gridDim.x * blockDim.x) use(i < first ? (int)i : (int)i + used - first);
}

// ---- positions and masks -------------------------------------------------------------------------------------------------
// Row i of a request stands at position len + depth(i) and its K and V lie at len + i.  Bit d of its word: it sees what lies d before that, its own at d = 0; all that lies
// 64 and more before it is seen.  Relative to the row's own place the words do not change when a tree is drafted level by level, a call each.
// A request begins with a chain of C rows (parent i - 1); those see all before them.  A later row goes up to it, in shared memory, and sees the whole chain up to
// where it arrives.  What lies 64 before must be its ancestor, so behind the chain there are at most 64 rows.
// Bound by latency: row_start, then the parents, then a walk as long as the tree is deep.
struct TableArgs {
    const int *lens, *row_start, *parent;
    int B, R;
    int *pos;
    unsigned long long *seen;
    int *state;
};
constexpr int TABLE_NT = 128;
__global__ void __launch_bounds__(TABLE_NT) tree_tables_kernel(const TableArgs a) {
    __shared__ int par[WORD], warp_first[TABLE_NT / 32];
    chain_wait();
    const int tid = threadIdx.x, b = blockIdx.x;
    each_other_row(a.row_start, a.B, a.R, [&](int r) { a.pos[r] = -1; a.seen[r] = 0ull; });
    int row0, n;
    rows_of(a.row_start, a.R, b, row0, n);
    const int len = a.lens[b];
    const int *parent = a.parent + row0;
    int first = n;                                                   // the first row that does not follow the one before it
    for (int i = tid; i < n; i += TABLE_NT)
        if (parent[i] != i - 1) { first = i; break; }
    first = __reduce_min_sync(0xffffffffu, first);
    if ((tid & 31) == 0) warp_first[tid >> 5] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < TABLE_NT / 32; ++w) first = min(first, warp_first[w]);
    const int C = first, tail = min(n - C, WORD);
    if (tid < tail) par[tid] = parent[C + tid];
    __syncthreads();
    bool bad = n - C > WORD || len < 0 || len > 0x7fffffff - n;
    int my_pos = -1;
    unsigned long long my_word = 0ull;
    if (tid < tail) {                                                // rows C .. n - 1, a thread each
        const int i = C + tid;
        int at = i, walked = 0;
        while (at >= C) {                                            // ends: every step goes to a smaller row
            my_word |= 1ull << (i - at);
            ++walked;
            const int up = par[at - C];
            if (up < -1 || up >= at) { bad = true; at = -1; break; }
            at = up;
        }
        bad |= at < i - WORD;
        if (i - at < WORD) my_word |= ~0ull << (i - at);             // the chain from row at up, and what was there before the call
        // a row that follows none of the request's sees what was there before the call, at i + 1 and more before it: i - at as well
        my_pos = len + walked + at;
    }
    bad = __syncthreads_or(bad);
    for (int i = tid; i < C; i += TABLE_NT) {
        a.pos[row0 + i] = bad ? -1 : len + i;
        a.seen[row0 + i] = bad ? 0ull : ~0ull;
    }
    for (int i = C + tid; i < n; i += TABLE_NT) {
        a.pos[row0 + i] = bad ? -1 : my_pos;
        a.seen[row0 + i] = bad ? 0ull : my_word;
    }
    if (tid == 0) a.state[b] = bad ? 1 : 0;
}

// ---- greedy: from row 0 on to the first child that is the full model's choice ----------------------------------------------
struct AgreeArgs {
    const int *best, *token, *parent, *row_start;
    int B, R;
    int *path, *accepted, *next;
};
constexpr int AGREE_NT = 128;
// A warp per request: 32 rows at a time, which of them are their parent's choice, then from each row kept to the first of its children that is.  (Of siblings with one token that is the first,
// whichever of them leads further.)  Bound by latency: three dependent loads, a vote a row kept: 24 requests of 25 rows 1.9 us, 1024 of 40 2.5, one of 1024 15.
__global__ void __launch_bounds__(AGREE_NT) tree_agree_kernel(const AgreeArgs a) {
    chain_wait();
    each_other_row(a.row_start, a.B, a.R, [&](int r) { a.path[r] = -1; });
    const int b = blockIdx.x * (AGREE_NT / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (b >= a.B) return;
    int row0, n;
    rows_of(a.row_start, a.R, b, row0, n);
    int node = 0, kept = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        int up = -1;
        bool agrees = false;
        if (i > 0 && i < n) {
            up = a.parent[row0 + i];
            agrees = up >= 0 && up < i && a.token[row0 + i] == a.best[row0 + up];
        }
        if (i < n) a.path[row0 + i] = i == 0 ? 0 : -1;
        for (;;) {
            const unsigned found = __ballot_sync(0xffffffffu, agrees && up == node);
            if (!found) break;
            node = i0 + __ffs(found) - 1;                            // its children come behind it
            ++kept;
            __syncwarp();
            if (lane == 0) a.path[row0 + kept] = node;               // kept <= node: within the rows written so far
        }
        __syncwarp();
    }
    if (lane == 0) {
        a.accepted[b] = kept;
        a.next[b] = n > 0 ? a.best[row0 + node] : -1;
    }
}

// ---- the kept path's K and V -----------------------------------------------------------------------------------------------
// K and V of row path[j] go from position len + path[j] to len + j, in every pool.  path is ascending, so path[j] >= j: in ascending order no row is overwritten
// before it is read.  A thread has 16 bytes of a head in some pools and moves them through all of the path's rows, MOVES loads ahead of their stores; threads share
// nothing.  Every moved value is read and written once: bound by memory, and by latency where few rows move.  With two / four pieces a thread in half / a quarter of the blocks, or two or
// eight loads ahead, 24 requests of 64 pools of 32 heads (30 MB) take 10 - 17 us for 9.
constexpr int KEEP_NT = 256, KEEP_POOLS = 256, KEEP_MOST = 64, MOVES = 4;
struct KeepArgs {
    const int *table, *lens, *row_start, *path;
    int B, R, max_pages, n_pages, page_shift, KV, pieces;            // pieces of 16 bytes of a head
    int n_pools;
    uint4 *pools[KEEP_POOLS];
};
__global__ void __launch_bounds__(KEEP_NT) keep_rows_kernel(const __grid_constant__ KeepArgs a) {
    __shared__ long long from[KEEP_MOST], to[KEEP_MOST];             // of head 0, in 16 bytes
    __shared__ int count;
    chain_wait();
    const int b = blockIdx.x, tid = threadIdx.x;
    int row0, n;
    rows_of(a.row_start, a.R, b, row0, n);
    const int len = a.lens[b];
    if (n <= 1 || len < 0) return;
    const long long head = (long long)a.pieces << a.page_shift;      // from one head of a page to the next
    auto place = [&](long long pos) {                                // -1: no page
        const long long idx = pos >> a.page_shift;
        if (idx >= a.max_pages) return -1ll;
        const int id = a.table[(size_t)b * a.max_pages + idx];
        if (id < 0 || id >= a.n_pages) return -1ll;
        return (long long)id * a.KV * head + (pos & ((1 << a.page_shift) - 1)) * a.pieces;
    };
    const int units = a.n_pools * a.KV * a.pieces;
    for (int j0 = 0; j0 < n; j0 += KEEP_MOST) {                      // hardly ever more than once
        __syncthreads();
        if (tid < 32) {                                              // the moves, in order
            int moves = 0;
            bool on = true;
            for (int h = 0; h < KEEP_MOST; h += 32) {
                const int j = j0 + h + tid;
                const int r = j < n ? a.path[row0 + j] : -1, before = j > 0 && j <= n ? a.path[row0 + j - 1] : -1;
                const unsigned ends = __ballot_sync(0xffffffffu, r <= before || r >= n);          // the path ends where it does not ascend
                const bool its = on && (ends == 0 || tid < __ffs(ends) - 1);
                long long src = -1, dst = -1;
                if (its && r != j) { src = place((long long)len + r); dst = place((long long)len + j); }
                const bool move = src >= 0 && dst >= 0;
                const unsigned all = __ballot_sync(0xffffffffu, move);
                if (move) {
                    const int at = moves + __popc(all & ((1u << tid) - 1));
                    from[at] = src;
                    to[at] = dst;
                }
                moves += __popc(all);
                on = on && ends == 0;
            }
            if (tid == 0) count = on ? moves : -1 - moves;
        }
        __syncthreads();
        const int c = count, moves = c < 0 ? -1 - c : c;
        if (moves > 0) {
            for (long long u = blockIdx.y * KEEP_NT + tid; u < units; u += (long long)gridDim.y * KEEP_NT) {
                const int h = (int)u / a.pieces;
                uint4 *p = a.pools[h / a.KV] + (h % a.KV) * head + (int)u % a.pieces;
                for (int m0 = 0; m0 < moves; m0 += MOVES) {
                    uint4 v[MOVES];
#pragma unroll
                    for (int m = 0; m < MOVES; ++m)
                        if (m0 + m < moves) v[m] = p[from[m0 + m]];
#pragma unroll
                    for (int m = 0; m < MOVES; ++m)
                        if (m0 + m < moves) p[to[m0 + m]] = v[m];
                }
            }
        }
        if (c < 0) return;
    }
}

}  // namespace trees
}  // namespace knnssd
