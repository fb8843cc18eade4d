// Which drafts of a tree the full model's distributions keep, and the token after them: speculative sampling with several drafts behind a row.
//
// From row `node` (first the request's row 0) its children are tested in row order.  w is what is left of p[node], Z its sum (1 as long as nothing was rejected: a
// row of p is a distribution):
//   drafts drawn from q[node], each by itself:  child c is kept iff u_c Z q[node](x_c) < w(x_c); else w <- max(0, w / Z - q[node]), Z <- sum w
//   drafts chosen, not drawn (no q):            child c is kept iff u_c Z < w(x_c);              else w(x_c) <- 0, Z <- sum w
// A kept child is the next node.  Where none is left the token after it is the smallest x with w_0 + .. + w_x > u_final sum(w), from p[node] if nothing is left of it.
// Either way the tokens are distributed as p has them.  Random numbers are inputs.
//
// A request is the work of a cluster of C blocks, each with a contiguous part of the ids.  All blocks take the same decisions from the same numbers: the tests need one value
// of p and of q a draft, fetched for all drafts at once at the start.  Only a rejection reads a row: a pass over the ids, a sum per warp, a meeting of the cluster.  The last pass's sums
// are the draw's: the block and the warp whose ids hold the crossing are known from them, the block walks that warp's ids.  Without q a node takes one pass whatever is
// rejected: the sum of all ids but its children's, to which the children not yet rejected are added (nothing is subtracted, so nothing cancels).
// Sums in 64 bits: what a test or a draw next to a border decides does not depend on the order of 150 thousand additions.
#pragma once

#include <climits>
#include <cooperative_groups.h>

#include "trees.cuh"

namespace knnssd {
namespace trees {

namespace cg = cooperative_groups;

constexpr int ACC_NT = 512, ACC_NW = ACC_NT / 32;
constexpr int ACC_ROWS = 1024;            // rows of a request that are looked at
constexpr int ACC_AHEAD = 8;              // values of a row that a thread has on their way

struct AcceptArgs {
    const float *p, *q;                   // [R][V]; q null: drafts chosen
    int V;
    const int *token, *parent, *row_start;
    int B, R;
    const float *u_accept, *u_final;
    int *path, *accepted, *next;
};

struct AcceptShared {
    double warp_sum[ACC_NW], slot[2][16], inv[ACC_ROWS];             // inv: 1 / Z of the rejections at the node
    float p_of[ACC_ROWS], q_of[ACC_ROWS], u[ACC_ROWS];               // of each row: its parent's p and q at its token, its uniform
    int parent[ACC_ROWS], token[ACC_ROWS];                           // parent -1: not to be tested
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The lowest row behind `last` whose parent is `node`; n: there is none.  The same in every warp.
__device__ __forceinline__ int next_child(const AcceptShared &sh, int n, int node, int last) {
    for (int i0 = (last + 1) & ~31; i0 < n; i0 += 32) {
        const int i = i0 + (threadIdx.x & 31);
        const unsigned found = __ballot_sync(0xffffffffu, i > last && i < n && sh.parent[i] == node);
        if (found) return i0 + __ffs(found) - 1;
    }
    return n;
}

// What a row's weights are: its values; what is left after `m` rejections of drafts drawn from q; its values without those of the children of `node`.
enum { ALL = 0, DRAWN = 1, CHOSEN = 2 };
struct Weights { const float *p, *q; int kind, m, node, n; };

// The ids among 32 from `base` on that are tokens of the node's children, as bits.  t0, t1: this lane's of the first 64 rows, -1 where it is no child's.
__device__ __forceinline__ unsigned childrens_ids(const AcceptShared &sh, const Weights &w, int t0, int t1, int base) {
    unsigned mine = 0;
    if (t0 >= base && t0 < base + 32) mine |= 1u << (t0 - base);
    if (t1 >= base && t1 < base + 32) mine |= 1u << (t1 - base);
    for (int i = 64 + (threadIdx.x & 31); i < w.n; i += 32)
        if (sh.parent[i] == w.node && sh.token[i] >= base && sh.token[i] < base + 32) mine |= 1u << (sh.token[i] - base);
    return __reduce_or_sync(0xffffffffu, mine);
}
__device__ __forceinline__ int child_token(const AcceptShared &sh, const Weights &w, int i) { return w.kind == CHOSEN && i < w.n && sh.parent[i] == w.node ? sh.token[i] : -1; }
__device__ __forceinline__ double weight_of(const AcceptShared &sh, const Weights &w, float p, float q) {
    double x = p;
    if (w.kind == DRAWN)
        for (int k = 0; k < w.m; ++k) x = fmax(fma(x, sh.inv[k], -(double)q), 0.0);
    return x;
}

// Ids of a warp's part of a range of `len`.
__device__ __forceinline__ int part_of(int len) { return ((len + ACC_NW - 1) / ACC_NW + 31) & ~31; }

// The sum of the weights of ids [lo, hi), a part per warp: sh.warp_sum.  Behind it the block has met.
__device__ __forceinline__ void sum_part(AcceptShared &sh, const Weights &w, int lo, int hi) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = part_of(hi - lo);
    const int i0 = (int)min((long long)hi, lo + (long long)warp * part), i1 = min(hi, i0 + part);
    const int t0 = child_token(sh, w, lane), t1 = child_token(sh, w, lane + 32);
    bool here = (t0 >= i0 && t0 < i1) || (t1 >= i0 && t1 < i1);
    for (int i = 64 + lane; i < w.n; i += 32) { const int t = child_token(sh, w, i); here |= t >= i0 && t < i1; }
    const bool some = __any_sync(0xffffffffu, here);                 // a child's token is among the warp's ids
    double s[2] = {0.0, 0.0};
    for (int base = i0; base < i1; base += 32 * ACC_AHEAD) {
        float p[ACC_AHEAD], q[ACC_AHEAD];
#pragma unroll
        for (int e = 0; e < ACC_AHEAD; ++e) {
            const int i = base + 32 * e + lane;
            p[e] = i < i1 ? w.p[i] : 0.f;
            q[e] = w.kind == DRAWN && i < i1 ? w.q[i] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < ACC_AHEAD; ++e) {
            const double x = weight_of(sh, w, p[e], q[e]);
            const bool out = some && (childrens_ids(sh, w, t0, t1, base + 32 * e) >> lane & 1);
            s[e & 1] += out ? 0.0 : x;
        }
    }
    const double all = warp_sum64(s[0] + s[1]);
    __syncthreads();                                                 // the sums before have been read
    if (lane == 0) sh.warp_sum[warp] = all;
    __syncthreads();
}

// The same over all ids, for all blocks of the cluster: their sums are in sh.slot[turn].
template <int C> __device__ __forceinline__ double sum_all(AcceptShared &sh, const Weights &w, int lo, int hi, int turn) {
    cg::cluster_group cluster = cg::this_cluster();
    sum_part(sh, w, lo, hi);
    if (threadIdx.x < C) {
        double mine = 0.0;
#pragma unroll
        for (int k = 0; k < ACC_NW; ++k) mine += sh.warp_sum[k];
        cluster.map_shared_rank(&sh, threadIdx.x)->slot[turn][cluster.block_rank()] = mine;
    }
    cluster.sync();
    double total = 0.0;
#pragma unroll
    for (int r = 0; r < C; ++r) total += sh.slot[turn][r];
    return total;
}

// By the block whose ids hold the crossing, behind a sum over its ids [lo, hi): the first id at which the running sum, `before` ahead of them, passes `target`.
__device__ __forceinline__ int find_id(AcceptShared &sh, const Weights &w, int lo, int hi, double before, double target) {
    for (;;) {
        int k = 0;
        double e = before;
        while (k < ACC_NW && !(e + sh.warp_sum[k] > target)) e += sh.warp_sum[k++];
        if (k == ACC_NW) {                                           // rounding hides it: the last id with weight
            target = INFINITY;
            while (k > 0 && !(sh.warp_sum[--k] > 0.0)) {}
        }
        before = e;
        const int part = part_of(hi - lo);
        lo = min(hi, lo + k * part);
        hi = min(hi, lo + part);
        if (hi - lo <= 128) break;
        sum_part(sh, w, lo, hi);
    }
    int token = -1;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x, t0 = child_token(sh, w, lane), t1 = child_token(sh, w, lane + 32);
        for (int base = lo; base < hi; base += 32) {
            const int i = base + lane;
            double x = i < hi ? weight_of(sh, w, w.p[i], w.kind == DRAWN ? w.q[i] : 0.f) : 0.0;
            if (w.kind == CHOSEN && (childrens_ids(sh, w, t0, t1, base) >> lane & 1)) x = 0.0;
            double upto = x;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double t = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += t;
            }
            const unsigned past = __ballot_sync(0xffffffffu, x > 0.0 && before + upto > target), some = __ballot_sync(0xffffffffu, x > 0.0);
            if (past) { token = base + __ffs(past) - 1; break; }
            if (some) token = base + 31 - __clz(some);
            before += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
    return token;
}

template <int C> __global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(ACC_NT) tree_accept_kernel(const AcceptArgs a) {
    chain_wait();
    __shared__ AcceptShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    cluster.barrier_arrive();                                        // every block has to run before another writes to its shared memory
    const int b = blockIdx.x / C, rank = (int)cluster.block_rank(), tid = threadIdx.x, lane = tid & 31, V = a.V;
    each_other_row(a.row_start, a.B, a.R, [&](int r) { a.path[r] = -1; });
    int row0, n_all;
    rows_of(a.row_start, a.R, b, row0, n_all);
    const int n = min(n_all, ACC_ROWS);
    for (int i = tid; i < n; i += ACC_NT) {
        const int up = a.parent[row0 + i], x = a.token[row0 + i];
        const bool tested = i > 0 && up >= 0 && up < i && x >= 0 && x < V;
        const size_t at = (size_t)(row0 + up) * V + x;
        sh.parent[i] = tested ? up : -1;
        sh.token[i] = x;
        sh.u[i] = a.u_accept[row0 + i];
        sh.p_of[i] = tested ? a.p[at] : 0.f;
        sh.q_of[i] = tested && a.q ? a.q[at] : 1.f;
    }
    if (rank == 0)
        for (int i = tid; i < n_all; i += ACC_NT) a.path[row0 + i] = i == 0 ? 0 : -1;
    __syncthreads();
    if (!a.q) {                                                      // a token that a sibling before it has: nothing is left of it when it is tested
        for (int t = tid; t < n * n; t += ACC_NT) {
            const int i = t / n, j = t % n;
            if (j < i && sh.parent[i] >= 0 && sh.parent[j] == sh.parent[i] && sh.token[j] == sh.token[i]) sh.p_of[i] = 0.f;
        }
        __syncthreads();
    }
    const float u_final = a.u_final[b];
    cluster.barrier_wait();
    // this block's ids
    const int S = ((V + C - 1) / C + 31) & ~31, lo = (int)min((long long)V, (long long)rank * S), hi = (int)min((long long)V, (long long)lo + S);
    int kept = 0, turn = 0;
    Weights w{a.p + (size_t)row0 * V, a.q ? a.q + (size_t)row0 * V : nullptr, ALL, 0, 0, n};
    double z = 1.0, total = -1.0;                                    // total: the sum that the last pass over the weights as they are gave; -1: there was none
    for (int last = 0; n > 0;) {
        const int c = next_child(sh, n, w.node, last);
        if (c == n) break;
        last = c;
        const double mine = weight_of(sh, w, sh.p_of[c], sh.q_of[c]);
        if ((double)sh.u[c] * z * (double)sh.q_of[c] < mine) {
            ++kept;
            if (rank == 0 && tid == 0) a.path[row0 + kept] = c;
            const size_t row = (size_t)(row0 + c) * V;
            w = Weights{a.p + row, a.q ? a.q + row : nullptr, ALL, 0, c, n};
            z = 1.0;
            total = -1.0;
        } else if (a.q) {
            __syncthreads();                                         // the tests before have read what is written next
            if (tid == 0) sh.inv[w.m] = 1.0 / z;
            __syncthreads();
            w.kind = DRAWN;
            ++w.m;
            z = total = sum_all<C>(sh, w, lo, hi, turn);
            turn ^= 1;
            if (!(z > 0.0)) break;                                   // nothing is left: no other child is kept
        } else {
            if (w.kind == ALL) {
                w.kind = CHOSEN;
                total = sum_all<C>(sh, w, lo, hi, turn);
                turn ^= 1;
            }
            double others = 0.0;                                     // the children behind this one
            for (int i = lane; i < n; i += 32)
                if (i > c && sh.parent[i] == w.node) others += sh.p_of[i];
            z = total + warp_sum64(others);
        }
    }
    if (n > 0) {
        if (!(total > 0.0)) {                                        // no rejection at this node, or nothing is left of its row
            w.kind = ALL;
            w.m = 0;
            total = sum_all<C>(sh, w, lo, hi, turn);
            turn ^= 1;
        }
        const double target = (double)u_final * total;
        double upto = 0.0, before = 0.0;
        int holder = -1;                                             // the block whose ids the running sum passes the target at
#pragma unroll
        for (int r = 0; r < C; ++r) {
            const double next = upto + sh.slot[turn ^ 1][r];
            if (holder < 0 && target >= 0.0 && next > target) { holder = r; before = upto; }
            upto = next;
        }
        if (rank == max(holder, 0)) {
            const int token = holder < 0 ? -1 : find_id(sh, w, lo, hi, before, target);
            if (tid == 0) a.next[b] = token;
        }
    } else if (rank == 0 && tid == 0) a.next[b] = -1;
    if (rank == 0 && tid == 0) a.accepted[b] = kept;
}

}  // namespace trees
}  // namespace knnssd
