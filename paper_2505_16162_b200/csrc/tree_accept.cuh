// Which drafts of a tree the full model's distributions keep, and the token after them: speculative sampling with several drafts behind a row.
//
// From row `node` (first the request's row 0) its children are tested in row order.  w is what is left of p[node], Z its sum (1 as long as nothing was rejected: a
// row of p is a distribution):
//   drafts drawn from q[node], each by itself:  child c is kept iff u_c Z q[node](x_c) < w(x_c); else w <- max(0, w / Z - q[node]), Z <- sum w
//   drafts chosen, not drawn (no q):            child c is kept iff u_c Z < w(x_c);              else w(x_c) <- 0, Z <- sum w
// A kept child is the next node.  Where none is left the token after it is the smallest x with w_0 + .. + w_x > u_final sum(w), from p[node] if nothing is left of it.
// Either way the tokens are distributed as p has them.  Random numbers are inputs.  A sum that is NaN keeps no further child and ends in no token.
//
// A request is the work of a cluster of C blocks, each with a contiguous part of the ids.  All blocks take the same decisions from the same numbers: the tests need one value
// of p and of q a draft, fetched for all drafts at once at the start.  Only a rejection reads a row: a pass over the ids, a sum per warp, a meeting of the cluster.  The last pass's sums
// are the draw's: the block and the warp whose ids hold the crossing are known from them, that block goes on in that warp's ids.  Without q a node takes one pass whatever is
// rejected: the sum of all ids but its children's, to which the children not yet rejected are added (nothing is subtracted, so nothing cancels).
// Sums in 64 bits: what a test or a draw next to a border decides does not depend on the order of 150 thousand additions.
#pragma once

#include <climits>
#include <cooperative_groups.h>

#include "trees.cuh"

namespace knnssd {
namespace trees {

namespace cg = cooperative_groups;

constexpr int ACC_NT = 256, ACC_NW = ACC_NT / 32;
constexpr int ACC_ROWS = 1024;            // rows of a request that are looked at
// Blocks of a request: as many as find room at once, and a thousand ids at least for each, below that a meeting of more blocks costs what they save.  1 / 8 / 16 of them: 24 requests
// of 25 rows and 32000 ids 25 / 12 / 14 us where drafts are drawn, 16 / 11 / 14 where they are chosen; of 152064 ids 86 / 23 / 17 and 37 / 14 / 15; 400 requests of 9 rows and 32000
// ids 39 / 66 / 130 and 23 / 55 / 117.  Where a block has more than 10 000 values to read they pay up to three and a half a processor (32 requests of 152064 ids, drawn, as 16
// blocks 22 us, as 8 28), else up to two.
inline int blocks_of(int requests, int vocab, bool drawn, int processors) {
    for (int c = 16; c > 1; c /= 2)
        if (2ll * requests * c <= (vocab * (drawn ? 2ll : 1ll) > 10000 * c ? 7 : 4) * processors && vocab >= 1000 * c) return c;
    return 1;
}

struct AcceptArgs {
    const float *p, *q;                   // [R][V]; q null: drafts chosen
    int V;
    const int *token, *parent, *row_start;
    int B, R;
    const float *u_accept, *u_final;
    int *path, *accepted, *next;
};

template <int C> struct AcceptShared {
    double slot[2][C * ACC_NW];                                      // the sums of all blocks' warps; the next pass's may come while these are read
    double part[ACC_NW];
    float p_of[ACC_ROWS], q_of[ACC_ROWS], u[ACC_ROWS];               // of each row: its parent's p and q at its token, its uniform
    alignas(16) int parent[ACC_ROWS], token[ACC_ROWS];                           // parent -1: not to be tested
    double sums[ACC_ROWS];                                           // of the rejections so far: the sum that the draft was held against; FAR: the one before over it
};

__device__ __forceinline__ double warp_sum64(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ double warp_upto64(double v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double t = __shfl_up_sync(0xffffffffu, v, o);
        if ((threadIdx.x & 31) >= o) v += t;
    }
    return v;
}

// The lowest row behind `last` whose parent is `node`; n: there is none.  The same in every warp.
__device__ __forceinline__ int next_child(const int *parent, int n, int node, int last) {
    for (int i0 = (last + 1) & ~31; i0 < n; i0 += 32) {
        const int i = i0 + (threadIdx.x & 31);
        const unsigned found = __ballot_sync(0xffffffffu, i > last && i < n && parent[i] == node);
        if (found) return i0 + __ffs(found) - 1;
    }
    return n;
}

// What a row's weights are: its values; what rejections of drafts drawn from q have left; its values without those of the children of `node`.
// Drafts drawn.  DRAWN: W = max(0, p - r q), r the sum of the sums S that the rejected drafts were held against (S = 1 at first): with W = S' w, S' the sum before, a draft is kept
// iff u S q < W, and W / S - q is positive where p - (r + S) q is.  One pass whatever came before, but each rejection makes S smaller by its Z, and the digits of p - r q that are
// left are those of r: it is held in two doubles.  While S >= SMALL they hold it exactly: an S ends at 2^-93, r is below 2^11.  FAR: below that (two dozen children that
// were rejected with a Z of a third, which drawn drafts are with a probability of SMALL) the recursion itself, w <- max(0, w / Z - q), `times` steps a value.
enum { ALL = 0, DRAWN = 1, CHOSEN = 2, FAR = 3 };
constexpr double SMALL = 0x1p-40;
struct Weights { const float *p, *q; int kind, node, n; double r, r_low; int times; double *sums; };
__device__ __forceinline__ double positive(double x) { return x < 0.0 ? 0.0 : x; }           // NaN stays
__device__ __forceinline__ double left_of(double r, double r_low, float p, float q) { return positive(fma(-r_low, (double)q, fma(-r, (double)q, (double)p))); }
__device__ __forceinline__ double far_left_of(const double *over_z, int times, float p, float q) {
    double x = p;
#pragma unroll 1
    for (int k = 0; k < times; ++k) x = positive(fma(x, over_z[k], -(double)q));
    return x;
}
__device__ __forceinline__ double drawn_left_of(const Weights &w, float p, float q) {
    return w.kind == FAR ? far_left_of(w.sums, w.times, p, q) : left_of(w.r, w.r_low, p, q);
}
// r + s, to the last bit of its second double.
__device__ __forceinline__ void add_to(double &r, double &r_low, double s) {
    const double sum = r + s, of_s = sum - r, low = (r - (sum - of_s)) + (s - of_s) + r_low;
    r = sum + low;
    r_low = low - (r - sum);
}
template <int C> __device__ __forceinline__ int child_token(const AcceptShared<C> &sh, const Weights &w, int i) { return i < w.n && sh.parent[i] == w.node ? sh.token[i] : -1; }

// A lane's share of a sum over ids [i0, i1), N values of a row on their way.  Pieces of code of their own: a round calls them from several places, and a block that comes to an
// instruction for the first time waits for it (unrolled in place, 32 values at a time and the draw's running sums with them: one row of 152064 ids 19 us for 7).
// A float's bits, moved to where a double has its own, are its value times 2^-896, zeros and subnormals included; the sum is scaled back.  Two integer operations, where a
// conversion takes 11 clocks a warp (a row of 152064 ids by one block: 32 us so, 24 with the bits).  What is not a finite number, or has a sign, comes to 2^-768 and more (no other
// float does, its sign or its exponent's bits see to it): then the sum is formed once more by conversions.
constexpr int OUTS = 4;                   // ids that a sum of values can leave out
constexpr double SCALED_BACK = 0x1p896, TOO_LARGE = 0x1p-768;
__device__ __forceinline__ double scaled(unsigned bits) { return __hiloint2double(bits >> 3, bits << 29); }
// Four ids from `id` on, those below `end`; zeros behind.
__device__ __forceinline__ void four(const float *p, int id, int end, bool aligned, unsigned (&v)[4]) {
    if (aligned && id + 4 <= end) {
        const uint4 w = __ldg(reinterpret_cast<const uint4 *>(p + id));
        v[0] = w.x; v[1] = w.y; v[2] = w.z; v[3] = w.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = id + j < end ? __float_as_uint(__ldg(p + id + j)) : 0u;
    }
}
static __device__ __noinline__ double sum_values(const float *p, int i0, int i1, int out0, int out1, int out2, int out3) {
    constexpr int N = 4;
    double s[2] = {0.0, 0.0};
    const bool aligned = (reinterpret_cast<uintptr_t>(p + i0) & 15u) == 0, outs = out0 < i1;
    const int first = i0 + 4 * (threadIdx.x & 31);
#pragma unroll 1
    for (int i = first; i < i1; i += 128 * N) {
        unsigned v[N][4];
#pragma unroll
        for (int e = 0; e < N; ++e) four(p, i + 128 * e, i1, aligned, v[e]);
        if (outs) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const unsigned d0 = out0 - i - 128 * e, d1 = out1 - i - 128 * e, d2 = out2 - i - 128 * e, d3 = out3 - i - 128 * e;
                if (min(min(d0, d1), min(d2, d3)) < 4u)
#pragma unroll
                    for (unsigned j = 0; j < 4; ++j)
                        if (j == d0 || j == d1 || j == d2 || j == d3) v[e][j] = 0u;
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j & 1] += scaled(v[e][j]);
    }
    if (s[0] + s[1] < TOO_LARGE) return (s[0] + s[1]) * SCALED_BACK;
    double t = 0.0;
#pragma unroll 1
    for (int i = first; i < i1; i += 128)
        for (int j = i; j < min(i + 4, i1); ++j) t += j == out0 || j == out1 || j == out2 || j == out3 ? 0.0 : (double)p[j];
    return t;
}
static __device__ __noinline__ double sum_left(const float *p, const float *q, double r, double r_low, int i0, int i1) {
    constexpr int N = 2;
    double s[2] = {0.0, 0.0};
    unsigned top = 0;
    const bool aligned = ((reinterpret_cast<uintptr_t>(p + i0) | reinterpret_cast<uintptr_t>(q + i0)) & 15u) == 0;
    const int first = i0 + 4 * (threadIdx.x & 31);
#pragma unroll 1
    for (int i = first; i < i1; i += 128 * N) {
        unsigned v[N][4], u[N][4];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            four(p, i + 128 * e, i1, aligned, v[e]);
            four(q, i + 128 * e, i1, aligned, u[e]);
        }
#pragma unroll
        for (int e = 0; e < N; ++e)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const double y = scaled(u[e][j]), x = fma(-r_low, y, fma(-r, y, scaled(v[e][j])));
                s[j & 1] += __double2hiint(x) < 0 ? 0.0 : x;
                top = max(top, u[e][j]);
            }
    }
    if (top < 0x7f800000u && s[0] + s[1] < TOO_LARGE) return (s[0] + s[1]) * SCALED_BACK;
    double t = 0.0;
#pragma unroll 1
    for (int i = first; i < i1; i += 128)
        for (int j = i; j < min(i + 4, i1); ++j) t += left_of(r, r_low, p[j], q[j]);
    return t;
}
static __device__ __noinline__ double sum_far(const float *p, const float *q, const double *over_z, int times, int i0, int i1) {
    double t = 0.0;
#pragma unroll 1
    for (int i = i0 + (threadIdx.x & 31); i < i1; i += 32) t += far_left_of(over_z, times, p[i], q[i]);
    return t;
}
// Whether an id is the token of a child, for the 32 ids from `base` on.
template <int C> __device__ __forceinline__ bool childs_id(const AcceptShared<C> &sh, const Weights &w, int base) {
    unsigned out = 0;
    for (int i = threadIdx.x & 31; i < w.n; i += 32) {
        const int t = child_token(sh, w, i);
        if (t >= base && t < base + 32) out |= 1u << (t - base);
    }
    return __reduce_or_sync(0xffffffffu, out) >> (threadIdx.x & 31) & 1;
}
// The lowest token of a child above `id`; INT_MAX: none is.
template <int C> __device__ __forceinline__ int next_token(const AcceptShared<C> &sh, const Weights &w, int id) {
    int t = INT_MAX;
    for (int i = threadIdx.x & 31; i < w.n; i += 32) {
        const int x = child_token(sh, w, i);
        if (x > id) t = min(t, x);
    }
    return __reduce_min_sync(0xffffffffu, t);
}
// The sum of the weights of ids [i0, i1), by a warp.
template <int C> __device__ __forceinline__ double sum_of(const AcceptShared<C> &sh, const Weights &w, int i0, int i1) {
    double s = 0.0;
    if (w.kind == DRAWN) s = sum_left(w.p, w.q, w.r, w.r_low, i0, i1);
    else if (w.kind == FAR) s = sum_far(w.p, w.q, w.sums, w.times, i0, i1);
    else {
        for (int from = i0, to; from < i1; from = to) {              // runs of ids with OUTS of the children's tokens among them, or all
            int out[OUTS];
#pragma unroll
            for (int k = 0, t = from - 1; k < OUTS; ++k) out[k] = t = w.kind == CHOSEN && t < i1 ? next_token(sh, w, t) : INT_MAX;
            to = out[OUTS - 1] < i1 ? min(i1, next_token(sh, w, out[OUTS - 1])) : i1;
            s += sum_values(w.p, from, to, out[0], out[1], out[2], out[3]);
        }
    }
    return warp_sum64(s);
}

// Ids of a warp's part of a range of `len`, and where warp k's begins.
__device__ __forceinline__ int part_of(int len) { return ((len + ACC_NW - 1) / ACC_NW + 31) & ~31; }
__device__ __forceinline__ int part_at(int lo, int hi, int k) { return (int)min((long long)hi, lo + (long long)k * part_of(hi - lo)); }

// The sum of the weights over all ids, [lo, hi) this block's: a part a warp, whose sum goes to all blocks; then the cluster meets.
template <int C> __device__ __forceinline__ double sum_all(AcceptShared<C> &sh, const Weights &w, int lo, int hi, int turn) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const double mine = sum_of(sh, w, part_at(lo, hi, warp), part_at(lo, hi, warp + 1));
    if constexpr (C > 1) {
        cg::cluster_group cluster = cg::this_cluster();
        if (lane < C) cluster.map_shared_rank(&sh, lane)->slot[turn][cluster.block_rank() * ACC_NW + warp] = mine;
        cluster.sync();
    } else {
        if (lane == 0) sh.slot[turn][warp] = mine;
        __syncthreads();
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < (C * ACC_NW + 31) / 32; ++i)
        if (C * ACC_NW >= 32 || lane < C * ACC_NW) s += sh.slot[turn][lane * ((C * ACC_NW + 31) / 32) + i];
    return __shfl_sync(0xffffffffu, warp_upto64(s), 31);
}

// Of N sums one behind the other, `before` ahead of them, the one in which the running sum passes `target`, and what is ahead of it.  The lanes' running sums are rounded
// otherwise than a lane's own: where the crossing lies between the two it is in the last sum up to there that is not zero, at its end (the target becomes infinite).  By a warp.
template <int N> __device__ __forceinline__ int crossing(const double *sums, double &before, double &target) {
    constexpr int PER = (N + 31) / 32;
    const int lane = threadIdx.x & 31;
    double own = 0.0;
    int last = -1;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (lane * PER + i < N) {
            const double v = sums[lane * PER + i];
            own += v;
            if (v > 0.0) last = lane * PER + i;
        }
    const double upto = before + warp_upto64(own);
    const unsigned past = __ballot_sync(0xffffffffu, upto > target);
    double e = __shfl_up_sync(0xffffffffu, upto, 1);
    if (lane == 0) e = before;
    int at = -1;
    if (past && lane == __ffs(past) - 1) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (at < 0 && lane * PER + i < N) {
                const double v = sums[lane * PER + i];
                if (e + v > target) at = lane * PER + i; else e += v;
            }
    }
    if (past) {
        at = __shfl_sync(0xffffffffu, at, __ffs(past) - 1);
        before = __shfl_sync(0xffffffffu, e, __ffs(past) - 1);
        if (at >= 0) return at;
        if (lane >= __ffs(past)) last = -1;
    }
    target = INFINITY;
    return max(0, __reduce_max_sync(0xffffffffu, last));
}

// By a block: the first of the ids [lo, hi) at which the running sum, `before` ahead of them, passes `target`; in one of its warps, the others get -1.
template <int C> __device__ __forceinline__ int find_id(AcceptShared<C> &sh, const Weights &w, int lo, int hi, double before, double target) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    while (hi - lo > ACC_NT) {
        const double mine = sum_of(sh, w, part_at(lo, hi, warp), part_at(lo, hi, warp + 1));
        __syncthreads();                                             // the sums before have been read
        if (lane == 0) sh.part[warp] = mine;
        __syncthreads();
        const int k = crossing<ACC_NW>(sh.part, before, target), at = part_at(lo, hi, k);
        hi = part_at(lo, hi, k + 1);
        lo = at;
    }
    const int base = lo + 32 * warp, id = base + lane;               // an id a thread
    double x = 0.0;
    if (id < hi) x = w.kind == DRAWN || w.kind == FAR ? drawn_left_of(w, w.p[id], w.q[id]) : (double)w.p[id];
    if (w.kind == CHOSEN && childs_id(sh, w, base)) x = 0.0;
    const double upto = warp_upto64(x);
    __syncthreads();
    if (lane == 31) sh.part[warp] = upto;
    __syncthreads();
    if (warp != crossing<ACC_NW>(sh.part, before, target)) return -1;
    const unsigned past = __ballot_sync(0xffffffffu, x > 0.0 && before + upto > target), some = __ballot_sync(0xffffffffu, x > 0.0);
    return past ? base + __ffs(past) - 1 : some ? base + 31 - __clz(some) : base;
}

// FAR's factors from the sums of a node's rejections, by a block.
static __device__ __noinline__ void recur(double *sums, int times) {
    static_assert(ACC_ROWS == 4 * ACC_NT, "four a thread");
    double f[4];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = i * ACC_NT + threadIdx.x;
        f[i] = k < times ? (k > 0 ? sums[k - 1] : 1.0) / sums[k] : 0.0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * ACC_NT + threadIdx.x < times) sums[i * ACC_NT + threadIdx.x] = f[i];
    __syncthreads();
}
// Whether a sibling before row i has its token.  Siblings lie behind their parent: a chain has none to look at.  A piece of code of its own, for the registers of the rest.  A call
// with 1024 rows of 32000 ids as a chain / all children of one 23 / 85 us (every pair of rows, a division each: 432 / 500).
static __device__ __noinline__ bool came_before(const int *parent, const int *token, int i) {
    const int up = parent[i], x = token[i];
    bool found = false;
#pragma unroll 2
    for (int j = (up + 1) & ~3; j < i; j += 4) {
        const int4 p = *reinterpret_cast<const int4 *>(parent + j), t = *reinterpret_cast<const int4 *>(token + j);
        found |= (p.x == up && t.x == x) || (j + 1 < i && p.y == up && t.y == x) || (j + 2 < i && p.z == up && t.z == x) || (j + 3 < i && p.w == up && t.w == x);
    }
    return found;
}
// Drafts chosen: of the children of w.node behind row c, which was rejected, the first that is kept; `rest`: the sum without all of the node's children.  n: none is.
// The sum that a child is held against is the rest and the children from it on: all are tested at once.  The same in every warp.  Where p at a child's token is not finite
// the rest becomes NaN: the children before that one are held against such a sum, those behind it would not be.
template <int C> __device__ __forceinline__ int first_kept(const AcceptShared<C> &sh, const Weights &w, int c, double &rest) {
    if (!isfinite(sh.p_of[c])) rest = NAN;
    const int lane = threadIdx.x & 31;
    auto p_of = [&](int i) { return i > c && i < w.n && sh.parent[i] == w.node ? (double)sh.p_of[i] : 0.0; };
    auto from_here_on = [&](double v) {                              // the sum over this lane and those behind it
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const double t = __shfl_down_sync(0xffffffffu, v, o);
            if (lane + o < 32) v += t;
        }
        return v;
    };
    static_assert(ACC_ROWS <= 32 * 32, "a lane for 32 rows");
    double later = 0.0;                                              // lane k: children among the rows from 32 (k + 1) on
    if (w.n > 32) {
        for (int k = 1; 32 * k < w.n; ++k) {
            const double s = warp_sum64(p_of(32 * k + lane));
            if (lane == k - 1) later = s;
        }
        later = from_here_on(later);
    }
    for (int k = (c + 1) / 32; 32 * k < w.n; ++k) {
        const int i = 32 * k + lane;
        const double mine = p_of(i), sum = rest + __shfl_sync(0xffffffffu, later, k) + from_here_on(mine);
        const unsigned found = __ballot_sync(0xffffffffu, i > c && i < w.n && sh.parent[i] == w.node && (double)sh.u[i] * sum < mine);
        if (__any_sync(0xffffffffu, !isfinite(mine))) {
            rest = NAN;
            break;
        }
        if (found) return 32 * k + __ffs(found) - 1;
    }
    return w.n;
}

template <int C> __global__ void __cluster_dims__(C, 1, 1) __launch_bounds__(ACC_NT, 3) tree_accept_kernel(const AcceptArgs a) {
    chain_wait();
    __shared__ AcceptShared<C> sh;
    cg::cluster_group cluster = cg::this_cluster();
    if (C > 1) cluster.barrier_arrive();                             // every block has to run before another writes to its shared memory
    const int b = blockIdx.x / C, rank = C > 1 ? (int)cluster.block_rank() : 0, tid = threadIdx.x, lane = tid & 31, V = a.V;
    each_other_row(a.row_start, a.B, a.R, [&](int r) { a.path[r] = -1; });
    int row0, n_all;
    rows_of(a.row_start, a.R, b, row0, n_all);
    const int n = min(n_all, ACC_ROWS);
    const int S = ((V + C - 1) / C + 31) & ~31;                      // ids of a block
    auto first_id = [&](int r) { return (int)min((long long)V, (long long)r * S); };
    const int lo = first_id(rank), hi = first_id(rank + 1);
    Weights w{a.p + (size_t)row0 * V, a.q ? a.q + (size_t)row0 * V : nullptr, ALL, 0, n, 0.0, 0.0, 0, sh.sums};
    const float u_final = a.u_final[b];
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
        for (int i = tid; i < n; i += ACC_NT)
            if (sh.parent[i] >= 0 && came_before(sh.parent, sh.token, i)) sh.p_of[i] = 0.f;
        __syncthreads();
    }
    if (C > 1) cluster.barrier_wait();
    int kept = 0, turn = 0;
    double z = 1.0, total = -1.0;                                    // total: the sum that the last pass over the weights as they are gave; -1: there was none
    int last = 0;
    auto step_to = [&](int c) {
        ++kept;
        if (rank == 0 && tid == 0) a.path[row0 + kept] = c;
        const size_t row = (size_t)(row0 + c) * V;
        w.p = a.p + row;
        w.q = a.q ? a.q + row : nullptr;
        w.kind = ALL;
        w.node = last = c;
        w.r = w.r_low = 0.0;
        w.sums += w.times;                                           // no place of them is written twice: some warp may still be at the test before
        w.times = 0;
        z = 1.0;
        total = -1.0;
    };
    for (bool more = true; n > 0;) {                                 // more: there may be children that can be kept
        const int c = more ? next_child(sh.parent, n, w.node, last) : n;
        if (c < n) {
            last = c;
            const double mine = w.kind == DRAWN || w.kind == FAR ? drawn_left_of(w, sh.p_of[c], sh.q_of[c]) : (double)sh.p_of[c];
            if ((double)sh.u[c] * z * (double)sh.q_of[c] < mine) {
                step_to(c);
                continue;
            }
            if (a.q) {
                if (tid == 0) w.sums[w.times] = w.kind == FAR ? 1.0 / z : z;
                ++w.times;
                if (w.kind == FAR) __syncthreads();
                else {
                    w.kind = DRAWN;
                    add_to(w.r, w.r_low, z);
                }
            } else w.kind = CHOSEN;
        } else {
            more = false;
            if (total > 0.0 || total != total) break;
            w.kind = ALL;                                            // no rejection at this node, or nothing is left of its row
        }
        for (;;) {
            z = total = sum_all<C>(sh, w, lo, hi, turn);
            turn ^= 1;
            if (w.kind != DRAWN || !(total < SMALL)) break;
            recur(w.sums, w.times);                                  // once more, by the recursion
            w.kind = FAR;
        }
        if (!more) break;
        if (w.kind == CHOSEN) {
            const int next = first_kept(sh, w, c, total);
            if (next < n) step_to(next); else more = false;
        } else more = total > 0.0;
    }
    if (n > 0) {
        double target = (double)u_final * total, before = 0.0;
        const bool drawn = target >= 0.0 && target < total;
        const int part = drawn ? crossing<C * ACC_NW>(sh.slot[turn ^ 1], before, target) : 0, holder = part / ACC_NW;
        if (rank == holder) {
            const int l = first_id(holder), h = first_id(holder + 1), k = part % ACC_NW;
            const int token = drawn ? find_id(sh, w, part_at(l, h, k), part_at(l, h, k + 1), before, target) : -1;
            if (drawn ? token >= 0 && lane == 0 : tid == 0) a.next[b] = token;
        }
    } else if (rank == 0 && tid == 0) a.next[b] = -1;
    if (rank == 0 && tid == 0) a.accepted[b] = kept;
}

}  // namespace trees
}  // namespace knnssd
