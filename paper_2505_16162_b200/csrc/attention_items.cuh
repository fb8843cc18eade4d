// How the attention operators share their work out: items, and equal runs of their positions.
//
// An item is (request, block of new rows, K/V head): the rows of a block times the query heads that
// share the head, over the positions that the block's last row sees.  The positions of all items, one item behind the other in request,
// block and head order, are cut into equal runs, one per worker (a warp or a block of the launch), whatever the lengths.  Where an item begins follows
// from the sums of the requests' costs and a closed form within a request, so every worker finds its own run from the lengths on the device.
// Parts of an item that several workers have are put together by merge_kernel.
#pragma once

#include "device_common.cuh"

namespace knnssd {
namespace attn {

constexpr int SLOTS = 2;                  // parts a worker may leave: of the item its run begins in, of the one it ends in

struct Args {
    const void *q;                        // [R][H][hd], rows q_stride elements apart
    void *out;                            // [R][H][hd]
    long long q_stride;
    const void *k, *v;                    // pages [n_pages][KV][page][hd]; packed: [R][KV][hd], rows k_stride / v_stride elements apart
    long long k_stride, v_stride;
    const int *table;                     // [B][max_pages]
    int max_pages, page_shift, n_pages;
    const int *lens, *row_start;          // [B] (packed: nullptr, nothing held), [B + 1]
    int B, R, H, KV;
    float scale_log2;                     // scale log2 e: the softmax runs in powers of two
    int gs, subs, nvh;                    // query heads of an item; items that share a K/V head's rows (heads of a group / gs); KV subs
    int tb;                               // new rows of a block (of half a block, where blocks have two halves)
    int pair;                             // the halves of a block take two heads of a request with few rows
    int extra;                            // positions that an item's beginning and end cost
    int most, least_run;                  // workers at most (no more than the launch has); positions a worker takes at least
    // parts of items: what worker w knows of the item its run begins in, and its parts' (m, l) [w][SLOTS][rows] and o [w][SLOTS][rows][hd]
    struct Part *parts;
    float2 *ml;
    float *o;
    // bounded waits (tensor kernel): where one that gives up leaves its code, after how many polls; tiles that a block's copies end after, those of each of the copying warps
    int *err;
    unsigned wait_limit, stop_after[2];
    const unsigned long long *seen;       // trees: [R], which of the 64 positions up to a row's own it sees
};

// Which positions a row of a tree sees: all that lie 64 and more before its own, and of those d = 0 .. 63 before it the ones whose bit d is set.
__device__ __forceinline__ bool tree_sees(unsigned long long word, int d) { return d >= 64 || (d >= 0 && (word >> d & 1)); }

// first: no run before this one begins within the item; [from, to): the run's positions of it; start: the item (-1: none)
struct Part { long long start; int first, kv, from, to, row0, rows, vh, paired; };

// A request's new rows n, what it held before, the block's rows tb and the items nvh per block.  HALVES: a block has two halves of a.tb rows each;
// where a request has no more rows than one of them, the halves may take two heads instead (paired).
struct Request { int n, held, row0, tb, nvh; bool paired; long long cost; };

template <bool HALVES> __device__ __forceinline__ Request request_here(const Args &a, int b) {
    Request r;
    const int r0 = min(max(a.row_start[b], 0), a.R), r1 = min(max(a.row_start[b + 1], 0), a.R);
    r.n = max(r1 - r0, 0);
    r.row0 = r0;
    r.held = a.lens ? (int)min((long long)max(a.lens[b], 0), (long long)a.max_pages << a.page_shift) : 0;
    r.paired = HALVES && a.pair && r.n <= a.tb;
    r.tb = HALVES && !r.paired ? 2 * a.tb : a.tb;
    r.nvh = r.paired ? (a.nvh + 1) / 2 : a.nvh;
    const long long whole = r.n / r.tb, left = r.n % r.tb, each = (long long)r.held + a.extra;
    r.cost = (whole * each + r.tb * (whole * (whole + 1) / 2) + (left ? each + r.n : 0)) * r.nvh;
    return r;
}

// The rows kernel keeps its code small (its warps run apart, each through all of it), the tensor kernel its registers.
static __device__ __noinline__ Request request_apart(const Args &a, int b) { return request_here<false>(a, b); }
template <bool HALVES> __device__ __forceinline__ Request request_of(const Args &a, int b) {
    if constexpr (HALVES) return request_here<true>(a, b);
    else return request_apart(a, b);
}

// An item and where it begins among all items' positions.
template <bool HALVES> struct Item {
    Request r;
    int b, rb, vh, kv;                    // kv: positions that the block's last row sees
    long long start;
    __device__ __forceinline__ void see() { kv = r.held + min(r.tb * (rb + 1), r.n); }
    __device__ __forceinline__ int tokens() const { return min(r.tb, r.n - rb * r.tb); }
    // the item behind this one; false when there is none
    __device__ __forceinline__ bool next(const Args &a) {
        start += kv + a.extra;
        if (++vh < r.nvh) return true;
        vh = 0;
        if (++rb * r.tb < r.n) { see(); return true; }
        rb = 0;
        while (++b < a.B) {
            r = request_of<HALVES>(a, b);
            if (r.cost > 0) { see(); return true; }
        }
        return false;
    }
};

// A block's view of the requests: the costs of N runs of them, summed, N threads.
template <int N> struct Costs {
    long long pfx[N + 1];
    long long warp_sum[N / 32];
};

template <bool HALVES, int N> __device__ __forceinline__ void sum_costs(const Args &a, Costs<N> &c) {
    const int tid = threadIdx.x, per = (a.B + N - 1) / N, lane = tid & 31;
    long long v = 0;
    if (tid < N) {
        for (int b = tid * per; b < min((tid + 1) * per, a.B); ++b) v += request_of<HALVES>(a, b).cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        if (lane == 31) c.warp_sum[tid >> 5] = v;
    }
    __syncthreads();
    if (tid < N) {
        for (int w = 0; w < tid >> 5; ++w) v += c.warp_sum[w];
        c.pfx[tid + 1] = v;
        if (tid == 0) c.pfx[0] = 0;
    }
    __syncthreads();
}

// The item that position x of all items' lies in; x < the sum.
template <bool HALVES, int N> __device__ __forceinline__ Item<HALVES> item_at(const Args &a, const Costs<N> &c, long long x) {
    int lo = 0, hi = N - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (c.pfx[mid + 1] > x) hi = mid; else lo = mid + 1;
    }
    Item<HALVES> it;
    it.start = c.pfx[lo];
    it.b = lo * ((a.B + N - 1) / N);
    for (;; ++it.b) {
        it.r = request_of<HALVES>(a, it.b);
        if (x < it.start + it.r.cost) break;
        it.start += it.r.cost;
    }
    // block rb begins at nvh (rb (held + extra) + tb rb (rb + 1) / 2)
    const long long at = x - it.start;
    auto before = [&](long long rb) { return it.r.nvh * (rb * ((long long)it.r.held + a.extra) + it.r.tb * (rb * (rb + 1) / 2)); };
    int r0 = 0, r1 = (it.r.n + it.r.tb - 1) / it.r.tb - 1;
    while (r0 < r1) {
        const int mid = (r0 + r1) >> 1;
        if (before(mid + 1) > at) r1 = mid; else r0 = mid + 1;
    }
    it.rb = r0;
    it.see();
    it.vh = (int)((at - before(r0)) / (it.kv + a.extra));
    it.start += before(r0) + (long long)it.vh * (it.kv + a.extra);
    return it;
}

// The run of worker w of W, and where position x cuts an item: at the next multiple of TP of it.
__device__ __forceinline__ long long run_start(long long total, int w, int W) { return min(total, ((total + W - 1) / W) * w); }
template <int TP, bool HALVES> __device__ __forceinline__ int cut(const Item<HALVES> &it, long long x) {
    return (int)(x <= it.start ? 0 : min((x - it.start + TP - 1) & ~(long long)(TP - 1), (long long)it.kv));
}
__device__ __forceinline__ int workers_of(const Args &a, long long total) { return (int)max(1ll, min((long long)a.most, total / a.least_run)); }

// What worker w leaves for the merge about the item that its run begins in.
template <int TP, bool HALVES> __device__ __forceinline__ void note_part(const Args &a, const Item<HALVES> &it, int w, int W, long long total, long long x0, long long x1) {
    Part p;
    p.start = it.start;
    p.from = cut<TP>(it, x0); p.to = cut<TP>(it, x1); p.kv = it.kv;
    p.first = p.from > 0 && p.from < it.kv && run_start(total, w - 1, W) <= it.start;
    p.row0 = it.r.row0 + it.rb * it.r.tb; p.rows = it.tokens(); p.vh = it.vh; p.paired = it.r.paired;
    a.parts[w] = p;
}

// Rows before the first request's and behind the last one's are nobody's: zeros.
template <typename T> __device__ __forceinline__ void clear_others(const Args &a, int hd, int thread, int threads) {
    const int first = min(max(a.row_start[0], 0), a.R), used = max(first, min(a.row_start[a.B], a.R)), others = first + a.R - used;
    if (others == 0) return;
    const long long row = (long long)a.H * hd, held = (used - first) * row;
    for (long long i = thread; i < others * row; i += threads) static_cast<T *>(a.out)[i < first * row ? i : i + held] = T(0);
}

// Row r of an item's rows (ROWS, two halves of ROWS / 2 where HALVES): the new row of the block and the query head; -1 where there is none.
template <bool HALVES, int ROWS> __device__ __forceinline__ void place_of(const Args &a, int tokens, int vh, bool paired, int r, int &token, int &head) {
    const int half = HALVES ? r / (ROWS / 2) : 0, rr = HALVES ? r % (ROWS / 2) : r;
    const int t = rr / a.gs, v = paired ? 2 * vh + half : vh;
    token = t < a.tb ? t + (paired ? 0 : half * a.tb) : -1;
    const int G = a.H / a.KV, kvh = v / a.subs, h = (v % a.subs) * a.gs + rr % a.gs;
    if (token >= tokens || v >= a.nvh || h >= G) token = -1;
    head = kvh * G + h;
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---- rows by the definition ------------------------------------------------------------------------------------------
// Where a position of a request's K/V head lies, in elements; false: it has no page.
template <int HD, bool PAGED> __device__ __forceinline__ bool key_at(const Args &a, int b, int seq_row0, int kvh, int pos, size_t &k, size_t &v) {
    if (!PAGED) {
        k = (size_t)(seq_row0 + pos) * a.k_stride + (size_t)kvh * HD;
        v = (size_t)(seq_row0 + pos) * a.v_stride + (size_t)kvh * HD;
        return true;
    }
    const int idx = pos >> a.page_shift, id = idx < a.max_pages ? a.table[(size_t)b * a.max_pages + idx] : -1;
    if (id < 0 || id >= a.n_pages) return false;
    k = v = ((((size_t)id * a.KV + kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * HD;
    return true;
}
// N words, by as many bytes at a time as they are a multiple of.
template <int N> __device__ __forceinline__ void read_words(const void *p, uint32_t (&w)[N]) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 u = __ldg(static_cast<const uint4 *>(p) + i / 4);
            w[i] = u.x; w[i + 1] = u.y; w[i + 2] = u.z; w[i + 3] = u.w;
        }
    } else if constexpr (N == 2) {
        const uint2 u = __ldg(static_cast<const uint2 *>(p));
        w[0] = u.x; w[1] = u.y;
    } else w[0] = __ldg(static_cast<const uint32_t *>(p));
}
template <int N> __device__ __forceinline__ void read_values(const float *p, float (&v)[N]) {
    uint32_t w[N];
    read_words(p, w);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __uint_as_float(w[i]);
}
template <int N> __device__ __forceinline__ void read_values(const bf16_t *p, float (&v)[N]) {
    uint32_t w[N / 2];
    read_words(p, w);
#pragma unroll
    for (int i = 0; i < N; i += 2) { v[i] = __uint_as_float(w[i / 2] << 16); v[i + 1] = __uint_as_float(w[i / 2] & 0xffff0000u); }
}

// A row of an item: its place among all rows and its head, the positions from .. to - 1 that it is about, where its result goes, and its own position.
struct Row { int b, seq_row0, row, head, from, to; bool whole; size_t slot; int last; };

// The same row from nothing but the positions that it sees, in ordinary fp32 arithmetic: whatever IEEE makes of values that are not finite.  A warp
// together, a score a lane, then HD / 32 dimensions a lane.  For rows that the matrix instructions cannot do; never on finite inputs.
template <int HD, typename QT, typename KT, bool PAGED, bool TREE> __device__ __noinline__ void row_by_definition(const Args &a, const Row r) {
    constexpr int D = HD / 32, N = 16 / (int)sizeof(KT);             // dimensions a lane; values of 16 bytes of a key
    const int lane = threadIdx.x & 31, kvh = r.head / (a.H / a.KV);
    const QT *q = static_cast<const QT *>(a.q) + (size_t)r.row * a.q_stride + (size_t)r.head * HD;
    const KT *kp = static_cast<const KT *>(a.k), *vp = static_cast<const KT *>(a.v) + lane * D;
    const unsigned long long word = TREE ? a.seen[r.row] : 0ull;
    float o[D], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < D; ++j) o[j] = 0.f;
#pragma unroll 1
    for (int p0 = r.from; p0 < r.to; p0 += 32) {
        size_t k = 0, v = 0;
        const bool there = p0 + lane < r.to && (!TREE || tree_sees(word, r.last - p0 - lane)) && key_at<HD, PAGED>(a, r.b, r.seq_row0, kvh, p0 + lane, k, v);
        float s = -INFINITY;
        if (there) {
            s = 0.f;
#pragma unroll 4
            for (int i = 0; i < HD; i += N) {
                float x[N], y[N];
                read_values(q + i, x);
                read_values(kp + k + i, y);
#pragma unroll
                for (int j = 0; j < N; ++j) s = fmaf(x[j], y[j], s);
            }
            s *= a.scale_log2;
        }
        const unsigned some = __ballot_sync(0xffffffffu, there);
        const float mn = fmaxf(m, warp_max(s)), base = mn == -INFINITY ? 0.f : mn, f = exp2_approx(m - base), p = there ? exp2_approx(s - base) : 0.f;
        m = mn;
        l = l * f + warp_sum(p);
        bool nan = true;
#pragma unroll
        for (int j = 0; j < D; ++j) { o[j] *= f; nan &= o[j] != o[j]; }
        if (l != l || __all_sync(0xffffffffu, nan)) break;                 // that stays so
#pragma unroll 8
        for (int u = 0; u < 32; ++u) {
            const float pu = __shfl_sync(0xffffffffu, p, u);
            const size_t vu = __shfl_sync(0xffffffffu, (unsigned long long)v, u);
            if (!(some >> u & 1)) continue;
            float y[D];
            read_values(vp + vu, y);
#pragma unroll
            for (int j = 0; j < D; ++j) o[j] = fmaf(pu, y[j], o[j]);
        }
    }
    const float inv = !r.whole ? 1.f : l == 0.f ? 0.f : 1.0f / l;
    if (!r.whole && lane == 0) a.ml[r.slot] = make_float2(m, l);
#pragma unroll
    for (int j = 0; j < D; ++j) {
        if (!r.whole) a.o[r.slot * HD + lane * D + j] = o[j];
        else if constexpr (sizeof(QT) == 2) static_cast<QT *>(a.out)[((size_t)r.row * a.H + r.head) * HD + lane * D + j] = float_to_bf16_rne(o[j] * inv);
        else static_cast<QT *>(a.out)[((size_t)r.row * a.H + r.head) * HD + lane * D + j] = o[j] * inv;
    }
}

// Items in parts.  Block (w, j) does eight rows at a time of the item that worker w's run is the first to begin within: the part of worker w - 1
// and those behind it until the item's end, in their order.  Of few rows each has several of the block's eight warps, which share its parts out;
// a warp's lanes share the parts' (m, l) out, then hd / 32 dimensions each.  The grid has as many j as the host believes there to be
// rows, of either half; if there are more, a block goes on to them.  With as many as 256 rows need, whatever there is: 4 requests of 16 rows and 50
// positions 23 us for 18, 33 of 2 rows 20 for 16, 2 of 35 361 positions 37 for 30 (12000 packed tokens 723 for 726: five blocks an SM either way).
template <int HD, typename QT, bool HALVES, int ROWS>
__global__ void __launch_bounds__(256, 5) merge_kernel(const Args a) {
    constexpr int D = HD / 32, HALF = HALVES ? ROWS / 2 : ROWS;
    __shared__ float2 ml_of[8];
    __shared__ float o_of[8][HD];
    chain_wait();
    const int w = blockIdx.x + 1, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Part p = a.parts[w];
    if (!p.first) return;
    const int step = HALVES ? gridDim.y / 2 : gridDim.y, half = blockIdx.y / step;
    // the half's rows that can be live; place_of leaves out those of them that are not
    const int rows = min(HALF, (HALVES && !p.paired ? min(a.tb, p.rows - half * a.tb) : p.rows) * a.gs);
    for (int r0 = blockIdx.y % step * 8; r0 < rows; r0 += step * 8) {
        const int here = min(8, rows - r0);
        const int share = here > 4 ? 1 : here > 2 ? 2 : here > 1 ? 4 : 8;            // warps a row
        const int r = half * HALF + r0 + warp / share, mine = warp % share;
        int token = -1, head = 0;
        if (warp / share < here) place_of<HALVES, ROWS>(a, p.rows, p.vh, p.paired, r, token, head);
        // part i: of run w - 1 + i, as long as the runs begin in this item
        auto slot = [&](int i) { return ((size_t)(w - 1 + i) * SLOTS + (i == 0 ? 1 : 0)) * ROWS + r; };
        const int most = gridDim.x + 2 - w;
        float o[D], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int i = 0; i < D; ++i) o[i] = 0.f;
        for (int i0 = mine * 32; token >= 0; i0 += 32 * share) {
            const int i = i0 + lane;
            bool its = i < most, there = its;                            // there: not cut away
            if (its && i > 0) {
                const Part *q = a.parts + w - 1 + i;
                its = q->start == p.start;
                there = its && q->from < q->to;
            }
            const unsigned all = __ballot_sync(0xffffffffu, its);
            const int n = all == 0xffffffffu ? 32 : __ffs(~all) - 1;      // lanes up to the first that is not of the item
            there = there && lane < n;
            const float2 v = there ? a.ml[slot(i)] : make_float2(-INFINITY, 0.f);
            const float mn = fmaxf(m, warp_max(v.x)), base = mn == -INFINITY ? 0.f : mn;
            const float f = exp2_approx(v.x - base), old = exp2_approx(m - base);
            l = l * old + warp_sum(v.y * f);
#pragma unroll
            for (int j = 0; j < D; ++j) o[j] *= old;
            m = mn;
            const unsigned some = __ballot_sync(0xffffffffu, there);
#pragma unroll 8
            for (int u = 0; u < n; ++u) {
                const float fu = __shfl_sync(0xffffffffu, f, u);
                float d[D];
#pragma unroll
                for (int j = 0; j < D; ++j) d[j] = 0.f;
                if (some >> u & 1) {
                    const float *src = a.o + slot(i0 + u) * HD + lane * D;
                    if constexpr (D == 4) {
                        const float4 v4 = *reinterpret_cast<const float4 *>(src);
                        d[0] = v4.x; d[1] = v4.y; d[2] = v4.z; d[3] = v4.w;
                    } else {
                        const float2 v2 = *reinterpret_cast<const float2 *>(src);
                        d[0] = v2.x; d[1] = v2.y;
                    }
                }
#pragma unroll
                for (int j = 0; j < D; ++j) o[j] = fmaf(fu, d[j], o[j]);
            }
            if (n < 32) break;
        }
        if (share > 1) {                                                 // the row's warps, in their order
            if (lane == 0) ml_of[warp] = make_float2(m, l);
#pragma unroll
            for (int j = 0; j < D; ++j) o_of[warp][lane * D + j] = o[j];
            __syncthreads();
            for (int u = 1; u < share && mine == 0; ++u) {
                const float2 v = ml_of[warp + u];
                const float mn = fmaxf(m, v.x), base = mn == -INFINITY ? 0.f : mn, f = exp2_approx(v.x - base), old = exp2_approx(m - base);
                m = mn;
                l = l * old + v.y * f;
#pragma unroll
                for (int j = 0; j < D; ++j) o[j] = o[j] * old + f * o_of[warp + u][lane * D + j];
            }
            __syncthreads();                                             // before the next rows
        }
        if (token < 0 || mine > 0) continue;
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        QT *d = static_cast<QT *>(a.out) + ((size_t)(p.row0 + token) * a.H + head) * HD + lane * D;
#pragma unroll
        for (int j = 0; j < D; j += 2) {
            if constexpr (sizeof(QT) == 2) *reinterpret_cast<uint32_t *>(d + j) = cvt_bf16x2(o[j] * inv, o[j + 1] * inv);
            else *reinterpret_cast<float2 *>(d + j) = make_float2(o[j] * inv, o[j + 1] * inv);
        }
    }
}

}  // namespace attn
}  // namespace knnssd
