// Attention of trees' rows by blocks: all rows over short contexts, and fp32 rows over fp32 pages of any.
//
// The mathematics is the rows kernel's (row_attention.cuh): up to 16 rows of a request that share a K/V head are an operand of m16n8k16 products, fp32 values are multiplied as three bf16 terms
// each, a row sees what its word says.  Here a block has the rows: they lie in shared memory as the products take them, its warps take 16 positions each in turn, K and V straight from the pages into
// the products' operands (any order of a head's dimensions serves a sum over them, and each is stored where it belongs), and put their parts together in shared memory.
// Fewer bits: the weights of bf16 rows are rounded to bf16 for the product with V (2^-8 relative at most), as the tensor kernel has them; sums are fp32.
//
// Short contexts: a block has an item whole, one launch does it all, without scratch.  Which it has follows from row_start alone: request b's blocks are those from row_start[b] / tb + b on, as many
// as row_start[b + 1] / tb - row_start[b] / tb + 1, which are enough for its rows whatever the requests before it have.  Bound by latency: rows, page, K and V, products, the parts.  Two requests of
// 13 rows, 4 fp32 heads of 64 over 96 positions 5.7 us, where the ways for long contexts take 17; one request of 12 rows, 32 bf16 heads over 300 positions 9.7 for 21.
//
// Else a block has an equal run of all items' positions, as in attention_items.cuh, and parts of items are put together by the merge.  fp32 pages: the rows kernel has room for one warp a
// scheduler beside their copies, here there are two: 8 requests of 25 rows, 40 heads over 1280 positions 191 us for 288 (2.2 TB/s; the terms of K and V and six products of each,
// 16 rows at a time), one of 8000 positions 81 for 117.  (bf16 pages stay with the rows kernel, whose copies run ahead: 94 us for 109.)
#pragma once

#include "attention_items.cuh"
#include "row_attention.cuh"

namespace knnssd {
namespace treerows {

using namespace attn;
using rowattn::mma;
using rowattn::terms_of;

constexpr int TP = 16, ROWS = 16;
// W: a short context's block has so many warps; 0: runs of positions, four warps.  Eight warps a processor either way.
template <int HD, typename QT, typename KT, int W> struct Lay {
    static constexpr int WARPS = W ? W : 4, NT = WARPS * 32, BLOCKS = 8 / WARPS;
    static constexpr int NQ = sizeof(QT) == 4 ? 3 : 1, NK = sizeof(KT) == 4 ? 3 : 1, KS = HD / 16;
    static constexpr int Q_BYTES = KS * NQ * 32 * 16, PART_BYTES = WARPS * ROWS * HD * (int)sizeof(float), ML_BYTES = WARPS * ROWS * (int)sizeof(float2);
    static constexpr int SMEM = Q_BYTES + PART_BYTES + ML_BYTES;
};

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

// Rows of an item: `live` of them, row r the query head h0 + r % heads of the request's new row row0 + r / heads, which stands at position seen0 + r / heads and sees nothing from kv on.
struct Tile { int b, row_first, row0, seen0, kv, kvh, h0, heads, live; };

// The rows' terms, dimension pair h of k-step s that lane t multiplies, as the products take them.
template <int HD, typename QT, typename KT, int W> __device__ __forceinline__ void put_rows(const Args &a, const Tile &m, uint4 *rows) {
    using L = Lay<HD, QT, KT, W>;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    auto dim_of = [&](int s, int h) { return sizeof(KT) == 2 ? 32 * (s >> 1) + 8 * t + 4 * (s & 1) + 2 * h : 16 * s + 4 * t + 2 * h; };
#pragma unroll
    for (int s0 = 0; s0 < L::KS; s0 += L::WARPS) {
        const int s = s0 + warp;
        if (s >= L::KS) break;
        uint32_t q[L::NQ][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * e + g;
            const bool on = r < m.live;
            const QT *p = static_cast<const QT *>(a.q) + (long long)(m.row0 + r / m.heads) * a.q_stride + (long long)(m.h0 + r % m.heads) * HD;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (sizeof(QT) == 2) q[0][2 * h + e] = on ? __ldg(reinterpret_cast<const uint32_t *>(p + dim_of(s, h))) : 0u;
                else {
                    uint32_t tm[L::NQ];
                    const float2 v = on ? __ldg(reinterpret_cast<const float2 *>(p + dim_of(s, h))) : make_float2(0.f, 0.f);
                    terms_of<L::NQ>(v.x, v.y, tm);
#pragma unroll
                    for (int i = 0; i < L::NQ; ++i) q[i][2 * h + e] = tm[i];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < L::NQ; ++i) rows[(s * L::NQ + i) * 32 + lane] = make_uint4(q[i][0], q[i][1], q[i][2], q[i][3]);
    }
}

// A warp's positions of [from, to): 16 of every 16 WARPS; its rows' sums to parts [row][HD] and ml [row].
template <int HD, typename QT, typename KT, int W>
__device__ __forceinline__ void attend(const Args &a, const Tile &m, int from, int to, const uint4 *rows, float *parts, float2 *ml) {
    using L = Lay<HD, QT, KT, W>;
    constexpr int NQ = L::NQ, NK = L::NK, NTILE = HD / 8, PER = 16 / (int)sizeof(KT), STEP = L::WARPS * TP;        // PER: values of 16 bytes
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    auto page_at = [&](int p) {
        const int idx = p >> a.page_shift, id = p < to && idx < a.max_pages ? __ldg(a.table + (size_t)m.b * a.max_pages + idx) : -1;
        return id < a.n_pages ? id : -1;
    };
    int page = page_at(from + warp * TP), last[2];
    unsigned long long word[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int r = 8 * e + g, tok = r / m.heads;
        last[e] = r < m.live ? m.seen0 + tok : -1;
        word[e] = r < m.live ? __ldg(a.seen + m.row0 + tok) : 0ull;
    }
    auto row_terms = [&](int s, int i, uint32_t (&q)[4]) {
        const uint4 v = rows[(s * NQ + i) * 32 + lane];
        q[0] = v.x; q[1] = v.y; q[2] = v.z; q[3] = v.w;
    };
    float o[NTILE][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NTILE; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    uint4 k4[2][HD / (4 * PER)];                                     // of position 8 i + g: 16 bytes at 4 PER c + PER t
    uint4 v4[4][HD / (8 * PER)];                                     // of positions 2t, 2t + 1, 2t + 8, 2t + 9: 16 bytes at 8 PER c + PER g
    // Of 16 positions from p on; what lies behind the last that counts, or has no page, is zero.
    auto base_of = [&](const void *pool, int p, int id) {
        return static_cast<const KT *>(pool) + ((((size_t)max(id, 0) * a.KV + m.kvh) << a.page_shift) + (p & ((1 << a.page_shift) - 1))) * HD;
    };
    auto load = [&](const KT *base, int there, int pos, int dim) {
        return pos < there ? __ldg(reinterpret_cast<const uint4 *>(base + pos * HD + dim)) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto load_k = [&](int p, int id) {
        const KT *base = base_of(a.k, p, id);
        const int there = id < 0 ? 0 : m.kv - p;
#pragma unroll
        for (int c = 0; c < HD / (4 * PER); ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) k4[i][c] = load(base, there, 8 * i + g, 4 * PER * c + PER * t);
    };
    auto load_v = [&](int p, int id) {
        const KT *base = base_of(a.v, p, id);
        const int there = id < 0 ? 0 : m.kv - p;
#pragma unroll
        for (int c = 0; c < HD / (8 * PER); ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) v4[i][c] = load(base, there, 2 * t + (i & 1) + 8 * (i >> 1), 8 * PER * c + PER * g);
    };
#pragma unroll 1
    for (int p = from + warp * TP; p < to; p += STEP) {
        const int id = page;
        page = page_at(p + STEP);
        load_k(p, id);
        if (NK == 1) load_v(p, id);
        float sp[2][3][4];                                           // sums of the scores: large terms of even and odd k-steps, small terms
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int u = 0; u < 3; ++u)
#pragma unroll
                for (int j = 0; j < 4; ++j) sp[i][u][j] = 0.f;
#pragma unroll
        for (int c = 0; c < HD / (4 * PER); ++c) {
            if constexpr (NK == 1) {
#pragma unroll
                for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        uint32_t q[4];
                        row_terms(2 * c + e, i, q);
#pragma unroll
                        for (int j = 0; j < 2; ++j) mma(sp[j][i ? 2 : e], q, e ? k4[j][c].z : k4[j][c].x, e ? k4[j][c].w : k4[j][c].y);
                    }
            } else {
                uint32_t b0[2][NK], b1[2][NK];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    terms_of<NK>(__uint_as_float(k4[j][c].x), __uint_as_float(k4[j][c].y), b0[j]);
                    terms_of<NK>(__uint_as_float(k4[j][c].z), __uint_as_float(k4[j][c].w), b1[j]);
                }
#pragma unroll
                for (int i = NQ - 1; i >= 0; --i) {
                    uint32_t q[4];
                    row_terms(c, i, q);
#pragma unroll
                    for (int u = NK - 1 - i; u >= 0; --u)
#pragma unroll
                        for (int j = 0; j < 2; ++j) mma(sp[j][i + u ? 2 : c & 1], q, b0[j][u], b1[j][u]);
                }
            }
        }
        if (NK != 1) load_v(p, id);
        uint32_t pf[NQ][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (sp[i >> 1][0][2 * e + (i & 1)] + sp[i >> 1][1][2 * e + (i & 1)] + sp[i >> 1][2][2 * e + (i & 1)]) * a.scale_log2;
            if (id < 0 || p + TP - 1 > m.seen0 - 64) {               // some row may not see all of these positions
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (id < 0 || !tree_sees(word[e], last[e] - p - 8 * (i >> 1) - 2 * t - (i & 1))) x[i] = -INFINITY;
            }
            float most = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            if (__any_sync(0xffffffffu, most > top[e])) {
                const float now = fmaxf(top[e], most), f = now == -INFINITY ? 1.f : exp2_approx(top[e] - now);
                top[e] = now;
                sum[e] *= f;
#pragma unroll
                for (int i = 0; i < NTILE; ++i) { o[i][2 * e] *= f; o[i][2 * e + 1] *= f; }
            }
            const float base = top[e] == -INFINITY ? 0.f : top[e];
#pragma unroll
            for (int i = 0; i < 4; ++i) { x[i] = exp2_approx(x[i] - base); sum[e] += x[i]; }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t tm[NQ];
                terms_of<NQ>(x[2 * h], x[2 * h + 1], tm);
#pragma unroll
                for (int i = 0; i < NQ; ++i) pf[i][2 * h + e] = tm[i];
            }
        }
        auto products = [&](int tile, const uint32_t (&b0)[2][NK], const uint32_t (&b1)[2][NK]) {            // tiles `tile` and `tile` + 1
            float d[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                for (int j = NK == 1 ? 0 : NK - 1 - i; j >= 0; --j)
#pragma unroll
                    for (int u = 0; u < 2; ++u) mma(d[u], pf[i], b0[u][j], b1[u][j]);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[tile + u][i] += d[u][i];
        };
        // tile PER c + i of the result: dimension 8 PER c + PER j + i in column j
#pragma unroll
        for (int c = 0; c < HD / (8 * PER); ++c) {
            const uint32_t w[4][4] = {{v4[0][c].x, v4[0][c].y, v4[0][c].z, v4[0][c].w}, {v4[1][c].x, v4[1][c].y, v4[1][c].z, v4[1][c].w},
                                      {v4[2][c].x, v4[2][c].y, v4[2][c].z, v4[2][c].w}, {v4[3][c].x, v4[3][c].y, v4[3][c].z, v4[3][c].w}};
            if constexpr (NK == 1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t b0[2][1] = {{low_halves(w[0][i], w[1][i])}, {high_halves(w[0][i], w[1][i])}};
                    const uint32_t b1[2][1] = {{low_halves(w[2][i], w[3][i])}, {high_halves(w[2][i], w[3][i])}};
                    products(PER * c + 2 * i, b0, b1);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint32_t b0[2][NK], b1[2][NK];
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        terms_of<NK>(__uint_as_float(w[0][i + z]), __uint_as_float(w[1][i + z]), b0[z]);
                        terms_of<NK>(__uint_as_float(w[2][i + z]), __uint_as_float(w[3][i + z]), b1[z]);
                    }
                    products(PER * c + i, b0, b1);
                }
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 1);
        sum[e] += __shfl_xor_sync(0xffffffffu, sum[e], 2);
        const int r = 8 * e + g;
        if (t == 0) ml[r] = make_float2(top[e], sum[e]);
#pragma unroll
        for (int i = 0; i < NTILE; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) parts[r * HD + 8 * PER * (i / PER) + PER * (2 * t + j) + i % PER] = o[i][2 * e + j];
    }
}

// The sums of `warps` warps together: the rows' results, or, of an item in parts, this block's part in `slot`.  HD / 4 threads a row.
template <int HD, typename QT, typename KT, int W>
__device__ __forceinline__ void together(const Args &a, const Tile &m, int from, int to, int warps, bool whole, size_t slot, const float *parts, const float2 *ml) {
    constexpr int LANES = HD / 4, NT = Lay<HD, QT, KT, W>::NT;
    const int tid = threadIdx.x, warp = tid >> 5;
    for (int r0 = 0; r0 < m.live; r0 += NT / LANES) {
        const int r = r0 + tid / LANES, d = tid % LANES * 4;
        bool odd = false;
        if (r < m.live) {
            float top = -INFINITY, sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < warps; ++w) top = fmaxf(top, ml[w * ROWS + r].x);
            const float base = top == -INFINITY ? 0.f : top;
            for (int w = 0; w < warps; ++w) {
                const float2 p = ml[w * ROWS + r];
                const float f = exp2_approx(p.x - base);
                const float4 x = *reinterpret_cast<const float4 *>(parts + (w * ROWS + r) * HD + d);
                sum = fmaf(p.y, f, sum);
                v[0] = fmaf(x.x, f, v[0]); v[1] = fmaf(x.y, f, v[1]); v[2] = fmaf(x.z, f, v[2]); v[3] = fmaf(x.w, f, v[3]);
            }
            const float inv = !whole ? 1.f : sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] *= inv; odd |= !isfinite(v[i]); }
            if (!whole) {
                *reinterpret_cast<float4 *>(a.o + (slot + r) * HD + d) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) a.ml[slot + r] = make_float2(top, sum);
            } else {
                QT *out = static_cast<QT *>(a.out) + ((size_t)(m.row0 + r / m.heads) * a.H + m.h0 + r % m.heads) * HD + d;
                if constexpr (sizeof(QT) == 2) *reinterpret_cast<uint2 *>(out) = make_uint2(cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]));
                else *reinterpret_cast<float4 *>(out) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
        // A row may be so only by the products: 0 times a V that is not finite and that it does not see, an infinity in three terms.  By the definition then.
        unsigned odds = __ballot_sync(0xffffffffu, odd);
        __syncwarp();                                                // behind the stores
        for (int i = 0; odds != 0 && i < 32 / LANES; ++i, odds = LANES < 32 ? odds >> (LANES & 31) : 0u) {
            const int row = r0 + warp * (32 / LANES) + i, last = m.seen0 + row / m.heads;
            if (odds & (LANES < 32 ? (1u << (LANES & 31)) - 1 : 0xffffffffu))
                row_by_definition<HD, QT, KT, true, true>(a, Row{m.b, m.row_first, m.row0 + row / m.heads, m.h0 + row % m.heads, from, min(last + 1, to), whole, slot + row, last});
        }
    }
}

template <int HD, typename QT, typename KT, int W>
__global__ void __launch_bounds__(Lay<HD, QT, KT, W>::NT, Lay<HD, QT, KT, W>::BLOCKS) tree_rows_kernel(const __grid_constant__ Args a) {
    using L = Lay<HD, QT, KT, W>;
    constexpr int NT = L::NT;
    extern __shared__ __align__(16) unsigned char smem[];
    uint4 *rows = reinterpret_cast<uint4 *>(smem);                   // [k-step][term][lane]
    float *parts = reinterpret_cast<float *>(smem + L::Q_BYTES);     // [warp][row][HD]
    float2 *ml = reinterpret_cast<float2 *>(smem + L::Q_BYTES + L::PART_BYTES);              // [warp][row]
    chain_wait();
    const int tid = threadIdx.x, warp = tid >> 5, G = a.H / a.KV;
    auto item = [&](const Tile &m, int from, int to, bool whole, size_t slot) {
        const int warps = min(L::WARPS, (to - from + TP - 1) / TP);
        put_rows<HD, QT, KT, W>(a, m, rows);
        __syncthreads();
        if (warp < warps) attend<HD, QT, KT, W>(a, m, from, to, rows, parts + warp * ROWS * HD, ml + warp * ROWS);
        __syncthreads();
        together<HD, QT, KT, W>(a, m, from, to, warps, whole, slot, parts, ml);
    };
    if constexpr (W > 0) {
        const int vh = blockIdx.x, y = blockIdx.y;
        clear_others<QT>(a, HD, (y * gridDim.x + vh) * NT + tid, gridDim.x * gridDim.y * NT);
        int upto = 0;                                                // requests whose blocks begin at this one or before
        for (int b0 = 0; b0 < a.B; b0 += NT) {
            const int b = b0 + tid;
            upto += __syncthreads_count(b < a.B && min(max(a.row_start[b], 0), a.R) / a.tb + b <= y);
        }
        const int b = max(upto - 1, 0), first = min(max(a.row_start[b], 0), a.R), n = max(min(max(a.row_start[b + 1], 0), a.R) - first, 0);
        const int tile = y - (first / a.tb + b);
        if (tile < 0 || tile * a.tb >= n) return;
        const int held = (int)min((long long)max(a.lens[b], 0), (long long)a.max_pages << a.page_shift);
        const int tokens = min(a.tb, n - tile * a.tb), seen0 = held + tile * a.tb, kvh = vh / a.subs, h0 = kvh * G + (vh % a.subs) * a.gs, heads = min(a.gs, (kvh + 1) * G - h0);
        item(Tile{b, first, first + tile * a.tb, seen0, seen0 + tokens, kvh, h0, heads, tokens * heads}, 0, seen0 + tokens, true, 0);
    } else {
        __shared__ Costs<NT> costs;
        sum_costs<false>(a, costs);
        clear_others<QT>(a, HD, blockIdx.x * NT + tid, gridDim.x * NT);
        const long long total = costs.pfx[NT];
        const int workers = workers_of(a, total), w = blockIdx.x;
        const long long x0 = w < workers ? run_start(total, w, workers) : 0, x1 = w < workers ? run_start(total, w + 1, workers) : 0;
        if (x0 >= x1) {
            if (tid == 0) { a.parts[w].first = 0; a.parts[w].start = -1; }
            return;
        }
        Item<false> it = item_at<false>(a, costs, x0);
        if (tid == 0) note_part<TP>(a, it, w, workers, total, x0, x1);
        for (bool more = true; more; more = it.next(a) && it.start < x1) {
            const int from = cut<TP>(it, x0), to = cut<TP>(it, x1);
            if (from >= to) continue;
            const int tokens = it.tokens(), kvh = it.vh / a.subs, h0 = kvh * G + (it.vh % a.subs) * a.gs, heads = min(a.gs, (kvh + 1) * G - h0);
            item(Tile{it.b, it.r.row0, it.r.row0 + it.rb * it.r.tb, it.kv - tokens, it.kv, kvh, h0, heads, tokens * heads}, from, to, from == 0 && to == it.kv,
                 ((size_t)w * SLOTS + (from > 0 ? 0 : 1)) * ROWS);
            __syncthreads();                                         // the next item's rows and sums come where these were
        }
    }
}

}  // namespace treerows
}  // namespace knnssd
