// Attention of the new rows of many requests over their positions, for any of the library's types.
//
// Row i of request b stands at position held_b + i and looks at the positions 0 .. held_b + i:
//   s_j = scale q . k_j,   m = max_j s_j,   l = sum_j exp(s_j - m),   o = sum_j exp(s_j - m) v_j / l
// in one pass over the positions with m, l and o running: when m grows, l and o are multiplied by exp(m_old - m_new).  A row that
// sees nothing gives zeros.
//
// An item is (request, block of new rows, K/V head): the rows of a block times the query heads that share the head are up to
// 16 MB rows of one operand (m16n8k16 products), so K and V are read once for all of them.  The positions of all items, in order, are
// cut into equal runs, one per warp of the launch: whatever the lengths, every warp reads the same amount.  A warp streams its run
// through a ring of its own in shared memory (16-byte asynchronous copies, 16 positions a stage) and runs on from item to item without
// meeting another warp.  An item that several warps have parts of is put together by merge_kernel from the parts' (m, l, o).
//
// Types: fp32 values are multiplied as three bf16 terms each (24 bits), the products with terms i + j < 3 in fp32 sums: what an fp32 sum
// over the rounded inputs gives.  bf16 queries are answered in bf16, and their p is rounded to bf16 once (relative error 2^-8 of each
// term at most; in a sum of many it comes to less than the rounding of the result).
#pragma once

#include "attention_items.cuh"

namespace knnssd {
namespace rowattn {

using namespace attn;

constexpr int TP = 16;                    // positions of a stage; pages and items begin at multiples of it

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there) {
    const int n = there ? 16 : 0;                                    // 0: the 16 bytes become zeros
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t p) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(p));
    return v;
}
__device__ __forceinline__ void ldsm4t(uint32_t p, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(p));
}
// (v0, v1) as N bf16 pairs whose sums they are (N = 1: rounded to nearest).
template <int N> __device__ __forceinline__ void terms_of(float v0, float v1, uint32_t (&t)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        t[i] = cvt_bf16x2(v0, v1);
        if (i + 1 < N) { v0 -= __uint_as_float(t[i] << 16); v1 -= __uint_as_float(t[i] & 0xffff0000u); }
    }
}

template <int HD, typename KT> struct Ring {
    static constexpr int ROW = HD * (int)sizeof(KT), CHUNKS = ROW / 16;      // bytes and 16-byte pieces of a position
    static constexpr int STAGE = 2 * TP * ROW;                               // K, then V
    static constexpr int STAGES = STAGE >= 16384 ? 3 : STAGE >= 8192 ? 3 : 6;
    static constexpr int WARPS = STAGE >= 16384 ? 4 : 8;
    static constexpr int SMEM = WARPS * STAGES * STAGE;
    // Pieces of a position are kept permuted, so that what eight lanes fetch together lies in different banks: K is read by lanes of two
    // positions x four pieces; V as 8 x 8 matrices of eight positions (bf16), or by lanes of four positions x two pieces (fp32).
    __device__ static __forceinline__ int kswz(int p, int c) { return c ^ ((p & 1) << 2); }
    __device__ static __forceinline__ int vswz(int p, int c) { return sizeof(KT) == 2 ? c ^ (p & 7) : c ^ (((p >> 1) & 3) << 1); }
};

template <int HD, typename QT, typename KT, bool PAGED, int MB>
__global__ void __launch_bounds__(Ring<HD, KT>::WARPS * 32, 1) rows_kernel(const Args a) {
    using Rg = Ring<HD, KT>;
    constexpr int NT = Rg::WARPS * 32, NQ = sizeof(QT) == 4 ? 3 : 1, NK = sizeof(KT) == 4 ? 3 : 1, KS = HD / 16, NTILE = HD / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Costs<NT> costs;
    __shared__ int hole_of[Rg::WARPS][Rg::STAGES];
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    sum_costs<false>(a, costs);
    if (a.clear) clear_tail<QT>(a, HD, blockIdx.x * NT + threadIdx.x, gridDim.x * NT);
    const long long total = costs.pfx[NT];
    const int W = workers_of(a, total, gridDim.x * Rg::WARPS);
    // neighbouring runs go to different SMs: a short launch spreads over the chip
    const int w = warp * gridDim.x + blockIdx.x;
    const long long x0 = w < W ? run_start(total, w, W) : 0, x1 = w < W ? run_start(total, w + 1, W) : 0;
    if (x0 >= x1) {
        if (lane == 0) { a.parts[w].first = 0; a.parts[w].start = -1; }
        return;
    }
    Item<false> in = item_at<false>(a, costs, x0);                   // the item whose positions are being fetched
    Item<false> it = in;                                             // the item at work
    if (lane == 0) note_part<TP>(a, it, w, W, total, x0, x1);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * Rg::STAGES * Rg::STAGE;

    // ---- fetching -------------------------------------------------------------------------------------------------
    int at = cut<TP>(in, x0), until = cut<TP>(in, x1);
    bool more = true;
    int pid = 0;                                                     // the page of the next 16 positions
    auto settle = [&]() {                                            // on to the next positions that are this warp's
        while (more && at >= until) {
            more = in.next(a) && in.start < x1;
            if (more) { at = 0; until = cut<TP>(in, x1); }
        }
        if (PAGED && more) {
            const int idx = at >> a.page_shift;
            pid = idx < a.max_pages ? __ldg(a.table + (size_t)in.b * a.max_pages + idx) : -1;
        }
    };
    settle();
    int stage_in = 0;
    auto fetch = [&]() {
        if (more) {
            const uint32_t dst = ring + stage_in * Rg::STAGE;
            const int kvh = in.vh / a.subs;
            const bool there = !PAGED || (pid >= 0 && pid < a.n_pages);
            const unsigned char *kp, *vp;
            size_t kstep, vstep;
            if (PAGED) {
                const size_t e = ((((size_t)(there ? pid : 0) * a.KV + kvh) << a.page_shift) + (at & ((1 << a.page_shift) - 1))) * Rg::ROW;
                kp = static_cast<const unsigned char *>(a.k) + e; vp = static_cast<const unsigned char *>(a.v) + e;
                kstep = vstep = Rg::ROW;
            } else {
                kp = static_cast<const unsigned char *>(a.k) + ((size_t)(in.r.row0 + at) * a.k_stride + (size_t)kvh * HD) * sizeof(KT);
                vp = static_cast<const unsigned char *>(a.v) + ((size_t)(in.r.row0 + at) * a.v_stride + (size_t)kvh * HD) * sizeof(KT);
                kstep = a.k_stride * sizeof(KT); vstep = a.v_stride * sizeof(KT);
            }
#pragma unroll
            for (int i = lane; i < TP * Rg::CHUNKS; i += 32) {
                const int p = i / Rg::CHUNKS, c = i % Rg::CHUNKS;
                const bool ok = there && at + p < in.kv;             // what no row of the block sees is not read: zeros
                copy16(dst + p * Rg::ROW + Rg::kswz(p, c) * 16, ok ? kp + p * kstep + c * 16 : static_cast<const unsigned char *>(a.k), ok);
                copy16(dst + TP * Rg::ROW + p * Rg::ROW + Rg::vswz(p, c) * 16, ok ? vp + p * vstep + c * 16 : static_cast<const unsigned char *>(a.v), ok);
            }
            if (PAGED && lane == 0) hole_of[warp][stage_in] = !there;
            at += TP;
            settle();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage_in == Rg::STAGES) stage_in = 0;
    };
    for (int i = 0; i < Rg::STAGES - 1; ++i) fetch();

    // ---- working ----------------------------------------------------------------------------------------------------
    int stage = 0;
    bool any = true;
    while (any) {
        const int from = cut<TP>(it, x0), to = cut<TP>(it, x1);
        if (from < to) {
            const int row0 = it.r.row0 + it.rb * it.r.tb, tokens = it.tokens(), kvh = it.vh / a.subs, G = a.H / a.KV;
            const int h0 = kvh * G + (it.vh % a.subs) * a.gs, heads = min(a.gs, (kvh + 1) * G - h0), live = tokens * heads;
            const int seen0 = it.kv - tokens;                        // position of the block's first row
            // dimension pair h of k-step s that lane t multiplies: any order serves a dot product, this one makes 16-byte reads of K
            auto dim_of = [&](int s, int h) { return sizeof(KT) == 2 ? 32 * (s >> 1) + 8 * t + 4 * (s & 1) + 2 * h : 16 * s + 4 * t + 2 * h; };
            uint32_t qf[MB][KS][NQ][4];
            int last[MB][2];                                         // the last position a row sees; -1: no such row
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 16 * mb + 8 * e + g, tok = r / heads;
                    const bool on = r < live;
                    last[mb][e] = on ? seen0 + tok : -1;
                    const QT *qp = static_cast<const QT *>(a.q) + (long long)(row0 + tok) * a.q_stride + (long long)(h0 + r % heads) * HD;
#pragma unroll
                    for (int s = 0; s < KS; ++s)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t tm[NQ];
                            if (NQ == 1) {
                                tm[0] = on ? __ldg(reinterpret_cast<const uint32_t *>(qp + dim_of(s, h))) : 0u;
                            } else {
                                const float2 v = on ? __ldg(reinterpret_cast<const float2 *>(qp + dim_of(s, h))) : make_float2(0.f, 0.f);
                                terms_of<NQ>(v.x, v.y, tm);
                            }
#pragma unroll
                            for (int i = 0; i < NQ; ++i) qf[mb][s][i][2 * h + e] = tm[i];
                        }
                }
            float o[MB][NTILE][4], m[MB][2], l[MB][2];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
                for (int n = 0; n < NTILE; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[mb][n][i] = 0.f;
#pragma unroll
                for (int e = 0; e < 2; ++e) { m[mb][e] = -INFINITY; l[mb][e] = 0.f; }
            }
            for (int p = from; p < to; p += TP) {
                asm volatile("cp.async.wait_group %0;" ::"n"(Rg::STAGES - 2) : "memory");
                __syncwarp();
                const bool hole = PAGED && hole_of[warp][stage] != 0;
                const uint32_t kb = ring + stage * Rg::STAGE, vb = kb + TP * Rg::ROW;
                fetch();                                             // into the stage that the positions before have left
                // The tensor cores add to a sum by truncation.  Where fp32 is answered a sum gets few such additions: the small terms have a sum of
                // their own, and the 16 positions' share of o is added to it by an ordinary addition.
                constexpr int NS = NQ == 1 ? 2 : 3;                  // sums of the scores, all independent chains
                float sp[MB][2][NS][4];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int u = 0; u < NS; ++u)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sp[mb][n][u][i] = 0.f;
#pragma unroll
                for (int c = 0; c < HD / 32; ++c)
#pragma unroll
                    for (int n = 0; n < 2; ++n) {
                        const int pos = 8 * n + g;
                        if constexpr (NK == 1) {
                            const uint4 w = lds16(kb + pos * Rg::ROW + Rg::kswz(pos, 4 * c + t) * 16);
#pragma unroll
                            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                for (int i = NQ - 1; i >= 0; --i) {
                                    mma(sp[mb][n][i ? 2 : 0], qf[mb][2 * c][i], w.x, w.y);
                                    mma(sp[mb][n][i ? 2 : 1], qf[mb][2 * c + 1][i], w.z, w.w);
                                }
                        } else {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint4 w = lds16(kb + pos * Rg::ROW + Rg::kswz(pos, 8 * c + 4 * e + t) * 16);
                                uint32_t b0[NK], b1[NK];
                                terms_of<NK>(__uint_as_float(w.x), __uint_as_float(w.y), b0);
                                terms_of<NK>(__uint_as_float(w.z), __uint_as_float(w.w), b1);
#pragma unroll
                                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                    for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                                        for (int j = NK - 1 - i; j >= 0; --j) mma(sp[mb][n][i + j ? 2 : e], qf[mb][2 * c + e][i], b0[j], b1[j]);
                            }
                        }
                    }
                float s[MB][2][4];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int n = 0; n < 2; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[mb][n][i] = sp[mb][n][0][i] + sp[mb][n][1][i] + (NS == 3 ? sp[mb][n][NS - 1][i] : 0.f);
                const bool ragged = hole || p + TP - 1 > seen0;      // some row does not see all of these positions
                uint32_t pf[MB][NQ][4];
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x[i] = s[mb][i >> 1][2 * e + (i & 1)] * a.scale_log2;
                            if (ragged && (hole || p + 8 * (i >> 1) + 2 * t + (i & 1) > last[mb][e])) x[i] = -INFINITY;
                        }
                        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        if (__any_sync(0xffffffffu, top > m[mb][e])) {
                            const float mn = fmaxf(m[mb][e], top), f = mn == -INFINITY ? 1.f : exp2_approx(m[mb][e] - mn);
                            m[mb][e] = mn;
                            l[mb][e] *= f;
#pragma unroll
                            for (int n = 0; n < NTILE; ++n) { o[mb][n][2 * e] *= f; o[mb][n][2 * e + 1] *= f; }
                        }
                        const float base = m[mb][e] == -INFINITY ? 0.f : m[mb][e];
#pragma unroll
                        for (int i = 0; i < 4; ++i) { x[i] = exp2_approx(x[i] - base); l[mb][e] += x[i]; }
                        uint32_t tm[NQ];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            terms_of<NQ>(x[2 * h], x[2 * h + 1], tm);
#pragma unroll
                            for (int i = 0; i < NQ; ++i) pf[mb][i][2 * h + e] = tm[i];
                        }
                    }
                // Where the positions are the block's own, a row's p is 0 for those behind it - and 0 times a V that is not finite is not: rows
                // that see such a position must not disturb the ones that do not.
                bool odd = false;
                auto products = [&](int n, const uint32_t (&b0)[NK], const uint32_t (&b1)[NK]) {
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        if constexpr (NQ == 1) {
                            mma(o[mb][n], pf[mb][0], b0[0], b1[0]);
                        } else {
                            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                                for (int j = NK == 1 ? 0 : NK - 1 - i; j >= 0; --j) mma(d, pf[mb][i], b0[j], b1[j]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[mb][n][i] += d[i];
                        }
                    }
                };
                // the same, position by position, into the rows that see it
                auto products_apart = [&](int n, const uint32_t (&b0)[NK], const uint32_t (&b1)[NK]) {
                    for (int q = 0; q < TP && p + q < it.kv; ++q) {
                        const int reg = q >> 3, half = q & 1;
                        const bool mine = ((q & 7) >> 1) == t;
                        uint32_t c0[NK], c1[NK];
#pragma unroll
                        for (int j = 0; j < NK; ++j) {
                            const uint32_t keep = half ? 0xffff0000u : 0x0000ffffu;
                            c0[j] = mine && reg == 0 ? b0[j] & keep : 0u;
                            c1[j] = mine && reg == 1 ? b1[j] & keep : 0u;
                        }
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) {
                            float d[4] = {o[mb][n][0], o[mb][n][1], o[mb][n][2], o[mb][n][3]};
#pragma unroll
                            for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                                for (int j = NK == 1 ? 0 : NK - 1 - i; j >= 0; --j) mma(d, pf[mb][i], c0[j], c1[j]);
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (p + q <= last[mb][e]) { o[mb][n][2 * e] = d[2 * e]; o[mb][n][2 * e + 1] = d[2 * e + 1]; }
                        }
                    }
                };
                if (ragged && tokens > 1) {
                    bool bad = false;
                    for (int i = lane; i < TP * Rg::CHUNKS; i += 32) {
                        const uint4 w = lds16(vb + i * 16);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            bad |= (u[j] & 0x7f800000u) == 0x7f800000u;
                            if (NK == 1) bad |= (u[j] & 0x7f80u) == 0x7f80u;
                        }
                    }
                    odd = __any_sync(0xffffffffu, bad);
                }
                if constexpr (NK == 1) {
#pragma unroll
                    for (int n2 = 0; n2 < NTILE / 2; ++n2) {         // matrices: positions 0..7 and 8..15 of 8 dimensions, then of the next 8
                        uint32_t r[4];
                        const int pos = (lane & 7) + ((lane >> 3) & 1) * 8;
                        ldsm4t(vb + pos * Rg::ROW + Rg::vswz(pos, 2 * n2 + (lane >> 4)) * 16, r);
                        const uint32_t x0[1] = {r[0]}, x1[1] = {r[1]}, y0[1] = {r[2]}, y1[1] = {r[3]};
                        if (!odd) { products(2 * n2, x0, x1); products(2 * n2 + 1, y0, y1); }
                        else { products_apart(2 * n2, x0, x1); products_apart(2 * n2 + 1, y0, y1); }
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) {              // four dimensions 32 c + 4 g + i of positions 2t, 2t + 1, 2t + 8, 2t + 9
                        uint4 w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int pos = 2 * t + (i & 1) + 8 * (i >> 1);
                            w[i] = lds16(vb + pos * Rg::ROW + Rg::vswz(pos, 8 * c + g) * 16);
                        }
                        const uint32_t u[4][4] = {{w[0].x, w[0].y, w[0].z, w[0].w}, {w[1].x, w[1].y, w[1].z, w[1].w},
                                                  {w[2].x, w[2].y, w[2].z, w[2].w}, {w[3].x, w[3].y, w[3].z, w[3].w}};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t b0[NK], b1[NK];
                            terms_of<NK>(__uint_as_float(u[0][i]), __uint_as_float(u[1][i]), b0);
                            terms_of<NK>(__uint_as_float(u[2][i]), __uint_as_float(u[3][i]), b1);
                            if (!odd) products(4 * c + i, b0, b1);
                            else products_apart(4 * c + i, b0, b1);
                        }
                    }
                }
                if (++stage == Rg::STAGES) stage = 0;
            }
            // ---- the rows' ends ----------------------------------------------------------------------------------------
            // o[mb][n][2 e + i] is dimension col(n, i) of row 16 mb + 8 e + g
            auto col = [&](int n, int i) { return NK == 1 ? 8 * n + 2 * t + i : 32 * (n >> 2) + 4 * (2 * t + i) + (n & 3); };
            const bool whole = from == 0 && to == it.kv;
            const size_t slot = ((size_t)w * SLOTS + (from > 0 ? 0 : 1)) * (16 * MB);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float ls = l[mb][e];
                    ls += __shfl_xor_sync(0xffffffffu, ls, 1);
                    ls += __shfl_xor_sync(0xffffffffu, ls, 2);
                    const int r = 16 * mb + 8 * e + g;
                    if (r >= live) continue;
                    if (whole) {
                        const float inv = ls == 0.f ? 0.f : 1.0f / ls;
                        QT *d = static_cast<QT *>(a.out) + ((size_t)(row0 + r / heads) * a.H + h0 + r % heads) * HD;
#pragma unroll
                        for (int n = 0; n < NTILE; ++n) {
                            const float v0 = o[mb][n][2 * e] * inv, v1 = o[mb][n][2 * e + 1] * inv;
                            if constexpr (NQ == 1) {
                                *reinterpret_cast<uint32_t *>(d + col(n, 0)) = cvt_bf16x2(v0, v1);
                            } else if constexpr (NK == 1) {
                                *reinterpret_cast<float2 *>(d + col(n, 0)) = make_float2(v0, v1);
                            } else {
                                d[col(n, 0)] = v0; d[col(n, 1)] = v1;
                            }
                        }
                    } else {
                        if (t == 0) a.ml[slot + r] = make_float2(m[mb][e], ls);
                        float *d = a.o + (slot + r) * HD;
#pragma unroll
                        for (int n = 0; n < NTILE; ++n)
#pragma unroll
                            for (int i = 0; i < 2; ++i) d[col(n, i)] = o[mb][n][2 * e + i];
                    }
                }
        }
        any = it.next(a) && it.start < x1;
    }
}

}  // namespace rowattn
}  // namespace knnssd
