// Attention of fp32 rows over pages or over packed prompts.
//
// Row i of request b stands at position held_b + i and looks at the positions 0 .. held_b + i:
//   s_j = scale q . k_j,   m = max_j s_j,   l = sum_j exp(s_j - m),   o = sum_j exp(s_j - m) v_j / l
// in one pass over the positions with m, l and o running: when m grows, l and o are multiplied by exp(m_old - m_new).  A row that
// sees nothing gives zeros.
//
// An item's rows (new rows times the query heads that share the K/V head) are up to 16 rows of one operand (m16n8k16 products), so K and V are
// read once for all of them.  A worker is a warp: it streams its run of the positions through a ring of its own in shared memory (16-byte
// asynchronous copies, 16 positions a stage) and runs on from item to item without meeting another warp.
//
// fp32 values are multiplied as three bf16 terms each (24 bits), the products with terms i + j < 3: what an fp32 sum over the rounded inputs
// gives.  The tensor cores add to a sum by truncation; a sum gets few such additions: the small terms of the scores have a sum of their own, and
// the 16 positions' share of o is added to it by an ordinary addition.  Infinities have no terms: a row whose sums are not finite is done again by the
// definition, a row at a time (9 prompts of 3001 fp32 tokens in all with an infinite V every 64 rows 0.53 ms for 0.04).
//
// Measured: 8 requests of 5 rows and 40 heads over 1280 bf16 positions 55 us, 3.8 TB/s (60 % of a copy's): bound by what a warp issues - the terms, the
// products and the exponentials of 16 positions take the two warps of a scheduler about as long as a copy of them does - and by the ends of items.
// One request of 31 009 positions 40 us, 9 prompts of 3001 fp32 tokens in all 38.
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
// (v0, v1) as N bf16 pairs whose sums they are.
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
    static constexpr int STAGES = STAGE >= 8192 ? 3 : 6;                     // as many bytes on their way as the shared memory holds: 192 KB an SM
    static constexpr int WARPS = STAGE >= 16384 ? 4 : 8;
    static constexpr int SMEM = WARPS * STAGES * STAGE;
    // Pieces of a position are kept permuted, so that what eight lanes fetch together lies in different banks: K is read by lanes of two
    // positions x four pieces; V as 8 x 8 matrices of eight positions (bf16), or by lanes of four positions x two pieces (fp32).
    __device__ static __forceinline__ int kswz(int p, int c) { return c ^ ((p & 1) << 2); }
    __device__ static __forceinline__ int vswz(int p, int c) { return sizeof(KT) == 2 ? c ^ (p & 7) : c ^ (((p >> 1) & 3) << 1); }
};

template <int HD, typename KT, bool PAGED>
__global__ void __launch_bounds__(Ring<HD, KT>::WARPS * 32, 1) rows_kernel(const __grid_constant__ Args a) {
    using Rg = Ring<HD, KT>;
    constexpr int NT = Rg::WARPS * 32, NQ = 3, NK = sizeof(KT) == 4 ? 3 : 1, KS = HD / 16, NTILE = HD / 8;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ Costs<NT> costs;
    __shared__ int hole_of[Rg::WARPS][Rg::STAGES];
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    sum_costs<false>(a, costs);
    clear_others<float>(a, HD, blockIdx.x * NT + threadIdx.x, gridDim.x * NT);
    const long long total = costs.pfx[NT];
    const int W = workers_of(a, total);
    // neighbouring runs go to different SMs: a short launch spreads over the chip
    const int w = warp * gridDim.x + blockIdx.x;
    const long long x0 = w < W ? run_start(total, w, W) : 0, x1 = w < W ? run_start(total, w + 1, W) : 0;
    if (x0 >= x1) {
        if (lane == 0 && w < a.most) { a.parts[w].first = 0; a.parts[w].start = -1; }
        return;
    }
    Item<false> in = item_at<false>(a, costs, x0);                   // the item whose positions are being fetched
    Item<false> it = in;                                             // the item at work
    if (lane == 0) note_part<TP>(a, it, w, W, total, x0, x1);
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * Rg::STAGES * Rg::STAGE;

    // ---- fetching -------------------------------------------------------------------------------------------------
    // Copy i of the warp brings 16 bytes a lane: piece `chunk` of position i PER + sub (or of the position's second half, where a position has
    // more than 32 pieces: none here).
    constexpr int PER = 32 / Rg::CHUNKS > 0 ? 32 / Rg::CHUNKS : 1, N = TP * Rg::CHUNKS / 32;
    const int chunk = lane % Rg::CHUNKS, sub = lane / Rg::CHUNKS;
    int at = cut<TP>(in, x0), until = cut<TP>(in, x1);
    bool more = true;
    int pid = 0;                                                     // the page of the next 16 positions
    const unsigned char *kp = nullptr, *vp = nullptr;                // packed: this lane's piece of the item's first position
    auto settle = [&](bool fresh) {                                  // on to the next positions that are this warp's
        while (more && at >= until) {
            more = in.next(a) && in.start < x1;
            if (more) { at = 0; until = cut<TP>(in, x1); fresh = true; }
        }
        if (!more) return;
        if (PAGED) {
            const int idx = at >> a.page_shift;
            pid = idx < a.max_pages ? __ldg(a.table + (size_t)in.b * a.max_pages + idx) : -1;
        } else if (fresh) {
            const size_t head = (size_t)(in.vh / a.subs) * Rg::ROW + chunk * 16;
            kp = static_cast<const unsigned char *>(a.k) + (size_t)(in.r.row0 + sub) * a.k_stride * sizeof(KT) + head;
            vp = static_cast<const unsigned char *>(a.v) + (size_t)(in.r.row0 + sub) * a.v_stride * sizeof(KT) + head;
        }
    };
    settle(true);
    int stage_in = 0;
    uint32_t kat[N], vat[N];                                         // where copy i's pieces go in a stage
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = i * PER + sub;
        kat[i] = p * Rg::ROW + Rg::kswz(p, chunk) * 16;
        vat[i] = TP * Rg::ROW + p * Rg::ROW + Rg::vswz(p, chunk) * 16;
    }
    auto fetch = [&]() {
        if (more) {
            const uint32_t dst = ring + stage_in * Rg::STAGE;
            const bool there = !PAGED || (pid >= 0 && pid < a.n_pages);
            const unsigned char *ks, *vs;
            size_t kstep, vstep;
            if (PAGED) {
                const size_t e = ((((size_t)(there ? pid : 0) * a.KV + in.vh / a.subs) << a.page_shift) + (at & ((1 << a.page_shift) - 1)) + sub) * Rg::ROW + chunk * 16;
                ks = static_cast<const unsigned char *>(a.k) + e; vs = static_cast<const unsigned char *>(a.v) + e;
                kstep = vstep = PER * Rg::ROW;
            } else {
                kstep = (size_t)a.k_stride * sizeof(KT); vstep = (size_t)a.v_stride * sizeof(KT);
                ks = kp + at * kstep; vs = vp + at * vstep;
                kstep *= PER; vstep *= PER;
            }
            const int seen = there ? in.kv - at - sub : 0;           // positions from this lane's first on that the block sees: the others become zeros
            if (__all_sync(0xffffffffu, seen >= TP)) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    copy16(dst + kat[i], ks, true);
                    copy16(dst + vat[i], vs, true);
                    ks += kstep; vs += vstep;
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const bool ok = i * PER < seen;
                    copy16(dst + kat[i], ok ? ks : static_cast<const unsigned char *>(a.k), ok);
                    copy16(dst + vat[i], ok ? vs : static_cast<const unsigned char *>(a.v), ok);
                    ks += kstep; vs += vstep;
                }
            }
            if (PAGED && lane == 0) hole_of[warp][stage_in] = !there;
            at += TP;
            settle(false);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage_in == Rg::STAGES) stage_in = 0;
    };
#pragma unroll 1
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
            uint32_t qf[KS][NQ][4];
            int last[2];                                             // the last position a row sees; -1: no such row
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * e + g, tok = r / heads;
                const bool on = r < live;
                last[e] = on ? seen0 + tok : -1;
                const float *qp = static_cast<const float *>(a.q) + (long long)(row0 + tok) * a.q_stride + (long long)(h0 + r % heads) * HD;
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t tm[NQ];
                        const float2 v = on ? __ldg(reinterpret_cast<const float2 *>(qp + dim_of(s, h))) : make_float2(0.f, 0.f);
                        terms_of<NQ>(v.x, v.y, tm);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) qf[s][i][2 * h + e] = tm[i];
                    }
            }
            float o[NTILE][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int n = 0; n < NTILE; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
#pragma unroll 1
            for (int p = from; p < to; p += TP) {
                asm volatile("cp.async.wait_group %0;" ::"n"(Rg::STAGES - 2) : "memory");
                __syncwarp();
                const bool hole = PAGED && hole_of[warp][stage] != 0;
                const uint32_t kb = ring + stage * Rg::STAGE, vb = kb + TP * Rg::ROW;
                fetch();                                             // into the stage that the positions before have left
                float sp[2][3][4];                                   // sums of the scores: large terms of even and odd k-steps, small terms
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int u = 0; u < 3; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sp[n][u][i] = 0.f;
#pragma unroll
                for (int c = 0; c < HD / 32; ++c) {                  // products that follow one another go to different sums
                    if constexpr (NK == 1) {
                        uint4 k4[2];
#pragma unroll
                        for (int n = 0; n < 2; ++n) k4[n] = lds16(kb + (8 * n + g) * Rg::ROW + Rg::kswz(g, 4 * c + t) * 16);
#pragma unroll
                        for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
#pragma unroll
                                for (int n = 0; n < 2; ++n) mma(sp[n][i ? 2 : e], qf[2 * c + e][i], e ? k4[n].z : k4[n].x, e ? k4[n].w : k4[n].y);
                    } else {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            uint32_t b0[2][NK], b1[2][NK];
#pragma unroll
                            for (int n = 0; n < 2; ++n) {
                                const uint4 k4 = lds16(kb + (8 * n + g) * Rg::ROW + Rg::kswz(g, 8 * c + 4 * e + t) * 16);
                                terms_of<NK>(__uint_as_float(k4.x), __uint_as_float(k4.y), b0[n]);
                                terms_of<NK>(__uint_as_float(k4.z), __uint_as_float(k4.w), b1[n]);
                            }
#pragma unroll
                            for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                                for (int j = NK - 1 - i; j >= 0; --j)
#pragma unroll
                                    for (int n = 0; n < 2; ++n) mma(sp[n][i + j ? 2 : e], qf[2 * c + e][i], b0[n][j], b1[n][j]);
                        }
                    }
                }
                const bool ragged = hole || p + TP - 1 > seen0;      // some row does not see all of these positions
                uint32_t pf[NQ][4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[i] = (sp[i >> 1][0][2 * e + (i & 1)] + sp[i >> 1][1][2 * e + (i & 1)] + sp[i >> 1][2][2 * e + (i & 1)]) * a.scale_log2;
                    if (ragged) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (hole || p + 8 * (i >> 1) + 2 * t + (i & 1) > last[e]) x[i] = -INFINITY;
                    }
                    float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    if (__any_sync(0xffffffffu, top > m[e])) {
                        const float mn = fmaxf(m[e], top), f = mn == -INFINITY ? 1.f : exp2_approx(m[e] - mn);
                        m[e] = mn;
                        l[e] *= f;
#pragma unroll
                        for (int n = 0; n < NTILE; ++n) { o[n][2 * e] *= f; o[n][2 * e + 1] *= f; }
                    }
                    const float base = m[e] == -INFINITY ? 0.f : m[e];
#pragma unroll
                    for (int i = 0; i < 4; ++i) { x[i] = exp2_approx(x[i] - base); l[e] += x[i]; }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t tm[NQ];
                        terms_of<NQ>(x[2 * h], x[2 * h + 1], tm);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) pf[i][2 * h + e] = tm[i];
                    }
                }
                auto products = [&](int n, const uint32_t (&b0)[2][NK], const uint32_t (&b1)[2][NK]) {       // of 16 dimensions: tiles n and n + 1
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
                        for (int i = 0; i < 4; ++i) o[n + u][i] += d[u][i];
                };
                if constexpr (NK == 1) {
#pragma unroll
                    for (int n2 = 0; n2 < NTILE / 2; ++n2) {         // matrices: positions 0..7 and 8..15 of 8 dimensions, then of the next 8
                        uint32_t r[4];
                        const int pos = (lane & 7) + ((lane >> 3) & 1) * 8;
                        ldsm4t(vb + pos * Rg::ROW + Rg::vswz(pos, 2 * n2 + (lane >> 4)) * 16, r);
                        const uint32_t b0[2][1] = {{r[0]}, {r[2]}}, b1[2][1] = {{r[1]}, {r[3]}};
                        products(2 * n2, b0, b1);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) {              // four dimensions 32 c + 4 g + i of positions 2t, 2t + 1, 2t + 8, 2t + 9
                        uint4 v4[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int pos = 2 * t + (i & 1) + 8 * (i >> 1);
                            v4[i] = lds16(vb + pos * Rg::ROW + Rg::vswz(pos, 8 * c + g) * 16);
                        }
                        const uint32_t u[4][4] = {{v4[0].x, v4[0].y, v4[0].z, v4[0].w}, {v4[1].x, v4[1].y, v4[1].z, v4[1].w},
                                                  {v4[2].x, v4[2].y, v4[2].z, v4[2].w}, {v4[3].x, v4[3].y, v4[3].z, v4[3].w}};
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            uint32_t b0[2][NK], b1[2][NK];
#pragma unroll
                            for (int z = 0; z < 2; ++z) {
                                terms_of<NK>(__uint_as_float(u[0][i + z]), __uint_as_float(u[1][i + z]), b0[z]);
                                terms_of<NK>(__uint_as_float(u[2][i + z]), __uint_as_float(u[3][i + z]), b1[z]);
                            }
                            products(4 * c + i, b0, b1);
                        }
                    }
                }
                if (++stage == Rg::STAGES) stage = 0;
            }
            // ---- the rows' ends ----------------------------------------------------------------------------------------
            // o[n][2 e + i] is dimension col(n, i) of row 8 e + g
            auto col = [&](int n, int i) { return NK == 1 ? 8 * n + 2 * t + i : 32 * (n >> 2) + 4 * (2 * t + i) + (n & 3); };
            const bool whole = from == 0 && to == it.kv;
            const size_t slot = ((size_t)w * SLOTS + (from > 0 ? 0 : 1)) * 16;
            unsigned odd[2];                                         // lanes with a sum of row 8 e + g that is not finite
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float bad[2] = {0.f, 0.f};                           // 0 times the sums: not 0 where one is not finite
#pragma unroll
                for (int n = 0; n < NTILE; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) bad[i] = fmaf(o[n][2 * e + i], 0.f, bad[i]);
                odd[e] = __ballot_sync(0xffffffffu, bad[0] + bad[1] != 0.f);
                float ls = l[e];
                ls += __shfl_xor_sync(0xffffffffu, ls, 1);
                ls += __shfl_xor_sync(0xffffffffu, ls, 2);
                const int r = 8 * e + g;
                if (r >= live) continue;
                const float f = !whole ? 1.f : ls == 0.f ? 0.f : 1.0f / ls;
                float *d = whole ? static_cast<float *>(a.out) + ((size_t)(row0 + r / heads) * a.H + h0 + r % heads) * HD : a.o + (slot + r) * HD;
                if (!whole && t == 0) a.ml[slot + r] = make_float2(m[e], ls);
#pragma unroll
                for (int n = 0; n < NTILE; ++n) {
                    if constexpr (NK == 1) {
                        *reinterpret_cast<float2 *>(d + col(n, 0)) = make_float2(o[n][2 * e] * f, o[n][2 * e + 1] * f);
                    } else {
                        d[col(n, 0)] = o[n][2 * e] * f;
                        d[col(n, 1)] = o[n][2 * e + 1] * f;
                    }
                }
            }
            // Such a row may be so only by the products: 0 times a V that is not finite and that the row does not see, an infinity (or a value that bf16 rounds
            // to one) in three terms.
            if (odd[0] | odd[1]) {
                __syncwarp();                                        // behind the other lanes' stores
                for (int r = 0; r < live; ++r)
                    if (odd[r >> 3] >> (4 * (r & 7)) & 15u)
                        row_by_definition<HD, float, KT, PAGED>(a, Row{it.b, it.r.row0, row0 + r / heads, h0 + r % heads, from, min(seen0 + r / heads + 1, to), whole, slot + r});
            }
        }
        any = it.next(a) && it.start < x1;
    }
}

}  // namespace rowattn
}  // namespace knnssd
