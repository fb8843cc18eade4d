// Attention of trees' rows over short contexts: one launch, no scratch.
//
// The mathematics is the rows kernel's (row_attention.cuh): up to 16 rows of a request that share a K/V head are an operand of m16n8k16 products, fp32 values are multiplied as three bf16 terms
// each, a row sees what its word says.  Here a block has all positions of its rows: its eight warps take 16 of them in turn, K and V straight from the pages into the products'
// operands (any order of a head's dimensions serves a sum over them, and each is stored where it belongs), and put their parts together in shared memory.
//
// Which of the requests' rows a block has follows from row_start alone: request b's blocks are those from row_start[b] / tb + b on, as many as row_start[b + 1] / tb - row_start[b] / tb + 1, which
// are enough for its rows whatever the requests before it have.
#pragma once

#include "attention_items.cuh"
#include "row_attention.cuh"

namespace knnssd {
namespace shortattn {

using namespace attn;
using rowattn::mma;
using rowattn::terms_of;

constexpr int TP = 16, ROWS = 16, WARPS = 8, NT = WARPS * 32;

template <int HD> constexpr int smem_bytes() { return WARPS * ROWS * (HD * (int)sizeof(float) + (int)sizeof(float2)); }

__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

template <int HD, typename QT, typename KT>
__global__ void __launch_bounds__(NT, 1) short_kernel(const __grid_constant__ Args a) {
    constexpr int NQ = sizeof(QT) == 4 ? 3 : 1, NK = sizeof(KT) == 4 ? 3 : 1, KS = HD / 16, NTILE = HD / 8;
    constexpr int PER = 16 / (int)sizeof(KT);                        // values of 16 bytes
    extern __shared__ __align__(16) unsigned char smem[];
    float *parts = reinterpret_cast<float *>(smem);                  // [warp][row][HD]
    float2 *ml = reinterpret_cast<float2 *>(smem + WARPS * ROWS * HD * sizeof(float));       // [warp][row]
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, vh = blockIdx.x, y = blockIdx.y;
    clear_others<QT>(a, HD, (y * gridDim.x + vh) * NT + tid, gridDim.x * gridDim.y * NT);
    int upto = 0;                                                    // requests whose blocks begin at this one or before
    for (int b0 = 0; b0 < a.B; b0 += NT) {
        const int b = b0 + tid;
        upto += __syncthreads_count(b < a.B && min(max(a.row_start[b], 0), a.R) / a.tb + b <= y);
    }
    const int b = max(upto - 1, 0), row_first = min(max(a.row_start[b], 0), a.R), n = max(min(max(a.row_start[b + 1], 0), a.R) - row_first, 0);
    const int tile = y - (row_first / a.tb + b);
    if (tile < 0 || tile * a.tb >= n) return;
    const int held = (int)min((long long)max(a.lens[b], 0), (long long)a.max_pages << a.page_shift);
    const int tokens = min(a.tb, n - tile * a.tb), seen0 = held + tile * a.tb, kv = seen0 + tokens, row0 = row_first + tile * a.tb;
    const int G = a.H / a.KV, kvh = vh / a.subs, h0 = kvh * G + (vh % a.subs) * a.gs, heads = min(a.gs, (kvh + 1) * G - h0), live = tokens * heads;
    const int warps = min(WARPS, (kv + TP - 1) / TP);
    if (warp < warps) {
        auto page_at = [&](int p) {
            const int idx = p >> a.page_shift, id = p < kv && idx < a.max_pages ? __ldg(a.table + (size_t)b * a.max_pages + idx) : -1;
            return id < a.n_pages ? id : -1;
        };
        int page = page_at(warp * TP);
        // the rows: dimension pair h of k-step s that lane t multiplies
        auto dim_of = [&](int s, int h) { return sizeof(KT) == 2 ? 32 * (s >> 1) + 8 * t + 4 * (s & 1) + 2 * h : 16 * s + 4 * t + 2 * h; };
        uint32_t qf[KS][NQ][4];
        int last[2];
        unsigned long long word[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * e + g, tok = r / heads;
            const bool on = r < live;
            last[e] = on ? seen0 + tok : -1;
            word[e] = on ? __ldg(a.seen + row0 + tok) : 0ull;
            const QT *qp = static_cast<const QT *>(a.q) + (long long)(row0 + tok) * a.q_stride + (long long)(h0 + r % heads) * HD;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (sizeof(QT) == 2) qf[s][0][2 * h + e] = on ? __ldg(reinterpret_cast<const uint32_t *>(qp + dim_of(s, h))) : 0u;
                    else {
                        uint32_t tm[NQ];
                        const float2 v = on ? __ldg(reinterpret_cast<const float2 *>(qp + dim_of(s, h))) : make_float2(0.f, 0.f);
                        terms_of<NQ>(v.x, v.y, tm);
#pragma unroll
                        for (int i = 0; i < NQ; ++i) qf[s][i][2 * h + e] = tm[i];
                    }
                }
        }
        float o[NTILE][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NTILE; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
#pragma unroll 1
        for (int p = warp * TP; p < kv; p += WARPS * TP) {
            const int id = page;
            page = page_at(p + WARPS * TP);
            const size_t at = ((((size_t)max(id, 0) * a.KV + kvh) << a.page_shift) + (p & ((1 << a.page_shift) - 1))) * HD;
            const KT *kp = static_cast<const KT *>(a.k) + at, *vp = static_cast<const KT *>(a.v) + at;
            const int there = id < 0 ? 0 : kv - p;                   // positions that count; the others are zeros
            auto load = [&](const KT *from, int pos, int dim) {
                return pos < there ? __ldg(reinterpret_cast<const uint4 *>(from + pos * HD + dim)) : make_uint4(0u, 0u, 0u, 0u);
            };
            float sp[2][3][4];                                       // sums of the scores: large terms of even and odd k-steps, small terms
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int u = 0; u < 3; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sp[i][u][j] = 0.f;
            uint4 k4[2][HD / (4 * PER)];                             // of position 8 i + g: 16 bytes at 4 PER c + PER t
#pragma unroll
            for (int c = 0; c < HD / (4 * PER); ++c)
#pragma unroll
                for (int i = 0; i < 2; ++i) k4[i][c] = load(kp, 8 * i + g, 4 * PER * c + PER * t);
            uint4 v4[4][HD / (8 * PER)];                             // of positions 2t, 2t + 1, 2t + 8, 2t + 9: 16 bytes at 8 PER c + PER g
            if constexpr (NK == 1) {
#pragma unroll
                for (int c = 0; c < HD / (8 * PER); ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v4[i][c] = load(vp, 2 * t + (i & 1) + 8 * (i >> 1), 8 * PER * c + PER * g);
            }
#pragma unroll
            for (int c = 0; c < HD / (4 * PER); ++c) {
                if constexpr (NK == 1) {
#pragma unroll
                    for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
#pragma unroll
                            for (int j = 0; j < 2; ++j) mma(sp[j][i ? 2 : e], qf[2 * c + e][i], e ? k4[j][c].z : k4[j][c].x, e ? k4[j][c].w : k4[j][c].y);
                } else {
                    uint32_t b0[2][NK], b1[2][NK];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        terms_of<NK>(__uint_as_float(k4[j][c].x), __uint_as_float(k4[j][c].y), b0[j]);
                        terms_of<NK>(__uint_as_float(k4[j][c].z), __uint_as_float(k4[j][c].w), b1[j]);
                    }
#pragma unroll
                    for (int i = NQ - 1; i >= 0; --i)
#pragma unroll
                        for (int u = NK - 1 - i; u >= 0; --u)
#pragma unroll
                            for (int j = 0; j < 2; ++j) mma(sp[j][i + u ? 2 : c & 1], qf[c][i], b0[j][u], b1[j][u]);
                }
            }
            if constexpr (NK != 1) {
#pragma unroll
                for (int c = 0; c < HD / (8 * PER); ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v4[i][c] = load(vp, 2 * t + (i & 1) + 8 * (i >> 1), 8 * PER * c + PER * g);
            }
            uint32_t pf[NQ][4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = (sp[i >> 1][0][2 * e + (i & 1)] + sp[i >> 1][1][2 * e + (i & 1)] + sp[i >> 1][2][2 * e + (i & 1)]) * a.scale_log2;
                    if (id < 0 || !tree_sees(word[e], last[e] - p - 8 * (i >> 1) - 2 * t - (i & 1))) x[i] = -INFINITY;
                }
                float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                if (__any_sync(0xffffffffu, top > m[e])) {
                    const float mn = fmaxf(m[e], top), f = mn == -INFINITY ? 1.f : exp2_approx(m[e] - mn);
                    m[e] = mn;
                    l[e] *= f;
#pragma unroll
                    for (int i = 0; i < NTILE; ++i) { o[i][2 * e] *= f; o[i][2 * e + 1] *= f; }
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
            auto products = [&](int tile, const uint32_t (&b0)[2][NK], const uint32_t (&b1)[2][NK]) {        // tiles `tile` and `tile` + 1
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
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
            l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
            const int r = 8 * e + g;
            if (t == 0) ml[warp * ROWS + r] = make_float2(m[e], l[e]);
            float *to = parts + (warp * ROWS + r) * HD;
#pragma unroll
            for (int i = 0; i < NTILE; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) to[8 * PER * (i / PER) + PER * (2 * t + j) + i % PER] = o[i][2 * e + j];
        }
    }
    __syncthreads();
    // ---- the warps' parts together: HD / 4 threads a row
    constexpr int LANES = HD / 4;
    for (int r0 = 0; r0 < live; r0 += NT / LANES) {
        const int r = r0 + tid / LANES, d = tid % LANES * 4;
        bool odd = false;
        if (r < live) {
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
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] *= inv; odd |= !isfinite(v[i]); }
            QT *to = static_cast<QT *>(a.out) + ((size_t)(row0 + r / heads) * a.H + h0 + r % heads) * HD + d;
            if constexpr (sizeof(QT) == 2) *reinterpret_cast<uint2 *>(to) = make_uint2(cvt_bf16x2(v[0], v[1]), cvt_bf16x2(v[2], v[3]));
            else *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
        }
        // A row may be so only by the products: 0 times a V that is not finite and that it does not see, an infinity in three terms.  By the definition then.
        unsigned odds = __ballot_sync(0xffffffffu, odd);
        __syncwarp();                                                // behind the stores
        for (int i = 0; odds != 0 && i < 32 / LANES; ++i, odds = LANES < 32 ? odds >> (LANES & 31) : 0u) {
            const int row = r0 + (warp * 32) / LANES + i, last = seen0 + row / heads;
            if (odds & (LANES < 32 ? (1u << (LANES & 31)) - 1 : 0xffffffffu))
                row_by_definition<HD, QT, KT, true, true>(a, Row{b, row_first, row0 + row / heads, h0 + row % heads, 0, last + 1, true, 0, last});
        }
    }
}

}  // namespace shortattn
}  // namespace knnssd
