// Attention of many new rows on the 5th-generation tensor cores: bf16 queries over pages or over packed prompts.
//
// The mathematics is the rows kernel's.  A block of a launch (one per SM) takes two halves of 128 rows (query heads that share a K/V head times
// new rows) through the positions 128 at a time:
//
//   warp 8       brings q, K and V in by TMA (128-byte swizzle), a ring of 128-position tiles ahead of the products
//   warp 9       issues the products: S = q K^T into tensor memory, O += P V with P read from tensor memory and V as the
//                transposed operand straight from its row-major tile
//   warps 0 - 3  the softmax of the first half, a row per thread: scores out of tensor memory, exponentials, P back as bf16 over them
//   warps 4 - 7  the same for the second half
//
// While one half's exponentials are formed the tensor cores do the other half's products, in the order S0 S1 | PV0 S0' PV1 S1' | ..  O stays in tensor
// memory; it is multiplied only when a row's maximum has grown by more than 2^8 since the reference its exponentials are taken against
// (their sums stay far inside fp32, and bf16 rounds relatively), which hardly ever happens after the first positions.
// Both halves share the K/V tiles; where a request has no more rows than one half, the halves are two K/V heads with tiles of their own.
//
// Every wait is bounded; one that gives up sets the error word and all warps leave, after their copies have landed.
#pragma once

#include <cuda.h>

#include "attention_items.cuh"

namespace knnssd {
namespace tcattn {

using namespace attn;

constexpr int KEYS = 128, HALF_ROWS = 128, ROWS = 256;
constexpr int SOFT_WARPS = 8, NT = (SOFT_WARPS + 4) * 32, LOAD_WARP = 8, MMA_WARP = 9;
constexpr int SOFT_REGS = 216, OTHER_REGS = 72;     // 2 x 128 x 216 + 128 x 72 = 384 x 168, what the block is launched with
constexpr int NCOST = 128;
constexpr int BAND = KEYS * 128;          // bytes of 64 dimensions of a tile: rows of 128 bytes, swizzled
constexpr int INFO = 16;                  // steps whose page masks are kept
constexpr unsigned WAIT_LIMIT = 1000000u;
constexpr float GROWTH = 8.f;
constexpr int TMEM_COLS = 512, O_COL = 256;

template <int HD> struct Lay {
    static constexpr int TILE = KEYS * HD * 2, BANDS = HD / 64;
    static constexpr int TILES = HD == 128 ? 5 : 10;
    static constexpr int SMEM = (2 + TILES) * TILE + 1024;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t b, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(count)); }
__device__ __forceinline__ void bar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t b, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(b), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(b), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool bar_wait(uint32_t b, uint32_t parity, volatile int *quit, int *err, int code) {
    if (bar_try(b, parity)) return true;
    for (unsigned spins = 0; !bar_try(b, parity);) {
        if (*quit) return false;
        if (++spins > WAIT_LIMIT) {
            *quit = 1;
            atomicExch(err, code);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ uint32_t elect() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one;
}
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y),
                 "r"(z)
                 : "memory");
}
// Shared-memory operand descriptors, 128-byte swizzle: address / 16 in bits 0 .. 13, leading offset / 16 in 16 .. 29, stride offset / 16 in
// 32 .. 45, version 1 in 46 .. 47, swizzle mode 2 in 61 .. 63.  Rows are 128 bytes, eight of them (1024 bytes) the stride.  Read along
// the dimensions (q, K): the leading offset plays no part.  Read along the positions (V, the transposed operand): it leads to the next 64 dimensions.
__device__ __forceinline__ uint64_t desc_of(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(BAND >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// fp32 sums, bf16 operands, M = 128, N columns; transposed: the second operand is read along its rows.
__host__ __device__ constexpr uint32_t idesc_of(int n, bool transposed) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (transposed ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add, uint32_t one) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(idesc), "r"(add), "r"(one)
                 : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add, uint32_t one) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b),
                 "r"(idesc), "r"(add), "r"(one)
                 : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar, uint32_t one) {
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(one) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define KNNSSD_R32(X, r) X(r[0]), X(r[1]), X(r[2]), X(r[3]), X(r[4]), X(r[5]), X(r[6]), X(r[7]), X(r[8]), X(r[9]), X(r[10]), X(r[11]), X(r[12]), X(r[13]), X(r[14]), X(r[15]), \
    X(r[16]), X(r[17]), X(r[18]), X(r[19]), X(r[20]), X(r[21]), X(r[22]), X(r[23]), X(r[24]), X(r[25]), X(r[26]), X(r[27]), X(r[28]), X(r[29]), X(r[30]), X(r[31])
#define KNNSSD_OUT(x) "=r"(x)
#define KNNSSD_IN(x) "r"(x)
#define KNNSSD_IO(x) "+r"(x)
// 32 columns of this thread's lane of tensor memory; the values are there after wait_ld() and settle().
__device__ __forceinline__ void tmem_ld(uint32_t t, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, "
                 "%25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : KNNSSD_R32(KNNSSD_OUT, r)
                 : "r"(t)
                 : "memory");
}
__device__ __forceinline__ void settle(uint32_t (&r)[32]) { asm volatile("" : KNNSSD_R32(KNNSSD_IO, r)::"memory"); }
__device__ __forceinline__ void tmem_st(uint32_t t, const uint32_t (&r)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, "
                 "%25, %26, %27, %28, %29, %30, %31};" ::KNNSSD_R32(KNNSSD_IN, r),
                 "r"(t)
                 : "memory");
}

// What a run has of an item: steps (tiles of KEYS positions) j0 .. of either half; a half without rows, or whose rows end before, has none.
struct Job {
    int from, to, j0, n[2], steps, seen0, tokens;
    bool paired;
    __device__ __forceinline__ Job(const Args &a, const Item<true> &it, long long x0, long long x1) {
        from = cut<KEYS>(it, x0); to = cut<KEYS>(it, x1);
        j0 = from / KEYS;
        tokens = it.tokens();
        seen0 = it.kv - tokens;
        paired = it.paired();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int end = paired ? it.kv : min(it.kv, seen0 + (h + 1) * a.tb);
            const bool rows = h == 0 || (paired ? 2 * it.vh + 1 < a.nvh : tokens > a.tb);
            n[h] = rows && from < to ? max(0, (min(to, end) + KEYS - 1) / KEYS - j0) : 0;
        }
        steps = max(n[0], n[1]);
    }
};

// A row whose sums are not finite, where that may have come from a position that it does not see (0 times a V that is not finite): the same
// from the positions that it does see, one by one.  Positions behind the block's last are zero in the tiles, so only the block's own
// positions can do it.  Never on finite inputs.
template <int HD, bool PAGED>
__device__ __forceinline__ void mend_row(const Args &a, int b, int seq_row0, int from, int tile_end, int kv, int token_row, int head, int last, bool whole, size_t slot) {
    const int kvh = head / (a.H / a.KV);
    auto place = [&](int pos, size_t &k, size_t &v) {
        if (!PAGED) {
            k = (size_t)(seq_row0 + pos) * a.k_stride + (size_t)kvh * HD;
            v = (size_t)(seq_row0 + pos) * a.v_stride + (size_t)kvh * HD;
            return true;
        }
        const int idx = pos >> a.page_shift, id = idx < a.max_pages ? a.table[(size_t)b * a.max_pages + idx] : -1;
        if (id < 0 || id >= a.n_pages) return false;
        k = v = ((((size_t)id * a.KV + kvh) << a.page_shift) + (pos & ((1 << a.page_shift) - 1))) * HD;
        return true;
    };
    const bf16_t *kp = static_cast<const bf16_t *>(a.k), *vp = static_cast<const bf16_t *>(a.v);
    bool disturbed = false;
    size_t k, v;
#pragma unroll 1
    for (int pos = max(last + 1, from); pos < min(tile_end, kv) && !disturbed; ++pos)
        if (place(pos, k, v)) {
#pragma unroll 1
            for (int i = 0; i < HD; ++i) disturbed |= (vp[v + i] & 0x7f80u) == 0x7f80u;
        }
    if (!disturbed) return;
    const bf16_t *q = static_cast<const bf16_t *>(a.q) + (size_t)token_row * a.q_stride + (size_t)head * HD;
    float o[HD], m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int i = 0; i < HD; ++i) o[i] = 0.f;
#pragma unroll 1
    for (int pos = from; pos <= last && pos < tile_end; ++pos) {
        if (!place(pos, k, v)) continue;
        float s = 0.f;
#pragma unroll 1
        for (int i = 0; i < HD; ++i) s = fmaf(bf16_bits_to_float(q[i]), bf16_bits_to_float(kp[k + i]), s);
        s *= a.scale_log2;
        const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn, f = exp2_approx(m - base), p = exp2_approx(s - base);
        m = mn;
        l = l * f + p;
#pragma unroll 1
        for (int i = 0; i < HD; ++i) o[i] = fmaf(p, bf16_bits_to_float(vp[v + i]), o[i] * f);
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll 1
    for (int i = 0; i < HD; ++i) {
        if (whole) static_cast<bf16_t *>(a.out)[((size_t)token_row * a.H + head) * HD + i] = float_to_bf16_rne(o[i] * inv);
        else a.o[slot * HD + i] = o[i];
    }
    if (!whole) a.ml[slot] = make_float2(m, l);
}

template <int HD, bool PAGED>
__global__ void __launch_bounds__(NT, 1) tensor_kernel(const Args a, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                        const __grid_constant__ CUtensorMap vmap) {
    using L = Lay<HD>;
    extern __shared__ unsigned char raw[];
    __shared__ Costs<NCOST> costs;
    __shared__ uint64_t bars[2 + 2 + 2 * L::TILES + 2 + 2 + 2];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int quit;
    __shared__ volatile unsigned info[INFO];                         // the 16-position groups of a step's tile that have a page
    const uint32_t smem = (smem_addr(raw) + 1023u) & ~1023u, q_tile = smem, ring = smem + 2 * L::TILE;
    const uint32_t q_full = smem_addr(bars), q_empty = q_full + 16, kv_full = q_empty + 16, kv_empty = kv_full + 8 * L::TILES, s_full = kv_empty + 8 * L::TILES,
                   p_full = s_full + 16, o_full = p_full + 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        quit = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(q_full + 8 * i, 1); bar_init(q_empty + 8 * i, 1);
            bar_init(s_full + 8 * i, 2); bar_init(p_full + 8 * i, 4); bar_init(o_full + 8 * i, 1);
        }
        for (int i = 0; i < L::TILES; ++i) { bar_init(kv_full + 8 * i, 1); bar_init(kv_empty + 8 * i, 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        fence_before();
    }
    chain_wait();
    sum_costs<true>(a, costs);                                       // has the block's barriers
    fence_after();
    const uint32_t tmem = tmem_base;
    if (a.clear) clear_tail<bf16_t>(a, HD, blockIdx.x * NT + tid, gridDim.x * NT);
    const long long total = costs.pfx[NCOST];
    const int w = blockIdx.x, W = total > 0 ? workers_of(a, total, gridDim.x) : 0;
    const long long x0 = w < W ? run_start(total, w, W) : 0, x1 = w < W ? run_start(total, w + 1, W) : 0;
    if (x0 >= x1) {
        if (tid == 0) { a.parts[w].first = 0; a.parts[w].start = -1; }
    } else {
        Item<true> it = item_at<true>(a, costs, x0);
        if (tid == 0) note_part<KEYS>(a, it, w, W, total, x0, x1);
        const uint32_t one = elect();
        bool ok = true, more = true;

        if (warp >= SOFT_WARPS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(OTHER_REGS));
        if (warp == LOAD_WARP) {
            // ---- copies ------------------------------------------------------------------------------------------------
            unsigned fills = 0, qfills[2] = {0, 0}, step0 = 0;
            const int piece = PAGED ? min(1 << a.page_shift, KEYS) : KEYS, pieces = KEYS / piece;
            int id = -1, next_id = -1;                               // lane i: the page of piece i of the tile, of the one behind it
            auto page_of = [&](int j) {
                const int pos = j * KEYS + lane * piece;
                if (lane >= pieces || pos >= it.kv || (pos >> a.page_shift) >= a.max_pages) return -1;
                const int p = __ldg(a.table + (size_t)it.b * a.max_pages + (pos >> a.page_shift));
                return p < a.n_pages ? p : -1;
            };
            auto put = [&](const CUtensorMap *map, int vh, int j, int page, bool note, unsigned step) {
                const unsigned slot = fills % L::TILES, turn = fills / L::TILES;
                ok = ok && bar_wait(kv_empty + 8 * slot, (turn & 1) ^ 1, &quit, a.err, 201);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; return; }
                const uint32_t dst = ring + slot * L::TILE, bar = kv_full + 8 * slot;
                const int kvh = vh / a.subs;
                if (PAGED) {
                    const unsigned there = __ballot_sync(0xffffffffu, page >= 0);
                    if (lane == 0) {
                        if (note) {
                            unsigned groups = 0;
                            for (int i = 0; i < pieces; ++i)
                                if (there >> i & 1) groups |= ((1u << (piece / 16)) - 1) << (i * (piece / 16));
                            info[step % INFO] = groups;
                        }
                        bar_expect(bar, __popc(there) * piece * HD * 2);
                    }
                    __syncwarp();
                    if (page >= 0) {
                        const int in_page = (j * KEYS + lane * piece) & ((1 << a.page_shift) - 1);
                        const int y = ((page * a.KV + kvh) << a.page_shift) + in_page;
#pragma unroll
                        for (int b = 0; b < L::BANDS; ++b) tma_2d(dst + b * BAND + lane * piece * 128, map, 64 * b, y, bar);
                    }
                } else if (lane == 0) {
                    bar_expect(bar, L::TILE);
#pragma unroll
                    for (int b = 0; b < L::BANDS; ++b) tma_3d(dst + b * BAND, map, 64 * b, kvh, it.r.row0 + j * KEYS, bar);
                }
                ++fills;
            };
            while (more && ok) {
                const Job job(a, it, x0, x1);
                const int v0 = job.paired ? 2 * it.vh : it.vh, v1 = job.paired ? v0 + 1 : v0;
                if (PAGED && job.steps) { id = page_of(job.j0); next_id = page_of(job.j0 + 1); }
                // the first tile's K before q: the ring has room while q waits for the products of the item before
                auto k_of = [&](int s, int page) {
                    if (!job.paired) put(&kmap, v0, job.j0 + s, page, true, step0 + s);
                };
                for (int h = 0; h < 2 && ok; ++h)
                    if (job.n[h]) {
                        ok = bar_wait(q_empty + 8 * h, (qfills[h] & 1) ^ 1, &quit, a.err, 202);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        if (lane == 0) {
                            const int vh = h ? v1 : v0, h0 = vh / a.subs * (a.H / a.KV) + vh % a.subs * a.gs;
                            const int row = it.r.row0 + it.rb * it.r.tb + (job.paired ? 0 : h * a.tb);
                            bar_expect(q_full + 8 * h, a.tb * a.gs * HD * 2);
#pragma unroll
                            for (int b = 0; b < L::BANDS; ++b) tma_3d(q_tile + h * L::TILE + b * BAND, &qmap, 64 * b, h0, row, q_full + 8 * h);
                        }
                        ++qfills[h];
                        if (h == 0 && ok) { if (job.paired) put(&kmap, v0, job.j0, id, true, step0); else k_of(0, id); }
                        if (h == 1 && ok) { if (job.paired) put(&kmap, v1, job.j0, id, false, step0); else if (!job.n[0]) k_of(0, id); }
                    }
                for (int s = 0; s < job.steps && ok; ++s) {
                    const int j = job.j0 + s;
                    const bool again = s + 1 < job.steps;
                    if (!job.paired) {
                        put(&vmap, v0, j, id, false, 0);
                        if (again && ok) k_of(s + 1, next_id);
                    } else {
                        put(&vmap, v0, j, id, false, 0);
                        if (again && ok) put(&kmap, v0, j + 1, next_id, true, step0 + s + 1);
                        if (job.n[1] && ok) put(&vmap, v1, j, id, false, 0);
                        if (job.n[1] && again && ok) put(&kmap, v1, j + 1, next_id, false, 0);
                    }
                    if (PAGED) { id = next_id; next_id = page_of(j + 2); }
                }
                step0 += job.steps;
                more = it.next(a) && it.start < x1;
            }
            // every copy has landed and every product has let go of its tile before the block goes
            for (unsigned i = fills > L::TILES ? fills - L::TILES : 0; i < fills; ++i) {
                const unsigned slot = i % L::TILES, parity = i / L::TILES & 1;
                if (ok) ok = bar_wait(kv_empty + 8 * slot, parity, &quit, a.err, 203);
                if (!ok)
                    for (unsigned spins = 0; spins < WAIT_LIMIT && !bar_try(kv_full + 8 * slot, parity); ++spins) {}
            }
            for (int h = 0; h < 2; ++h)
                if (qfills[h]) {
                    if (ok) ok = bar_wait(q_empty + 8 * h, (qfills[h] - 1) & 1, &quit, a.err, 204);
                    if (!ok)
                        for (unsigned spins = 0; spins < WAIT_LIMIT && !bar_try(q_full + 8 * h, (qfills[h] - 1) & 1); ++spins) {}
                }
        } else if (warp == MMA_WARP) {
            // ---- products ------------------------------------------------------------------------------------------------
            constexpr uint32_t S_DESC = idesc_of(KEYS, false), O_DESC = idesc_of(HD, true);
            unsigned uses = 0, q_uses[2] = {0, 0}, p_uses[2] = {0, 0}, step0 = 0;
            auto tile_there = [&](unsigned use) { ok = ok && bar_wait(kv_full + 8 * (use % L::TILES), use / L::TILES & 1, &quit, a.err, 205); return ok; };
            auto scores = [&](int h, unsigned use) {
                if (lane == 0) bar_arrive(s_full + 8 * h);           // hands on what the copies' warp noted of the tile
                fence_after();
                const uint32_t q = q_tile + h * L::TILE, k = ring + use % L::TILES * L::TILE;
#pragma unroll
                for (int i = 0; i < HD / 16; ++i)
                    mma_ss(tmem + h * KEYS, desc_of(q + (i >> 2) * BAND + (i & 3) * 32), desc_of(k + (i >> 2) * BAND + (i & 3) * 32), S_DESC, i > 0, one);
                commit(s_full + 8 * h, one);
            };
            // What lies behind the last position that the block sees, and what has no page, must be zero in V: its p is 0, and 0 times what happens
            // to lie there need not be.
            auto clean = [&](unsigned use, int valid, unsigned groups) {
                if (valid >= KEYS && groups == 0xffu) return;
                const uint32_t v = ring + use % L::TILES * L::TILE;
                for (int i = lane; i < KEYS * 8; i += 32) {
                    const int row = i >> 3;
                    if (row < valid && (groups >> (row >> 4) & 1)) continue;
#pragma unroll
                    for (int b = 0; b < L::BANDS; ++b)
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v + b * BAND + i * 16), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            };
            auto values = [&](int h, unsigned use, bool add) {
                ok = ok && bar_wait(p_full + 8 * h, p_uses[h]++ & 1, &quit, a.err, 206);
                if (!ok) return;
                fence_after();
                const uint32_t v = ring + use % L::TILES * L::TILE;
#pragma unroll
                for (int i = 0; i < KEYS / 16; ++i)
                    mma_ts(tmem + O_COL + h * HD, tmem + h * KEYS + 8 * i, desc_of(v + i * 2048), O_DESC, add || i > 0, one);
                commit(o_full + 8 * h, one);
            };
            auto let_go = [&](unsigned use) { commit(kv_empty + 8 * (use % L::TILES), one); };
            while (more && ok) {
                const Job job(a, it, x0, x1);
                unsigned k_use[2] = {0, 0}, v_use[2] = {0, 0};
                auto score_step = [&](int h, int s) {
                    if (job.paired || h == 0 || job.n[0] <= s) k_use[h] = uses++; else k_use[h] = k_use[0];
                    if (s == 0) ok = ok && bar_wait(q_full + 8 * h, q_uses[h]++ & 1, &quit, a.err, 207);
                    if (!ok || !tile_there(k_use[h])) { ok = false; return; }
                    scores(h, k_use[h]);
                    if (s + 1 == job.n[h]) commit(q_empty + 8 * h, one);
                    if (job.paired || h == 1 || job.n[1] <= s) let_go(k_use[h]);
                };
                for (int h = 0; h < 2 && ok; ++h)
                    if (job.n[h]) score_step(h, 0);
                for (int s = 0; s < job.steps && ok; ++s) {
                    const int valid = it.kv - (job.j0 + s) * KEYS;
                    for (int h = 0; h < 2 && ok; ++h) {
                        if (job.n[h] <= s) continue;
                        const bool own_tile = job.paired || h == 0 || job.n[0] <= s;
                        if (own_tile) v_use[h] = uses++; else v_use[h] = v_use[0];
                        if (!tile_there(v_use[h])) break;
                        if (own_tile) clean(v_use[h], valid, PAGED ? info[(step0 + s) % INFO] : 0xffu);
                        values(h, v_use[h], s > 0);
                        if (!ok) break;
                        if (job.paired || h == 1 || job.n[1] <= s) let_go(v_use[h]);
                        if (s + 1 < job.n[h]) score_step(h, s + 1);
                    }
                }
                step0 += job.steps;
                more = it.next(a) && it.start < x1;
            }
        }
        } else {
            // ---- softmax ---------------------------------------------------------------------------------------------------
            asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFT_REGS));
            const int h = warp >> 2, r = h * HALF_ROWS + (warp & 3) * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), s_at = lanes + h * KEYS, o_at = lanes + O_COL + h * HD;
            unsigned s_uses = 0, o_uses = 0, step0 = 0;
            while (more && ok) {
                const Job job(a, it, x0, x1);
                int token, head;
                place_of<true, ROWS>(a, job.tokens, it.vh, job.paired, r, token, head);
                const int last = token >= 0 ? job.seen0 + token : -1, first_last = job.seen0 + (job.paired ? 0 : h * a.tb);
                const size_t row = (size_t)(it.r.row0 + it.rb * it.r.tb + (token < 0 ? 0 : token)) * a.H + head;
                const bool live = __any_sync(0xffffffffu, token >= 0);
                float m = -INFINITY, l = 0.f;
                for (int s = 0; s < job.n[h] && ok; ++s) {
                    const int k0 = (job.j0 + s) * KEYS;
                    ok = bar_wait(s_full + 8 * h, s_uses++ & 1, &quit, a.err, 208);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    if (!live) {                                     // none of the warp's rows is anyone's: what is in P there stays there
                        __syncwarp();
                        if (lane == 0) bar_arrive(p_full + 8 * h);
                        ++o_uses;
                        continue;
                    }
                    fence_after();
                    uint32_t x[4][32];
#pragma unroll
                    for (int i = 0; i < 4; ++i) tmem_ld(s_at + 32 * i, x[i]);
                    wait_ld();
#pragma unroll
                    for (int i = 0; i < 4; ++i) settle(x[i]);
                    const unsigned groups = PAGED ? info[(step0 + s) % INFO] : 0xffu;
                    const bool ragged = k0 + KEYS - 1 > first_last || groups != 0xffu;
                    if (ragged) {
                        const int see = last - k0;                   // the row sees keys 0 .. see of the tile
#pragma unroll
                        for (int i = 0; i < KEYS; ++i)
                            if (i > see || !(groups >> (i >> 4) & 1)) x[i >> 5][i & 31] = 0xff800000u;
                    }
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < KEYS; ++i) top = fmaxf(top, __uint_as_float(x[i >> 5][i & 31]));
                    const float grown = top == -INFINITY ? -INFINITY : top * a.scale_log2;
                    const bool over = grown > m + GROWTH;            // the first positions a row sees: m is -inf
                    if (__any_sync(0xffffffffu, over)) {
                        const float f = over ? exp2_approx(m - grown) : 1.f;
                        if (over) { m = grown; l *= f; }
                        if (s > 0) {
                            ok = bar_wait(o_full + 8 * h, (o_uses - 1) & 1, &quit, a.err, 209);
                            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                            fence_after();
#pragma unroll
                            for (int c = 0; c < HD / 32; ++c) {
                                uint32_t o[32];
                                tmem_ld(o_at + 32 * c, o);
                                wait_ld();
                                settle(o);
#pragma unroll
                                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                tmem_st(o_at + 32 * c, o);
                            }
                        }
                    }
                    const float base = m == -INFINITY ? 0.f : m;
                    uint32_t p[2][32];
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < KEYS; i += 2) {
                        float u = exp2_approx(fmaf(__uint_as_float(x[i >> 5][i & 31]), a.scale_log2, -base));
                        float v = exp2_approx(fmaf(__uint_as_float(x[(i + 1) >> 5][(i + 1) & 31]), a.scale_log2, -base));
                        if (ragged) {                                // also where scale is 0
                            const int see = last - k0;
                            const bool gone = !(groups >> (i >> 4) & 1);
                            if (i > see || gone) u = 0.f;
                            if (i + 1 > see || gone) v = 0.f;
                        }
                        sum[(i >> 1) & 3] += u + v;
                        p[i >> 6][(i >> 1) & 31] = cvt_bf16x2(u, v);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_st(s_at, p[0]);
                    tmem_st(s_at + 32, p[1]);
                    wait_st();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_full + 8 * h);
                    ++o_uses;
                }
                if (!ok) break;
                // ---- the row's end
                const bool whole = job.from == 0 && job.to == it.kv;
                if (job.n[h]) {
                    ok = bar_wait(o_full + 8 * h, (o_uses - 1) & 1, &quit, a.err, 210);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    fence_after();
                }
                if (live && (job.n[h] || (job.from < job.to && !whole))) {
                    const float f = whole ? (l == 0.f ? 0.f : 1.0f / l) : 1.f;
                    const size_t slot = ((size_t)w * SLOTS + (job.from > 0 ? 0 : 1)) * ROWS + r;
                    bool odd = false;
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t o[32];
                        if (job.n[h]) {
                            tmem_ld(o_at + 32 * c, o);
                            wait_ld();
                            settle(o);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0u;
                        }
                        if (token < 0) continue;
#pragma unroll
                        for (int i = 0; i < 32; ++i) odd |= (o[i] & 0x7f800000u) == 0x7f800000u;
                        if (whole) {
                            bf16_t *d = static_cast<bf16_t *>(a.out) + row * HD + 32 * c;
#pragma unroll
                            for (int i = 0; i < 32; i += 8) {
                                uint4 v;
                                v.x = cvt_bf16x2(__uint_as_float(o[i]) * f, __uint_as_float(o[i + 1]) * f);
                                v.y = cvt_bf16x2(__uint_as_float(o[i + 2]) * f, __uint_as_float(o[i + 3]) * f);
                                v.z = cvt_bf16x2(__uint_as_float(o[i + 4]) * f, __uint_as_float(o[i + 5]) * f);
                                v.w = cvt_bf16x2(__uint_as_float(o[i + 6]) * f, __uint_as_float(o[i + 7]) * f);
                                *reinterpret_cast<uint4 *>(d + i) = v;
                            }
                        } else {
                            float *d = a.o + slot * HD + 32 * c;
#pragma unroll
                            for (int i = 0; i < 32; i += 4)
                                *reinterpret_cast<uint4 *>(d + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                        }
                    }
                    if (token >= 0 && !whole) a.ml[slot] = make_float2(m, l);
                    if (odd && token >= 0) mend_row<HD, PAGED>(a, it.b, it.r.row0, job.from, min(job.to, (job.j0 + job.n[h]) * KEYS), it.kv, it.r.row0 + it.rb * it.r.tb + token, head, last, whole, slot);
                    fence_before();
                }
                step0 += job.steps;
                more = it.next(a) && it.start < x1;
            }
        }
        fence_before();
    }
    __syncthreads();
    if (warp == MMA_WARP) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

}  // namespace tcattn
}  // namespace knnssd
