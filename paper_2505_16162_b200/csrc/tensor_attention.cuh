// Attention of many new rows on the 5th-generation tensor cores: bf16 queries over pages or over packed prompts.
//
// The mathematics is the rows kernel's.  A block of a launch (one per SM) takes two halves of 128 rows (query heads that share a K/V head times
// new rows) through the positions, in tiles of 128 and steps of 64:
//
//   warp 8       brings q, K and V in, a ring of tiles ahead of the products (K and V of pages: a second warp with it)
//   warps 9, 10  issue the products of a half each: S = q K^T into tensor memory, O += P V with P read from tensor memory and V as the
//                transposed operand straight from its row-major tile
//   warps 0 - 3  the softmax of the first half, a row per thread: scores out of tensor memory, exponentials, P back as bf16 over them
//   warps 4 - 7  the same for the second half
//
// Each half has two score buffers of 64 columns: while the softmax works on one step the scores of the next are formed in the other, so
// that neither the softmax nor the tensor cores wait out the other's latency (with one buffer of 128 columns a step of 128 positions
// took softmax + products, 3900 .. 4700 clocks, one half's softmax under the other half's products).  O stays in tensor memory; it is multiplied
// only when a row's maximum has grown by more than 2^8 since the reference its exponentials are taken against (their sums stay far inside
// fp32, and bf16 rounds relatively), which hardly ever happens after the first positions.
// Both halves share the K/V tiles; where a request has no more rows than one half, the halves are two K/V heads with tiles of their own.
//
// Measured, in a row of calls from a cool start / for seconds on end, when the chip runs at its power limit (1.6 - 1.7 GHz):
//   12000 packed tokens in 4 prompts, 40 heads (8 of K/V)    680 - 710 / 792 us, 1.1 / 0.96 PFLOP/s: the exponentials (8 clocks a warp for each value
//                                                           of its rows) and what stands beside them in the softmax, then power
//   2 requests of 5 rows, 240 000 positions in all            155 - 174 / 187 us, 5.4 - 6.0 / 5.0 TB/s: memory, then power
//   64 requests of 1 row over 2304 positions                 122 - 133 / 144 us, 4.6 - 5.0 / 4.2 TB/s: 3.5 items a CTA, 5 - 8 thousand clocks at each one's ends
//   24 requests of 64 rows of trees over 3000 positions      232 - 244 / 282 us, 4.9 - 5.2 / 4.3 TB/s: memory, then power
//
// Fewer bits: P is rounded to bf16 (2^-8 relative at most), as the products take it, a quarter of it comes from a cubic of 7.5e-5, and O's sums in tensor memory
// round towards zero.  Against 64 bits, with the result's own rounding, 1.8e-3 .. 2.3e-3 for 1.7e-3 by that rounding alone.
//
// Every wait is bounded; one that gives up sets the error word, all warps leave after their copies have landed and their products are done, and the rows of the
// block's run become NaN.
#pragma once

#include <cuda.h>

#include "attention_items.cuh"

namespace knnssd {
namespace tcattn {

using namespace attn;

constexpr int KEYS = 128, SUB = 64, HALF_ROWS = 128, ROWS = 256;      // positions of a tile, and of a step of the softmax
constexpr int SOFT_WARPS = 8, LOAD_WARP = 8, MMA_WARP = 9;      // pages: the second loader is the warp behind the products'
__host__ __device__ constexpr int loaders_of(bool paged) { return paged ? 2 : 1; }
__host__ __device__ constexpr int threads_of(bool paged) { return (SOFT_WARPS + 2 + loaders_of(paged)) * 32; }
constexpr int PIECE = KEYS / 2;           // positions of a page that a copy brings at most: both loaders have some of a tile
constexpr int NCOST = 128;
constexpr int BAND = KEYS * 128;          // bytes of 64 dimensions of a tile: rows of 128 bytes, swizzled
constexpr int INFO = 16;                  // steps whose page masks are kept
constexpr unsigned WAIT_LIMIT = 1000000u;
constexpr float GROWTH = 8.f;
// One pair in four takes its powers of two from the multiply-add units (a cubic, below): with none / one in eight / one in four / three in eight 12000 packed
// tokens take 750 / 739 / 709 / 726 us.  8 clocks a warp's ex2 against 3.2 for a packed multiply-add.
constexpr int CUBIC = 1, CUBIC_OF = 4;
constexpr int TMEM_COLS = 512, O_COL = 256;

template <int HD> struct Lay {
    static constexpr int TILE = KEYS * HD * 2, BANDS = HD / 64;
    // Eight rows of 64 dimensions, 1024 bytes, are what the swizzle turns.  K and V of packed rows lie as the queries, all rows of 64 dimensions and then the next 64; of pages the next
    // 64 dimensions of eight rows lie behind them, so that one copy brings a page.
    __host__ __device__ static constexpr int group(bool paged) { return paged ? 1024 * BANDS : 1024; }       // from eight rows to the next
    __host__ __device__ static constexpr int band(bool paged) { return paged ? 1024 : BAND; }                // from 64 dimensions to the next
    static constexpr int TILES = HD == 128 ? 5 : 10;
    static constexpr int SMEM = (2 + TILES) * TILE + 1024;
};

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint32_t b, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(b), "r"(count)); }
__device__ __forceinline__ void bar_arrive(uint32_t b) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(b) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(b), "r"(parity) : "memory");
    return ok != 0;
}
// The polls are a piece of code of their own: the warps' loops, each its own way through the kernel, are shorter for it (12000 packed tokens 703 us with them in
// every wait, 682 so).
static __device__ __noinline__ bool bar_poll(uint32_t b, uint32_t parity, volatile int *quit, unsigned limit, int *err, int code) {
    for (unsigned spins = 0; !bar_try(b, parity);) {
        if (*quit) return false;
        if (++spins > limit) {
            *quit = 1;
            atomicExch(err, code);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool bar_wait(uint32_t b, uint32_t parity, volatile int *quit, const Args &a, int code) {
    return bar_try(b, parity) || bar_poll(b, parity, quit, a.wait_limit, a.err, code);
}
// The same for a warp as a whole: all lanes go on, or none.
__device__ __forceinline__ bool warp_wait(uint32_t b, uint32_t parity, volatile int *quit, const Args &a, int code) {
    return __all_sync(0xffffffffu, bar_wait(b, parity, quit, a, code));
}
// For what is on its way and comes whatever else the block does: copies, products.
__device__ __forceinline__ void bar_settle(uint32_t b, uint32_t parity) {
    for (unsigned spins = 0; spins < WAIT_LIMIT && !bar_try(b, parity); ++spins) {}
}
// One thread of the warp, which goes through them as a whole (a branch on the lane costs some 100 clocks per copy: its operands are moved to
// uniform registers one by one); `one` is 1 in that thread and 0 in the others.
__device__ __forceinline__ uint32_t elect() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one;
}
__device__ __forceinline__ void bar_expect_if(uint32_t b, uint32_t bytes, uint32_t one) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(b), "r"(bytes), "r"(one) : "memory");
}
// Groups of eight rows from `group` on, all dimensions.
__device__ __forceinline__ void tma_groups(uint32_t dst, const CUtensorMap *map, int group, uint32_t bar, uint32_t one) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t"
                 "@p cp.async.bulk.tensor.4d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %3, %3, %4}], [%2];\n\t}" ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(group),
                 "r"(one)
                 : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar, uint32_t one) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
                 "@p cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n\t}" ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y),
                 "r"(z), "r"(one)
                 : "memory");
}
// Shared-memory operand descriptors, 128-byte swizzle: address / 16 in bits 0 .. 13, leading offset / 16 in 16 .. 29, stride offset / 16 in
// 32 .. 45, version 1 in 46 .. 47, swizzle mode 2 in 61 .. 63.  Rows are 128 bytes, from eight of them to the next the stride.  Read along
// the dimensions (q, K): the leading offset plays no part.  Read along the positions (V, the transposed operand): it leads to the next 64 dimensions.
// The constant upper half, and the lower half.
__host__ __device__ constexpr uint32_t desc_upper(int group) { return ((uint32_t)group >> 4) | (1u << 14) | (2u << 29); }
__device__ __forceinline__ uint32_t desc_of(uint32_t addr, int band) { return (addr >> 4) | ((uint32_t)(band >> 4) << 16); }
// fp32 sums, bf16 operands, M = 128, N columns; transposed: the second operand is read along its rows.
__host__ __device__ constexpr uint32_t idesc_of(int n, bool transposed) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (transposed ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// A row of products as one piece of code, so that their operands differ from one another by constants; one thread of the warp issues them.
#define KNNSSD_SS(Q, K) "add.u32 x, %1, " Q ";\n\tadd.u32 y, %2, " K ";\n\tmov.b64 da, {x, %5};\n\tmov.b64 db, {y, %6};\n\t"
#define KNNSSD_SS_FIRST "{\n\t.reg .pred q;\n\t.reg .b64 da, db;\n\t.reg .b32 x, y;\n\telect.sync _|q, 0xffffffff;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %6};\n\t" \
    "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, 0;\n\t"
#define KNNSSD_SS_NEXT(Q, K) KNNSSD_SS(Q, K) "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, 1;\n\t"
#define KNNSSD_SS_LAST "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t}"
// S (128 x 64) = q k^T over HD dimensions: steps of 16 are 32 bytes apart, the second 64 dimensions a band further; then bar is told.
template <int HD, bool PAGED> __device__ __forceinline__ void mma_scores(uint32_t d, uint32_t q, uint32_t k, uint32_t idesc, uint32_t bar) {
    constexpr uint32_t q_upper = desc_upper(1024), k_upper = desc_upper(Lay<HD>::group(PAGED));
    static_assert(BAND >> 4 == 1024, "as written below");
    if constexpr (HD == 128 && PAGED)
        asm volatile(KNNSSD_SS_FIRST KNNSSD_SS_NEXT("2", "2") KNNSSD_SS_NEXT("4", "4") KNNSSD_SS_NEXT("6", "6") KNNSSD_SS_NEXT("1024", "64") KNNSSD_SS_NEXT("1026", "66")
                     KNNSSD_SS_NEXT("1028", "68") KNNSSD_SS_NEXT("1030", "70") KNNSSD_SS_LAST ::"r"(d), "r"(q), "r"(k), "r"(idesc), "r"(bar), "r"(q_upper), "r"(k_upper)
                     : "memory");
    else if constexpr (HD == 128)
        asm volatile(KNNSSD_SS_FIRST KNNSSD_SS_NEXT("2", "2") KNNSSD_SS_NEXT("4", "4") KNNSSD_SS_NEXT("6", "6") KNNSSD_SS_NEXT("1024", "1024") KNNSSD_SS_NEXT("1026", "1026")
                     KNNSSD_SS_NEXT("1028", "1028") KNNSSD_SS_NEXT("1030", "1030") KNNSSD_SS_LAST ::"r"(d), "r"(q), "r"(k), "r"(idesc), "r"(bar), "r"(q_upper), "r"(k_upper)
                     : "memory");
    else
        asm volatile(KNNSSD_SS_FIRST KNNSSD_SS_NEXT("2", "2") KNNSSD_SS_NEXT("4", "4") KNNSSD_SS_NEXT("6", "6") KNNSSD_SS_LAST ::"r"(d), "r"(q), "r"(k), "r"(idesc), "r"(bar),
                     "r"(q_upper), "r"(k_upper)
                     : "memory");
}
#define KNNSSD_TS_NEXT(A, B) "add.u32 x, %1, " A ";\n\tadd.u32 y, %2, " B ";\n\tmov.b64 db, {y, %5};\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %3, 1;\n\t"
#define KNNSSD_TS_FIRST "{\n\t.reg .pred q, a;\n\t.reg .b64 db;\n\t.reg .b32 x, y;\n\telect.sync _|q, 0xffffffff;\n\tsetp.ne.b32 a, %4, 0;\n\tmov.b64 db, {%2, %5};\n\t" \
    "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, a;\n\t"
#define KNNSSD_TS_LAST "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t}"
// O (128 x HD) += P V over 64 positions: P 8 columns a step of 16, V two groups of eight rows.  add 0: the first product begins the sum.  Then bar is told.
template <int HD, bool PAGED> __device__ __forceinline__ void mma_values(uint32_t d, uint32_t p, uint32_t v, uint32_t idesc, uint32_t add, uint32_t bar) {
    constexpr int group = Lay<HD>::group(PAGED);
    static_assert(group == 1024 || group == 2048, "as written below");
    if constexpr (group == 2048)
        asm volatile(KNNSSD_TS_FIRST KNNSSD_TS_NEXT("8", "256") KNNSSD_TS_NEXT("16", "512") KNNSSD_TS_NEXT("24", "768") KNNSSD_TS_LAST ::"r"(d), "r"(p), "r"(v), "r"(idesc), "r"(add),
                     "r"(desc_upper(group)), "r"(bar)
                     : "memory");
    else
        asm volatile(KNNSSD_TS_FIRST KNNSSD_TS_NEXT("8", "128") KNNSSD_TS_NEXT("16", "256") KNNSSD_TS_NEXT("24", "384") KNNSSD_TS_LAST ::"r"(d), "r"(p), "r"(v), "r"(idesc), "r"(add),
                     "r"(desc_upper(group)), "r"(bar)
                     : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

#define KNNSSD_R32(X, r) X(r[0]), X(r[1]), X(r[2]), X(r[3]), X(r[4]), X(r[5]), X(r[6]), X(r[7]), X(r[8]), X(r[9]), X(r[10]), X(r[11]), X(r[12]), X(r[13]), X(r[14]), X(r[15]), \
    X(r[16]), X(r[17]), X(r[18]), X(r[19]), X(r[20]), X(r[21]), X(r[22]), X(r[23]), X(r[24]), X(r[25]), X(r[26]), X(r[27]), X(r[28]), X(r[29]), X(r[30]), X(r[31])
#define KNNSSD_R16(X, r) X(r[0]), X(r[1]), X(r[2]), X(r[3]), X(r[4]), X(r[5]), X(r[6]), X(r[7]), X(r[8]), X(r[9]), X(r[10]), X(r[11]), X(r[12]), X(r[13]), X(r[14]), X(r[15])
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

__device__ __forceinline__ void tmem_st16(uint32_t t, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::KNNSSD_R16(KNNSSD_IN, r), "r"(t)
                 : "memory");
}

// ---- pairs of fp32 values: two operations an instruction -------------------------------------------------------------
__device__ __forceinline__ uint64_t pair_of(uint32_t a, uint32_t b) {
    uint64_t p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "r"(a), "r"(b));
    return p;
}
__device__ __forceinline__ uint64_t pair_of(float a, float b) { return pair_of(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ void split(uint64_t p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// The largest of three; NaN where one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// 2^x of two values on the multiply-add units: x = n + f with n the nearest whole number (added to 1.5 2^23 it is the sum's low bits), 2^f by a
// cubic (minimax of the relative error on [-1/2, 1/2] by Lawson's weighted least squares: 7.5e-5, a fiftieth of what rounding to bf16
// does at most), and n added to the exponent.  At x = -126.999 the exponent ends at 0 and what is left, 6e-4 2^-126, is 0 as bf16: below that, and for what a
// row does not see, there is no weight at all.  (With 2^n as a factor instead, 0 for n = -127, packed prompts and long contexts take 1 % longer.)  NaN gives 0
// as well.
__device__ __forceinline__ void exp2_cubic(uint64_t x, float &a, float &b) {
    float x0, x1;
    split(x, x0, x1);
    x = pair_of(fmaxf(x0, -126.999f), fmaxf(x1, -126.999f));
    const uint64_t n = add2(x, pair_of(12582912.f, 12582912.f)), f = fma2(add2(n, pair_of(-12582912.f, -12582912.f)), pair_of(-1.f, -1.f), x);
    uint64_t y = fma2(f, pair_of(0.0551716685295105f, 0.0551716685295105f), pair_of(0.2426111251115799f, 0.2426111251115799f));
    y = fma2(f, y, pair_of(0.6932609677314758f, 0.6932609677314758f));
    y = fma2(f, y, pair_of(0.9999280571937561f, 0.9999280571937561f));
    float y0, y1, n0, n1;
    split(y, y0, y1);
    split(n, n0, n1);
    a = __uint_as_float(__float_as_uint(y0) + (__float_as_uint(n0) << 23));
    b = __uint_as_float(__float_as_uint(y1) + (__float_as_uint(n1) << 23));
}

// Lane 4 i + j has row j of a 4 x 4 square of 16-byte pieces; afterwards it has column j.
__device__ __forceinline__ void turn4(uint4 (&v)[4], int lane) {
    auto swap = [&](uint4 &a, uint4 &b, int by) {                    // the lanes with the bit give a and take into it, the others b
        const bool up = lane & by;
        uint4 t = up ? a : b;
        t.x = __shfl_xor_sync(0xffffffffu, t.x, by); t.y = __shfl_xor_sync(0xffffffffu, t.y, by);
        t.z = __shfl_xor_sync(0xffffffffu, t.z, by); t.w = __shfl_xor_sync(0xffffffffu, t.w, by);
        if (up) a = t; else b = t;
    };
    swap(v[0], v[1], 1);
    swap(v[2], v[3], 1);
    swap(v[0], v[2], 2);
    swap(v[1], v[3], 2);
}

// What a run has of an item: n[h] steps of SUB positions from tile j0 on for either half; a half without rows, or whose rows end before, has none.
struct Job {
    int from, to, j0, n[2], tiles, seen0, tokens;
    bool paired;
    __device__ __forceinline__ Job(const Args &a, const Item<true> &it, long long x0, long long x1) {
        from = cut<KEYS>(it, x0); to = cut<KEYS>(it, x1);
        j0 = from / KEYS;
        tokens = it.tokens();
        seen0 = it.kv - tokens;
        paired = it.r.paired;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int end = paired ? it.kv : min(it.kv, seen0 + (h + 1) * a.tb);
            const bool rows = h == 0 || (paired ? 2 * it.vh + 1 < a.nvh : tokens > a.tb);
            n[h] = rows && from < to ? max(0, (min(to, end) + SUB - 1) / SUB - from / SUB) : 0;
        }
        tiles = (max(n[0], n[1]) + KEYS / SUB - 1) / (KEYS / SUB);
    }
};

// Row rr of half h of an item; token -1: there is none.
struct Mine {
    int token, head, last, row, steps;
    bool whole;
    __device__ __forceinline__ Mine(const Args &a, const Item<true> &it, const Job &job, int h, int my_token, int my_head) {
        const int G = a.H / a.KV, v = job.paired ? 2 * it.vh + h : it.vh, kvh = a.subs == 1 ? v : v / a.subs, hh = (a.subs == 1 ? 0 : v % a.subs * a.gs) + my_head;
        token = my_token + (job.paired ? 0 : h * a.tb);
        if (my_token < 0 || token >= job.tokens || v >= a.nvh || hh >= G) token = -1;
        head = kvh * G + hh;
        last = token >= 0 ? job.seen0 + token : -1;
        row = it.r.row0 + it.rb * it.r.tb + (token < 0 ? 0 : token);
        steps = h ? job.n[1] : job.n[0];
        whole = job.from == 0 && job.to == it.kv;
    }
};

// Rows of the block's run whose sums are not finite, where that may have come from a position that they do not see (0 times a V that is not
// finite): the same by the definition, a row a warp.  Positions behind an item's last are zero in the tiles, so only the item's own new positions can
// do it.  Never on finite inputs.  It comes behind the block's last item, when no wait is left that could run out meanwhile: 12000 packed tokens with such a V
// every 64 rows take 170 ms for 0.79, two requests of 120 thousand positions with one each 8.0 for 0.24.
template <int HD, bool PAGED, bool TREE> __device__ __noinline__ void mend_rows(const Args &a, const Costs<NCOST> &costs, int w, long long x0, long long x1) {
    constexpr int PIECES = HD / 8;                                   // 16-byte pieces of a position
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    Item<true> it = item_at<true>(a, costs, x0);
    do {
        const Job job(a, it, x0, x1);
        for (int r = warp; r < ROWS; r += warps) {
            const int h = r / HALF_ROWS, rr = r % HALF_ROWS;
            const Mine mine(a, it, job, h, rr / a.gs < a.tb ? rr / a.gs : -1, rr % a.gs);
            if (mine.token < 0 || mine.steps == 0) continue;
            const size_t slot = ((size_t)w * SLOTS + (job.from > 0 ? 0 : 1)) * ROWS + r;
            const bf16_t *out = static_cast<const bf16_t *>(a.out) + ((size_t)mine.row * a.H + mine.head) * HD;
            bool odd = false, disturbed = false;
            for (int i = lane; i < HD; i += 32) odd |= !isfinite(mine.whole ? bf16_bits_to_float(out[i]) : a.o[slot * HD + i]);
            if (!__any_sync(0xffffffffu, odd)) continue;
            const int end = min(min(job.to, job.from + mine.steps * SUB), it.kv), hidden = max(mine.last + (TREE ? -63 : 1), job.from);
            const unsigned long long word = TREE ? a.seen[mine.row] : 0ull;
            for (int i = lane; i < (end - hidden) * PIECES; i += 32) {
                size_t k, v;
                if (TREE && tree_sees(word, mine.last - hidden - i / PIECES)) continue;
                if (!key_at<HD, PAGED>(a, it.b, it.r.row0, mine.head / (a.H / a.KV), hidden + i / PIECES, k, v)) continue;
                float y[8];
                read_values(static_cast<const bf16_t *>(a.v) + v + i % PIECES * 8, y);
#pragma unroll
                for (int j = 0; j < 8; ++j) disturbed |= !isfinite(y[j]);
            }
            if (__any_sync(0xffffffffu, disturbed))
                row_by_definition<HD, bf16_t, bf16_t, PAGED, TREE>(a, Row{it.b, it.r.row0, mine.row, mine.head, job.from, min(mine.last + 1, end), mine.whole, slot, mine.last});
        }
    } while (it.next(a) && it.start < x1);
}

// A wait of the block gave up: the rows of its run are NaN, those of cut items by their parts.
template <int HD> __device__ __noinline__ void spoil_rows(const Args &a, const Costs<NCOST> &costs, int w, long long x0, long long x1) {
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5, lane = threadIdx.x & 31;
    Item<true> it = item_at<true>(a, costs, x0);
    do {
        const Job job(a, it, x0, x1);
        for (int r = warp; r < ROWS; r += warps) {
            const int rr = r % HALF_ROWS;
            const Mine mine(a, it, job, r / HALF_ROWS, rr / a.gs < a.tb ? rr / a.gs : -1, rr % a.gs);
            if (mine.token < 0 || job.from >= job.to) continue;
            bf16_t *out = static_cast<bf16_t *>(a.out) + ((size_t)mine.row * a.H + mine.head) * HD;
            if (!mine.whole) {
                if (lane == 0) a.ml[((size_t)w * SLOTS + (job.from > 0 ? 0 : 1)) * ROWS + r] = make_float2(0.f, __int_as_float(0x7fffffff));
            } else {
                for (int i = lane; i < HD; i += 32) out[i] = 0x7fff;
            }
        }
    } while (it.next(a) && it.start < x1);
}

// K and V come from pages or from packed rows.
template <int HD, bool PAGED, bool TREE = false>
__global__ void __launch_bounds__(threads_of(PAGED), 1) tensor_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                                                        const __grid_constant__ CUtensorMap vmap) {
    using L = Lay<HD>;
    constexpr int GROUP = L::group(PAGED), NEXT_BAND = L::band(PAGED);
    extern __shared__ unsigned char raw[];
    __shared__ Costs<NCOST> costs;
    __shared__ uint64_t bars[2 + 2 + 2 * L::TILES + 4 + 4 + 4 + 2];    // s_full, p_full and o_full: [half][buffer]
    __shared__ uint32_t tmem_base;
    __shared__ volatile int quit, odd;                               // a wait gave up; some row is not finite
    __shared__ volatile unsigned info[INFO];                         // the 16-position groups of a step's tile that have a page
    __shared__ volatile unsigned filled[2];                          // tiles that a loader has filled its part of, when it is done
    const uint32_t smem = (smem_addr(raw) + 1023u) & ~1023u, q_tile = smem, ring = smem + 2 * L::TILE;
    const uint32_t q_full = smem_addr(bars), q_empty = q_full + 16, kv_full = q_empty + 16, kv_empty = kv_full + 8 * L::TILES, s_full = kv_empty + 8 * L::TILES,
                   p_full = s_full + 32, o_full = p_full + 32, all_done = o_full + 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        quit = odd = 0;
        for (int i = 0; i < 2; ++i) {
            bar_init(q_full + 8 * i, 1); bar_init(q_empty + 8 * i, 1); bar_init(all_done + 8 * i, 1);
            for (int b = 0; b < 2; ++b) { bar_init(o_full + 8 * (2 * i + b), 1); bar_init(s_full + 8 * (2 * i + b), 2); bar_init(p_full + 8 * (2 * i + b), 4); }
        }
        for (int i = 0; i < L::TILES; ++i) { bar_init(kv_full + 8 * i, loaders_of(PAGED)); bar_init(kv_empty + 8 * i, 2); }
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
    clear_others<bf16_t>(a, HD, blockIdx.x * blockDim.x + tid, gridDim.x * blockDim.x);
    const long long total = costs.pfx[NCOST];
    const int w = blockIdx.x, W = total > 0 ? workers_of(a, total) : 0;
    const long long x0 = w < W ? run_start(total, w, W) : 0, x1 = w < W ? run_start(total, w + 1, W) : 0;
    if (x0 >= x1) {
        if (tid == 0) { a.parts[w].first = 0; a.parts[w].start = -1; }
    } else {
        Item<true> it = item_at<true>(a, costs, x0);
        if (tid == 0) note_part<KEYS>(a, it, w, W, total, x0, x1);
        bool ok = true, more = true;

        if (warp == LOAD_WARP || warp >= MMA_WARP + 2) {
            // ---- copies ------------------------------------------------------------------------------------------------
            // By TMA: packed rows one copy for 64 dimensions of a tile; pages one copy for each of a tile's, two of the larger ones, shared out between two warps, since a copy takes the
            // issuing warp some 100 clocks: 64 requests of 16 rows over pages of 16 / 32 / 64 / 128 positions 134 / 128 / 126 / 124 us, by one warp 171 / 138 / 129 / 128, by 16-byte
            // copies of four warps 146 whatever the pages.  What has no page is not copied.
            const int loader = warp == LOAD_WARP ? 0 : 1;
            const uint32_t one = elect();
            unsigned fills = 0, slot = 0, turn_of = 0, qfills[2] = {0, 0}, step0 = 0;      // slot, turn_of: the ring's next tile
            const int piece = min(1 << a.page_shift, PIECE), pieces = KEYS / piece;
            int id = -1, next_id = -1;                               // pages: lane i: the page of piece i of the tile, of the one behind it
            auto page_of = [&](int j) {
                const int pos = j * KEYS + lane * piece;
                if (lane >= pieces || pos >= it.kv || (pos >> a.page_shift) >= a.max_pages) return -1;
                const int p = __ldg(a.table + (size_t)it.b * a.max_pages + (pos >> a.page_shift));
                return p < a.n_pages ? p : -1;
            };
            while (more && ok) {
                const Job job(a, it, x0, x1);
                // tiles in the order of their use (see the products)
                const bool own = job.paired && job.n[0] > 0 && job.n[1] > 0;
                const int T = job.tiles, total_tiles = (own ? 4 : 2) * T;
                if (PAGED && T) { id = page_of(job.j0); next_id = page_of(job.j0 + 1); }
                const int until = (int)min((unsigned)total_tiles, a.stop_after[loader] - fills);      // fewer in a test of the waits alone
#pragma unroll 1
                for (int i = 0; i < until && ok; ++i) {
                    // half i's q before tile i: the first K is on its way while q waits for the products of the item before
                    if (i < 2 && loader == 0 && (i ? job.n[1] : job.n[0]) > 0) {
                        ok = warp_wait(q_empty + 8 * i, (qfills[i] & 1) ^ 1, &quit, a, 202);
                        if (!ok) break;
                        const int vh = job.paired ? 2 * it.vh + i : it.vh, h0 = a.subs == 1 ? vh * a.gs : vh / a.subs * (a.H / a.KV) + vh % a.subs * a.gs;
                        const int row = it.r.row0 + it.rb * it.r.tb + (job.paired ? 0 : i * a.tb);
                        bar_expect_if(q_full + 8 * i, a.tb * a.gs * HD * 2, one);
#pragma unroll
                        for (int b = 0; b < L::BANDS; ++b) tma_3d(q_tile + i * L::TILE + b * BAND, &qmap, 64 * b, h0, row, q_full + 8 * i, one);
                        ++qfills[i];
                    }
                    bool is_k, second = false;
                    int t;
                    if (own) {
                        const int r = (i - 2) & 3;
                        t = (i - 2) >> 2;
                        const bool end = t == T - 1;                 // V of both halves, no K behind them
                        is_k = i < 2 || (!end && (r & 1));
                        second = i < 2 ? i == 1 : end ? r == 1 : r >= 2;
                        t = i < 2 ? 0 : t + is_k;
                    } else {
                        is_k = !(i & 1);
                        t = i >> 1;
                    }
                    const bool ahead = is_k && t > 0;                // K of the tile behind the one whose V goes by
                    ok = warp_wait(kv_empty + 8 * slot, (turn_of & 1) ^ 1, &quit, a, 201);
                    if (!ok) break;
                    const uint32_t dst = ring + slot * L::TILE, bar = kv_full + 8 * slot;
                    const int vh = job.paired ? 2 * it.vh + second : it.vh, kvh = a.subs == 1 ? vh : vh / a.subs;
                    const int page = ahead ? next_id : id;
                    const unsigned there = PAGED ? __ballot_sync(0xffffffffu, page >= 0) : 0u;
                    if (PAGED && is_k && !second && lane == 0 && loader == 0) {
                        unsigned groups = 0;
                        const unsigned each = (1u << (piece / 16)) - 1;
                        for (int g = 0; g < pieces; ++g)
                            if (there >> g & 1) groups |= each << (g * (piece / 16));
                        info[(step0 + t) % INFO] = groups;
                    }
                    if (PAGED && ahead && (second || !own)) { id = next_id; next_id = page_of(job.j0 + t + 1); }
                    const CUtensorMap *map = is_k ? &kmap : &vmap;
                    if (PAGED) {
                        __syncwarp();                                // behind the note: the arrival that goes with it hands it on
                        bar_expect_if(bar, __popc(there & (0x55555555u << loader)) * piece * HD * 2, one);
                        const int group = (((page * a.KV + kvh) << (a.page_shift - 3))) + ((((job.j0 + t) * KEYS + lane * piece) & ((1 << a.page_shift) - 1)) >> 3);
                        for (int g = loader; g < pieces; g += 2) tma_groups(dst + g * piece * HD * 2, map, __shfl_sync(0xffffffffu, group, g), bar, there >> g & one);
                    } else {
                        bar_expect_if(bar, L::TILE, one);
#pragma unroll
                        for (int b = 0; b < L::BANDS; ++b) tma_3d(dst + b * NEXT_BAND, map, 64 * b, kvh, it.r.row0 + (job.j0 + t) * KEYS, bar, one);
                    }
                    ++fills;
                    if (++slot == L::TILES) { slot = 0; ++turn_of; }
                }
                ok &= until == total_tiles;
                step0 += T;
                more = it.next(a) && it.start < x1;
            }
            if (PAGED) {                                             // where one loader gave up the other's tiles still have to be full: it arrives for those that it left out
                // (at most a turn of the ring: for a tile in a place for the second time the other has waited for its products, and they for both).  Their rows are lost.
                if (lane == 0) filled[loader] = fills;
                __syncwarp();
                asm volatile("bar.sync 1, 64;" ::: "memory");
                const unsigned all = max(filled[0], filled[1]);
                if (fills < all && lane == 0 && !quit) {
                    quit = 1;
                    atomicExch(a.err, 211);
                }
                for (; fills < all; ++fills)
                    if (lane == 0) bar_arrive(kv_full + 8 * (fills % L::TILES));
            }
            // every copy has landed and every product has let go of its tile before the block goes
            for (unsigned i = fills > L::TILES ? fills - L::TILES : 0; i < fills; ++i) {
                const unsigned slot = i % L::TILES, parity = i / L::TILES & 1;
                if (ok) ok = warp_wait(kv_empty + 8 * slot, parity, &quit, a, 203);
                if (!ok) bar_settle(kv_full + 8 * slot, parity);
            }
            for (int h = 0; h < 2; ++h)
                if (qfills[h]) {
                    if (ok) ok = warp_wait(q_empty + 8 * h, (qfills[h] - 1) & 1, &quit, a, 204);
                    if (!ok) bar_settle(q_full + 8 * h, (qfills[h] - 1) & 1);
                }
        } else if (warp >= MMA_WARP) {
            // ---- products ------------------------------------------------------------------------------------------------
            // A warp per half: its own instructions, some 150 a step next to 640 clocks of products, bound the loop where one warp served both.
            // Of the half two steps are under way: while the softmax works on one, the scores of the other are formed.
            constexpr uint32_t S_DESC = idesc_of(SUB, false), O_DESC = idesc_of(HD, true), SUB_STEP = SUB / 8 * GROUP >> 4;
            const int h = warp - MMA_WARP;
            const uint32_t q_desc = desc_of(q_tile + h * L::TILE, BAND), s_col = tmem + h * KEYS, o_col = tmem + O_COL + h * HD;
            const uint32_t my_s = s_full + 16 * h, my_p = p_full + 16 * h, my_o = o_full + 16 * h, my_q = q_full + 8 * h, my_q_empty = q_empty + 8 * h;
            unsigned slot = 0, phase = 0, q_phase = 0, step0 = 0;    // slot, phase: the ring's next tile
            unsigned sb = 0, vbuf = 0, p_phase = 0;                  // the buffers that scores go to and p comes from, p's phase
            // Either half goes through every tile of the ring, waits for it and lets it go, whether it has a use for it or not: a half that left the
            // other's tiles out could be a turn of the ring ahead, where a barrier's parity no longer tells one phase from the next.
            unsigned walked = 0;
            auto there = [&]() {
                if (ok) ok = warp_wait(kv_full + 8 * slot, phase, &quit, a, 205);
            };
            auto onward = [&]() {
                ++walked;
                if (++slot == L::TILES) { slot = 0; phase ^= 1; }
            };
            auto pass = [&](unsigned tiles) {
                for (; tiles > 0 && ok; --tiles) {
                    there();
                    if (ok && lane == 0) bar_arrive(kv_empty + 8 * slot);
                    onward();
                }
            };
            auto take = [&](uint32_t &tile, uint32_t &bar) {
                there();
                tile = ring + slot * L::TILE;
                bar = kv_empty + 8 * slot;
                onward();
            };
            // What lies behind the last position that the block sees, and what has no page, must be zero in V: its p is 0, and 0 times what happens
            // to lie there need not be.  (Where the halves share the tile both do it.)
            auto clean = [&](uint32_t v, int valid, unsigned groups) {
                for (int i = lane; i < KEYS * 8; i += 32) {
                    const int row = i >> 3;
                    if (row < valid && (groups >> (row >> 4) & 1)) continue;
#pragma unroll
                    for (int b = 0; b < L::BANDS; ++b)
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v + (row >> 3) * GROUP + b * NEXT_BAND + (i & 63) * 16), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            };
            while (more && ok) {
                const Job job(a, it, x0, x1);
                const int n = h ? job.n[1] : job.n[0], other = h ? job.n[0] : job.n[1], T = job.tiles;
                // Tiles come as K0 V0 K1 V1 .., where the halves have tiles of their own (A, B) as KA0 KB0 VA0 KA1 VB0 KB1 VA1 ..
                const bool own = job.paired && n > 0 && other > 0;
                walked = 0;
                uint32_t k = 0, k_bar = 0, v = 0, v_bar = 0;
                auto scores = [&](int u) {
                    if ((u & 1) == 0) {
                        if (own && h && u == 0) pass(1);
                        take(k, k_bar);
                    }
                    if (!ok) return;
                    const uint32_t bar = my_s + 8 * sb;
                    if (lane == 0) bar_arrive(bar);                  // hands on what the copies' warp noted of the tile
                    fence_after();
                    mma_scores<HD, PAGED>(s_col + sb * SUB, q_desc, desc_of(k, NEXT_BAND) + (u & 1) * SUB_STEP, S_DESC, bar);
                    sb ^= 1;
                    if (u + 1 == n) commit(my_q_empty);
                    if ((u & 1) || u + 1 == n) commit(k_bar);
                };
                if (n > 0) {
                    if (ok) ok = warp_wait(my_q, q_phase, &quit, a, 207);
                    q_phase ^= 1;
                    scores(0);
                    if (n > 1 && ok) scores(1);
                    for (int u = 0; u < n && ok; ++u) {
                        if ((u & 1) == 0) {
                            const int t = u >> 1;
                            if (own) pass(h ? (t == T - 1 ? 1 : 2) : (t == 0 ? 1 : 2));
                            take(v, v_bar);
                            const int valid = it.kv - (job.j0 + t) * KEYS;
                            const unsigned groups = PAGED ? info[(step0 + t) % INFO] : 0xffu;
                            if (ok && (valid < KEYS || groups != 0xffu)) clean(v, valid, groups);
                        }
                        if (ok) ok = warp_wait(my_p + 8 * vbuf, p_phase, &quit, a, 206);
                        if (!ok) break;
                        fence_after();
                        mma_values<HD, PAGED>(o_col, s_col + vbuf * SUB, desc_of(v, NEXT_BAND) + (u & 1) * SUB_STEP, O_DESC, u > 0, my_o + 8 * vbuf);
                        p_phase ^= vbuf;
                        vbuf ^= 1;
                        if ((u & 1) || u + 1 == n) commit(v_bar);
                        if (u + 2 < n) scores(u + 2);
                    }
                }
                pass((own ? 4 : 2) * T - walked);
                step0 += T;
                more = it.next(a) && it.start < x1;
            }
            // no product of this warp is at work when it leaves, whoever gave up
            commit(all_done + 8 * h);
            bar_settle(all_done + 8 * h, 0);
        } else {
            // ---- softmax ---------------------------------------------------------------------------------------------------
            const int h = warp >> 2, r = h * HALF_ROWS + (warp & 3) * 32 + lane;
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16), o_at = lanes + O_COL + h * HD;
            unsigned done = 0, step0 = 0;                            // steps of this half
            bool odd_rows = false;                                   // one of this thread's rows is not finite
            const int rr = r % HALF_ROWS, my_head = rr % a.gs, my_token = rr / a.gs < a.tb ? rr / a.gs : -1;      // as place_of
            while (more && ok) {
                const Job job(a, it, x0, x1);
                const Mine mine(a, it, job, h, my_token, my_head);
                const int token = mine.token, last = mine.last, row = mine.row * a.H + mine.head, steps = mine.steps;
                const int first_last = job.seen0 + (job.paired ? 0 : h * a.tb);
                const bool live = __any_sync(0xffffffffu, token >= 0);
                const unsigned long long word = TREE && token >= 0 ? __brevll(__ldg(a.seen + mine.row)) : 0ull;      // bit 63 - d: the position d before the row's own
                float m = -INFINITY, l = 0.f;
                for (int u = 0; u < steps && ok; ++u, ++done) {
                    const uint32_t bar = 8 * (2 * h + (done & 1)), s_at = lanes + h * KEYS + (done & 1) * SUB;
                    const int k0 = job.from + u * SUB;
                    ok = warp_wait(s_full + bar, done >> 1 & 1, &quit, a, 208);
                    if (!ok) break;
                    if (!live) {                                     // none of the warp's rows is anyone's: what is in P there stays there
                        __syncwarp();
                        if (lane == 0) bar_arrive(p_full + bar);
                        continue;
                    }
                    fence_after();
                    uint32_t x[2][32];
                    tmem_ld(s_at, x[0]);
                    tmem_ld(s_at + 32, x[1]);
                    wait_ld();
                    settle(x[0]);
                    settle(x[1]);
                    const unsigned groups = PAGED ? info[(step0 + (u >> 1)) % INFO] >> (4 * (u & 1)) & 15u : 15u;
                    if (k0 + SUB - 1 > first_last - (TREE ? 64 : 0) || groups != 15u) {            // what a row does not see is made -inf
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int n = last - k0 - 32 * c;        // the row sees keys 0 .. n of the 32
                            uint32_t seen = n >= 31 ? 0xffffffffu : n < 0 ? 0u : (2u << n) - 1;
                            if (TREE && n < 64 + 31) {               // some of the 32 are less than 64 positions before the row's own, or behind it
                                const int s = 63 - n;                // the word's bit of the first one
                                seen = s >= 64 ? 0u : s >= 0 ? (uint32_t)(word >> s) : (uint32_t)(word << -s) | ((1u << -s) - 1);
                            }
                            if (PAGED) seen &= ((groups >> (2 * c) & 1) ? 0xffffu : 0u) | ((groups >> (2 * c) & 2) ? 0xffff0000u : 0u);
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (!(seen >> i & 1)) x[c][i] = 0xff800000u;
                        }
                    }
                    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < SUB; i += 2) tops[(i >> 1) & 3] = max3(tops[(i >> 1) & 3], __uint_as_float(x[i >> 5][i & 31]), __uint_as_float(x[i >> 5][(i & 31) + 1]));
                    const float top = max3(max3(tops[0], tops[1], tops[2]), tops[3], tops[3]);
                    const float grown = top == -INFINITY ? -INFINITY : top * a.scale_log2;
                    const bool over = grown > m + GROWTH;            // the first positions a row sees: m is -inf
                    if (__any_sync(0xffffffffu, over)) {
                        const float f = over ? exp2_approx(m - grown) : 1.f;
                        if (over) { m = grown; l *= f; }
                        if (u > 0) {
                            ok = warp_wait(o_full + 8 * (2 * h + (done - 1 & 1)), (done - 1) >> 1 & 1, &quit, a, 209);
                            if (!ok) break;
                            fence_after();
#pragma unroll 1
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
                    // A score that is NaN or +inf makes the row NaN (inf - inf).  Its weight need not show it, the cubic has no NaN: l does, from here on.
                    if (!(top < INFINITY)) l = __int_as_float(0x7fffffff);
                    const float base = m == -INFINITY ? 0.f : m;
                    uint64_t sums[2] = {0, 0};
                    const uint64_t scale2 = pair_of(a.scale_log2, a.scale_log2), base2 = pair_of(-base, -base);
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < SUB; i += 2) {
                        const uint64_t e = fma2(pair_of(x[i >> 5][i & 31], x[i >> 5][(i & 31) + 1]), scale2, base2);
                        float y0, y1;
                        if ((i >> 1) % CUBIC_OF < CUBIC) {
                            exp2_cubic(e, y0, y1);
                        } else {
                            split(e, y0, y1);
                            y0 = exp2_approx(y0);
                            y1 = exp2_approx(y1);
                        }
                        sums[(i >> 1) & 1] = add2(sums[(i >> 1) & 1], pair_of(y0, y1));
                        p[i >> 1] = cvt_bf16x2(y0, y1);
                    }
                    tmem_st(s_at, p);
                    float sum0, sum1;
                    split(add2(sums[0], sums[1]), sum0, sum1);
                    l += sum0 + sum1;
                    wait_st();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(p_full + bar);
                }
                if (!ok) break;
                // ---- the rows' ends
                const bool whole = mine.whole;
                if (steps) {
                    ok = warp_wait(o_full + 8 * (2 * h + (done - 1 & 1)), (done - 1) >> 1 & 1, &quit, a, 210);
                    if (!ok) break;
                    fence_after();
                }
                if (live && (steps || (job.from < job.to && !whole))) {
                    const bool none = m == -INFINITY && l == l;      // the row has seen nothing
                    if (none) l = 0.f;
                    const float f = none ? 0.f : whole ? __fdividef(1.0f, l) : 1.f;
                    const size_t slot = ((size_t)w * SLOTS + (job.from > 0 ? 0 : 1)) * ROWS;
                    // Lane 4 i + j takes the j-th 16 bytes of each of the rows 4 i .. 4 i + 3: a store of the warp is eight runs of 64 bytes, where a row
                    // per lane is 32 half sectors (the end of an item took 9000 clocks, its stores in the way of the other warps').
                    int at[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        at[i] = __shfl_sync(0xffffffffu, whole ? row : r, (lane & ~3) + i);
                        if (__shfl_sync(0xffffffffu, token, (lane & ~3) + i) < 0) at[i] = -1;
                    }
                    float bad[2] = {0.f, 0.f};                       // 0 times the sums: not 0 where one is not finite
#pragma unroll 1
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t o[32];
                        if (steps) {
                            tmem_ld(o_at + 32 * c, o);
                            wait_ld();
                            settle(o);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = 0u;
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) bad[i & 1] = fmaf(__uint_as_float(o[i]), 0.f, bad[i & 1]);
                        if (whole) {
                            uint4 v[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t *p = o + 8 * i;
                                v[i].x = cvt_bf16x2(__uint_as_float(p[0]) * f, __uint_as_float(p[1]) * f);
                                v[i].y = cvt_bf16x2(__uint_as_float(p[2]) * f, __uint_as_float(p[3]) * f);
                                v[i].z = cvt_bf16x2(__uint_as_float(p[4]) * f, __uint_as_float(p[5]) * f);
                                v[i].w = cvt_bf16x2(__uint_as_float(p[6]) * f, __uint_as_float(p[7]) * f);
                            }
                            turn4(v, lane);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (at[i] >= 0) *reinterpret_cast<uint4 *>(static_cast<bf16_t *>(a.out) + (size_t)at[i] * HD + 32 * c + 8 * (lane & 3)) = v[i];
                        } else {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                uint4 v[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = make_uint4(o[16 * e + 4 * i], o[16 * e + 4 * i + 1], o[16 * e + 4 * i + 2], o[16 * e + 4 * i + 3]);
                                turn4(v, lane);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (at[i] >= 0) *reinterpret_cast<uint4 *>(a.o + (slot + at[i]) * HD + 32 * c + 16 * e + 4 * (lane & 3)) = v[i];
                            }
                        }
                    }
                    if (token >= 0 && !whole) a.ml[slot + r] = make_float2(m, l);
                    odd_rows |= token >= 0 && bad[0] + bad[1] != 0.f;
                    fence_before();
                }
                step0 += job.tiles;
                more = it.next(a) && it.start < x1;
            }
            if (odd_rows) odd = 1;
        }
        fence_before();
    }
    __syncthreads();
    if (warp == MMA_WARP) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
    if (quit) spoil_rows<HD>(a, costs, w, x0, x1);
    else if (odd) mend_rows<HD, PAGED, TREE>(a, costs, w, x0, x1);
}

}  // namespace tcattn
}  // namespace knnssd
