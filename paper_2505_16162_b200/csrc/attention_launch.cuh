// Host side that the attention operators share: checks of arguments and the launches of their kernels.
#pragma once

#include "../../include/knnssd.h"
#include "host_common.cuh"
#include "row_attention.cuh"
#include "tensor_attention.cuh"
#include "tensor_maps.cuh"
#include "tree_rows.cuh"

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstdint>

namespace knnssd {

// The word of the current device that the bounded waits of the tensor-core attention report to, until knnssd_attention_status takes it.
int *attention_err_ptr();
// What knnssd_debug_attention_timeout sets: polls of a wait, tiles that the copies of a block's first and second copying warp end after.
extern std::atomic<unsigned> g_wait_limit, g_stop_after[2];

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }

inline knnssd_status launched() { return cudaGetLastError() == cudaSuccess ? KNNSSD_OK : KNNSSD_ERR_CUDA; }

// Dynamic shared memory of a kernel on the current device, set once per device.
template <typename K> bool allow_smem(K kernel, int bytes, bool (&done)[kMaxDevices]) {
    const int dev = current_device_slot();
    if (done[dev]) return true;
    const ApartFromCapture apart;
    done[dev] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    return done[dev];
}

// The parts of items that `workers` of a launch may leave, `rows` rows each: one piece of scratch.
inline bool get_parts(Scratch &mem, attn::Args &a, int workers, int rows, int hd) {
    const size_t slots = (size_t)workers * attn::SLOTS * rows, o_bytes = slots * hd * sizeof(float), ml_bytes = slots * sizeof(float2);
    unsigned char *p = nullptr;
    if (!mem.get(&p, o_bytes + ml_bytes + (size_t)workers * sizeof(attn::Part))) return false;
    a.o = reinterpret_cast<float *>(p);
    a.ml = reinterpret_cast<float2 *>(p + o_bytes);
    a.parts = reinterpret_cast<attn::Part *>(p + o_bytes + ml_bytes);
    return true;
}

// Rows that share a K/V head, up to `most` of them a block's: a.gs of its heads, a.subs blocks for all of them, a.tb new rows.
inline void share_heads(attn::Args &a, int most) {
    const int G = a.H / a.KV;
    a.gs = (G + (G + most - 1) / most - 1) / ((G + most - 1) / most);
    a.subs = (G + a.gs - 1) / a.gs;
    a.nvh = a.KV * a.subs;
    a.tb = most / a.gs;
}

template <int HD, typename KT, bool PAGED, bool TREE = false> knnssd_status launch_rows(attn::Args a, cudaStream_t s) {
    using Rg = rowattn::Ring<HD, KT>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = rowattn::rows_kernel<HD, KT, PAGED, TREE>;
    if (!allow_smem(kernel, Rg::SMEM, configured)) return KNNSSD_ERR_CUDA;
    constexpr int most = 16;
    share_heads(a, most);
    // An item's beginning and end in positions, and what a warp takes at least: extra 0 / 64 / 256: 9 prompts of 3001 tokens 50 / 42 / 55 us, 8 requests
    // of 5 new rows 56 / 58 / 66; least_run 16 / 32 / 64 / 256: 2 requests of 1851 positions 33 / 24 / 22 / -, one of 96 15 / 15 / 15 / 29.
    a.extra = 64;
    a.least_run = 64;
    // Parts an item may be in, on average over the call's items, as the merge takes them 32 at a time: at most 32 / 64 / 128 / any number (296): one request
    // of 31 009 positions 85 / 51 / 40 / 56 us, two of 74 011 205 / 119 / 87 / 105.  A long item beside short ones is in more, up to all workers: 31 009
    // positions and 40 times 100, 8 heads on one of K/V, 85 us for 41 alone; 4 heads of their own 31 for 35.  A bound by the longest item instead (41, 41)
    // cost short prompts 4 % for the search.
    const int ctas = sm_count();
    a.most = (int)std::min((long long)ctas * Rg::WARPS, 128ll * a.nvh * std::max(a.B, a.R / a.tb));
    Scratch mem(s);
    if (!get_parts(mem, a, a.most, most, HD)) return KNNSSD_ERR_CUDA;
    launch_chained(kernel, dim3(ctas), dim3(Rg::WARPS * 32), Rg::SMEM, s, a);
    launch_chained(attn::merge_kernel<HD, float, false, 16>, dim3(a.most - 1, (a.tb * a.gs + 7) / 8), dim3(256), 0, s, a);
    return launched();
}

// most_rows: the rows that a request is believed to have at most.
template <int HD, bool PAGED, bool TREE = false> knnssd_status launch_tensor(attn::Args a, int most_rows, cudaStream_t s) {
    using L = tcattn::Lay<HD>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = tcattn::tensor_kernel<HD, PAGED, TREE>;
    a.err = attention_err_ptr();
    a.wait_limit = g_wait_limit; a.stop_after[0] = g_stop_after[0]; a.stop_after[1] = g_stop_after[1];
    if (!a.err || !allow_smem(kernel, L::SMEM, configured)) return KNNSSD_ERR_CUDA;
    share_heads(a, tcattn::HALF_ROWS);
    const int ctas = sm_count();
    // An item's beginning and end cost a CTA some 5 to 8 thousand clocks, as much as these positions: with 0 / 384 / 1024, 24 short prompts take
    // 88 / 34 / 33 us and 12000 tokens in 4 prompts 935 / 709 / 750.
    a.extra = 384;
    // What a CTA takes at least: with 64 / 512 / 2048, 6 requests of 13 thousand positions take 33 / 32 / 42 us, 24 short prompts 34 / 34 / 39.
    a.least_run = 512;
    // Two heads a block where there are items enough for all CTAs either way: half as many beginnings and ends, half as many pieces.  1440 items
    // of one row 44 -> 33 us, 768 of about 100 rows 43 -> 35, 512 of one row and 200 positions 46 -> 43; but 16 of 35 thousand positions 35 -> 45,
    // 128 of 50 positions 22 -> 25.  One answer for the call: a head's positions cost a pair twice the reading, and a mix of both is uneven.
    a.most = ctas;
    a.pair = (long long)a.B * a.nvh >= 2ll * ctas;
    CUtensorMap qm{}, km{}, vm{};
    const cuuint64_t qs[3] = {HD, (cuuint64_t)a.H, (cuuint64_t)a.R}, qst[2] = {HD * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t qb[3] = {64, (cuuint32_t)a.gs, (cuuint32_t)a.tb};
    bool made = bf16_map(&qm, a.q, 3, qs, qst, qb);
    if (PAGED) {                                                     // groups of eight rows, the rows' 64 dimensions apart from one another
        const int page = 1 << a.page_shift;
        const cuuint64_t ks[4] = {64, 8, HD / 64, (cuuint64_t)a.n_pages * a.KV * page / 8}, kst[3] = {HD * 2, 128, HD * 16};
        const cuuint32_t kb[4] = {64, 8, HD / 64, (cuuint32_t)(page < tcattn::PIECE ? page : tcattn::PIECE) / 8};
        made = made && bf16_map(&km, a.k, 4, ks, kst, kb) && bf16_map(&vm, a.v, 4, ks, kst, kb);
    } else {
        const cuuint64_t ks[3] = {HD, (cuuint64_t)a.KV, (cuuint64_t)a.R}, kst[2] = {HD * 2, (cuuint64_t)a.k_stride * 2}, vst[2] = {HD * 2, (cuuint64_t)a.v_stride * 2};
        const cuuint32_t kb[3] = {64, 1, tcattn::KEYS};
        made = made && bf16_map(&km, a.k, 3, ks, kst, kb) && bf16_map(&vm, a.v, 3, ks, vst, kb);
    }
    if (!made) return KNNSSD_ERR_CUDA;
    Scratch mem(s);
    if (!get_parts(mem, a, ctas, tcattn::ROWS, HD)) return KNNSSD_ERR_CUDA;
    launch_chained(kernel, dim3(ctas), dim3(tcattn::threads_of(PAGED)), L::SMEM, s, a, qm, km, vm);
    launch_chained(attn::merge_kernel<HD, bf16_t, true, tcattn::ROWS>, dim3(ctas - 1, 2 * ((std::min(a.tb, most_rows) * a.gs + 7) / 8)), dim3(256), 0, s, a);
    return launched();
}

// Trees over short contexts: whether a block for 16 rows and all positions that the table has room for is the sooner way, and with how many warps (0: it is not), by microseconds that were
// measured.
// bf16 pages: a block of eight warps, one a processor at a time, takes 3 and, for 128 positions of 128 dimensions, 0.8 (bf16 rows) or 1.45 (fp32); of four warps, two a processor, 3.5 and
// 2.2 times that.  The ways that share positions out take 16 to 20 whatever the sizes and then some 7 GB of pages a millisecond.  8 / 4 warps / shared out: one request of 48
// rows, 32 bf16 heads and 300 positions 10 / 14 / 24 us, 8 requests of 12 rows 18 / 14 / 34; 32 requests of 60 positions 36 / - / 30.
// fp32 pages: always eight warps; 1 and, for each round of blocks (between their number a processor and that rounded up, as processors end apart), 2 and 2.4 for 128 positions of
// 128 dimensions, 0.7 of that for 64.  Shared out 23 (64 dimensions: 16) and 1.5 a block of a processor for the same.  Over 1500 calls of 1 to 90 requests, tables of 32 to 2048 positions, full
// or not, the way taken is 1.3 to 2 % longer than the sooner one, where it is short and not at most 1.4 times, where it is shared out and hardly filled 1.7 times as long.  From two blocks a
// processor on the two are within 5 % of one another on average (8 requests of 25 rows, 40 heads, 1280 positions 174 / 191: shared out).  Whole / shared out: 22 requests of 64 rows, 8 heads on 2 of 64 dimensions, 80 positions 22 / 24 us; 3 of 48,
// 32 heads on 4, 480 positions 35 / 44; 1 of 8, 40 heads, 1472 positions 42 / 27; 5 of 2, 32 heads, 1424 positions 88 / 68.
inline int short_warps(attn::Args a, int dtype, int cache_dtype, int hd) {
    share_heads(a, treerows::ROWS);
    const long long positions = (long long)a.max_pages << a.page_shift, tiles = (long long)a.R / a.tb + a.B;
    const double blocks = (double)tiles * a.nvh / sm_count();
    if (blocks > 8.0 || positions > 2048) return 0;                  // beyond what the figures are of
    if (cache_dtype == 0) {
        const double part = (hd == 64 ? 0.7 : 1.0) * positions / 128.0, rounds = (std::ceil(blocks) + std::max(1.0, blocks)) / 2;
        return 1.0 + rounds * (2.0 + 2.4 * part) < (hd == 64 ? 16.0 : 23.0) + 1.5 * blocks * part ? 8 : 0;
    }
    const double step = hd / 128.0 * (dtype == 0 ? 1.45 : 0.8) * positions / 128.0;
    const double eight = 3.0 + std::ceil(blocks) * (3.0 + step), four = 3.0 + std::max(1.0, blocks / 2) * (3.5 + 2.2 * step);
    const double shared = (dtype == 0 && hd == 64 ? 16.0 : 20.0) + (double)a.B * a.KV * positions * hd * 4.0 / 7e6;
    if (std::min(eight, four) >= shared) return 0;
    return eight <= four ? 8 : 4;
}
template <int HD, typename QT, typename KT, int W> knnssd_status launch_short_of(attn::Args a, cudaStream_t s) {
    using L = treerows::Lay<HD, QT, KT, W>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = treerows::tree_rows_kernel<HD, QT, KT, W>;
    if (!allow_smem(kernel, L::SMEM, configured)) return KNNSSD_ERR_CUDA;
    share_heads(a, treerows::ROWS);
    launch_chained(kernel, dim3(a.nvh, a.R / a.tb + a.B), dim3(L::NT), L::SMEM, s, a);
    return launched();
}
template <int HD> knnssd_status launch_short(const attn::Args &a, int dtype, int cache_dtype, int warps, cudaStream_t s) {
    if (cache_dtype == 0) return launch_short_of<HD, float, float, 8>(a, s);
    if (dtype == 0) return warps == 8 ? launch_short_of<HD, float, bf16_t, 8>(a, s) : launch_short_of<HD, float, bf16_t, 4>(a, s);
    return warps == 8 ? launch_short_of<HD, bf16_t, bf16_t, 8>(a, s) : launch_short_of<HD, bf16_t, bf16_t, 4>(a, s);
}
template <int HD> knnssd_status launch_tree_rows(attn::Args a, cudaStream_t s) {
    using L = treerows::Lay<HD, float, float, 0>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = treerows::tree_rows_kernel<HD, float, float, 0>;
    if (!allow_smem(kernel, L::SMEM, configured)) return KNNSSD_ERR_CUDA;
    share_heads(a, treerows::ROWS);
    // As above.  extra 0 / 64 / 128 / 256 / 512: 24 requests of 13 rows and 300 to 1700 positions 202 / 193 / 186 / 189 / 204 us, 32 of 6 and 100 to 700 161 / 131 / 124 / 132 / 142, one of 25
    // and 8000 126 / 122 / 122 / 122 / 127; least_run 64 / 128 / 256 / 512: one of 1 row and 3000 36 / 36 / 36 / 46, 3 of 48 and 900 38 / 38 / 38 / 42, two of 13 and 200 and 90 in a wide table
    // 13 / 15 / 18 / 24 (short_warps' figures of the shared-out way are of 256), the others the same.
    a.extra = 128;
    a.least_run = 256;
    a.most = (int)std::min((long long)L::BLOCKS * sm_count(), 128ll * a.nvh * std::max(a.B, a.R / a.tb));
    Scratch mem(s);
    if (!get_parts(mem, a, a.most, treerows::ROWS, HD)) return KNNSSD_ERR_CUDA;
    launch_chained(kernel, dim3(a.most), dim3(L::NT), L::SMEM, s, a);
    launch_chained(attn::merge_kernel<HD, float, false, treerows::ROWS>, dim3(a.most - 1, (a.tb * a.gs + 7) / 8), dim3(256), 0, s, a);
    return launched();
}

// The scale of scores in powers of two.  A scale of zero (equal weights) is taken as next to nothing: what a row does not see is -inf times it.
inline float log2_scale(float scale) { return scale > 1e-36f ? scale * 1.4426950408889634f : 1e-36f; }

// Types and head counts that the attention operators and the store share.
inline knnssd_status check_heads(int dtype, int cache_dtype, int n_heads, int n_kv_heads, int head_dim) {
    if ((dtype != 0 && dtype != 1) || (cache_dtype != 0 && cache_dtype != 1) || n_heads < 1 || n_kv_heads < 1) return KNNSSD_ERR_INVALID_ARG;
    if ((dtype == 1 && cache_dtype == 0) || (head_dim != 64 && head_dim != 128) || n_heads % n_kv_heads != 0 || n_heads > 65535) return KNNSSD_ERR_SHAPE;
    return KNNSSD_OK;
}
inline knnssd_status check_pages(int page_size, int max_pages, int n_pages) {
    if (page_size < 1 || max_pages < 1 || n_pages < 1) return KNNSSD_ERR_INVALID_ARG;
    if (page_size < 16 || !power_of_two(page_size)) return KNNSSD_ERR_SHAPE;
    if ((long long)(max_pages + 1ll) * page_size > INT_MAX / 2 || (long long)n_pages * page_size > INT_MAX) return KNNSSD_ERR_CAPACITY;
    return KNNSSD_OK;
}

// Attention of new rows over pages, its arguments checked; seen_dev: trees, else nullptr.
template <bool TREE>
knnssd_status paged_attention(const void *q_dev, int dtype, int n_rows, long long q_stride, int n_heads, int n_kv_heads, int head_dim, const void *k_pages_dev,
                              const void *v_pages_dev, int cache_dtype, int page_size, int n_pages, const int *table_dev, int max_pages, const int *lens_dev,
                              const int *row_start_dev, const unsigned long long *seen_dev, int n_requests, int max_fresh, float scale, void *out_dev, void *cuda_stream) {
    if (n_rows < 0 || n_requests < 1 || max_fresh < 0 || !std::isfinite(scale) || scale < 0.f) return KNNSSD_ERR_INVALID_ARG;
    if (knnssd_status st = check_heads(dtype, cache_dtype, n_heads, n_kv_heads, head_dim); st != KNNSSD_OK) return st;
    if (knnssd_status st = check_pages(page_size, max_pages, n_pages); st != KNNSSD_OK) return st;
    if (n_rows > INT_MAX / 2 || (long long)n_rows * n_heads > INT_MAX) return KNNSSD_ERR_CAPACITY;
    if (n_rows == 0) return KNNSSD_OK;
    if (!q_dev || !k_pages_dev || !v_pages_dev || !table_dev || !lens_dev || !row_start_dev || (TREE && !seen_dev) || !out_dev) return KNNSSD_ERR_INVALID_ARG;
    if (q_stride < (long long)n_heads * head_dim || q_stride % (dtype ? 8 : 4) != 0 || !aligned16(q_dev) || !aligned16(k_pages_dev) || !aligned16(v_pages_dev) || !aligned16(out_dev) ||
        (TREE && (reinterpret_cast<uintptr_t>(seen_dev) & 7u)))
        return KNNSSD_ERR_SHAPE;
    attn::Args a{};
    a.q = q_dev; a.out = out_dev; a.q_stride = q_stride;
    a.k = k_pages_dev; a.v = v_pages_dev;
    a.table = table_dev; a.max_pages = max_pages; a.n_pages = n_pages;
    while ((1 << a.page_shift) < page_size) ++a.page_shift;
    a.lens = lens_dev; a.row_start = row_start_dev; a.B = n_requests; a.R = n_rows; a.H = n_heads; a.KV = n_kv_heads;
    a.scale_log2 = log2_scale(scale);
    a.seen = seen_dev;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    try {
        if constexpr (TREE)
            if (const int warps = short_warps(a, dtype, cache_dtype, head_dim))
                return head_dim == 128 ? launch_short<128>(a, dtype, cache_dtype, warps, s) : launch_short<64>(a, dtype, cache_dtype, warps, s);
        if (dtype == 1) {
            const int most_rows = max_fresh > 0 ? std::min(max_fresh, a.R) : a.R;
            // a coordinate of the copies, eight rows, has 31 bits
            if ((long long)n_pages * n_kv_heads > INT_MAX / (page_size / 8)) return KNNSSD_ERR_CAPACITY;
            return head_dim == 128 ? launch_tensor<128, true, TREE>(a, most_rows, s) : launch_tensor<64, true, TREE>(a, most_rows, s);
        }
        if constexpr (TREE)
            if (cache_dtype == 0) return head_dim == 128 ? launch_tree_rows<128>(a, s) : launch_tree_rows<64>(a, s);
        if (head_dim == 128) return cache_dtype == 0 ? launch_rows<128, float, true>(a, s) : launch_rows<128, bf16_t, true, TREE>(a, s);
        return cache_dtype == 0 ? launch_rows<64, float, true>(a, s) : launch_rows<64, bf16_t, true, TREE>(a, s);
    } catch (...) { return KNNSSD_ERR_CUDA; }
}

}  // namespace knnssd
