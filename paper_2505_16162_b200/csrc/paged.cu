// Host side of the operators for many requests on one paged K/V cache: block tables and slot maps, rotary embedding into pages, attention
// of new rows over pages, attention over packed prompts.  The C ABI is declared in include/knnssd.h.
#include "../../include/knnssd.h"
#include "host_common.cuh"
#include "page_tables.cuh"
#include "row_attention.cuh"
#include "tensor_attention.cuh"
#include "tensor_maps.cuh"

#include <atomic>
#include <climits>
#include <cmath>
#include <cstdint>

using namespace knnssd;

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }

knnssd_status launched() { return cudaGetLastError() == cudaSuccess ? KNNSSD_OK : KNNSSD_ERR_CUDA; }

// Dynamic shared memory of a kernel on the current device, set once per device.
template <typename K> bool allow_smem(K kernel, int bytes, bool (&done)[kMaxDevices]) {
    const int dev = current_device_slot();
    if (done[dev]) return true;
    const ApartFromCapture apart;
    done[dev] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    return done[dev];
}

// The parts of items that `workers` of a launch may leave, `rows` rows each: one piece of scratch.
bool get_parts(Scratch &mem, attn::Args &a, int workers, int rows, int hd) {
    const size_t slots = (size_t)workers * attn::SLOTS * rows, o_bytes = slots * hd * sizeof(float), ml_bytes = slots * sizeof(float2);
    unsigned char *p = nullptr;
    if (!mem.get(&p, o_bytes + ml_bytes + (size_t)workers * sizeof(attn::Part))) return false;
    a.o = reinterpret_cast<float *>(p);
    a.ml = reinterpret_cast<float2 *>(p + o_bytes);
    a.parts = reinterpret_cast<attn::Part *>(p + o_bytes + ml_bytes);
    return true;
}

template <int HD, typename KT, bool PAGED> knnssd_status launch_rows(attn::Args a, cudaStream_t s) {
    using Rg = rowattn::Ring<HD, KT>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = rowattn::rows_kernel<HD, KT, PAGED>;
    if (!allow_smem(kernel, Rg::SMEM, configured)) return KNNSSD_ERR_CUDA;
    const int G = a.H / a.KV, most = 16;
    a.gs = (G + (G + most - 1) / most - 1) / ((G + most - 1) / most);
    a.subs = (G + a.gs - 1) / a.gs;
    a.nvh = a.KV * a.subs;
    a.tb = most / a.gs;
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

// The word of the current device that the bounded waits of the tensor-core attention report to, until knnssd_attention_status takes it.
__device__ int g_attention_err;
int *attention_err_ptr() {
    static int *addr[kMaxDevices] = {};
    static std::mutex mu;
    const int dev = current_device_slot();
    std::lock_guard<std::mutex> lock(mu);
    if (!addr[dev]) {
        const ApartFromCapture apart;
        cudaGetSymbolAddress(reinterpret_cast<void **>(&addr[dev]), g_attention_err);
    }
    return addr[dev];
}
__global__ void take_word_kernel(int *word, int *to) { *to = atomicExch(word, 0); }

// What knnssd_debug_attention_timeout sets: polls of a wait, tiles that a block's copies end after.
std::atomic<unsigned> g_wait_limit{tcattn::WAIT_LIMIT}, g_stop_after{~0u};

// most_rows: the rows that a request is believed to have at most.
template <int HD, int MODE> knnssd_status launch_tensor(attn::Args a, int most_rows, cudaStream_t s) {
    using L = tcattn::Lay<HD>;
    static bool configured[kMaxDevices] = {};
    const auto kernel = tcattn::tensor_kernel<HD, MODE>;
    a.err = attention_err_ptr();
    a.wait_limit = g_wait_limit; a.stop_after = g_stop_after;
    if (!a.err || !allow_smem(kernel, L::SMEM, configured)) return KNNSSD_ERR_CUDA;
    const int G = a.H / a.KV, most = tcattn::HALF_ROWS;
    a.gs = (G + (G + most - 1) / most - 1) / ((G + most - 1) / most);
    a.subs = (G + a.gs - 1) / a.gs;
    a.nvh = a.KV * a.subs;
    a.tb = most / a.gs;
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
    if (MODE == tcattn::TILED) {
        const int page = 1 << a.page_shift;
        const cuuint64_t ks[2] = {HD, (cuuint64_t)a.n_pages * a.KV * page}, kst[1] = {HD * 2};
        const cuuint32_t kb[2] = {64, (cuuint32_t)(page < tcattn::KEYS ? page : tcattn::KEYS)};
        made = made && bf16_map(&km, a.k, 2, ks, kst, kb) && bf16_map(&vm, a.v, 2, ks, kst, kb);
    } else if (MODE == tcattn::PACKED) {
        const cuuint64_t ks[3] = {HD, (cuuint64_t)a.KV, (cuuint64_t)a.R}, kst[2] = {HD * 2, (cuuint64_t)a.k_stride * 2}, vst[2] = {HD * 2, (cuuint64_t)a.v_stride * 2};
        const cuuint32_t kb[3] = {64, 1, tcattn::KEYS};
        made = made && bf16_map(&km, a.k, 3, ks, kst, kb) && bf16_map(&vm, a.v, 3, ks, vst, kb);
    }
    if (!made) return KNNSSD_ERR_CUDA;
    Scratch mem(s);
    if (!get_parts(mem, a, ctas, tcattn::ROWS, HD)) return KNNSSD_ERR_CUDA;
    launch_chained(kernel, dim3(ctas), dim3(tcattn::threads_of(MODE == tcattn::COPIED)), L::SMEM, s, a, qm, km, vm);
    launch_chained(attn::merge_kernel<HD, bf16_t, true, tcattn::ROWS>, dim3(ctas - 1, 2 * ((std::min(a.tb, most_rows) * a.gs + 7) / 8)), dim3(256), 0, s, a);
    return launched();
}

template <int HD> knnssd_status launch_paged_rows(const attn::Args &a, int cache_dtype, cudaStream_t s) {
    return cache_dtype == 0 ? launch_rows<HD, float, true>(a, s) : launch_rows<HD, bf16_t, true>(a, s);
}

template <int HD> void launch_rotary(const pages::RotaryArgs &a, int dtype, int cache_dtype, cudaStream_t s) {
    const dim3 grid(a.n_rows), block(a.n_rows > pages::ROT_ROWS ? pages::ROT_FEW : pages::ROT_MANY);
    if (dtype == 1) launch_chained(pages::rotary_store_kernel<HD, bf16_t, bf16_t>, grid, block, 0, s, a);
    else if (cache_dtype == 1) launch_chained(pages::rotary_store_kernel<HD, float, bf16_t>, grid, block, 0, s, a);
    else launch_chained(pages::rotary_store_kernel<HD, float, float>, grid, block, 0, s, a);
}

// The scale of scores in powers of two.  A scale of zero (equal weights) is taken as next to nothing: what a row does not see is -inf times it.
float log2_scale(float scale) { return scale > 1e-36f ? scale * 1.4426950408889634f : 1e-36f; }

// Types and head counts that the attention operators and the store share.
knnssd_status check_heads(int dtype, int cache_dtype, int n_heads, int n_kv_heads, int head_dim) {
    if ((dtype != 0 && dtype != 1) || (cache_dtype != 0 && cache_dtype != 1) || n_heads < 1 || n_kv_heads < 1) return KNNSSD_ERR_INVALID_ARG;
    if ((dtype == 1 && cache_dtype == 0) || (head_dim != 64 && head_dim != 128) || n_heads % n_kv_heads != 0 || n_heads > 65535) return KNNSSD_ERR_SHAPE;
    return KNNSSD_OK;
}
knnssd_status check_pages(int page_size, int max_pages, int n_pages) {
    if (page_size < 1 || max_pages < 1 || n_pages < 1) return KNNSSD_ERR_INVALID_ARG;
    if (page_size < 16 || !power_of_two(page_size)) return KNNSSD_ERR_SHAPE;
    if ((long long)(max_pages + 1ll) * page_size > INT_MAX / 2 || (long long)n_pages * page_size > INT_MAX) return KNNSSD_ERR_CAPACITY;
    return KNNSSD_OK;
}

}  // namespace

extern "C" {

knnssd_status knnssd_page_tables(const int *lens_dev, const int *fresh_dev, int n_requests, int page_size, int max_pages, int n_pages, int *owned_dev, int *table_dev,
                                 int *free_pages_dev, int *free_count_dev, int max_rows, int *row_start_dev, int *row_request_dev, int *row_pos_dev, int *row_slot_dev,
                                 int *info_dev, void *cuda_stream) {
    if (!lens_dev || !fresh_dev || !owned_dev || !table_dev || !free_pages_dev || !free_count_dev || !row_start_dev || !info_dev || n_requests < 1 || max_rows < 0 ||
        (max_rows > 0 && (!row_request_dev || !row_pos_dev || !row_slot_dev)))
        return KNNSSD_ERR_INVALID_ARG;
    if (const knnssd_status st = check_pages(page_size, max_pages, n_pages); st != KNNSSD_OK) return st;
    if (n_requests > pages::MAX_REQUESTS || (long long)n_requests * max_pages > INT_MAX) return KNNSSD_ERR_CAPACITY;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    static bool configured[kMaxDevices] = {};
    if (!allow_smem(pages::plan_kernel, pages::plan_smem(pages::MAX_REQUESTS), configured)) return KNNSSD_ERR_CUDA;
    pages::PlanArgs a{lens_dev, fresh_dev, n_requests, page_size, max_pages, n_pages, owned_dev, table_dev, free_pages_dev, free_count_dev, max_rows,
                      row_start_dev, row_request_dev, row_pos_dev, row_slot_dev, info_dev, max_rows <= pages::ROWS_HERE};
    launch_chained(pages::plan_kernel, dim3(1), dim3(pages::NT), pages::plan_smem(n_requests), s, a);
    if (!a.rows_here) launch_chained(pages::map_rows_kernel, dim3((max_rows + pages::ROWS_NT - 1) / pages::ROWS_NT), dim3(pages::ROWS_NT), 0, s, a);
    return launched();
}

knnssd_status knnssd_rotary_store(const void *qkv_dev, int dtype, int n_rows, long long row_stride, int n_heads, int n_kv_heads, int head_dim, const float *cos_sin_dev,
                                  int n_positions, const int *row_pos_dev, const int *row_slot_dev, int page_size, int n_pages, void *q_dev,
                                  void *k_rows_dev, void *k_pages_dev, void *v_pages_dev, int cache_dtype, void *cuda_stream) {
    if (n_rows < 0 || n_positions < 1) return KNNSSD_ERR_INVALID_ARG;
    if (knnssd_status st = check_heads(dtype, cache_dtype, n_heads, n_kv_heads, head_dim); st != KNNSSD_OK) return st;
    if (knnssd_status st = check_pages(page_size, 1, n_pages); st != KNNSSD_OK) return st;
    if (n_rows == 0) return KNNSSD_OK;
    if (!qkv_dev || !cos_sin_dev || !row_pos_dev || !row_slot_dev || !q_dev || !k_pages_dev || !v_pages_dev) return KNNSSD_ERR_INVALID_ARG;
    const long long width = ((long long)n_heads + 2ll * n_kv_heads) * head_dim;
    if (row_stride < width || row_stride % (dtype ? 8 : 4) != 0 || !aligned16(qkv_dev) || !aligned16(cos_sin_dev) || !aligned16(q_dev) || !aligned16(k_rows_dev) ||
        !aligned16(k_pages_dev) || !aligned16(v_pages_dev))
        return KNNSSD_ERR_SHAPE;
    pages::RotaryArgs a{qkv_dev, row_stride, n_rows, n_heads, n_kv_heads, n_positions, reinterpret_cast<const float2 *>(cos_sin_dev), row_pos_dev, row_slot_dev, page_size,
                        n_pages * page_size, q_dev, k_rows_dev, k_pages_dev, v_pages_dev};
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    if (head_dim == 128) launch_rotary<128>(a, dtype, cache_dtype, s);
    else launch_rotary<64>(a, dtype, cache_dtype, s);
    return launched();
}

knnssd_status knnssd_paged_attention(const void *q_dev, int dtype, int n_rows, long long q_stride, int n_heads, int n_kv_heads, int head_dim, const void *k_pages_dev,
                                     const void *v_pages_dev, int cache_dtype, int page_size, int n_pages, const int *table_dev, int max_pages, const int *lens_dev,
                                     const int *row_start_dev, int n_requests, int max_fresh, float scale, void *out_dev, void *cuda_stream) {
    if (n_rows < 0 || n_requests < 1 || max_fresh < 0 || !std::isfinite(scale) || scale < 0.f) return KNNSSD_ERR_INVALID_ARG;
    if (knnssd_status st = check_heads(dtype, cache_dtype, n_heads, n_kv_heads, head_dim); st != KNNSSD_OK) return st;
    if (knnssd_status st = check_pages(page_size, max_pages, n_pages); st != KNNSSD_OK) return st;
    if (n_rows > INT_MAX / 2 || (long long)n_rows * n_heads > INT_MAX) return KNNSSD_ERR_CAPACITY;
    if (n_rows == 0) return KNNSSD_OK;
    if (!q_dev || !k_pages_dev || !v_pages_dev || !table_dev || !lens_dev || !row_start_dev || !out_dev) return KNNSSD_ERR_INVALID_ARG;
    if (q_stride < (long long)n_heads * head_dim || q_stride % (dtype ? 8 : 4) != 0 || !aligned16(q_dev) || !aligned16(k_pages_dev) || !aligned16(v_pages_dev) || !aligned16(out_dev))
        return KNNSSD_ERR_SHAPE;
    attn::Args a{};
    a.q = q_dev; a.out = out_dev; a.q_stride = q_stride;
    a.k = k_pages_dev; a.v = v_pages_dev;
    a.table = table_dev; a.max_pages = max_pages; a.n_pages = n_pages;
    while ((1 << a.page_shift) < page_size) ++a.page_shift;
    a.lens = lens_dev; a.row_start = row_start_dev; a.B = n_requests; a.R = n_rows; a.H = n_heads; a.KV = n_kv_heads;
    a.scale_log2 = log2_scale(scale);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    try {
        if (dtype == 1) {
            const int most_rows = max_fresh > 0 ? std::min(max_fresh, a.R) : a.R;
            // a coordinate of the TMA has 31 bits
            if (page_size >= 64 && (long long)n_pages * page_size * n_kv_heads <= INT_MAX)
                return head_dim == 128 ? launch_tensor<128, tcattn::TILED>(a, most_rows, s) : launch_tensor<64, tcattn::TILED>(a, most_rows, s);
            return head_dim == 128 ? launch_tensor<128, tcattn::COPIED>(a, most_rows, s) : launch_tensor<64, tcattn::COPIED>(a, most_rows, s);
        }
        return head_dim == 128 ? launch_paged_rows<128>(a, cache_dtype, s) : launch_paged_rows<64>(a, cache_dtype, s);
    } catch (...) { return KNNSSD_ERR_CUDA; }
}

knnssd_status knnssd_packed_attention(const void *q_dev, const void *k_dev, const void *v_dev, int dtype, int n_rows, long long q_stride, long long k_stride,
                                      long long v_stride, int n_heads, int n_kv_heads, int head_dim, const int *row_start_dev, int n_requests, float scale, void *out_dev,
                                      void *cuda_stream) {
    if (n_rows < 0 || n_requests < 1 || !std::isfinite(scale) || scale < 0.f) return KNNSSD_ERR_INVALID_ARG;
    if (knnssd_status st = check_heads(dtype, dtype, n_heads, n_kv_heads, head_dim); st != KNNSSD_OK) return st;
    if (n_rows > INT_MAX / 2 || (long long)n_rows * n_heads > INT_MAX) return KNNSSD_ERR_CAPACITY;
    if (n_rows == 0) return KNNSSD_OK;
    if (!q_dev || !k_dev || !v_dev || !row_start_dev || !out_dev) return KNNSSD_ERR_INVALID_ARG;
    const int per16 = dtype ? 8 : 4;
    const long long kv_width = (long long)n_kv_heads * head_dim;
    if (q_stride < (long long)n_heads * head_dim || k_stride < kv_width || v_stride < kv_width || q_stride % per16 || k_stride % per16 || v_stride % per16 || !aligned16(q_dev) ||
        !aligned16(k_dev) || !aligned16(v_dev) || !aligned16(out_dev))
        return KNNSSD_ERR_SHAPE;
    attn::Args a{};
    a.q = q_dev; a.out = out_dev; a.q_stride = q_stride;
    a.k = k_dev; a.v = v_dev; a.k_stride = k_stride; a.v_stride = v_stride;
    a.row_start = row_start_dev; a.B = n_requests; a.R = n_rows; a.H = n_heads; a.KV = n_kv_heads;
    a.scale_log2 = log2_scale(scale);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    try {
        if (dtype == 1) {
            return head_dim == 128 ? launch_tensor<128, tcattn::PACKED>(a, a.R, s) : launch_tensor<64, tcattn::PACKED>(a, a.R, s);
        }
        return head_dim == 128 ? launch_rows<128, float, false>(a, s) : launch_rows<64, float, false>(a, s);
    } catch (...) { return KNNSSD_ERR_CUDA; }
}

knnssd_status knnssd_attention_status(void *cuda_stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(s, &capturing) != cudaSuccess || capturing != cudaStreamCaptureStatusNone) {
        cudaGetLastError();
        return KNNSSD_ERR_CUDA;
    }
    try {
        int *word = attention_err_ptr(), *taken = nullptr, code = 0;
        Scratch mem(s);
        if (!word || !mem.get(&taken, 1)) return KNNSSD_ERR_CUDA;
        take_word_kernel<<<1, 1, 0, s>>>(word, taken);
        if (launched() != KNNSSD_OK || cudaMemcpyAsync(&code, taken, sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
            cudaGetLastError();
            return KNNSSD_ERR_CUDA;
        }
        return code ? KNNSSD_ERR_TIMEOUT : KNNSSD_OK;
    } catch (...) { return KNNSSD_ERR_CUDA; }
}

knnssd_status knnssd_debug_attention_timeout(unsigned spin_limit, unsigned tiles) {
    if (spin_limit > tcattn::WAIT_LIMIT) return KNNSSD_ERR_INVALID_ARG;
    g_wait_limit = spin_limit ? spin_limit : tcattn::WAIT_LIMIT;
    g_stop_after = spin_limit ? tiles : ~0u;
    return KNNSSD_OK;
}

}  // extern "C"
