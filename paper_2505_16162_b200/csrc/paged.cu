// Host side of the operators for many requests on one paged K/V cache: block tables and slot maps, rotary embedding into pages, attention
// of new rows over pages, attention over packed prompts.  The C ABI is declared in include/knnssd.h.
#include "../../include/knnssd.h"
#include "host_common.cuh"
#include "attention_launch.cuh"
#include "page_tables.cuh"

#include <atomic>
#include <climits>
#include <cmath>
#include <cstdint>

using namespace knnssd;

std::atomic<unsigned> knnssd::g_wait_limit{tcattn::WAIT_LIMIT}, knnssd::g_stop_after[2]{~0u, ~0u};

namespace {

__device__ int g_attention_err;
__global__ void take_word_kernel(int *word, int *to) { *to = atomicExch(word, 0); }

template <int HD> void launch_rotary(const pages::RotaryArgs &a, int dtype, int cache_dtype, cudaStream_t s) {
    const dim3 grid(a.n_rows), block(a.n_rows > pages::ROT_ROWS ? pages::ROT_FEW : pages::ROT_MANY);
    if (dtype == 1) launch_chained(pages::rotary_store_kernel<HD, bf16_t, bf16_t>, grid, block, 0, s, a);
    else if (cache_dtype == 1) launch_chained(pages::rotary_store_kernel<HD, float, bf16_t>, grid, block, 0, s, a);
    else launch_chained(pages::rotary_store_kernel<HD, float, float>, grid, block, 0, s, a);
}

}  // namespace

int *knnssd::attention_err_ptr() {
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
    return paged_attention<false>(q_dev, dtype, n_rows, q_stride, n_heads, n_kv_heads, head_dim, k_pages_dev, v_pages_dev, cache_dtype, page_size, n_pages, table_dev, max_pages,
                                  lens_dev, row_start_dev, nullptr, n_requests, max_fresh, scale, out_dev, cuda_stream);
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
            return head_dim == 128 ? launch_tensor<128, false>(a, a.R, s) : launch_tensor<64, false>(a, a.R, s);
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
    const unsigned only = tiles & (KNNSSD_DEBUG_ONLY_FIRST | KNNSSD_DEBUG_ONLY_SECOND), after = tiles & ~only;
    g_stop_after[0] = spin_limit && only != KNNSSD_DEBUG_ONLY_SECOND ? after : ~0u;
    g_stop_after[1] = spin_limit && only != KNNSSD_DEBUG_ONLY_FIRST ? after : ~0u;
    return KNNSSD_OK;
}

}  // extern "C"
