// Host side of the operators for drafts that branch: tables of a tree's rows, attention, acceptance, and the kept rows' K and V.  The C ABI is declared in
// include/knnssd.h.
#include "../../include/knnssd.h"
#include "attention_launch.cuh"
#include "tree_accept.cuh"
#include "trees.cuh"

using namespace knnssd;

namespace {

template <int C> knnssd_status launch_accept(const trees::AcceptArgs &a, cudaStream_t s) {
    if (C > 8) {                                                     // more blocks a cluster than every device has
        static bool allowed[kMaxDevices] = {};
        const int dev = current_device_slot();
        if (!allowed[dev]) {
            const ApartFromCapture apart;
            allowed[dev] = cudaFuncSetAttribute(trees::tree_accept_kernel<C>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
            if (!allowed[dev]) { cudaGetLastError(); return KNNSSD_ERR_CUDA; }
        }
    }
    launch_chained(trees::tree_accept_kernel<C>, dim3(C * a.B), dim3(trees::ACC_NT), 0, s, a);
    return launched();
}

}  // namespace

extern "C" {

knnssd_status knnssd_tree_tables(const int *lens_dev, const int *row_start_dev, const int *row_parent_dev, int n_requests, int n_rows, int *row_pos_dev,
                                 unsigned long long *row_seen_dev, int *request_state_dev, void *cuda_stream) {
    if (!lens_dev || !row_start_dev || !request_state_dev || n_requests < 1 || n_rows < 0 || (n_rows > 0 && (!row_parent_dev || !row_pos_dev || !row_seen_dev)))
        return KNNSSD_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(row_seen_dev) & 7u) return KNNSSD_ERR_SHAPE;
    launch_chained(trees::tree_tables_kernel, dim3(n_requests), dim3(trees::TABLE_NT), 0, reinterpret_cast<cudaStream_t>(cuda_stream),
                   trees::TableArgs{lens_dev, row_start_dev, row_parent_dev, n_requests, n_rows, row_pos_dev, row_seen_dev, request_state_dev});
    return launched();
}

knnssd_status knnssd_tree_attention(const void *q_dev, int dtype, int n_rows, long long q_stride, int n_heads, int n_kv_heads, int head_dim, const void *k_pages_dev,
                                    const void *v_pages_dev, int cache_dtype, int page_size, int n_pages, const int *table_dev, int max_pages, const int *lens_dev,
                                    const int *row_start_dev, const unsigned long long *row_seen_dev, int n_requests, int max_fresh, float scale, void *out_dev,
                                    void *cuda_stream) {
    return paged_attention<true>(q_dev, dtype, n_rows, q_stride, n_heads, n_kv_heads, head_dim, k_pages_dev, v_pages_dev, cache_dtype, page_size, n_pages, table_dev, max_pages,
                                 lens_dev, row_start_dev, row_seen_dev, n_requests, max_fresh, scale, out_dev, cuda_stream);
}

knnssd_status knnssd_tree_accept(const float *p_dev, const float *q_dev_or_null, int vocab, const int *row_token_dev, const int *row_parent_dev, const int *row_start_dev,
                                 int n_requests, int n_rows, const float *u_accept_dev, const float *u_final_dev, int *path_dev, int *n_accepted_dev, int *next_token_dev,
                                 void *cuda_stream) {
    if (!row_start_dev || !u_final_dev || !n_accepted_dev || !next_token_dev || n_requests < 1 || n_rows < 0 || vocab < 1 ||
        (n_rows > 0 && (!p_dev || !row_token_dev || !row_parent_dev || !u_accept_dev || !path_dev)))
        return KNNSSD_ERR_INVALID_ARG;
    if (vocab > KNNSSD_MAX_VOCAB || n_requests > KNNSSD_MAX_REQUESTS) return KNNSSD_ERR_CAPACITY;
    const trees::AcceptArgs a{p_dev, q_dev_or_null, vocab, row_token_dev, row_parent_dev, row_start_dev, n_requests, n_rows, u_accept_dev, u_final_dev, path_dev, n_accepted_dev, next_token_dev};
    cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
    switch (trees::blocks_of(n_requests, vocab, q_dev_or_null != nullptr, sm_count())) {
    case 16: return launch_accept<16>(a, s);
    case 8: return launch_accept<8>(a, s);
    case 4: return launch_accept<4>(a, s);
    case 2: return launch_accept<2>(a, s);
    default: return launch_accept<1>(a, s);
    }
}

knnssd_status knnssd_tree_agree(const int *row_best_dev, const int *row_token_dev, const int *row_parent_dev, const int *row_start_dev, int n_requests, int n_rows,
                                int *path_dev, int *n_accepted_dev, int *next_token_dev, void *cuda_stream) {
    if (!row_start_dev || !n_accepted_dev || !next_token_dev || n_requests < 1 || n_rows < 0 ||
        (n_rows > 0 && (!row_best_dev || !row_token_dev || !row_parent_dev || !path_dev)))
        return KNNSSD_ERR_INVALID_ARG;
    constexpr int PER = trees::AGREE_NT / 32;
    launch_chained(trees::tree_agree_kernel, dim3((n_requests + PER - 1) / PER), dim3(trees::AGREE_NT), 0, reinterpret_cast<cudaStream_t>(cuda_stream),
                   trees::AgreeArgs{row_best_dev, row_token_dev, row_parent_dev, row_start_dev, n_requests, n_rows, path_dev, n_accepted_dev, next_token_dev});
    return launched();
}

knnssd_status knnssd_keep_rows(void *const *pools_host, int n_pools, int cache_dtype, int n_kv_heads, int head_dim, int page_size, int n_pages, const int *table_dev,
                               int max_pages, const int *lens_dev, const int *row_start_dev, const int *path_dev, int n_requests, int n_rows, void *cuda_stream) {
    if (n_pools < 1 || !pools_host || n_requests < 1 || n_rows < 0) return KNNSSD_ERR_INVALID_ARG;
    if (knnssd_status st = check_heads(0, cache_dtype, n_kv_heads, n_kv_heads, head_dim); st != KNNSSD_OK) return st;
    if (knnssd_status st = check_pages(page_size, max_pages, n_pages); st != KNNSSD_OK) return st;
    for (int i = 0; i < n_pools; ++i) {
        if (!pools_host[i]) return KNNSSD_ERR_INVALID_ARG;
        if (!aligned16(pools_host[i])) return KNNSSD_ERR_SHAPE;
    }
    if (n_rows == 0) return KNNSSD_OK;
    if (!table_dev || !lens_dev || !row_start_dev || !path_dev) return KNNSSD_ERR_INVALID_ARG;
    trees::KeepArgs a{};
    a.table = table_dev; a.lens = lens_dev; a.row_start = row_start_dev; a.path = path_dev;
    a.B = n_requests; a.R = n_rows; a.max_pages = max_pages; a.n_pages = n_pages; a.KV = n_kv_heads;
    a.pieces = head_dim * (cache_dtype ? 2 : 4) / 16;
    while ((1 << a.page_shift) < page_size) ++a.page_shift;
    for (int done = 0; done < n_pools; done += a.n_pools) {
        a.n_pools = std::min(n_pools - done, trees::KEEP_POOLS);
        for (int i = 0; i < a.n_pools; ++i) a.pools[i] = static_cast<uint4 *>(pools_host[done + i]);
        const long long units = (long long)a.n_pools * n_kv_heads * a.pieces;
        launch_chained(trees::keep_rows_kernel, dim3(n_requests, (unsigned)std::min((units + trees::KEEP_NT - 1) / trees::KEEP_NT, 65535ll)), dim3(trees::KEEP_NT), 0,
                       reinterpret_cast<cudaStream_t>(cuda_stream), a);
    }
    return launched();
}

}  // extern "C"
