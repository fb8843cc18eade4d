// Pages of many requests: block tables, the free stack, slots of new rows, and the rows' way into the pages.
//
// A pool holds n_pages pages of `page` positions each; a request's positions 0 .. len - 1 lie in the pages that its row of the block
// table names, page p holding positions p page .. p page + page - 1.  A page's K (and V) values are [kv head][position][head_dim]: the
// cache of the decode passes cut into pieces, a head's piece contiguous.
#pragma once

#include "device_common.cuh"

namespace knnssd {
namespace pages {

constexpr int NT = 1024;                  // threads of the planning block
constexpr int MAX_REQUESTS = 8192;        // three prefixes of 32 KB each in shared memory
constexpr int ROWS_NT = 256;
// Rows up to which the planning block maps them itself, rather than a second launch over the whole chip: 120 / 500 / 1000 / 2000 / 4000 rows in
// 7.2 / 7.6 / 8.0 / 9.5 / 12.2 us by itself, 8.7 / 9.5 / 10.0 / 10.6 / 11.5 with the launch; 30 000 rows 49 and 14.
constexpr int ROWS_HERE = 3200;

enum { SHORT_OF_PAGES = 1, TABLE_FULL = 2, TOO_MANY_ROWS = 4, BAD_STATE = 8 };

struct PlanArgs {
    const int *lens, *fresh;
    int n_requests, page, max_pages, n_pages;
    int *owned, *table, *free_pages, *free_count;
    int max_rows;
    int *row_start, *row_request, *row_pos, *row_slot, *info;
    int rows_here;                        // the planning block maps the rows too
};

__host__ __device__ __forceinline__ int plan_smem(int n_requests) { return 3 * (n_requests + 1) * (int)sizeof(int); }

// First index of the ascending pfx[1 .. n] whose value is above x, i.e. the request that item x belongs to; x < pfx[n].
template <typename T> __device__ __forceinline__ int owner_of(const T *pfx, int n, T x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (pfx[mid + 1] > x) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// Request, position and slot of row r; total: rows that there are, later ones get -1.
__device__ __forceinline__ void map_row(const PlanArgs &a, const int *start, int total, int r) {
    int b = -1, pos = -1, slot = -1;
    if (r < total) {
        b = owner_of(start, a.n_requests, r);
        pos = a.lens[b] + r - start[b];
        const int id = a.table[(size_t)b * a.max_pages + pos / a.page];
        if (id >= 0 && id < a.n_pages) slot = id * a.page + pos % a.page;
    }
    a.row_request[r] = b;
    a.row_pos[r] = pos;
    a.row_slot[r] = slot;
}

// One block: what every request needs, takes and gives back (three prefix sums in request order), then the pages, then - where there are
// few - the rows.  Surplus pages are pushed before new ones are popped, both in request and page order, so that page k of all that are taken
// is entry count + given - 1 - k of the stack.  Nothing of the state changes unless everything fits.
// Bound by latency: three loads deep for the sums, two for the pages, two for the rows.
__global__ void __launch_bounds__(NT) plan_kernel(const PlanArgs a) {
    extern __shared__ int sm[];
    int *start = sm, *take = start + a.n_requests + 1, *give = take + a.n_requests + 1;
    __shared__ long long w_rows[NT / 32], w_take[NT / 32], w_give[NT / 32];
    __shared__ int w_bad[NT / 32];
    chain_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.n_requests;
    const int per = (n + NT - 1) / NT, b0 = min(tid * per, n), b1 = min(b0 + per, n);
    const int count = *a.free_count;
    int bad = count < 0 || count > a.n_pages ? BAD_STATE : 0;
    auto request = [&](int b, long long &rows, long long &need, int &have) {
        const int len = a.lens[b], fresh = a.fresh[b];
        have = a.owned[b];
        if (len < 0 || fresh < -1 || have < 0 || have > a.max_pages) { bad |= BAD_STATE; rows = 0; need = have = 0; return; }
        rows = fresh > 0 ? fresh : 0;
        need = fresh < 0 ? 0 : ((long long)len + rows + a.page - 1) / a.page;
        if (need > a.max_pages) bad |= TABLE_FULL;
    };
    long long rows = 0, taken = 0, given = 0;
    for (int b = b0; b < b1; ++b) {
        long long r, need;
        int have;
        request(b, r, need, have);
        rows += r;
        if (need > have) taken += need - have; else given += have - need;
    }
    const long long own[3] = {rows, taken, given};
    long long incl[3] = {rows, taken, given};
#pragma unroll
    for (int o = 1; o < 32; o <<= 1)
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const long long v = __shfl_up_sync(0xffffffffu, incl[i], o);
            if (lane >= o) incl[i] += v;
        }
    bad = (int)__reduce_or_sync(0xffffffffu, (unsigned)bad);
    if (lane == 31) { w_rows[warp] = incl[0]; w_take[warp] = incl[1]; w_give[warp] = incl[2]; w_bad[warp] = bad; }
    __syncthreads();
    long long before[3] = {incl[0] - own[0], incl[1] - own[1], incl[2] - own[2]}, total[3] = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const long long v[3] = {w_rows[w], w_take[w], w_give[w]};
        bad |= w_bad[w];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (w < warp) before[i] += v[i];
            total[i] += v[i];
        }
    }
    // the same in every thread from here on
    if (total[0] > a.max_rows) bad |= TOO_MANY_ROWS;
    if (count + total[2] > a.n_pages) bad |= BAD_STATE;
    else if (!(bad & BAD_STATE) && total[1] > count + total[2]) bad |= SHORT_OF_PAGES;
    const int n_rows = bad ? 0 : (int)total[0];
    if (!bad) {
        for (int b = b0; b < b1; ++b) {
            long long r, need;
            int have;
            request(b, r, need, have);
            start[b] = (int)before[0]; take[b] = (int)before[1]; give[b] = (int)before[2];
            before[0] += r;
            if (need > have) before[1] += need - have; else before[2] += have - need;
            a.row_start[b] = start[b];
        }
        if (tid == 0) { start[n] = (int)total[0]; take[n] = (int)total[1]; give[n] = (int)total[2]; a.row_start[n] = (int)total[0]; }
    } else {
        for (int b = tid; b <= n; b += NT) a.row_start[b] = 0;
    }
    if (tid == 0) {
        a.info[0] = n_rows;
        a.info[1] = bad ? 0 : (int)total[1];
        a.info[2] = bad ? 0 : (int)total[2];
        a.info[3] = bad;
    }
    __syncthreads();
    if (!bad) {
        const int T = (int)total[1], G = (int)total[2];
        auto need_of = [&](int b) { const int f = a.fresh[b]; return f < 0 ? 0 : (a.lens[b] + f + a.page - 1) / a.page; };
        for (int j = tid; j < G; j += NT) {
            const int b = owner_of(give, n, j);
            int *e = a.table + (size_t)b * a.max_pages + need_of(b) + (j - give[b]);
            a.free_pages[count + j] = *e;
            *e = -1;
        }
        __syncthreads();
        for (int k = tid; k < T; k += NT) {
            const int b = owner_of(take, n, k);
            a.table[(size_t)b * a.max_pages + a.owned[b] + (k - take[b])] = a.free_pages[count + G - 1 - k];
        }
        __syncthreads();
        for (int b = b0; b < b1; ++b) a.owned[b] = need_of(b);
        if (tid == 0) *a.free_count = count + G - T;
    }
    if (a.rows_here)
        for (int r = tid; r < a.max_rows; r += NT) map_row(a, start, n_rows, r);
}

// The rows of a large plan, over the whole chip.
__global__ void __launch_bounds__(ROWS_NT) map_rows_kernel(const PlanArgs a) {
    chain_wait();
    const int r = blockIdx.x * ROWS_NT + threadIdx.x;
    if (r < a.max_rows) map_row(a, a.row_start, a.row_start[a.n_requests], r);
}

// ---- rotary embedding of new rows, K and V into their pages ----------------------------------------------------------
// A row of qkv is [n_heads + 2 n_kv_heads][hd]: q, k and v heads.  With (c, s) of the row's position and dimension i < hd / 2,
//   x'[i] = c x[i] - s x[i + hd/2],  x'[i + hd/2] = c x[i + hd/2] + s x[i]
// for q and k, in fp32; q goes to q_out (and K to k_rows, for attention over whole prompts), K and V, rounded to the cache's type (to nearest
// even), to the row's slot.  Every value is read and written once: bound by memory.  A thread takes 16 bytes of either half of a head; the
// threads of a block keep their dimensions from head to head, so the row's (c, s) are loaded once.
struct RotaryArgs {
    const void *qkv;
    long long row_stride;                 // elements
    int n_rows, n_heads, n_kv_heads, n_positions;
    const float2 *cos_sin;                // [n_positions][hd / 2]
    const int *row_pos, *row_slot;
    int page, n_slots;                    // n_slots = n_pages page
    void *q_out, *k_rows, *k_pages, *v_pages;      // k_rows: the rotated K heads by rows, or null
};
// A block does a row.  Few rows are done soonest by many threads each, many rows by few threads with more in flight each: 120 rows of 120 heads by 256 /
// 128 / 64 threads 6.1 / 6.6 / 10.2 us, 8192 rows of 56 heads 48.2 / 42.0 / 39.7 (6.0 TB/s).
constexpr int ROT_FEW = 64, ROT_MANY = 256, ROT_ROWS = 1024, AHEAD = 4;

// 16 bytes that are read once: not kept in L1.
__device__ __forceinline__ uint4 ld_stream16(const void *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <int N> __device__ __forceinline__ void load_row(const float *p, float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const uint4 w = __ldg(reinterpret_cast<const uint4 *>(p + i));
        v[i] = __uint_as_float(w.x); v[i + 1] = __uint_as_float(w.y); v[i + 2] = __uint_as_float(w.z); v[i + 3] = __uint_as_float(w.w);
    }
}
// The values of 16 bytes.
__device__ __forceinline__ void unpack(uint4 w, float (&v)[4], const float *) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void unpack(uint4 w, float (&v)[8], const bf16_t *) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[2 * j] = __uint_as_float(u[j] << 16); v[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u); }
}
template <int N> __device__ __forceinline__ void store_row(float *p, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
template <int N> __device__ __forceinline__ void store_row(bf16_t *p, const float (&v)[N]) {
    uint32_t u[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) u[j] = cvt_bf16x2(v[2 * j], v[2 * j + 1]);
    if (N == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(u[0], u[1]);
    else
#pragma unroll
        for (int j = 0; j + 3 < N / 2; j += 4) *reinterpret_cast<uint4 *>(p + 2 * j) = make_uint4(u[j], u[j + 1], u[j + 2], u[j + 3]);
}

template <int HD, typename XT, typename CT>
__global__ void __launch_bounds__(ROT_MANY) rotary_store_kernel(const RotaryArgs a) {
    constexpr int N = 16 / (int)sizeof(XT), PER_HEAD = HD / 2 / N;       // values of a half that a thread takes; threads of a head
    chain_wait();
    const int row = blockIdx.x, i0 = (threadIdx.x % PER_HEAD) * N;
    const int pos = a.row_pos[row], slot = a.row_slot[row];
    const bool live = pos >= 0 && pos < a.n_positions, stored = live && slot >= 0 && slot < a.n_slots;
    float cs[2 * N];
    if (live) load_row(reinterpret_cast<const float *>(a.cos_sin + (size_t)pos * (HD / 2) + i0), cs);
    const XT *x = static_cast<const XT *>(a.qkv) + (size_t)row * a.row_stride;
    const int heads = a.n_heads + 2 * a.n_kv_heads;
    const size_t page = stored ? slot / a.page : 0, off = stored ? slot % a.page : 0;
    const int STEP = blockDim.x / PER_HEAD;
    for (int h0 = threadIdx.x / PER_HEAD; h0 < heads; h0 += AHEAD * STEP) {
        uint4 lo[AHEAD], hi[AHEAD];                                  // AHEAD heads' halves on their way at once
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int h = h0 + u * STEP;
            lo[u] = hi[u] = make_uint4(0u, 0u, 0u, 0u);
            if (live && h < heads) {
                lo[u] = ld_stream16(x + (size_t)h * HD + i0);
                hi[u] = ld_stream16(x + (size_t)h * HD + HD / 2 + i0);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int h = h0 + u * STEP;
            const bool is_q = h < a.n_heads, is_v = h >= a.n_heads + a.n_kv_heads;
            if (h >= heads || (!is_q && !stored && (is_v || !a.k_rows))) continue;
            float v0[N], v1[N];
            unpack(lo[u], v0, (const XT *)nullptr);
            unpack(hi[u], v1, (const XT *)nullptr);
            if (live && !is_v)
#pragma unroll
                for (int i = 0; i < N; ++i) rotate_pair(v0[i], v1[i], make_float2(cs[2 * i], cs[2 * i + 1]));
            if (is_q) {
                XT *d = static_cast<XT *>(a.q_out) + ((size_t)row * a.n_heads + h) * HD + i0;
                store_row(d, v0);
                store_row(d + HD / 2, v1);
                continue;
            }
            if (!is_v && a.k_rows) {
                XT *d = static_cast<XT *>(a.k_rows) + ((size_t)row * a.n_kv_heads + h - a.n_heads) * HD + i0;
                store_row(d, v0);
                store_row(d + HD / 2, v1);
            }
            if (stored) {
                const int kv = is_v ? h - a.n_heads - a.n_kv_heads : h - a.n_heads;
                CT *d = static_cast<CT *>(is_v ? a.v_pages : a.k_pages) + ((page * a.n_kv_heads + kv) * a.page + off) * HD + i0;
                store_row(d, v0);
                store_row(d + HD / 2, v1);
            }
        }
    }
}

}  // namespace pages
}  // namespace knnssd
