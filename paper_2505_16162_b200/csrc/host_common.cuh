// What the host sides of the library's operators share: the scratch pool and the tables per device.  One instance for all source files.
#pragma once

#include <cuda_runtime.h>

#include <mutex>
#include <vector>

namespace knnssd {

// ---- scratch of the stand-alone operators --------------------------------------------------------------------------
// One memory pool per device that keeps at most kPoolKeep bytes between calls (what it holds beyond that goes back to the
// driver at every synchronisation, all of it when a context is destroyed): a cudaMalloc / cudaFree pair cost 100 .. 1000 us
// a call, next to kernels of 10 .. 50 us.  Allocations are ordered on the caller's stream, so any number of threads and
// streams may call at once.
// 96 MB hold the largest scratch of a contraction in pieces (prefill_host.cuh: 72 MB of chunk sums) and the planes of its rows: with
// 64, knnssd_gemm_split over 5120 x 13824 weights mapped memory on every call (77 rows 336 us, with 96 129; 1024 rows 488, 275).
constexpr unsigned long long kPoolKeep = 96ull << 20;

// What a call sets up once (pools, addresses, attributes) is no part of a capture that its thread may be in: within this, such calls are let through
// rather than end it.
struct ApartFromCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    ApartFromCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ~ApartFromCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
    ApartFromCapture(const ApartFromCapture &) = delete;
};

struct DevicePools {
    std::mutex mu;
    cudaMemPool_t pool[64] = {};
    bool tried[64] = {};
    // The pool of the current device; nullptr where the device has none.
    cudaMemPool_t current() {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
        std::lock_guard<std::mutex> lock(mu);
        if (!tried[dev]) {
            tried[dev] = true;
            const ApartFromCapture apart;
            int has = 0;
            cudaMemPoolProps props{};
            props.allocType = cudaMemAllocationTypePinned;
            props.location.type = cudaMemLocationTypeDevice;
            props.location.id = dev;
            unsigned long long keep = kPoolKeep;
            if (cudaDeviceGetAttribute(&has, cudaDevAttrMemoryPoolsSupported, dev) != cudaSuccess || !has ||
                cudaMemPoolCreate(&pool[dev], &props) != cudaSuccess)
                pool[dev] = nullptr;
            else
                cudaMemPoolSetAttribute(pool[dev], cudaMemPoolAttrReleaseThreshold, &keep);
            cudaGetLastError();
        }
        return pool[dev];
    }
};
inline DevicePools &device_pools() {
    static DevicePools *pools = new DevicePools();      // never destroyed: a thread may still call at process exit
    return *pools;
}

// The buffers of one call.  They are given back in stream order when it ends, whichever way it ends.
struct Scratch {
    cudaStream_t s;
    cudaMemPool_t pool;
    std::vector<void *> held;
    explicit Scratch(cudaStream_t stream) : s(stream), pool(device_pools().current()) {}
    Scratch(const Scratch &) = delete;
    template <typename T> bool get(T **p, size_t count) {
        void *q = nullptr;
        const cudaError_t e = pool ? cudaMallocFromPoolAsync(&q, count * sizeof(T), pool, s) : cudaMalloc(&q, count * sizeof(T));
        if (e != cudaSuccess) { cudaGetLastError(); return false; }
        held.push_back(q);
        *p = static_cast<T *>(q);
        return true;
    }
    ~Scratch() {
        for (void *q : held) {
            if (pool) cudaFreeAsync(q, s);
            else cudaFree(q);
        }
    }
};

constexpr int kMaxDevices = 64;

// Index of the current device in the per-device tables below (0 if it cannot be read or is out of range).
inline int current_device_slot() {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) dev = 0;
    return dev;
}

// Multiprocessors of the current device.
inline int sm_count() {
    int dev = 0, n = 148;
    if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    return n;
}

}  // namespace knnssd
