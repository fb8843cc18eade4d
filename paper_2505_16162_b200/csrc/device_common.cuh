// Device helpers that every kernel of the library may use: chained launches, bf16 conversions, rotary pairs, warp sums.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace knnssd {

typedef unsigned short bf16_t;  // raw bf16 bit pattern

// Kernels that follow one another closely are launched with programmatic stream serialisation: a kernel may be set up on
// the SMs while the one before it still runs.  Each of them lets its successor come and then waits until the one before it
// has finished and its writes are visible, before it touches any memory; with an ordinary launch both do nothing.
// (A verification pass of an fp32 model, run as 36 kernels of 2 .. 10 us: 279 -> 217 us; a prompt of 77 rows, 8 layers of the 7B widths:
// 1.68 -> 1.62 ms.)
__device__ __forceinline__ void chain_wait() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}
// Launch of a kernel that calls chain_wait() before it touches memory.  (The prompt pass's contractions and its head fetch weights before: in a
// chain that an ordinary launch has begun, nothing on the stream before the chain is still at work.)
template <typename... P, typename... A>
void launch_chained(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, A... args) {
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = s; cfg.attrs = &attr; cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

// The GPU's nanosecond timer.  Calls that return a device time have it stamped by their first and their last kernel, into pinned words: two
// events and their difference took 7.3 us of a call, next to 9.3 for a launch and the wait for it.
__device__ __forceinline__ unsigned long long globaltimer_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

__device__ __forceinline__ float bf16_bits_to_float(unsigned int b) { return __uint_as_float(b << 16); }

// Round to nearest even on the bit pattern.  A NaN stays a NaN (the integer rounding alone would carry the all-ones
// NaN over into -0, and a non-finite activation would silently turn into zeros downstream).
__device__ __forceinline__ bf16_t float_to_bf16_rne(float f) {
    const unsigned int u = __float_as_uint(f);
    const unsigned int r = (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
    return (bf16_t)((u & 0x7FFFFFFFu) > 0x7F800000u ? 0x7FC0u : r);
}

// (v0, v1) -> packed bf16 pair (v0 in the low half), round to nearest even; hi part and what is left of it
__device__ __forceinline__ uint32_t cvt_bf16x2(float v0, float v1) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(v1), "f"(v0));
    return r;
}
__device__ __forceinline__ void split_pair(float v0, float v1, uint32_t &hi, uint32_t &lo) {
    hi = cvt_bf16x2(v0, v1);
    lo = cvt_bf16x2(v0 - __uint_as_float(hi << 16), v1 - __uint_as_float(hi & 0xffff0000u));
}

// Rotary embedding of a pair by (cos, sin) = c.  The rounding is spelled out: left to the compiler, the prompt pass's contraction and
// rope_kv_rows_kernel fused other products of the second sum, and a row's K depended on which of them a launch's sizes chose.
__device__ __forceinline__ void rotate_pair(float &a, float &b, float2 c) {
    const float ra = __fmaf_rn(a, c.x, -__fmul_rn(b, c.y));
    b = __fmaf_rn(b, c.x, __fmul_rn(a, c.y));
    a = ra;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

}  // namespace knnssd
