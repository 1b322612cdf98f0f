// share.h -- how the threads of a workgroup share out many things, with counters that hold at
// the largest numbers.  Plain C++: tests run it on the host.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

// body(x) for a thread's share of n things: the first one and every step-th from there.  Where n is
// within a step of INT_MAX a 32-bit counter would pass it and go on from the negative numbers.
template <typename Body>
__host__ __device__ __forceinline__ void each_of(int64_t n, uint32_t first, uint32_t step, Body&& body) {
    for (int64_t x = first; x < n; x += step) body(x);
}

// How many blocks of `block` n things fill, up to n = INT_MAX.
__host__ __device__ __forceinline__ int32_t blocks_of(int32_t n, int32_t block) {
    return (int32_t)(((uint32_t)n + (uint32_t)block - 1) / (uint32_t)block);
}

// body(k, e) for a thread's share of the entries e < used of the rows k < rows: of the places
// k * used + e, the first one and every step-th from there.  That number passes 32 bits for long
// rows (64 of 2^26 entries), so the thread's place is kept as row and entry: e + step % used is
// below 2 * used, and used below 2^31.  It also takes one division where every place took one.
template <typename Body>
__host__ __device__ __forceinline__ void each_entry(uint32_t used, uint32_t rows, uint32_t first, uint32_t step, Body&& body) {
    if (used == 0) return;
    const uint32_t dk = step / used, de = step - dk * used;
    uint32_t k = first / used, e = first - k * used;
    while (k < rows) {
        body(k, e);
        k += dk;
        e += de;
        if (e >= used) {
            e -= used;
            ++k;
        }
    }
}

}  // namespace
