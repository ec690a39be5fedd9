// Figures that workgroups leave in memory for each other within one launch: device-scope stores and loads of pairs, performed past the dies'
// caches.  A reader knows by a ticket, drawn after the writer's stores have been acknowledged, that they are there.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bl {

__device__ __forceinline__ float2 read_figure(float2* at) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<unsigned long long*>(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}
__device__ __forceinline__ void leave_figure(float2* at, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(at), (unsigned long long)__float_as_uint(x) | (unsigned long long)__float_as_uint(y) << 32,
                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace bl
