// qmm_async.cuh -- copies from global into shared memory that run beside the thread (cp.async) and their groups.
#pragma once

#include <stdint.h>

namespace qmm {

__device__ __forceinline__ void async16(uint32_t to, const void* from, int bytes)            // bytes < 16: the rest becomes zero
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void async4(uint32_t to, const void* from, int bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

}  // namespace qmm
