// Host-side helpers that both libraries use.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Launches a kernel; the result is this launch's own.  (`<<<>>>` drops it, and hipGetLastError, asked behind it, also tells of calls of
// anybody's that have failed on this thread before: a step that runs would be taken for one that does not.)
template <typename T> struct as_is { using type = T; };
template <typename... P>
hipError_t launch(void (*kernel)(P...), dim3 grid, int threads, size_t lds, hipStream_t st, const typename as_is<P>::type&... arguments)
{
    void* args[] = {const_cast<void*>(static_cast<const void*>(&arguments))...};
    const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3((unsigned)threads), args, lds, st);
    if (e != hipSuccess) (void)hipGetLastError();       // (nor is it left for others)
    return e;
}

}  // namespace
