// Loads and stores of 16 bytes that the copy kernels share (device code).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace kvl {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
// Every buffer is device (or device-mapped) memory: say so, so that the
// compiler emits global_load / global_store rather than flat accesses.
typedef const v4u __attribute__((address_space(1))) *gsrc_t;
typedef v4u __attribute__((address_space(1))) *gdst_t;

template <bool NT>
__device__ __forceinline__ v4u load16(gsrc_t p) {
    if (NT) return __builtin_nontemporal_load(p);
    return *p;
}

// Store with a cache policy.  The compiler only offers the non-temporal hint;
// the system-scope write-through forms (sc1) are written out as instructions.
// A store needs no wait: nothing here reads what it wrote.  The s_nop after a written-out
// store covers the one hazard the compiler cannot see through the asm: a vector-ALU write to the
// store's data registers in the next two issue slots (it handles that itself for stores it
// emits; in a loop the next instruction may well be such a write).
template <int SP>
__device__ __forceinline__ void store16(gdst_t p, v4u v) {
    if (SP == 0) *p = v;
    else if (SP == 1) __builtin_nontemporal_store(v, p);
    else if (SP == 2) asm volatile("global_store_dwordx4 %0, %1, off sc1\n\ts_nop 1" : : "v"(p), "v"(v) : "memory");
    else asm volatile("global_store_dwordx4 %0, %1, off sc1 nt\n\ts_nop 1" : : "v"(p), "v"(v) : "memory");
}

}  // namespace kvl
