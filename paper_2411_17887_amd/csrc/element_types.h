// The floating element types of the operators on tokens, and what their entry points ask of sizes and pointers.
#ifndef TCUSCAN_ELEMENT_TYPES_H
#define TCUSCAN_ELEMENT_TYPES_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/tcuscan.h"

namespace {

typedef _Float16 f16_t;
typedef __bf16   bf16_t;

// An element type is named by the dtype whose input it is, also where a kernel is named by it.
constexpr int kF16 = TCUSCAN_F16_F32, kF32 = TCUSCAN_F32_F32, kBF16 = TCUSCAN_BF16_F32;
template <int DT> struct Elem;
template <> struct Elem<kF16>  { typedef f16_t T; };
template <> struct Elem<kF32>  { typedef float T; };
template <> struct Elem<kBF16> { typedef bf16_t T; };

inline size_t elem_bytes(int dt) { return dt == kF32 ? 4 : dt == kF16 || dt == kBF16 ? 2 : 0; }

// Workgroups of `threads` that one launch holds: HIP takes fewer than 2^32 threads.  Calls beyond it are refused before anything is enqueued.
constexpr size_t most_groups(size_t threads) { return 0xFFFFFFFFu / threads; }

// Raised where a device array holds an offset, slot or token number that is out of range (chain_layout.h: the header's first word).
constexpr uint32_t kFaultBadIndex = 2u;
__device__ __forceinline__ void raise_fault(void *ws, uint32_t fault)
{
    if (ws) __hip_atomic_store((uint32_t *)ws, fault, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace

#endif
