// What the tiled matrix products share: loads from memory straight to LDS, waits,
// constant indices for registers, and how many workgroups the GPU holds.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <exception>
#include <map>
#include <mutex>
#include <type_traits>
#include <utility>

#include "sa_conv_device.h"
#include "sa_host.h"

namespace sa {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kMaxLds = 160 * 1024;

__device__ inline int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a raw buffer of `bytes` at base, both wavefront-uniform
__device__ inline i32x4 buffer_at(uint64_t base, uint32_t bytes) {
    return i32x4{uni((int)(uint32_t)base), uni((int)((uint32_t)(base >> 32) & 0xffffu)), uni((int)bytes), kRsrcWord3};
}

// 16 bytes per lane straight from memory to LDS: lane i's land at lds + AT + 16 * i.
// Inline asm: after the compiler's own LDS-DMA builtin every LDS read waits for
// all loads in flight.  The statement has no outputs; the waits are wait_vm().
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <int AT>
__device__ inline void dma16(i32x4 r, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(voff),
                 "s"(r), "s"(soff), "n"(AT)
                 : "memory", "scc", "m0");
}
// The same with 4 bytes per lane, at lds + AT + 4 * i.
template <int AT>
__device__ inline void dma4(i32x4 r, uint32_t voff, uint32_t soff, uint32_t lds) {
    asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(voff),
                 "s"(r), "s"(soff), "n"(AT)
                 : "memory", "scc", "m0");
}
#pragma clang diagnostic pop
template <int N>
__device__ inline void wait_vm() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// this wavefront's LDS accesses done, then the workgroup's barrier
__device__ inline void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// f(j) with j, below N, as a constant: registers cannot be indexed
template <int N, typename F>
__device__ inline void pick(int j, F &&f) {
    if constexpr (N > 0) {
        if (j == N - 1) f(std::integral_constant<int, N - 1>{});
        else pick<N - 1>(j, f);
    }
}

// f(0), .. f(N - 1) with constants
template <int N, int I = 0, typename F>
__device__ inline void each(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

// Workgroups of `kern` (nt threads, lds bytes) that the GPU holds at once; raises
// the kernel's LDS limit on the first call per device.
inline int resident(const void *kern, int nt, int lds, int *groups) try {
    static std::mutex mu;
    static std::map<std::pair<const void *, int>, int> known;
    int dev = 0;
    if (int rc = check_hip(hipGetDevice(&dev), "matrix product: current device")) return rc;
    std::lock_guard<std::mutex> lock(mu);
    const auto it = known.find({kern, dev});
    if (it != known.end()) {
        *groups = it->second;
        return SA_OK;
    }
    if (int rc = check_hip(hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds), "matrix product: LDS"))
        return rc;
    int per_cu = 0, cus = 0;
    if (int rc = check_hip(hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kern, nt, lds), "matrix product: occupancy"))
        return rc;
    if (int rc = check_hip(hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev), "matrix product: CU count"))
        return rc;
    *groups = std::max(1, per_cu) * std::max(1, cus);
    known[{kern, dev}] = *groups;
    return SA_OK;
} catch (const std::exception &) {  // no exception leaves a C entry
    return fail(SA_E_HIP, "matrix product: out of host memory");
}

}  // namespace
}  // namespace sa
