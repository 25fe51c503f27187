// Element types and matrix instructions of the operators' kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace ii {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using f32x16 = __attribute__((ext_vector_type(16))) float;
using u32x2 = __attribute__((ext_vector_type(2))) uint32_t;
using u32x4 = __attribute__((ext_vector_type(4))) uint32_t;
using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
using f16x2 = __attribute__((ext_vector_type(2))) _Float16;
using bf16x4 = __attribute__((ext_vector_type(4))) __bf16;
using f16x4 = __attribute__((ext_vector_type(4))) _Float16;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using s16x4 = __attribute__((ext_vector_type(4))) short;

template <class T>
struct Vec;
template <>
struct Vec<__bf16> {
    using x2 = bf16x2;
    using x4 = bf16x4;
    using x8 = bf16x8;
};
template <>
struct Vec<_Float16> {
    using x2 = f16x2;
    using x4 = f16x4;
    using x8 = f16x8;
};

// 16 rows of a times 16 rows of b over 32 elements: lane l holds elements
// 8 (l / 16) .. + 8 of row l mod 16 of each, and of the sum rows
// 4 (l / 16) + r of a against row l mod 16 of b.
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
// 32 rows of a times 32 rows of b over 16 elements: lane l holds elements
// 8 (l / 32) .. + 8 of row l mod 32, and of the sum rows
// 8 (r / 4) + 4 (l / 32) + r mod 4 of a against row l mod 32 of b.
__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

using Rsrc = __amdgpu_buffer_rsrc_t;

// Memory from base on for buffer instructions, which take 32-bit offsets and
// give zeros past its end.
__device__ inline Rsrc buffer(const void* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0,
                                             (int)(uint32_t)min(bytes, (int64_t)0xffffffffll),
                                             0x00020000);
}

// Workgroups that share a result leave their parts in global memory; the last
// to arrive joins them, in the order of their places. The workgroups run on
// XCDs whose L2 caches do not see each other, so parts are written and read by
// instructions of device scope (sc1), which go past those caches. Nothing else
// passes between the workgroups, so it is enough that a wave's writes have
// arrived before it counts itself: a fence of device scope would also write
// back the whole L2, which took 130 us where 512 workgroups of a 20 us kernel
// did it.
constexpr int kDeviceScope = 16;
__device__ inline void leave_part(Rsrc parts, uint32_t offset, f32x4 v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, v), parts, (int)offset, 0,
                                           kDeviceScope);
}
__device__ inline f32x4 take_part(Rsrc parts, uint32_t offset) {
    return __builtin_bit_cast(
        f32x4, __builtin_amdgcn_raw_buffer_load_b128(parts, (int)offset, 0, kDeviceScope));
}
// Whether this workgroup is the last of `parts`; the counter is zero again
// then. Called by every thread, after the parts were left.
__device__ inline bool arrive_last(uint32_t* counter, uint32_t parts) {
    __shared__ uint32_t before;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        before = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == parts - 1)
            __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    asm volatile("" ::: "memory");  // parts are taken after this
    return before == parts - 1;
}

}  // namespace ii
