/* A HIP runtime in which every address is device memory of one allocation and no
 * kernel can be launched: what an operator's checks let through ends in
 * hipErrorNoDevice, what they refuse in its own code. */
#include <hip/hip_runtime_api.h>
#include <string.h>

static hipError_t last = hipSuccess;

hipError_t hipPointerGetAttributes(hipPointerAttribute_t* a, const void* at) {
    memset(a, 0, sizeof *a);
    a->type = hipMemoryTypeDevice;
    a->devicePointer = (void*)at;
    return hipSuccess;
}

hipError_t hipMemGetAddressRange(hipDeviceptr_t* base, size_t* size, hipDeviceptr_t at) {
    (void)at;
    *base = 0;
    *size = (size_t)1 << 62;
    return hipSuccess;
}

/* the first step of a launch; after an error the others are left out */
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    (void)grid, (void)block, (void)lds, (void)stream;
    return last = hipErrorNoDevice;
}

hipError_t hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void** args, size_t lds,
                           hipStream_t stream) {
    (void)kernel, (void)grid, (void)block, (void)args, (void)lds, (void)stream;
    return last = hipErrorNoDevice;
}

hipError_t hipGetLastError(void) {
    const hipError_t e = last;
    last = hipSuccess;
    return e;
}
