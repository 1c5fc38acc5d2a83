// The stand-in HIP runtime of ../../hoststub, with what the operators' host
// code uses besides.
#pragma once
#include "../../hoststub/hip/hip_runtime.h"

#define __host__
#define __device__
#define hipStreamPerThread ((hipStream_t)2)
struct int4 {
    int x, y, z, w;
};

// Waits for the device are counted, and events answer as the test says.
#define hipErrorNotReady ((hipError_t)600)
extern "C" hipError_t hipEventQuery(hipEvent_t e);
extern "C" hipError_t opstub_device_synchronize();
extern "C" hipError_t opstub_host_free(void *p);
#define hipDeviceSynchronize opstub_device_synchronize
#define hipHostFree opstub_host_free
