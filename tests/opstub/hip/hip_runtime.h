// The stand-in HIP runtime of ../../hoststub, with what the operators' host
// code uses besides.
#pragma once
#include "../../hoststub/hip/hip_runtime.h"

#define __host__
#define __device__
struct int4 {
    int x, y, z, w;
};
