// 256 bytes of zeros in device memory: what direct transfers from each lane's
// own address read where there is nothing.  Included by the HIP kernels only.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mssa {
namespace {

__device__ __attribute__((aligned(256))) const uint32_t zero_row[64] = {};

}  // namespace
}  // namespace mssa
