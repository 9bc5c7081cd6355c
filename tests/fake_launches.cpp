// The HIP runtime of fake_hip.cpp, which refuses launches that the real one refuses for their size, and counts all.
#include <hip/hip_runtime.h>

#define hipLaunchKernel any_launch
#include "fake_hip.cpp"
#undef hipLaunchKernel

namespace {
int launches = 0, too_large = 0;
}

extern "C" {
int fake_launches() { return launches; }
int fake_too_large() { return too_large; }
hipError_t hipLaunchKernel(const void *kernel, dim3 grid, dim3 block, void **args, size_t lds, hipStream_t s)
{
    ++launches;
    // a dimension holds fewer than 2^32 threads, a work-group at most 160 KiB of local memory
    if (static_cast<uint64_t>(grid.x) * block.x >= (1ull << 32) || lds > 160 * 1024) {
        ++too_large;
        return last = hipErrorInvalidConfiguration;
    }
    return any_launch(kernel, grid, block, args, lds, s);
}
}
