// Launches of kernels by a handle that is asked for once a device, where a call's host time counts: with 200 bytes of arguments 2.9 us for 3.4 by the kernel's symbol, which is looked up
// in each launch.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>

namespace mp {

template <auto kKernel>
struct Launch;
template <class... P, void (*kKernel)(P...)>
struct Launch<kKernel> {
    static hipError_t on(dim3 grid, dim3 block, hipStream_t s, P... args)
    {
        constexpr int kDevices = 16;
        static std::atomic<hipFunction_t> handles[kDevices];
        int device;
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) return e;
        hipFunction_t f = device < kDevices ? handles[device].load(std::memory_order_relaxed) : nullptr;
        if (!f) {
            e = hipGetFuncBySymbol(&f, reinterpret_cast<const void*>(kKernel));
            if (e != hipSuccess) return e;
            if (device < kDevices) handles[device].store(f, std::memory_order_relaxed);      // (the same whoever stores it)
        }
        void* of[] = {&args...};
        return hipModuleLaunchKernel(f, grid.x, grid.y, grid.z, block.x, block.y, block.z, 0, s, of, nullptr);
    }
};

}  // namespace mp
