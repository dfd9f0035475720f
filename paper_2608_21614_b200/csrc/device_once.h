// Set-up that a device needs once (function attributes, driver entry points) before the first launch of a kernel.
#ifndef SAEM_DEVICE_ONCE_H_
#define SAEM_DEVICE_ONCE_H_

#include <atomic>

#include <cuda_runtime_api.h>

namespace saem {

struct DeviceOnce {
    std::atomic<bool> ready[64];            // static: zero at the start
};
// Runs `set_up` unless it has succeeded on the current device before.  The device counts as ready only afterwards, so
// that a second thread's first call never launches before the attributes are there, and a failure is tried again; two
// threads may both run `set_up`, which therefore has to bear being run twice.
template <class F>
inline cudaError_t once_on_device(DeviceOnce& once, F set_up) {
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (known && once.ready[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t s = set_up();
    if (s == cudaSuccess && known) once.ready[dev].store(true, std::memory_order_release);
    return s;
}

}  // namespace saem

#endif  // SAEM_DEVICE_ONCE_H_
