// Host-side helpers shared by the C ABI's files.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cstring>
#include <vector>

namespace gd {

// Restores the caller's current device on scope exit.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = prev == dev || hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

// The integer a C caller passed for an enum parameter.  A C caller may pass
// any int; in C++ reading an enum object that holds a value outside the
// enumeration is undefined, so the bytes are copied out instead and checked
// as an int.
template <typename E>
int enum_int(const E* e) {
    static_assert(sizeof(E) == sizeof(int), "C enums are int-sized");
    int v;
    std::memcpy(&v, e, sizeof v);
    return v;
}

// Device memory of a handle, freed with it.
struct DeviceMemory {
    std::vector<void*> held;
    ~DeviceMemory() {
        for (void* p : held) (void)hipFree(p);
    }
    template <typename T>
    bool alloc(T** p, size_t count) {
        void* q = nullptr;
        held.reserve(held.size() + 1);
        if (hipMalloc(&q, std::max<size_t>(count, 1) * sizeof(T)) != hipSuccess) {
            (void)hipGetLastError();  // the caller is told; the next launch must not find it
            return false;
        }
        held.push_back(q);
        *p = static_cast<T*>(q);
        return true;
    }
    template <typename T>
    bool upload(T** p, const std::vector<T>& v) {
        if (!alloc(p, v.size())) return false;
        return v.empty() || hipMemcpy(*p, v.data(), v.size() * sizeof(T), hipMemcpyHostToDevice) == hipSuccess;
    }
};

}  // namespace gd
