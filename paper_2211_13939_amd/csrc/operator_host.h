// What the operators' host code (norm.cpp, linear8.cpp, cross.cpp) has in common: the arena's checks, and the device that an object belongs to.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "hostutil.h"

namespace tts {

inline int check_arena(const void* dev_arena, size_t arena_bytes, size_t needed, int* device)
{
    if (!dev_arena) return fail(TTS_E_INVAL, "null argument");
    if (arena_bytes < needed) return fail(TTS_E_INVAL, "arena has %zu bytes, %zu needed", arena_bytes, needed);
    if ((uintptr_t)dev_arena % 256) return fail(TTS_E_INVAL, "arena must be 256-byte aligned");
    hipPointerAttribute_t attr;
    if (hipPointerGetAttributes(&attr, dev_arena) != hipSuccess || attr.type != hipMemoryTypeDevice) {
        (void)hipGetLastError();
        return fail(TTS_E_INVAL, "arena is not device memory");
    }
    *device = attr.device;
    return TTS_OK;
}

// The object's device is current while this lives: a stream takes launches of its own device alone.
class OnDevice {
public:
    explicit OnDevice(int device)
    {
        err = hipGetDevice(&was_);
        if (err == hipSuccess && was_ != device) {
            err = hipSetDevice(device);
            moved_ = err == hipSuccess;
        }
    }
    OnDevice(const OnDevice&) = delete;
    ~OnDevice()
    {
        if (moved_) (void)hipSetDevice(was_);
    }
    hipError_t err;

private:
    int was_ = -1;
    bool moved_ = false;
};

inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
inline int dtype_bytes(int dtype) { return dtype == TTS_DTYPE_BF16 ? 2 : 4; }
inline bool is_dtype(int dtype) { return dtype == TTS_DTYPE_F32 || dtype == TTS_DTYPE_BF16; }

}  // namespace tts
