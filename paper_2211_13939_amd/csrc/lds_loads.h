// A load from memory straight into LDS, written out: of the builtin the compiler does not know which of two buffers it fills, and waits for it in front of every read of the other.  It has no
// registers to come back to; what it brings is there behind a wait that the caller writes.  m0, where it goes, is its own: it sets it itself, and its old value is no longer there.
//
// A vector instruction that reads a scalar register needs five wait states behind a vector instruction that wrote it (v_readfirstlane, or v_readlane, which is how spilled scalar registers come back).
// The compiler keeps them ahead of loads of its own, but does not look into these, so the base is passed on by a scalar instruction, which needs none.  It stands where m0 needs a wait state.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tts {

// BYTES a lane, from a wave's address and a lane's offset
template <int BYTES> __device__ __forceinline__ void to_lds_from(const void* base, uint32_t offset, uint32_t to)
{
    static_assert(BYTES == 16 || BYTES == 4, "");
    uint32_t m0;
    uint64_t at;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %1, %4\n\tglobal_load_lds_dwordx4 %3, %1" : "={m0}"(m0), "=&s"(at) : "s"(to), "v"(offset), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 m0, %2\n\ts_mov_b64 %1, %4\n\tglobal_load_lds_dword %3, %1" : "={m0}"(m0), "=&s"(at) : "s"(to), "v"(offset), "s"(base) : "memory");
}

}  // namespace tts
