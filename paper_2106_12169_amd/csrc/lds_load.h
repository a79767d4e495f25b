// Global memory straight to LDS, 16 bytes a lane.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace apnn {

typedef uint32_t v4u_t __attribute__((ext_vector_type(4)));

// Raw buffer descriptor (base, no stride, byte count, 32-bit raw data format).
__device__ __forceinline__ v4u_t make_raw_desc(const void *base, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(base);
    v4u_t d;
    d[0] = static_cast<uint32_t>(a);
    d[1] = static_cast<uint32_t>(a >> 32) & 0xFFFFu;
    d[2] = bytes;
    d[3] = 0x00020000u;
    return d;
}

// Global memory -> LDS, 16 bytes per lane, no registers in between: lane l's data
// lands at LDS byte address lds_base + 16 l (lds_base is wave-uniform and travels
// in M0); a lane whose offset lies outside the descriptor deposits zeros.  Written
// as an instruction sequence of its own so that completion is tracked only by the
// explicit vmcnt waits of the caller (a compiler that knows about the LDS write
// would wait for it before every later LDS read, which serialises the pipeline).
__device__ __forceinline__ void load_to_lds_16(v4u_t desc, uint32_t lds_base, uint32_t voffset, int soffset)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds_base), "v"(voffset), "s"(desc), "s"(soffset)
                 : "memory", "m0");
}

// Between LDS accesses of one wave to memory of its own: the hardware keeps them in order, the compiler has to as well.
__device__ __forceinline__ void lds_in_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}

}  // namespace apnn
