// The paged cache of 4-bit codes: geometry and checks shared by the entry points that write and read it.
#pragma once
#include "dense.h"

#include <type_traits>

namespace apnn {

// Checks a cache description; APNN_OK or the failure of entry point `who`.
int check_cache(const char *who, const apnn_kv_cache *c);

// Row of (token slot, head) in the code and scale arrays.
__host__ __device__ __forceinline__ int64_t cache_row(int64_t slot, int head, int heads, int page_shift)
{
    return (((slot >> page_shift) * heads + head) << page_shift) + (slot & ((1 << page_shift) - 1));
}

// f(integral constant D) for the supported sizes
template <class F> int by_channels(int D, F &&f)
{
    switch (D) {
        case 64: return f(std::integral_constant<int, 64>{});
        case 96: return f(std::integral_constant<int, 96>{});
        case 128: return f(std::integral_constant<int, 128>{});
        default: return f(std::integral_constant<int, 256>{});
    }
}

inline int shift_of(int power_of_two) { return __builtin_ctz(static_cast<unsigned>(power_of_two)); }

}  // namespace apnn
