// pk_i8.hpp -- element types and unaligned 16-byte accesses shared by the
// 8-bit operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/pk.h"

namespace pk {

typedef __bf16 bf16;
typedef _Float16 f16;

// E elements of T in one 16-byte access that needs only T's own alignment:
// one instruction whatever the address, so that rows of any length and stride
// take the same code.
template <typename T, int E = 16 / (int)sizeof(T)>
struct Pack {
    typedef T V __attribute__((ext_vector_type(E)));
    typedef V U __attribute__((aligned(sizeof(T))));
};

// An fp32 result in T.  The compiler would fold an fp16 conversion and the
// operation before it into one instruction, which leaves out the rounding to
// fp32, for some elements of a lane and not for others: a result's last bit would
// depend on its column and on the tile.
template <typename T>
__device__ __forceinline__ T rounded(float x)
{
    if constexpr (sizeof(T) == 2 && !__is_same(T, bf16)) asm("" : "+v"(x));
    return (T)x;
}

inline int dtype_size(int dtype)
{
    return dtype == PK_F32 ? 4 : dtype == PK_BF16 || dtype == PK_F16 ? 2 : 0;
}

}  // namespace pk
