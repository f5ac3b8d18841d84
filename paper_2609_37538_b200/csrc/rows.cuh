// What the kernels that write rows and those that read them share.
#pragma once
#include <cuda_fp16.h>

#include "rows.h"

namespace avsg {

// Cosine and sine (times the rotation's scale) of pair i at a position.  The angle of a far position has many whole turns, which
// 32 bits would leave no digits behind: they are taken off in 64 bits, and half turns go on in 32.
__device__ __forceinline__ void rotation(const RopeParams& r, uint32_t pair, int32_t position, float& c, float& s)
{
    const double t = (double)position * r.turns[pair];
    sincospif(2.f * (float)(t - rint(t)), &s, &c);
    c *= r.scale;
    s *= r.scale;
}

// The two numbers of a byte of e2m1, the low half first.
__device__ __forceinline__ __half2 e2m1_pair(uint32_t byte)
{
    uint32_t two;
    asm("{\n\t.reg .b8 b;\n\tcvt.u8.u32 b, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(two) : "r"(byte));
    return *reinterpret_cast<const __half2*>(&two);
}

}  // namespace avsg
