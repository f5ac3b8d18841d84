// avsg_append: rows of new positions, rotated and (for AVSG_ROW_FP8 / AVSG_ROW_FP4) quantised on their way into the cache.
//
// One pass: a warp per position.  A lane holds 16 consecutive numbers of the latent, so that a scale's group is 8 lanes (e4m3) or
// 2 (e2m1), its largest magnitude 3 or 1 shuffles away, and the row leaves as one run of 512 or 256 bytes; lane i turns pair i of the
// rotated part.  Bounded by the bytes (1152 in, a row out) for chunks of a prompt, by the launch and one trip to memory for a decode
// step's few rows.
//
// A code is the nearest to number / scale itself: with scale = largest / 448 the quotients of numbers of few bits lie next to ties by
// the thousand (168.000002 between 160 and 176), and rounded to 32 bits first they would become ties: see sticky_quotient().
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "avsg_kernels.cuh"
#include "rows.h"
#include "rows.cuh"

namespace avsg {

namespace {

constexpr uint32_t WARPS = 4;

template <uint32_t TYPE>
__device__ __forceinline__ float number(const uint8_t* p, uint32_t i)
{
    if constexpr (TYPE == AVSG_TYPE_BF16) return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
    else if constexpr (TYPE == AVSG_TYPE_FP16) return __half2float(reinterpret_cast<const __half*>(p)[i]);
    else return reinterpret_cast<const float*>(p)[i];
}

// A lane's 16 numbers.
template <uint32_t TYPE>
__device__ __forceinline__ void sixteen(const uint8_t* p, float (&x)[16])
{
    constexpr int BYTES = TYPE == AVSG_TYPE_FP32 ? 64 : 32;
    __align__(16) uint4 w[BYTES / 16];
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = number<TYPE>(reinterpret_cast<const uint8_t*>(w), i);
}

// Two numbers at a time.
__device__ __forceinline__ float2 product(float2 a, float2 b)
{
    float2 c;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(c)) : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
    return c;
}
__device__ __forceinline__ float2 sum_of_product(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(d))
        : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)), "l"(reinterpret_cast<const uint64_t&>(c)));
    return d;
}

// x / s such that a later rounding to few bits rounds the exact quotient: cut off towards zero, with the last bit set if anything was
// cut (a quotient that is not a number of few bits is then none of their midpoints either).  r is 1 / s; q is within one step of the
// quotient after one correction, and what is left, x - q s, says by its sign on which side of it.  (s is -scale here, 2^-40 or more in
// magnitude: what is left of a quotient that matters, down to 2^-33 s, must not become zero.)
__device__ __forceinline__ float2 sticky_quotients(float2 x, float2 s, float2 r)
{
    float2 q = product(x, r);
    q = sum_of_product(sum_of_product(q, s, x), r, q);
    const float2 left = sum_of_product(q, s, x);
    auto one = [](float x, float q, float left) {
        const uint32_t bits = __float_as_uint(q);
        const uint32_t cut = (__float_as_uint(left) ^ bits) >> 31;      // the quotient is smaller than q: one step back
        return copysignf(left == 0.f ? q : __uint_as_float((bits - cut) | 1u), x);        // (a zero keeps its sign)
    };
    return make_float2(one(x.x, q.x, left.x), one(x.y, q.y, left.y));
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// The numbers that the row stands for, for the caller that reads them at once.
__device__ __forceinline__ void put_values(uint8_t* to, uint32_t lane, const float (&x)[16])
{
    uint4 w[2];
    uint32_t* v = reinterpret_cast<uint32_t*>(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bf16_pair(x[2 * i], x[2 * i + 1]);
    reinterpret_cast<uint4*>(to + lane * 32)[0] = w[0];
    reinterpret_cast<uint4*>(to + lane * 32)[1] = w[1];
}

}  // namespace

// (16 blocks an SM, 32 registers a thread, where the numbers come in 16 bits: 16.6 us for 32768 rows of e4m3 where 40 registers take 17.1)
template <uint32_t FORMAT, uint32_t TYPE>
__global__ void __launch_bounds__(WARPS * 32, TYPE == AVSG_TYPE_FP32 ? 12 : 16) avsg_append_kernel(const __grid_constant__ AppendParams p)
{
    const uint32_t lane = threadIdx.x & 31u;
    const uint32_t at = blockIdx.x * WARPS + (threadIdx.x >> 5);
    const uint32_t table = at / p.n_tokens, token = at - table * p.n_tokens;
    if (table >= p.n_launch) return;
    const int32_t position = p.positions[at];
    // (numbers are asked for before the position is known: padding is rare)
    const uint8_t* latent = p.latent + table * p.latent_stride[0] + token * p.latent_stride[1];
    const uint8_t* part = p.rope_part + table * p.rope_stride[0] + token * p.rope_stride[1];

    // the rotated part: lane i has pair i
    const uint32_t first = p.rope.halves ? lane : 2u * lane, second = p.rope.halves ? lane + 32u : 2u * lane + 1u;
    float a = number<TYPE>(part, first), b = number<TYPE>(part, second);
    float x[16];
    sixteen<TYPE>(latent + lane * (TYPE == AVSG_TYPE_FP32 ? 64u : 32u), x);
    const int32_t row = p.rows ? p.rows[at] : position;
    if (position < 0 || row < 0) return;
    if ((uint32_t)row >= p.limit[table]) {
        if (lane == 0 && p.status) atomicOr(p.status, ST_BAD_ID);
        return;
    }
    uint8_t* out = reinterpret_cast<uint8_t*>(p.base[table]) + (uint64_t)row * p.stride16[table] * 16u;
    uint8_t* values = p.values ? p.values + (uint64_t)at * (LATENT + ROPE) * 2u : nullptr;
    if (p.rope.on) {
        float c, s;
        rotation(p.rope, lane, position, c, s);
        const float turned = a * c - b * s;
        b = a * s + b * c;
        a = turned;
    }
    auto put_rope = [&](uint8_t* to) {
        if (p.rope.halves) {
            reinterpret_cast<__nv_bfloat16*>(to)[first] = __float2bfloat16_rn(a);
            reinterpret_cast<__nv_bfloat16*>(to)[second] = __float2bfloat16_rn(b);
        } else {
            reinterpret_cast<uint32_t*>(to)[lane] = bf16_pair(a, b);
        }
    };
    put_rope(out + row_bytes_of(FORMAT) - 2u * ROPE);
    if (values) put_rope(values + 2u * LATENT);

    if constexpr (FORMAT == AVSG_ROW_BF16) {
        put_values(out, lane, x);
    } else {
        // Largest magnitude of the scale's group, as bits: they order like the magnitudes, with infinity and NaN above all.
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(x[i]) & 0x7FFFFFFFu);
        constexpr uint32_t LANES = (FORMAT == AVSG_ROW_FP8 ? FP8_GROUP : FP4_GROUP) / 16u;
#pragma unroll
        for (uint32_t o = 1; o < LANES; o <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
        if constexpr (FORMAT == AVSG_ROW_FP8) {
            const float scale = most >= 0x7F800000u ? __uint_as_float(most)
                                                    : fmaxf(__fdiv_rn(__uint_as_float(most), 448.f), 1.17549435e-38f);
            // Where the group is tiny, numbers and scale go up by the same power of two, which leaves the quotients as they are.
            float divisor = scale;
            if (scale < 9.09494701772928237915e-13f) {                            // 2^-40
                divisor *= 18446744073709551616.f;                                // 2^64
#pragma unroll
                for (int i = 0; i < 16; ++i) x[i] *= 18446744073709551616.f;
            }
            const float inverse = __frcp_rn(divisor);
            uint4 code;
            __nv_fp8x2_storage_t* c = reinterpret_cast<__nv_fp8x2_storage_t*>(&code);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                c[i] = __nv_cvt_float2_to_fp8x2(sticky_quotients(make_float2(x[2 * i], x[2 * i + 1]), make_float2(-divisor, -divisor), make_float2(inverse, inverse)),
                                                __NV_SATFINITE, __NV_E4M3);
            reinterpret_cast<uint4*>(out)[lane] = code;
            if (lane % LANES == 0) reinterpret_cast<float*>(out + LATENT)[lane / LANES] = scale;
            if (values)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 v = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(c[i], __NV_E4M3)));
                x[2 * i] = v.x * scale;
                x[2 * i + 1] = v.y * scale;
            }
        } else {
            // floor(log2) is the exponent field; the division by a power of two is exact
            const int e = max((int)(most >> 23) - 127 - 2, -127);
            const bool odd = most >= 0x7F800000u;
            const float inverse = ldexpf(1.f, -e);
            uint2 code = make_uint2(0u, 0u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t two = odd ? 0u : __nv_cvt_float2_to_fp4x2(make_float2(x[2 * i] * inverse, x[2 * i + 1] * inverse), __NV_E2M1, cudaRoundNearest);
                (i < 4 ? code.x : code.y) |= two << (i % 4 * 8);
            }
            reinterpret_cast<uint2*>(out)[lane] = code;
            // the row's 16 scale bytes leave as four words
            const uint32_t byte = odd ? 255u : (uint32_t)(e + 127);
            uint32_t word = __shfl_sync(0xffffffffu, byte, (2u * lane) & 31u);
            word |= __shfl_down_sync(0xffffffffu, word, 1) << 8;
            word |= __shfl_down_sync(0xffffffffu, word, 2) << 16;
            if (lane < 16u && lane % 4u == 0) reinterpret_cast<uint32_t*>(out + LATENT / 2u)[lane / 4u] = word;
            const float twice = odd ? __uint_as_float(0x7FC00000u) : ldexpf(1.f, e + 1);       // (the scale itself may be 2^-127)
            if (values)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 v = __half22float2(e2m1_pair((i < 4 ? code.x : code.y) >> (i % 4 * 8) & 255u));
                x[2 * i] = 0.5f * v.x * twice;
                x[2 * i + 1] = 0.5f * v.y * twice;
            }
        }
    }
    if (values) put_values(values, lane, x);
}

namespace {
using Kernel = void (*)(const AppendParams);
template <uint32_t FORMAT>
Kernel of_type(uint32_t type)
{
    return type == AVSG_TYPE_BF16 ? avsg_append_kernel<FORMAT, AVSG_TYPE_BF16>
         : type == AVSG_TYPE_FP16 ? avsg_append_kernel<FORMAT, AVSG_TYPE_FP16> : avsg_append_kernel<FORMAT, AVSG_TYPE_FP32>;
}
Kernel append_kernel(uint32_t format, uint32_t type)
{
    return format == AVSG_ROW_BF16 ? of_type<AVSG_ROW_BF16>(type) : format == AVSG_ROW_FP8 ? of_type<AVSG_ROW_FP8>(type) : of_type<AVSG_ROW_FP4>(type);
}
}  // namespace

cudaError_t append_prepare()
{
    for (uint32_t f = AVSG_ROW_BF16; f <= AVSG_ROW_FP4; ++f)
        for (uint32_t t = AVSG_TYPE_BF16; t <= AVSG_TYPE_FP32; ++t) {
            cudaFuncAttributes at;                                        // (asking loads the kernel)
            const cudaError_t e = cudaFuncGetAttributes(&at, append_kernel(f, t));
            if (e != cudaSuccess) return e;
        }
    return cudaSuccess;
}

cudaError_t launch_append(const AppendParams& p, uint32_t format, uint32_t type, cudaStream_t stream)
{
    const uint64_t tokens = (uint64_t)p.n_launch * p.n_tokens;
    void* args[] = {const_cast<AppendParams*>(&p)};
    return cudaLaunchKernel(append_kernel(format, type), dim3((uint32_t)((tokens + WARPS - 1) / WARPS)), dim3(WARPS * 32), args, 0, stream);
}

}  // namespace avsg
