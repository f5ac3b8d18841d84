// avsg_attend, the plain way: a block per query head, softmax over the selected rows in chunks with a running maximum and sum.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "avsg_kernels.cuh"
#include "rows.cuh"

namespace avsg {

namespace {

constexpr uint32_t CHUNK = 128;         // rows at a time = threads

__device__ __forceinline__ float bf16_at(const uint8_t* p, uint32_t i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]); }

template <uint32_t FORMAT>
__device__ __forceinline__ float latent_at(const uint8_t* row, uint32_t d)
{
    if constexpr (FORMAT == AVSG_ROW_BF16) {
        return bf16_at(row, d);
    } else if constexpr (FORMAT == AVSG_ROW_FP8) {
        return __half2float(__half(__nv_cvt_fp8_to_halfraw(row[d], __NV_E4M3))) * reinterpret_cast<const float*>(row + LATENT)[d / FP8_GROUP];
    } else {
        const uint32_t e = row[LATENT / 2 + d / FP4_GROUP];
        const float scale = e == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(1.f, (int)e - 127);
        return __half2float(__half(__nv_cvt_fp4_to_halfraw(row[d / 2] >> (d % 2 * 4), __NV_E2M1))) * scale;
    }
}

}  // namespace

template <uint32_t FORMAT, int CAP>
__global__ void __launch_bounds__(CHUNK) avsg_attend_kernel(const __grid_constant__ AttendParamsT<CAP> p)
{
    __shared__ float q[LATENT + ROPE], weight[CHUNK], part[4];
    __shared__ int32_t slot[CHUNK];
    const uint32_t t = threadIdx.x, item = blockIdx.x / p.heads, head = blockIdx.x % p.heads;
    const uint32_t table = item / p.n_tokens, token = item % p.n_tokens;
    const uint8_t* rows = p.buffer + (uint64_t)(p.mapped ? p.table_id[table] : table) * p.table_stride;
    const uint8_t* query = p.q + table * p.q_stride[0] + token * p.q_stride[1] + head * p.q_stride[2];
    for (uint32_t d = t; d < LATENT + ROPE; d += CHUNK) q[d] = bf16_at(query, d);
    __syncthreads();
    if (p.rope.on && t < 32u) {
        const uint32_t i = LATENT + (p.rope.halves ? t : 2u * t), j = LATENT + (p.rope.halves ? t + 32u : 2u * t + 1u);
        float c, s;
        rotation(p.rope, t, p.positions[item], c, s);
        const float a = q[i], b = q[j];
        q[i] = __bfloat162float(__float2bfloat16_rn(a * c - b * s));
        q[j] = __bfloat162float(__float2bfloat16_rn(a * s + b * c));
    }
    float most = -INFINITY, total = 0.f, out[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t from = 0; from < p.topk; from += CHUNK) {
        __syncthreads();
        const uint32_t k = from + t;
        int32_t s = -1;
        const uint64_t at = (uint64_t)item * p.topk + k;
        if (k < p.topk) {
            s = p.slots[at];
            if (s >= 0 && (uint32_t)s >= p.rows) { s = -1; if (p.status) atomicOr(p.status, ST_BAD_SLOT); }
            if (p.spans && s >= 0 && (p.ids[at] < p.spans[2 * item] || p.ids[at] >= p.spans[2 * item + 1])) s = -1;
        }
        float score = -INFINITY;
        if (s >= 0) {
            const uint8_t* row = rows + (uint64_t)s * p.row_stride;
            score = 0.f;
            for (uint32_t d = 0; d < LATENT; ++d) score += q[d] * latent_at<FORMAT>(row, d);
            for (uint32_t d = 0; d < ROPE; ++d) score += q[LATENT + d] * bf16_at(row + row_bytes_of(FORMAT) - 2 * ROPE, d);
            score *= p.scale;
            if (p.softcap > 0.f) score = p.softcap * (1.f - 2.f / (1.f + expf(2.f * score / p.softcap)));
            if (p.slopes) score += p.slopes[head] * (float)(p.ids[at] - p.positions[item]);
        }
        slot[t] = s;
        float chunk = score;
        for (int o = 16; o; o >>= 1) chunk = fmaxf(chunk, __shfl_xor_sync(0xffffffffu, chunk, o));
        if (t % 32 == 0) part[t / 32] = chunk;
        __syncthreads();
        chunk = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
        const float now = fmaxf(most, chunk), base = now == -INFINITY ? 0.f : now, keep = expf(most - base);
        most = now;
        weight[t] = s >= 0 ? expf(score - base) : 0.f;
        __syncthreads();
        total *= keep;
        for (int j = 0; j < 4; ++j) out[j] *= keep;
        for (uint32_t i = 0; i < CHUNK; ++i) {
            if (slot[i] < 0) continue;
            const uint8_t* row = rows + (uint64_t)slot[i] * p.row_stride;
            total += weight[i];
            for (int j = 0; j < 4; ++j) out[j] += weight[i] * latent_at<FORMAT>(row, t + CHUNK * j);
        }
    }
    __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(p.out + table * p.out_stride[0] + token * p.out_stride[1] + head * p.out_stride[2]);
    for (int j = 0; j < 4; ++j) to[t + CHUNK * j] = __float2bfloat16_rn(total == 0.f ? 0.f : out[j] / total);
    if (p.lse && t == 0) p.lse[(uint64_t)item * p.heads + head] = total == 0.f ? -INFINITY : most + logf(total);
}

namespace {
template <int CAP>
cudaError_t launch(const AttendParamsT<CAP>& p, uint32_t format, cudaStream_t stream)
{
    using Kernel = void (*)(const AttendParamsT<CAP>);
    const Kernel k = format == AVSG_ROW_BF16 ? (Kernel)avsg_attend_kernel<AVSG_ROW_BF16, CAP>
                   : format == AVSG_ROW_FP8 ? (Kernel)avsg_attend_kernel<AVSG_ROW_FP8, CAP> : (Kernel)avsg_attend_kernel<AVSG_ROW_FP4, CAP>;
    void* args[] = {const_cast<AttendParamsT<CAP>*>(&p)};
    return cudaLaunchKernel(k, dim3(p.n * p.n_tokens * p.heads), dim3(CHUNK), args, 0, stream);
}
}  // namespace

cudaError_t attend_prepare() { return cudaSuccess; }
cudaError_t launch_attend(const AttendParams& p, uint32_t format, cudaStream_t stream) { return launch(p, format, stream); }
cudaError_t launch_attend(const AttendParamsBig& p, uint32_t format, cudaStream_t stream) { return launch(p, format, stream); }

}  // namespace avsg
