// Rows whose inside the library knows (AVSG_ROW_*): the launches of the kernels that write and read them.
#pragma once
#include <cuda_runtime_api.h>
#include <stdint.h>

#include "avsg.h"

namespace avsg {

constexpr uint32_t LATENT = AVSG_LATENT_DIMS, ROPE = AVSG_ROPE_DIMS;
constexpr uint32_t FP8_GROUP = 128, FP4_GROUP = 32;             // numbers that share a scale
constexpr uint32_t ROWS_MAX_TABLES = 2048;                      // tables of one call

__host__ __device__ constexpr uint32_t row_bytes_of(uint32_t format)
{
    return format == AVSG_ROW_BF16 ? 1152u : format == AVSG_ROW_FP8 ? 656u : format == AVSG_ROW_FP4 ? 400u : 0u;
}

struct RopeParams {
    double turns[32];       // inv_freq / (2 pi): turns of a pair per position
    float scale;
    uint32_t halves, on;
};

RopeParams rope_params(const avsg_rope* r);

// Tables of one launch: their cache addresses travel as kernel arguments (128 of them stay below 4 KB).
constexpr int APPEND_MAX_TABLES = 128;
struct AppendParams {
    const uint8_t* latent; const uint8_t* rope_part;
    uint64_t latent_stride[2], rope_stride[2];
    const int32_t* positions; const int32_t* rows;
    uint8_t* values; uint32_t* status;
    uint32_t n_tokens, n_launch;
    RopeParams rope;
    uint64_t base[APPEND_MAX_TABLES];
    uint32_t stride16[APPEND_MAX_TABLES];       // bytes between rows / 16
    uint32_t limit[APPEND_MAX_TABLES];          // rows of the cache
};
cudaError_t append_prepare();
cudaError_t launch_append(const AppendParams& p, uint32_t format, uint32_t type, cudaStream_t stream);

constexpr int ATTEND_MAX_TABLES = 128;
struct AttendParams {
    const uint8_t* buffer;
    uint64_t table_stride; uint32_t row_stride; uint32_t rows;      // of a table
    const int32_t* slots; const int32_t* ids; const int32_t* positions; const int32_t* spans; const float* slopes;
    const uint8_t* q; uint64_t q_stride[3];
    uint8_t* out; uint64_t out_stride[3];
    float* lse; uint32_t* status;
    float scale, softcap, per_cap[2];           // 1 / (softcap log2(e)) is per_cap[0] x per_cap[1]
    uint32_t n, n_tokens, topk, heads;
    uint32_t groups, group_heads, cluster;      // set by launch_attend(): groups of heads, heads of one, blocks per query and group
    RopeParams rope;
    uint32_t mapped;                            // table_id holds the tables; else table i is i
    uint32_t table_id[ATTEND_MAX_TABLES];
};
cudaError_t attend_prepare();
cudaError_t launch_attend(AttendParams& p, uint32_t format, cudaStream_t stream);

// The parts of the two calls: the checks, and what follows them with a context's buffers and status word or the caller's own.
// The device that an array lies on (AVSG_EINVAL: on none).
int device_of(const void* p, int* device);
int check_append(const avsg_append_args* a);
int check_attend(const avsg_attend_args* a);
int append_run(const avsg_append_args* a, uint32_t* status, cudaStream_t stream);
int attend_run(const avsg_attend_args* a, const void* buffer, uint32_t rows, uint64_t row_stride, uint32_t* status, cudaStream_t stream);
int append_bare(const avsg_append_args* a, cudaStream_t stream);       // the calls without a context
int attend_bare(const avsg_attend_args* a, cudaStream_t stream);

}  // namespace avsg
