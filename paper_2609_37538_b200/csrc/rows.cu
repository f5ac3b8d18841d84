// avsg_append and avsg_attend: argument checks and the two calls without a context (with one: avsg_api.cu).
#include <float.h>
#include <math.h>
#include <mutex>
#include <string.h>

#include "rows.h"

namespace avsg {

namespace {

constexpr int MAX_DEVICES = 64;
std::mutex g_mutex;
bool g_ready[MAX_DEVICES] = {false};

bool aligned(const void* p, uint64_t to) { return (reinterpret_cast<uint64_t>(p) & (to - 1)) == 0; }

bool good_rope(const avsg_rope* r)
{
    for (double f : r->inv_freq) if (!isfinite(f)) return false;
    return isfinite(r->scale) && r->halves <= 1;
}

}  // namespace

// What a call without a context runs on: the device that one of its arrays lies on.
int device_of(const void* p, int* device)
{
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return AVSG_ECUDA; }
    if (at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) return AVSG_EINVAL;
    *device = at.device;
    return AVSG_OK;
}

namespace {

// The kernels write to a caller's status word only when something is wrong: where it lies is looked at in every call.
int check_status(const uint32_t* status, int device)
{
    int at = -1;
    if (!status) return AVSG_OK;
    const int rc = device_of(status, &at);
    return rc != AVSG_OK ? rc : at == device ? AVSG_OK : AVSG_EINVAL;
}

// Makes `device` current; its kernels are loaded by the first call on it.
struct OnDevice {
    int prev = -1, rc = AVSG_OK;
    bool other = false;
    explicit OnDevice(int device)
    {
        if (device < 0 || device >= MAX_DEVICES || cudaGetDevice(&prev) != cudaSuccess) { rc = AVSG_ECUDA; return; }
        other = prev != device;
        if (other && cudaSetDevice(device) != cudaSuccess) { rc = AVSG_ECUDA; return; }
        std::lock_guard<std::mutex> lock(g_mutex);
        if (!g_ready[device]) {
            if (append_prepare() != cudaSuccess || attend_prepare() != cudaSuccess) { cudaGetLastError(); rc = AVSG_ECUDA; return; }
            g_ready[device] = true;
        }
    }
    ~OnDevice() { if (other) cudaSetDevice(prev); }
};

}  // namespace

RopeParams rope_params(const avsg_rope* r)
{
    RopeParams p;
    memset(&p, 0, sizeof(p));
    if (!r) return p;
    for (int i = 0; i < 32; ++i) p.turns[i] = r->inv_freq[i] * 0.15915494309189533577;      // 1 / (2 pi)
    p.scale = r->scale; p.halves = r->halves; p.on = 1;
    return p;
}

int check_append(const avsg_append_args* a)
{
    if (!a || a->n == 0 || a->n_tokens == 0 || a->n > ROWS_MAX_TABLES || (uint64_t)a->n * a->n_tokens > 0x7FFFFFFFull) return AVSG_EINVAL;
    const uint64_t bytes = row_bytes_of(a->row_format);
    if (!bytes || a->type > AVSG_TYPE_FP32) return AVSG_EINVAL;
    if (!a->latent || !a->rope_part || !a->positions || !aligned(a->latent, 16) || !aligned(a->rope_part, 16)) return AVSG_EINVAL;
    if (!aligned(a->positions, 4) || !aligned(a->rows, 4) || !aligned(a->values, 16) || !aligned(a->status, 4)) return AVSG_EINVAL;
    for (int i = 0; i < 2; ++i) if (a->latent_stride[i] % 16 || a->rope_stride[i] % 16) return AVSG_EINVAL;
    if (a->kv_base ? a->kv != nullptr : (!a->kv || !aligned(a->kv, 16) || a->kv_table_stride % 16)) return AVSG_EINVAL;
    for (uint32_t i = 0; i < a->n; ++i) {
        if (a->kv_base && (!a->kv_base[i] || !aligned(a->kv_base[i], 16))) return AVSG_EINVAL;
        if (a->row_stride && (a->row_stride[i] % 16 || a->row_stride[i] < bytes || a->row_stride[i] > 0xFFFFFFFFull * 16)) return AVSG_EINVAL;
        if (a->kv_rows && a->kv_rows[i] > 0x80000000u) return AVSG_EINVAL;
    }
    if (a->rope && !good_rope(a->rope)) return AVSG_EINVAL;
    return AVSG_OK;
}

int append_run(const avsg_append_args* a, uint32_t* status, cudaStream_t stream)
{
    // Every address that the GPU cannot reach is refused before anything is launched.
    uint64_t base[ROWS_MAX_TABLES];
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return AVSG_ECUDA; }
    for (uint32_t i = 0; i < (a->kv_base ? a->n : 1u); ++i) {
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, a->kv_base ? a->kv_base[i] : a->kv) != cudaSuccess) { cudaGetLastError(); return AVSG_EINVAL; }
        if (at.type == cudaMemoryTypeUnregistered || !at.devicePointer || (at.type == cudaMemoryTypeDevice && at.device != device)) return AVSG_EINVAL;
        base[i] = reinterpret_cast<uint64_t>(at.devicePointer);
    }
    AppendParams p;
    p.rope = rope_params(a->rope);
    p.n_tokens = a->n_tokens; p.status = status;
    for (int i = 0; i < 2; ++i) { p.latent_stride[i] = a->latent_stride[i]; p.rope_stride[i] = a->rope_stride[i]; }
    const uint32_t bytes = row_bytes_of(a->row_format);
    for (uint32_t first = 0; first < a->n; first += APPEND_MAX_TABLES) {
        const uint32_t cnt = a->n - first < (uint32_t)APPEND_MAX_TABLES ? a->n - first : (uint32_t)APPEND_MAX_TABLES;
        const size_t skipped = (size_t)first * a->n_tokens;
        p.n_launch = cnt;
        p.latent = static_cast<const uint8_t*>(a->latent) + first * a->latent_stride[0];
        p.rope_part = static_cast<const uint8_t*>(a->rope_part) + first * a->rope_stride[0];
        p.positions = a->positions + skipped;
        p.rows = a->rows ? a->rows + skipped : nullptr;
        p.values = a->values ? static_cast<uint8_t*>(a->values) + skipped * (LATENT + ROPE) * 2 : nullptr;
        for (uint32_t i = 0; i < cnt; ++i) {
            p.base[i] = a->kv_base ? base[first + i] : base[0] + (first + i) * a->kv_table_stride;
            p.stride16[i] = (uint32_t)((a->row_stride ? a->row_stride[first + i] : bytes) / 16);
            p.limit[i] = a->kv_rows ? a->kv_rows[first + i] : 0x80000000u;
        }
        if (launch_append(p, a->row_format, a->type, stream) != cudaSuccess) { cudaGetLastError(); return AVSG_ECUDA; }
    }
    return AVSG_OK;
}

int check_attend(const avsg_attend_args* a)
{
    if (!a || a->n == 0 || a->n_tokens == 0 || a->topk == 0 || a->heads == 0 || a->n > ROWS_MAX_TABLES) return AVSG_EINVAL;
    if (!row_bytes_of(a->row_format)) return AVSG_EINVAL;
    if (a->heads > 1024 || (uint64_t)a->n * a->n_tokens > (1u << 24) || a->topk > (1u << 24)) return AVSG_EUNSUPPORTED;
    if (!a->slots || !a->q || !a->out || !aligned(a->slots, 4) || !aligned(a->q, 16) || !aligned(a->out, 16)) return AVSG_EINVAL;
    for (int i = 0; i < 3; ++i) if (a->q_stride[i] % 16 || a->out_stride[i] % 16) return AVSG_EINVAL;
    // (queries may be broadcast; outputs may not)
    if ((a->n > 1 && a->out_stride[0] == 0) || (a->n_tokens > 1 && a->out_stride[1] == 0) || (a->heads > 1 && a->out_stride[2] == 0)) return AVSG_EINVAL;
    if (!aligned(a->lse, 4) || !aligned(a->ids, 4) || !aligned(a->positions, 4) || !aligned(a->spans, 4) || !aligned(a->slopes, 4) || !aligned(a->status, 4))
        return AVSG_EINVAL;
    if (!isfinite(a->scale) || !isfinite(a->softcap) || a->softcap < 0.f || (a->softcap > 0.f && a->softcap < FLT_MIN)) return AVSG_EINVAL;
    if ((a->spans || a->slopes) && !a->ids) return AVSG_EINVAL;
    if ((a->slopes || a->rope) && !a->positions) return AVSG_EINVAL;
    if (a->rope && !good_rope(a->rope)) return AVSG_EINVAL;
    return AVSG_OK;
}

int attend_run(const avsg_attend_args* a, const void* buffer, uint32_t rows, uint64_t row_stride, uint32_t* status, cudaStream_t stream)
{
    AttendParams p;
    p.table_stride = (uint64_t)rows * row_stride; p.row_stride = (uint32_t)row_stride; p.rows = rows;
    p.slopes = a->slopes; p.status = status;
    for (int i = 0; i < 3; ++i) { p.q_stride[i] = a->q_stride[i]; p.out_stride[i] = a->out_stride[i]; }
    p.scale = a->scale; p.softcap = a->softcap;
    // (either factor, and a score times the first, stays within the range of normal floats for every cap)
    p.per_cap[0] = a->softcap >= 1.f ? 5.9604644775390625e-8f : 1.f;                        // 2^-24
    p.per_cap[1] = a->softcap > 0.f ? (float)(0.69314718055994530942 / a->softcap / p.per_cap[0]) : 0.f;
    p.n_tokens = a->n_tokens; p.topk = a->topk; p.heads = a->heads;
    p.rope = rope_params(a->rope);
    p.mapped = a->table_ids != nullptr;
    // Tables of a context travel as kernel arguments, as many as these hold to a launch; others need no list.
    const uint32_t most = a->table_ids ? (uint32_t)ATTEND_MAX_TABLES : a->n;
    for (uint32_t first = 0; first < a->n; first += most) {
        const size_t queries = (size_t)first * a->n_tokens, ids = queries * a->topk;
        p.n = a->n - first < most ? a->n - first : most;
        p.buffer = static_cast<const uint8_t*>(buffer);                                     // (first > 0: tables by their ids)
        p.slots = a->slots + ids; p.ids = a->ids ? a->ids + ids : nullptr;
        p.positions = a->positions ? a->positions + queries : nullptr; p.spans = a->spans ? a->spans + 2 * queries : nullptr;
        p.q = static_cast<const uint8_t*>(a->q) + first * a->q_stride[0]; p.out = static_cast<uint8_t*>(a->out) + first * a->out_stride[0];
        p.lse = a->lse ? a->lse + queries * a->heads : nullptr;
        if (a->table_ids) memcpy(p.table_id, a->table_ids + first, p.n * sizeof(uint32_t));
        if (launch_attend(p, a->row_format, stream) != cudaSuccess) { cudaGetLastError(); return AVSG_ECUDA; }
    }
    return AVSG_OK;
}

// The two calls without a context.
int append_bare(const avsg_append_args* a, cudaStream_t stream)
{
    int rc = check_append(a), device = -1;
    if (rc != AVSG_OK) return rc;
    if (a->table_ids) return AVSG_EINVAL;
    if ((rc = device_of(a->positions, &device)) != AVSG_OK || (rc = check_status(a->status, device)) != AVSG_OK) return rc;
    OnDevice on(device);
    if (on.rc != AVSG_OK) return on.rc;
    return append_run(a, a->status, stream);
}

int attend_bare(const avsg_attend_args* a, cudaStream_t stream)
{
    int rc = check_attend(a), device = -1;
    if (rc != AVSG_OK) return rc;
    const uint64_t bytes = row_bytes_of(a->row_format), stride = a->buffer_row_bytes ? a->buffer_row_bytes : bytes;
    if (a->table_ids || !a->buffer || !aligned(a->buffer, 16) || a->buffer_slots == 0 || a->buffer_slots > 0x80000000u) return AVSG_EINVAL;
    if (stride % 16 || stride < bytes || stride > 0xFFFFFFFFull) return AVSG_EINVAL;
    if ((rc = device_of(a->slots, &device)) != AVSG_OK || (rc = check_status(a->status, device)) != AVSG_OK) return rc;
    OnDevice on(device);
    if (on.rc != AVSG_OK) return on.rc;
    return attend_run(a, a->buffer, a->buffer_slots, stride, a->status, stream);
}

}  // namespace avsg

extern "C" uint32_t avsg_row_bytes(uint32_t row_format) { return avsg::row_bytes_of(row_format); }
