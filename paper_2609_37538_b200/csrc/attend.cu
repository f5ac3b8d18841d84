// avsg_attend on the matrix unit: a block (or a cluster of them) per query and group of up to 64 heads.
//
// For 64 selected rows at a time ("tile"), S = Q K^T (64 heads x 64 rows, 576 steps), softmax weights P with a running maximum, and
// O^T += V^T P^T (512 numbers x heads, 64 steps).  Rows are gathered, converted and laid out in shared memory ONCE, and serve both
// products: as K with lines along the sum, as V^T with lines along its rows, which the unit reads from the same bytes.  O is kept
// transposed so that its 512 numbers fill all 128 lanes four times over and heads, of which there may be few, are the free dimension.
//
// Formats.  bf16 rows are multiplied as they are, with bf16 weights.  e4m3 and 4-bit rows become fp16 numbers in units of a power of
// two of the row's own (put_row()): bf16 would round every element to 8 bits (error of the result 1.7 x that of its own last
// rounding), fp16 rounds an e4m3 times its scale to 11 and holds a 4-bit one exactly.  The row's unit goes onto its score in 32 bits, and onto its
// weight, which then is held in units of the largest row's.  Queries become fp16 in units of a power of two of the head's (exact: they have 8 bits).  The rotated
// 64 numbers are bf16 on both sides and have a product of their own.
//
// Warps: 0-3 softmax (16 heads each), 4-11 rows (each gathers 8 of a tile's 64, one tile ahead in registers), 12 issues the products.
// Two tiles in shared memory, two S in TMEM: the unit computes S of tile j + 1 while the weights of tile j are formed.
//
// A query's rows are split over a cluster's blocks where queries are few, tile by tile in turn; the blocks' sums are joined through
// distributed shared memory in a fixed order (same results on every run, no workspace).
#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "avsg_kernels.cuh"
#include "rows.cuh"
#include "tensor.cuh"

namespace avsg {

namespace {

constexpr uint32_t TILE = 64, GROUP = 64;                   // rows of a tile, most heads of a block
constexpr uint32_t SOFTMAX_WARPS = 4, ROW_WARPS = 8, THREADS = 32 * (SOFTMAX_WARPS + ROW_WARPS + 1);
constexpr uint32_t PIECE = 64 * 128;                        // 64 lines of 64 16-bit numbers
constexpr uint32_t PIECES = (LATENT + ROPE) / 64;           // of a row: 8 of the latent, 1 rotated
constexpr uint32_t MAX_CLUSTER = 8;

// Shared memory, in bytes.
constexpr uint32_t AT_Q = 0, AT_ROWS = PIECES * PIECE, AT_P = AT_ROWS + 2 * PIECES * PIECE, AT_INFO = AT_P + PIECE;
constexpr uint32_t AT_ALPHA = AT_INFO + 2 * TILE * 8, AT_MOST = AT_ALPHA + 2 * GROUP * 4, AT_TOTAL = AT_MOST + GROUP * 4, AT_UNIT = AT_TOTAL + GROUP * 4;
constexpr uint32_t AT_BARS = AT_UNIT + GROUP * 4, AT_MISC = AT_BARS + 8 * 8, SHARED_BYTES = AT_MISC + 96;
static_assert(SHARED_BYTES <= 232448, "more than a block can have");
// after the last product: O in 32 bits [heads][512] where the tiles were, and the blocks' shares in it behind
constexpr uint32_t AT_OUT = AT_ROWS, AT_SHARE = AT_OUT + GROUP * LATENT * 4;
static_assert(AT_SHARE + MAX_CLUSTER * GROUP * 4 <= AT_P, "");

// TMEM columns: O^T in four parts of 128 numbers, S of two tiles (latent part, rotated part)
constexpr uint32_t COL_OUT = 0, COL_S = 256, COL_ROT = 384, COLUMNS = 512;

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LAZY = 4.f;             // the maximum that weights refer to lags behind by up to this (log2): O is rescaled seldom
constexpr float ROOM = 2048.f;          // fp16 weights are multiplied by this: up to 2^(11 + 4) with a lagging maximum, whole to 2^-25
constexpr long long WAIT_CLOCKS = 1ll << 29;        // about 0.3 s: longer than any wait that ends

constexpr uint32_t LEAST_UNIT = 27u << 23;          // 2^-100: no row's unit is smaller, so that ratios of units stay finite

struct Misc {
    uint32_t tmem, failed;
    int32_t last[THREADS / 32];
    float unit;                         // largest row unit that O's weights refer to
};

// A warp waits, bounded: false (and the block's other waits end too) if nothing came.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile Misc* misc)
{
    if (__all_sync(0xffffffffu, barrier_done(bar, parity))) return true;
    const long long start = clock64();
    while (!__all_sync(0xffffffffu, barrier_done(bar, parity)))
        if (__any_sync(0xffffffffu, misc->failed || clock64() - start > WAIT_CLOCKS)) { misc->failed = 1; return false; }
    return true;
}

// What a lane of a row warp has of one row: every fourth 16-byte unit, and its scales.
template <uint32_t FORMAT>
struct RowPart {
    static constexpr int BODY = FORMAT == AVSG_ROW_BF16 ? 16 : FORMAT == AVSG_ROW_FP8 ? 8 : 4;
    uint4 body[BODY], rope[2], scales;
};

__device__ __forceinline__ uint4 zeros() { return make_uint4(0u, 0u, 0u, 0u); }

template <uint32_t FORMAT>
__device__ __forceinline__ void get_row(RowPart<FORMAT>& v, const uint8_t* row, uint32_t sub)
{
    const uint4* at = reinterpret_cast<const uint4*>(row);
    if (row == nullptr) {               // masked: zeros, so that nothing of it reaches a sum
#pragma unroll
        for (int i = 0; i < RowPart<FORMAT>::BODY; ++i) v.body[i] = zeros();
        v.rope[0] = v.rope[1] = v.scales = zeros();
        return;
    }
#pragma unroll
    for (int i = 0; i < RowPart<FORMAT>::BODY; ++i) v.body[i] = __ldg(at + 4 * i + sub);
    if constexpr (FORMAT != AVSG_ROW_BF16) v.scales = __ldg(at + 4 * RowPart<FORMAT>::BODY);
#pragma unroll
    for (int i = 0; i < 2; ++i) v.rope[i] = __ldg(at + (row_bytes_of(FORMAT) - 2 * ROPE) / 16 + 4 * i + sub);
}

__device__ __forceinline__ void put_unit(uint32_t piece, uint32_t line, uint32_t unit, uint4 v)
{
    asm volatile("st.shared::cta.v4.b32 [%0], {%1, %2, %3, %4};"
                 :: "r"(piece + line * 128u + ((unit ^ (line & 7u)) << 4)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint32_t bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

// 2^e as fp16, zero where that has no such number.
__device__ __forceinline__ uint32_t half_power(int e)
{
    const int field = e + 15;
    return field > 0 ? (uint32_t)field << 10 : field > -10 ? 1u << (field + 9) : 0u;
}

// Lays a lane's part of a row out as line `line` of a tile; returns the unit that its fp16 numbers are in (1 for bf16).
// The eight lanes of a store's phase have the eight lines of a piece: no two of them share a bank.
template <uint32_t FORMAT>
__device__ __forceinline__ float put_row(const RowPart<FORMAT>& v, uint32_t tile, uint32_t line, uint32_t sub)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) put_unit(tile + 8 * PIECE, line, 4 * i + sub, v.rope[i]);
    if constexpr (FORMAT == AVSG_ROW_BF16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) put_unit(tile + (i / 2) * PIECE, line, (i % 2) * 4 + sub, v.body[i]);
        return 1.f;
    } else if constexpr (FORMAT == AVSG_ROW_FP8) {
        // Unit: the power of two at or above the largest scale, / 128: numbers reach 448 x 128 = 57344.
        const uint32_t s[4] = {v.scales.x, v.scales.y, v.scales.z, v.scales.w};
        uint32_t most = LEAST_UNIT + (7u << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, s[i] & 0x7FFFFFFFu);
        if (most < 0x7F800000u) most = (most + 0x007FFFFFu) & 0xFF800000u;
        const uint32_t unit = most < 0x7F800000u ? most - (7u << 23) : most;
        const float inverse = __uint_as_float((254u << 23) - (unit & 0x7F800000u));
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            // scale / unit in two fp16 numbers: a code times it is rounded once, to 11 bits
            const float ratio = most < 0x7F800000u ? __uint_as_float(s[g]) * inverse : __uint_as_float(0x7FC00000u);
            const __half high = __float2half_rn(ratio), low = __float2half_rn(ratio - __half2float(high));
            const __half2 high2 = __half2half2(high), low2 = __half2half2(low);
#pragma unroll
            for (int i = 2 * g; i < 2 * g + 2; ++i) {
                const uint32_t w[4] = {v.body[i].x, v.body[i].y, v.body[i].z, v.body[i].w};
                uint32_t to[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const __half2 k = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[j / 2] >> (j % 2 * 16)), __NV_E4M3));
                    to[j] = bits(__hfma2(k, high2, __hmul2(k, low2)));
                }
                // numbers 16 (4 i + sub) ..: piece i, units 2 sub and 2 sub + 1
                put_unit(tile + i * PIECE, line, 2 * sub, make_uint4(to[0], to[1], to[2], to[3]));
                put_unit(tile + i * PIECE, line, 2 * sub + 1, make_uint4(to[4], to[5], to[6], to[7]));
            }
        }
        return __uint_as_float(unit);
    } else {
        // Unit: the largest scale / 2^13: numbers reach 6 x 8192 = 49152.  All products are exact.
        const uint32_t s[4] = {v.scales.x, v.scales.y, v.scales.z, v.scales.w};
        uint32_t most = __vmaxu4(__vmaxu4(s[0], s[1]), __vmaxu4(s[2], s[3]));
        most = __vmaxu4(most, most >> 16);
        most = max(most & 255u, most >> 8 & 255u);
        const int unit = max((int)most - 13, (int)(LEAST_UNIT >> 23));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t e = s[i] >> (8 * sub) & 255u;
            const uint32_t ratio = e == 255u ? 0x7E00u : half_power((int)e - unit);
            const uint32_t two = ratio | ratio << 16;
            const uint32_t w[4] = {v.body[i].x, v.body[i].y, v.body[i].z, v.body[i].w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t to[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] = bits(__hmul2(e2m1_pair(w[u] >> (8 * j) & 255u), *reinterpret_cast<const __half2*>(&two)));
                // numbers 32 (4 i + sub) + 8 u ..: piece 2 i + sub / 2, unit 4 (sub % 2) + u
                put_unit(tile + (2 * i + sub / 2) * PIECE, line, 4 * (sub % 2) + u, make_uint4(to[0], to[1], to[2], to[3]));
            }
        }
        return __uint_as_float((uint32_t)unit << 23);
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

}  // namespace

template <uint32_t FORMAT, bool SHAPED>
__global__ void __launch_bounds__(THREADS, 1) avsg_attend_kernel(const __grid_constant__ AttendParams p)
{
    constexpr bool HALF = FORMAT != AVSG_ROW_BF16;
    extern __shared__ __align__(1024) uint8_t shared[];
    const uint32_t base = shared_address(shared);
    Misc* misc = reinterpret_cast<Misc*>(shared + AT_MISC);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    // barriers: [0, 1] tile laid out, [2, 3] S there, [4] P there, [5, 6] tile and P read, [7] queries there
    const uint32_t bars = base + AT_BARS;

    const uint32_t rank = blockIdx.x % p.cluster, work = blockIdx.x / p.cluster;
    const uint32_t group = work % p.groups, item = work / p.groups;
    const uint32_t table = item / p.n_tokens, token = item - table * p.n_tokens;
    const uint32_t first_head = group * p.group_heads, heads = min(p.group_heads, p.heads - first_head);
    const uint32_t columns = (heads + 15u) & ~15u;
    const int32_t* slots = p.slots + (uint64_t)item * p.topk;
    const int32_t* ids = p.ids ? p.ids + (uint64_t)item * p.topk : nullptr;

    // The selection's last position: what is behind it (padding) costs nothing.
    int32_t last = -1;
    for (uint32_t k = threadIdx.x; k < p.topk; k += THREADS) if (slots[k] >= 0) last = (int32_t)k;
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) misc->last[warp] = last;
    if (threadIdx.x == 0) {
        misc->failed = 0;
        for (uint32_t i = 0; i < 2; ++i) { barrier_init(bars + 8 * i, ROW_WARPS * 32); barrier_init(bars + 8 * (2 + i), 1); barrier_init(bars + 8 * (5 + i), 1); }
        barrier_init(bars + 8 * 4, SOFTMAX_WARPS * 32);
        barrier_init(bars + 8 * 7, SOFTMAX_WARPS * 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == SOFTMAX_WARPS + ROW_WARPS) tmem_alloc(base + AT_MISC, COLUMNS);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&misc->tmem);
#pragma unroll
    for (uint32_t w = 0; w < THREADS / 32; ++w) last = max(last, misc->last[w]);
    const uint32_t all_tiles = (uint32_t)(last + 1 + (int32_t)TILE - 1) / TILE;
    const uint32_t tiles = all_tiles > rank ? (all_tiles - rank + p.cluster - 1) / p.cluster : 0u;       // rank, rank + cluster, ...

    if (warp < SOFTMAX_WARPS) {
        // ---- queries: warp w's 16 lines are its 16 heads ----
        float cosine = 1.f, sine = 0.f;
        const uint32_t first = p.rope.halves ? lane : 2u * lane, second = p.rope.halves ? lane + 32u : 2u * lane + 1u;
        if (p.rope.on) rotation(p.rope, lane, p.positions[item], cosine, sine);
        float* unit_of = reinterpret_cast<float*>(shared + AT_UNIT);
#pragma unroll 4
        for (uint32_t i = 0; i < 16; ++i) {
            const uint32_t h = warp * 16u + i;
            uint4 u[2] = {zeros(), zeros()};
            float a = 0.f, b = 0.f;
            if (h < heads) {
                const uint8_t* q = p.q + table * p.q_stride[0] + token * p.q_stride[1] + (first_head + h) * p.q_stride[2];
                u[0] = __ldg(reinterpret_cast<const uint4*>(q) + lane);
                u[1] = __ldg(reinterpret_cast<const uint4*>(q) + lane + 32);
                const __nv_bfloat16* r = reinterpret_cast<const __nv_bfloat16*>(q) + LATENT;
                a = __bfloat162float(r[first]);
                b = __bfloat162float(r[second]);
            }
            if (p.rope.on) {
                const float turned = a * cosine - b * sine;
                b = a * sine + b * cosine;
                a = turned;
            }
            auto put_bf16 = [&](uint32_t d, uint32_t at, float x) {
                *reinterpret_cast<__nv_bfloat16*>(shared + AT_Q + 8 * PIECE + at * 128u + (((d >> 3) ^ (at & 7u)) << 4) + (d & 7u) * 2u) = __float2bfloat16_rn(x);
            };
            put_bf16(first, h, a);
            put_bf16(second, h, b);
            if constexpr (HALF) {
                const uint32_t* w = reinterpret_cast<const uint32_t*>(u);
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) most = max(most, max(w[j] << 16 & 0x7FFF0000u, w[j] & 0x7FFF0000u));
                most = __reduce_max_sync(0xffffffffu, most);
                const uint32_t e = max(most >> 23, 14u);               // the largest becomes 2^13 or more, below 2^14
                const float inverse = __uint_as_float((267u - e) << 23);
                if (lane == 0) unit_of[h] = __uint_as_float((e - 13u) << 23);
                uint32_t* to = reinterpret_cast<uint32_t*>(u);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    to[j] = bits(__floats2half2_rn(__uint_as_float(w[j] << 16) * inverse, __uint_as_float(w[j] & 0xFFFF0000u) * inverse));
            }
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) put_unit(base + AT_Q + (lane / 8u + 4u * j) * PIECE, h, lane % 8u, u[j]);
        }
        fence_for_matrix_unit();
        barrier_arrive(bars + 8 * 7);

        // ---- softmax: a thread has 16 rows' scores of two heads ----
        __syncwarp();
        const uint32_t row[2] = {warp * 16u + lane / 4u, warp * 16u + lane / 4u + 8u};
        const bool mine = warp * 16u < columns;
        float factor[2], slope[2] = {0.f, 0.f};
        const float to_log2 = p.scale * LOG2E;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            factor[i] = HALF ? unit_of[row[i]] * to_log2 : to_log2;
            if (SHAPED && p.slopes && row[i] < heads) slope[i] = p.slopes[first_head + row[i]] * LOG2E;
        }
        const int32_t position = SHAPED && p.slopes ? p.positions[item] : 0;
        float most[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f}, unit = 0.f;
        for (uint32_t j = 0; j < tiles; ++j) {              // (also after a wait that failed: the warps meet at a barrier)
            const uint32_t b = j & 1u;
            wait(bars + 8 * (2 + b), j >> 1 & 1u, misc);
            tmem_after_sync();
            const float2* info = reinterpret_cast<const float2*>(shared + AT_INFO) + b * TILE;
            float s[32];
            float now = 0.f;                       // the tile's largest unit
            bool rescale = false;
            if (mine) {
                tmem_load_16x64(tmem + (warp * 32u << 16) + COL_S + 64 * b, s);
                if constexpr (HALF) {
                    float rotated[32];
                    tmem_load_16x64(tmem + (warp * 32u << 16) + COL_ROT + 64 * b, rotated);
                    tmem_loaded();
#pragma unroll
                    for (int g = 0; g < 8; ++g)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float r = info[8 * g + 2 * (lane % 4u) + i].x;
                            now = fmaxf(now, r);
                            s[4 * g + i] = s[4 * g + i] * (factor[0] * r) + rotated[4 * g + i] * to_log2;
                            s[4 * g + 2 + i] = s[4 * g + 2 + i] * (factor[1] * r) + rotated[4 * g + 2 + i] * to_log2;
                        }
                } else {
                    tmem_loaded();
#pragma unroll
                    for (int i = 0; i < 32; ++i) s[i] *= to_log2;
                }
                float tile_most[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int g = 0; g < 8; ++g)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 about = info[8 * g + 2 * (lane % 4u) + i];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            float& x = s[4 * g + 2 * k + i];
                            if constexpr (SHAPED) {
                                // cap x tanh(x / cap), by exp2 alone: off by 2^-22 of the cap at most, however small x is
                                if (p.softcap > 0.f) x = p.softcap * LOG2E * (1.f - 2.f / (1.f + exp2f(x * (2.f / p.softcap))));
                                if (p.slopes) x += slope[k] * (float)(__float_as_int(about.y) - position);
                            }
                            if (about.x == 0.f) x = -INFINITY;
                            tile_most[k] = fmaxf(tile_most[k], x);
                        }
                    }
                float keep[2] = {1.f, 1.f};
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    tile_most[k] = fmaxf(tile_most[k], __shfl_xor_sync(0xffffffffu, tile_most[k], 1));
                    tile_most[k] = fmaxf(tile_most[k], __shfl_xor_sync(0xffffffffu, tile_most[k], 2));
                    if (tile_most[k] > most[k] + LAZY || (most[k] == -INFINITY && tile_most[k] > -INFINITY)) {
                        keep[k] = exp2f(most[k] - tile_most[k]);
                        most[k] = tile_most[k];
                        total[k] *= keep[k];
                        rescale = true;
                    }
                }
                if constexpr (HALF) {
                    now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 1));
                    now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, 2));
                    if (now > unit) {
                        const float less = unit / now;
                        keep[0] *= less;
                        keep[1] *= less;
                        unit = now;
                        rescale = true;
                    }
                }
                if (lane % 4u == 0) {
                    float* alpha = reinterpret_cast<float*>(shared + AT_ALPHA) + b * GROUP;
                    alpha[row[0]] = keep[0];
                    alpha[row[1]] = keep[1];
                }
            }
            // Any head's reference moved: O is brought to the new ones before this tile's product is added.
            int any;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, 1, 128, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
                         : "=r"(any) : "r"((int)(rescale && j > 0)) : "memory");
            if (mine) {
                const float weight = HALF ? ROOM / fmaxf(unit, __uint_as_float(LEAST_UNIT)) : 1.f;
                uint32_t packed[16];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float from = most[k] == -INFINITY ? 0.f : most[k];
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        float w[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            w[i] = exp2f(s[4 * g + 2 * k + i] - from);
                            total[k] += w[i];
                            if constexpr (HALF) w[i] *= info[8 * g + 2 * (lane % 4u) + i].x * weight;
                        }
                        packed[8 * k + g] = HALF ? bits(__floats2half2_rn(w[0], w[1])) : bf16_pair(w[0], w[1]);
                    }
                }
                if (j > 0) wait(bars + 8 * (5 + (b ^ 1u)), (j - 1) >> 1 & 1u, misc);
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (uint32_t g = 0; g < 8; ++g)
                        *reinterpret_cast<uint32_t*>(shared + AT_P + row[k] * 128u + ((g ^ (row[k] & 7u)) << 4) + (lane % 4u) * 4u) = packed[8 * k + g];
                fence_for_matrix_unit();
            } else if (j > 0) {
                wait(bars + 8 * (5 + (b ^ 1u)), (j - 1) >> 1 & 1u, misc);
            }
            if (any) {
                tmem_after_sync();
                const float* alpha = reinterpret_cast<const float*>(shared + AT_ALPHA) + b * GROUP;
                for (uint32_t part = 0; part < 4; ++part)
                    for (uint32_t c = 0; c < columns; c += 16) {
                        float x[16];
                        const uint32_t at = tmem + (warp * 32u << 16) + COL_OUT + 64 * part + c;
                        tmem_load_32x16(at, x);
                        tmem_loaded();
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] *= alpha[c + i];
                        tmem_store_32x16(at, x);
                    }
                tmem_stored();
            }
            tmem_before_sync();
            barrier_arrive(bars + 8 * 4);
        }
        float* most_of = reinterpret_cast<float*>(shared + AT_MOST);
        float* total_of = reinterpret_cast<float*>(shared + AT_TOTAL);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            total[k] += __shfl_xor_sync(0xffffffffu, total[k], 1);
            total[k] += __shfl_xor_sync(0xffffffffu, total[k], 2);
            if (lane % 4u == 0) { most_of[row[k]] = most[k]; total_of[row[k]] = total[k]; }
        }
        if (threadIdx.x == 0) misc->unit = HALF ? unit / ROOM : 1.f;
    } else if (warp < SOFTMAX_WARPS + ROW_WARPS) {
        // ---- rows ----
        const uint32_t line = (warp - SOFTMAX_WARPS) * 8u + lane % 8u, sub = lane / 8u;
        const uint8_t* rows = p.buffer + (uint64_t)(p.mapped ? p.table_id[table] : table) * p.table_stride;
        int32_t begin = INT32_MIN, end = INT32_MAX;
        if (p.spans) { begin = p.spans[2 * item]; end = p.spans[2 * item + 1]; }
        struct Place { const uint8_t* row; int32_t id; };
        auto place = [&](uint32_t j) -> Place {
            Place to = {nullptr, 0};
            const uint64_t k = (uint64_t)(rank + j * p.cluster) * TILE + line;
            if (j >= tiles || k >= p.topk) return to;
            const int32_t slot = __ldg(slots + k);
            if (ids) to.id = __ldg(ids + k);
            if (slot < 0 || (p.spans && (to.id < begin || to.id >= end))) return to;
            if ((uint32_t)slot >= p.rows) { if (p.status) atomicOr(p.status, ST_BAD_SLOT); return to; }
            to.row = rows + (uint64_t)slot * p.row_stride;
            return to;
        };
        RowPart<FORMAT> part;
        Place here = place(0), next = place(1);
        get_row(part, here.row, sub);
        for (uint32_t j = 0; j < tiles; ++j) {
            const uint32_t b = j & 1u;
            if (j >= 2 && !wait(bars + 8 * (5 + b), (j - 2) >> 1 & 1u, misc)) break;
            const float unit = put_row(part, base + AT_ROWS + b * PIECES * PIECE, line, sub);
            if (sub == 0) reinterpret_cast<float2*>(shared + AT_INFO)[b * TILE + line] = make_float2(here.row ? unit : 0.f, __int_as_float(here.id));
            fence_for_matrix_unit();
            barrier_arrive(bars + 8 * b);
            here = next;
            get_row(part, here.row, sub);
            next = place(j + 2);
        }
    } else {
        // ---- products ----
        const uint32_t s_shape = product_shape(!HALF, 64, 64, false), rot_shape = product_shape(true, 64, 64, false);
        const uint32_t out_shape = product_shape(!HALF, 128, columns, true);
        bool ok = wait(bars + 8 * 7, 0, misc);
        auto scores = [&](uint32_t j) {
            const uint32_t b = j & 1u, tile = base + AT_ROWS + b * PIECES * PIECE;
            for (uint32_t c = 0; c < PIECES; ++c)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k) {
                    const uint64_t q = operand(base + AT_Q + c * PIECE + 32 * k, 16), r = operand(tile + c * PIECE + 32 * k, 16);
                    if (HALF && c == 8) multiply(tmem + COL_ROT + 64 * b, q, r, rot_shape, k > 0);
                    else multiply(tmem + COL_S + 64 * b, q, r, s_shape, c + k > 0);
                }
            products_done(bars + 8 * (2 + b));
        };
        auto sums = [&](uint32_t j) {
            const uint32_t b = j & 1u, tile = base + AT_ROWS + b * PIECES * PIECE;
            for (uint32_t part = 0; part < 4; ++part)
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    multiply(tmem + COL_OUT + 64 * part, operand(tile + 2 * part * PIECE + 2048 * k, PIECE), operand(base + AT_P + 32 * k, 16), out_shape, j + k > 0);
            products_done(bars + 8 * (5 + b));
        };
        for (uint32_t j = 0; j <= tiles && ok && tiles; ++j) {
            if (j < tiles) {
                ok = wait(bars + 8 * (j & 1u), j >> 1 & 1u, misc);
                tmem_after_sync();
                if (ok && lane == 0) scores(j);
                __syncwarp();
            }
            if (j > 0 && ok) {
                ok = wait(bars + 8 * 4, (j - 1) & 1u, misc);
                tmem_after_sync();
                if (ok && lane == 0) sums(j - 1);
                __syncwarp();
            }
        }
    }

    // ---- the block's sums to shared memory, and the cluster's blocks' together ----
    __syncwarp();
    if (tiles) wait(bars + 8 * (5 + ((tiles - 1) & 1u)), (tiles - 1) >> 1 & 1u, misc);
    tmem_after_sync();
    __syncwarp();
    if (warp < 8 && tiles) {
        float* out = reinterpret_cast<float*>(shared + AT_OUT);
        const uint32_t quarter = warp & 3u;
        for (uint32_t part = warp / 4u; part < 4u; part += 2)
            for (uint32_t c = 0; c < columns; c += 16) {
                float x[16];
                tmem_load_32x16(tmem + (quarter * 32u << 16) + COL_OUT + 64 * part + c, x);
                tmem_loaded();
#pragma unroll
                for (int i = 0; i < 16; ++i) out[(c + i) * LATENT + part * 128u + quarter * 32u + lane] = x[i];
            }
    }
    tmem_before_sync();
    __syncthreads();
    if (warp == SOFTMAX_WARPS + ROW_WARPS) {
        if (misc->failed) __nanosleep(100000);                  // (products that nobody waits for any more)
        __syncwarp();
        tmem_after_sync();
        tmem_free(tmem, COLUMNS);
    }
    if (p.cluster > 1) cluster_sync();
    float* share = reinterpret_cast<float*>(shared + AT_SHARE);
    if (threadIdx.x < heads) {
        const uint32_t h = threadIdx.x;
        float most = -INFINITY, total = 0.f;
        for (uint32_t c = 0; c < p.cluster; ++c) most = fmaxf(most, load_float(in_block(base + AT_MOST + 4 * h, c)));
        const float from = most == -INFINITY ? 0.f : most;
        for (uint32_t c = 0; c < p.cluster; ++c)
            total += load_float(in_block(base + AT_TOTAL + 4 * h, c)) * exp2f(load_float(in_block(base + AT_MOST + 4 * h, c)) - from);
        for (uint32_t c = 0; c < p.cluster; ++c) {
            const float t = load_float(in_block(base + AT_TOTAL + 4 * h, c)), m = load_float(in_block(base + AT_MOST + 4 * h, c));
            share[c * GROUP + h] = t == 0.f ? 0.f : exp2f(m - from) * load_float(in_block(base + AT_MISC + offsetof(Misc, unit), c)) / total;
        }
        if (rank == 0 && p.lse)
            p.lse[(uint64_t)item * p.heads + first_head + h] = total == 0.f ? -INFINITY : (most + log2f(total)) * 0.6931471805599453f;
    }
    __syncthreads();
    uint8_t* out = p.out + table * p.out_stride[0] + token * p.out_stride[1] + first_head * p.out_stride[2];
    if (!misc->failed)
        for (uint32_t u = rank * THREADS + threadIdx.x; u < heads * (LATENT / 8); u += p.cluster * THREADS) {
            const uint32_t h = u / (LATENT / 8), d = u % (LATENT / 8);
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (uint32_t c = 0; c < p.cluster; ++c) {
                const float w = share[c * GROUP + h];
                if (w == 0.f) continue;                         // (a block without rows has no sums either)
                const uint32_t at = in_block(base + AT_OUT + (h * LATENT + 8 * d) * 4u, c);
                const float4 v = load_float4(at), y = load_float4(at + 16);
                x[0] += w * v.x; x[1] += w * v.y; x[2] += w * v.z; x[3] += w * v.w;
                x[4] += w * y.x; x[5] += w * y.y; x[6] += w * y.z; x[7] += w * y.w;
            }
            *reinterpret_cast<uint4*>(out + h * p.out_stride[2] + 16 * d) =
                make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
        }
    else if (threadIdx.x == 0 && p.status) atomicOr(p.status, ST_WAIT_TIMEOUT);
    __syncthreads();
    if (p.cluster > 1) cluster_sync();                          // nobody leaves whose memory is still read
}

namespace {

using Kernel = void (*)(const AttendParams);
Kernel attend_kernel(uint32_t format, bool shaped)
{
    static const Kernel k[3][2] = {{avsg_attend_kernel<AVSG_ROW_BF16, false>, avsg_attend_kernel<AVSG_ROW_BF16, true>},
                                   {avsg_attend_kernel<AVSG_ROW_FP8, false>, avsg_attend_kernel<AVSG_ROW_FP8, true>},
                                   {avsg_attend_kernel<AVSG_ROW_FP4, false>, avsg_attend_kernel<AVSG_ROW_FP4, true>}};
    return k[format][shaped];
}

// Clusters of 2, 4, 8 blocks that a device runs at once (blocks of a cluster share a GPC), as found by attend_prepare().
constexpr int MAX_DEVICES = 64;
std::atomic<int> g_active[MAX_DEVICES][4];

cudaLaunchConfig_t config(uint32_t blocks, uint32_t cluster, cudaLaunchAttribute* attr, cudaStream_t stream)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(blocks); c.blockDim = dim3(THREADS); c.dynamicSmemBytes = SHARED_BYTES; c.stream = stream;
    attr->id = cudaLaunchAttributeClusterDimension;
    attr->val.clusterDim.x = cluster; attr->val.clusterDim.y = attr->val.clusterDim.z = 1;
    c.attrs = attr; c.numAttrs = cluster > 1 ? 1 : 0;
    return c;
}

}  // namespace

cudaError_t attend_prepare()
{
    int device = -1;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    for (uint32_t f = AVSG_ROW_BF16; f <= AVSG_ROW_FP4; ++f)
        for (int s = 0; s < 2; ++s)
            if ((e = cudaFuncSetAttribute(attend_kernel(f, s), cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED_BYTES)) != cudaSuccess) return e;
    if (device < 0 || device >= MAX_DEVICES) return cudaSuccess;                        // (then a block per query)
    for (int i = 1; i < 4; ++i) {
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t c = config(1u << i, 1u << i, &attr, nullptr);
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, attend_kernel(AVSG_ROW_FP8, false), &c) != cudaSuccess) { cudaGetLastError(); n = 0; }
        g_active[device][i] = n;
    }
    return cudaSuccess;
}

cudaError_t launch_attend(AttendParams& p, uint32_t format, cudaStream_t stream)
{
    p.groups = (p.heads + GROUP - 1) / GROUP;
    p.group_heads = (p.heads + p.groups - 1) / p.groups;
    const uint64_t work = (uint64_t)p.n * p.n_tokens * p.groups;
    // As many blocks per query as find room at once, each with a tile or more.
    int device = -1;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    p.cluster = 1;
    if (device >= 0 && device < MAX_DEVICES)
        for (uint32_t i = 3; i > 0; --i)
            if (work <= (uint64_t)g_active[device][i] && p.topk > TILE * ((1u << i) - 1u)) { p.cluster = 1u << i; break; }
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t c = config((uint32_t)(work * p.cluster), p.cluster, &attr, stream);
    void* args[] = {&p};
    return cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(attend_kernel(format, p.softcap > 0.f || p.slopes)), args);
}

}  // namespace avsg
