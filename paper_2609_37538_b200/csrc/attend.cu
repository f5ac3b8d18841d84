// avsg_attend on the matrix unit: a block (or a cluster of them) per query and group of up to 64 heads.
//
// For 64 selected rows at a time ("tile"), S = Q K^T (64 heads x 64 rows, 576 steps), softmax weights P with a running maximum, and
// O^T += V^T P^T (512 numbers x heads, 64 steps).  A row is gathered and laid out in shared memory ONCE and serves both products: as
// K with lines along the sum, as V^T with lines along its rows, which the unit reads from the same bytes.  O is kept transposed, so that its
// 512 numbers fill all 128 lanes four times over, and heads, of which there may be few, are the free dimension.
//
// Rows in 8 bits (e4m3; 4-bit ones become e4m3 on their way, in units of a power of two for each 128 numbers) are multiplied as they are,
// unscaled: nothing is rounded.  Their scales, one for 128 numbers, go onto the scores, which therefore come in four sums, and onto
// the weights, of which there are four for that reason.  The other operands are split into two e4m3 numbers each: a query's bf16 has 8
// significant bits, which two of 4 hold exactly (in units of a power of two of the head's, down to 2^-17 of its largest number); a weight keeps 8 bits, as in bf16,
// and no less than 2^-16 of the largest.  (fp16 operands, rows times their scales, rounded each score by 2^-12: 4e-4 on its logarithm's sum.)
// The two halves of a query are the 32 lanes that a warp reads, so that S has all 128 lanes and its products the unit's full rate.
// bf16 rows are multiplied as they are, with bf16 weights.  The rotated 64 numbers are bf16 on both sides.
//
// Warps: 0-7 softmax (two for each 16 heads, 32 rows each), 8-11 rows (asynchronous copies, two or three tiles in shared memory; 4 bits: through
// registers), 12 issues the products, whichever of the next tile's S and the last one's O can be next.
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
constexpr uint32_t SOFTMAX_WARPS = 8, ROW_WARPS = 4, WARPS = SOFTMAX_WARPS + ROW_WARPS + 1, THREADS = 32 * WARPS;
constexpr uint32_t PIECE = 64 * 128;                        // 64 lines
constexpr uint32_t MAX_CLUSTER = 8;
constexpr uint32_t SLOTS = 4;                               // sums S under way in TMEM

// How a format's rows, queries and weights lie in shared memory (bytes).
template <uint32_t FORMAT>
struct Layout {
    static constexpr bool BYTES = FORMAT != AVSG_ROW_BF16;
    static constexpr uint32_t BODY = BYTES ? 4 : 8;                             // pieces of the latent: 128 or 64 numbers a line
    static constexpr uint32_t BUFFERS = BYTES ? 3 : 2;                          // tiles
    static constexpr uint32_t SUMS = BYTES ? 5 : 1;                             // sums S of a tile
    static constexpr uint32_t TILE_BYTES = (BODY + 1) * PIECE;
    static constexpr uint32_t QUERY_PIECE = BYTES ? 2 * PIECE : PIECE;          // (two halves of each number)
    static constexpr uint32_t AT_Q = 0, AT_Q_ROPE = BODY * QUERY_PIECE, AT_TILES = AT_Q_ROPE + PIECE;
    // Weights: one set, or four of which the last takes the place of the tile's rotated numbers, read by then.
    static constexpr uint32_t AT_P = AT_TILES + BUFFERS * TILE_BYTES, AT_SMALL = AT_P + (BYTES ? 3 : 1) * PIECE;
    static constexpr uint32_t AT_SCALES = AT_SMALL, AT_PLACES = AT_SCALES + (BYTES ? BUFFERS * TILE * 16 : 0);
    static constexpr uint32_t AT_ALPHA = AT_PLACES + BUFFERS * TILE * 8, AT_UNIT = AT_ALPHA + GROUP * 4, AT_PEAK = AT_UNIT + (BYTES ? GROUP * 4 : 0);
    static constexpr uint32_t AT_BARS = AT_PEAK + 2 * GROUP * 4, AT_MISC = AT_BARS + 16 * 8, TOTAL = AT_MISC + 112;
    // once all products are through: O in 32 bits [heads][512], the blocks' shares in it, and the running maxima and sums
    static constexpr uint32_t AT_OUT = AT_TILES, AT_SHARE = AT_OUT + GROUP * LATENT * 4;
    static constexpr uint32_t AT_MOST = AT_PLACES, AT_SUM = AT_MOST + GROUP * 4;
    static_assert(AT_SHARE + MAX_CLUSTER * GROUP * 4 <= AT_SMALL && AT_SUM + 2 * GROUP * 4 <= AT_ALPHA && TOTAL <= 232448, "");
};
constexpr uint32_t SHARED_MOST = Layout<AVSG_ROW_BF16>::TOTAL > Layout<AVSG_ROW_FP8>::TOTAL ? Layout<AVSG_ROW_BF16>::TOTAL : Layout<AVSG_ROW_FP8>::TOTAL;

// Barriers, by their place: tile laid out, tile read (3 each); sum there, sum read (4 each); weights there; queries there.
constexpr uint32_t FULL = 0, FREE = 24, SUM_FULL = 48, SUM_FREE = 80, WEIGHTS = 112, QUERIES = 120;

// TMEM columns: O^T in four parts of 128 numbers, then the sums S.
constexpr uint32_t COL_OUT = 0, COL_S = 256, COLUMNS = 512;

constexpr float LOG2E = 1.4426950408889634f;
// The maximum that weights refer to lags behind by up to this (log2), so that O is rescaled seldom.  Weights in two e4m3 numbers are
// multiplied by ROOM: the largest is 32 to 256, of at most 448, and all are whole to 2^-10.
template <uint32_t FORMAT> constexpr float LAZY = Layout<FORMAT>::BYTES ? 3.f : 11.f;
constexpr float ROOM = 32.f;
constexpr float LEAST_UNIT = 7.888609052210118e-31f;        // 2^-100: what weights refer to while rows are zeros
constexpr long long WAIT_CLOCKS = 1ll << 29;                // about 0.3 s: longer than any wait that ends

struct Misc {
    uint32_t tmem, failed;
    int32_t last[WARPS];
    float scale_peak[2];                // largest scale of a tile's halves
    float unit;                         // what O's weights are multiples of
};
static_assert(sizeof(Misc) <= 112, "");

// A warp waits, bounded: false (and the block's other waits end too) if nothing came.
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile Misc* misc)
{
    if (__all_sync(0xffffffffu, barrier_done(bar, parity))) return true;
    const long long start = clock64();
    while (!__all_sync(0xffffffffu, barrier_done(bar, parity)))
        if (__any_sync(0xffffffffu, misc->failed || clock64() - start > WAIT_CLOCKS)) { misc->failed = 1; return false; }
    return true;
}

// A warp's lanes have done their part.
__device__ __forceinline__ void arrive(uint32_t bar, uint32_t lane)
{
    __syncwarp();
    if (lane == 0) barrier_arrive(bar);
}

__device__ __forceinline__ uint4 zeros() { return make_uint4(0u, 0u, 0u, 0u); }

__device__ __forceinline__ uint32_t place_of(uint32_t piece, uint32_t line, uint32_t unit) { return piece + line * 128u + ((unit ^ (line & 7u)) << 4); }

__device__ __forceinline__ void put16(uint32_t at, uint4 v)
{
    asm volatile("st.shared::cta.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void put4(uint32_t at, uint32_t v) { asm volatile("st.shared::cta.b32 [%0], %1;" :: "r"(at), "r"(v) : "memory"); }

// Two numbers as e4m3, and what that leaves of them as e4m3 again: high in the lower 16 bits.
__device__ __forceinline__ uint32_t split(__half2 x)
{
    const uint32_t high = __nv_cvt_halfraw2_to_fp8x2(__half2_raw(x), __NV_SATFINITE, __NV_E4M3);
    const __half2 left = __hsub2(x, __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)high, __NV_E4M3)));
    return high | (uint32_t)__nv_cvt_halfraw2_to_fp8x2(__half2_raw(left), __NV_SATFINITE, __NV_E4M3) << 16;
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A 4-bit row's units 4 i + sub (32 numbers with a scale of their own each), rotated numbers and scales, as a lane has them.
struct NibbleRow { uint4 body[4], rope[2], scales; };

__device__ __forceinline__ void get_nibbles(NibbleRow& v, const uint8_t* row, uint32_t sub)
{
    const uint4* at = reinterpret_cast<const uint4*>(row);
#pragma unroll
    for (int i = 0; i < 4; ++i) v.body[i] = row ? __ldg(at + 4 * i + sub) : zeros();
    v.scales = row ? __ldg(at + 16) : zeros();
#pragma unroll
    for (int i = 0; i < 2; ++i) v.rope[i] = row ? __ldg(at + 17 + 4 * i + sub) : zeros();
}

// Lays them out as e4m3: numbers 128 i .. of the row in units of 2^-6 of the largest of their four scales (up to 6 x 64 = 384; exact where
// a scale is no smaller than 2^-11 of that, else whole to 2^-10 units).  Eight lanes of a store have the eight lines of a piece: no two share a bank.
__device__ __forceinline__ float4 put_nibbles(const NibbleRow& v, uint32_t tile, uint32_t line, uint32_t sub)
{
    const uint32_t s[4] = {v.scales.x, v.scales.y, v.scales.z, v.scales.w};
    float unit[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t most = max(max(s[i] & 255u, s[i] >> 8 & 255u), max(s[i] >> 16 & 255u, s[i] >> 24));
        const uint32_t field = max((int)most - 6, 1);
        unit[i] = __uint_as_float(most == 255u ? 0x7FC00000u : field << 23);
        const int e = (int)(s[i] >> (8 * sub) & 255u) - (int)field + 15;            // of the ratio, as fp16
        const uint32_t one = e > 0 ? (uint32_t)e << 10 : e > -10 ? 1u << (e + 9) : 0u, ratio = one | one << 16;
        const uint32_t w[4] = {v.body[i].x, v.body[i].y, v.body[i].z, v.body[i].w};
        uint32_t to[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t four = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const __half2 x = __hmul2(e2m1_pair(w[j / 2] >> (16 * (j % 2) + 8 * k) & 255u), *reinterpret_cast<const __half2*>(&ratio));
                four |= (uint32_t)__nv_cvt_halfraw2_to_fp8x2(__half2_raw(x), __NV_SATFINITE, __NV_E4M3) << (16 * k);
            }
            to[j] = four;
        }
        put16(place_of(tile + i * PIECE, line, 2 * sub), make_uint4(to[0], to[1], to[2], to[3]));
        put16(place_of(tile + i * PIECE, line, 2 * sub + 1), make_uint4(to[4], to[5], to[6], to[7]));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) put16(place_of(tile + 4 * PIECE, line, 4 * i + sub), v.rope[i]);
    return make_float4(unit[0], unit[1], unit[2], unit[3]);
}

}  // namespace

template <uint32_t FORMAT, bool SHAPED>
__global__ void __launch_bounds__(THREADS, 1) avsg_attend_kernel(const __grid_constant__ AttendParams p)
{
    using L = Layout<FORMAT>;
    extern __shared__ __align__(1024) uint8_t shared[];
    const uint32_t base = shared_address(shared), bars = base + L::AT_BARS;
    Misc* misc = reinterpret_cast<Misc*>(shared + L::AT_MISC);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t rank = blockIdx.x % p.cluster, work = blockIdx.x / p.cluster;
    const uint32_t group = work % p.groups, item = work / p.groups;
    const uint32_t table = item / p.n_tokens, token = item - table * p.n_tokens;
    const uint32_t first_head = group * p.group_heads, heads = min(p.group_heads, p.heads - first_head);
    const uint32_t columns = (heads + 15u) & ~15u;
    // Head h is line 16 (h / in_quarter) + h % in_quarter of S: a quarter of TMEM's lanes, and two softmax warps, have in_quarter heads.
    const uint32_t in_quarter = (heads + 3u) / 4u, quarters = (heads + in_quarter - 1u) / in_quarter;
    const int32_t* slots = p.slots + (uint64_t)item * p.topk;
    const int32_t* ids = p.ids ? p.ids + (uint64_t)item * p.topk : nullptr;

    // Queries are asked for first: warp w has heads w, w + 13, ...
    constexpr uint32_t MINE = (GROUP + WARPS - 1) / WARPS;
    const uint32_t first = p.rope.halves ? lane : 2u * lane, second = p.rope.halves ? lane + 32u : 2u * lane + 1u;
    uint4 q[MINE][2];
    __nv_bfloat16 qa[MINE], qb[MINE];
    {
        const uint8_t* from = p.q + table * p.q_stride[0] + token * p.q_stride[1] + (uint64_t)first_head * p.q_stride[2];
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i) {
            const uint32_t h = warp + i * WARPS;
            if (h < heads) {
                const uint8_t* at = from + h * p.q_stride[2];
                const uint4* units = reinterpret_cast<const uint4*>(at);
                q[i][0] = __ldg(units + (L::BYTES ? 2u * lane : lane));
                q[i][1] = __ldg(units + (L::BYTES ? 2u * lane + 1u : lane + 32u));
                qa[i] = reinterpret_cast<const __nv_bfloat16*>(at)[LATENT + first];
                qb[i] = reinterpret_cast<const __nv_bfloat16*>(at)[LATENT + second];
            }
        }
    }
    // The selection's last position: what is behind it (padding) costs nothing.
    int32_t last = -1;
    for (uint32_t k = threadIdx.x; k < p.topk; k += THREADS) if (slots[k] >= 0) last = (int32_t)k;
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) misc->last[warp] = last;
    if (threadIdx.x == 0) {
        misc->failed = 0;
        for (uint32_t i = 0; i < 3; ++i) { barrier_init(bars + FULL + 8 * i, ROW_WARPS); barrier_init(bars + FREE + 8 * i, 1); }
        for (uint32_t i = 0; i < SLOTS; ++i) { barrier_init(bars + SUM_FULL + 8 * i, 1); barrier_init(bars + SUM_FREE + 8 * i, 2 * quarters); }
        barrier_init(bars + WEIGHTS, SOFTMAX_WARPS);
        barrier_init(bars + QUERIES, WARPS);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == WARPS - 1) tmem_alloc(base + L::AT_MISC, COLUMNS);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&misc->tmem);
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) last = max(last, misc->last[w]);
    const uint32_t all_tiles = (uint32_t)(last + 1 + (int32_t)TILE - 1) / TILE;
    const uint32_t tiles = all_tiles > rank ? (all_tiles - rank + p.cluster - 1) / p.cluster : 0u;       // rank, rank + cluster, ...

    // ---- queries ----
    {
        float cosine = 1.f, sine = 0.f;
        if (p.rope.on) rotation(p.rope, lane, p.positions[item], cosine, sine);
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i) {
            const uint32_t h = warp + i * WARPS, quarter = h / in_quarter, line = h - quarter * in_quarter;
            if (h >= heads) break;
            float a = __bfloat162float(qa[i]), b = __bfloat162float(qb[i]);
            if (p.rope.on) {
                const float turned = a * cosine - b * sine;
                b = a * sine + b * cosine;
                a = turned;
            }
            auto put_bf16 = [&](uint32_t d, float v) {
                *reinterpret_cast<__nv_bfloat16*>(shared + place_of(L::AT_Q_ROPE, 16u * quarter + line, d >> 3) + (d & 7u) * 2u) = __float2bfloat16_rn(v);
            };
            put_bf16(first, a);
            put_bf16(second, b);
            if constexpr (L::BYTES) {
                const uint32_t w[8] = {q[i][0].x, q[i][0].y, q[i][0].z, q[i][0].w, q[i][1].x, q[i][1].y, q[i][1].z, q[i][1].w};
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) most = max(most, max(w[j] << 16 & 0x7FFF0000u, w[j] & 0x7FFF0000u));
                most = __reduce_max_sync(0xffffffffu, most);
                const uint32_t e = max(most >> 23, 8u);                        // the largest becomes 2^7 or more, below 2^8
                const float inverse = __uint_as_float((261u - e) << 23);
                if (lane == 0) reinterpret_cast<float*>(shared + L::AT_UNIT)[h] = __uint_as_float(most >= 0x7F800000u ? 0x7FC00000u : (e - 7u) << 23);
                uint32_t high[4], low[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t x = split(__floats2half2_rn(__uint_as_float(w[2 * j] << 16) * inverse, __uint_as_float(w[2 * j] & 0xFFFF0000u) * inverse));
                    const uint32_t y = split(__floats2half2_rn(__uint_as_float(w[2 * j + 1] << 16) * inverse, __uint_as_float(w[2 * j + 1] & 0xFFFF0000u) * inverse));
                    high[j] = __byte_perm(x, y, 0x5410);
                    low[j] = __byte_perm(x, y, 0x7632);
                }
                const uint32_t piece = base + L::AT_Q + (lane / 8u) * L::QUERY_PIECE;
                put16(place_of(piece, 32u * quarter + line, lane % 8u), make_uint4(high[0], high[1], high[2], high[3]));
                put16(place_of(piece, 32u * quarter + 16u + line, lane % 8u), make_uint4(low[0], low[1], low[2], low[3]));
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 2; ++j) put16(place_of(base + L::AT_Q + (lane / 8u + 4u * j) * PIECE, 16u * quarter + line, lane % 8u), q[i][j]);
            }
        }
        fence_for_matrix_unit();
        arrive(bars + QUERIES, lane);
    }

    if (warp < SOFTMAX_WARPS) {
        // ---- softmax: a thread has 8 rows' scores of two heads, lines r and r + 8 of its quarter ----
        const uint32_t quarter = warp & 3u, half = warp >> 2, quad = lane & 3u;
        const bool busy = quarter < quarters;
        uint32_t head[2];
        bool real[2];
        float factor[2] = {0.f, 0.f}, slope[2] = {0.f, 0.f};
        const float to_log2 = p.scale * LOG2E;
        wait(bars + QUERIES, 0, misc);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t line = lane / 4u + 8u * k;
            head[k] = quarter * in_quarter + line;
            real[k] = line < in_quarter && head[k] < heads;
            if (real[k]) {
                factor[k] = L::BYTES ? reinterpret_cast<const float*>(shared + L::AT_UNIT)[head[k]] * to_log2 : to_log2;
                if (SHAPED && p.slopes) slope[k] = p.slopes[first_head + head[k]] * LOG2E;
            }
        }
        const bool two = in_quarter > 8u;                   // (else nobody has a second head)
        const int32_t position = SHAPED && p.slopes ? p.positions[item] : 0;
        float most[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f}, unit = LEAST_UNIT;
        const uint32_t lanes = tmem + (quarter * 32u << 16);
        for (uint32_t j = 0; j < tiles; ++j) {              // (also after a wait that failed: the warps meet at a barrier)
            const uint32_t b = j % L::BUFFERS;
            const float2* places = reinterpret_cast<const float2*>(shared + L::AT_PLACES) + b * TILE + 32u * half + 2u * quad;
            const float4* scales_at = reinterpret_cast<const float4*>(shared + L::AT_SCALES) + b * TILE + 32u * half + 2u * quad;
            float x[2][8], peak[2] = {-INFINITY, -INFINITY}, scale_peak = 0.f;
            float scale[L::BYTES ? 4 : 1][8];
            bool behind = false;
            if (busy) {
#pragma unroll
                for (uint32_t g = 0; g < L::SUMS; ++g) {
                    const uint32_t sum = j * L::SUMS + g, at = lanes + COL_S + 64 * (sum % SLOTS) + 32 * half;
                    wait(bars + SUM_FULL + 8 * (sum % SLOTS), sum / SLOTS & 1u, misc);
                    tmem_after_sync();
                    float s[16];
                    tmem_load_16x32(at, s);
                    if constexpr (L::BYTES) {
                        if (g == 0)
#pragma unroll
                            for (int c = 0; c < 8; ++c) {
                                const float4 v = scales_at[8 * (c / 2) + c % 2];
                                scale[0][c] = v.x; scale[1][c] = v.y; scale[2][c] = v.z; scale[3][c] = v.w;
                                scale_peak = fmaxf(scale_peak, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
                            }
                        if (g < 4) {
                            float low[16];
                            tmem_load_16x32(at + (16u << 16), low);
                            tmem_loaded();
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] += low[i];
                        } else {
                            tmem_loaded();
                        }
                    } else {
                        tmem_loaded();
                    }
                    tmem_before_sync();
                    arrive(bars + SUM_FREE + 8 * (sum % SLOTS), lane);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if (k == 1 && !two) continue;
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float v = s[4 * (c / 2) + 2 * k + c % 2];
                            if constexpr (!L::BYTES) x[k][c] = v * to_log2;
                            else if (g == 0) x[k][c] = v * scale[0][c];
                            else if (g < 4) x[k][c] += v * scale[g < 4 ? g : 0][c];
                            else x[k][c] = x[k][c] * factor[k] + v * to_log2;
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float2 place = places[8 * (c / 2) + c % 2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        if (k == 1 && !two) continue;
                        if constexpr (SHAPED) {
                            // cap x tanh(x / cap), by exp2 alone: off by 2^-22 of the cap at most, however small x is
                            if (p.softcap > 0.f) x[k][c] = p.softcap * LOG2E * (1.f - 2.f / (1.f + exp2f(x[k][c] * (2.f / p.softcap))));
                            if (p.slopes) x[k][c] += slope[k] * (float)(__float_as_int(place.y) - position);
                        }
                        if (place.x == 0.f) x[k][c] = -INFINITY;
                        peak[k] = fmaxf(peak[k], x[k][c]);
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == 1 && !two) continue;
                    peak[k] = fmaxf(peak[k], __shfl_xor_sync(0xffffffffu, peak[k], 1));
                    peak[k] = fmaxf(peak[k], __shfl_xor_sync(0xffffffffu, peak[k], 2));
                    if (real[k]) behind |= peak[k] > most[k] + LAZY<FORMAT> || (most[k] == -INFINITY && peak[k] > -INFINITY);
                }
                if constexpr (L::BYTES) behind |= scale_peak > unit;
            }
            // Weights would grow beyond their range: the references move, and O is brought to the new ones before it is added to.
            int any;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, 1, 256, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
                         : "=r"(any) : "r"((int)behind) : "memory");
            if (any) {
                float* peaks = reinterpret_cast<float*>(shared + L::AT_PEAK);
                if (busy && quad == 0) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) if (real[k]) peaks[half * GROUP + head[k]] = peak[k];
                }
                if (L::BYTES && quarter == 0) {
                    scale_peak = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(scale_peak)));        // (not negative)
                    if (lane == 0) misc->scale_peak[half] = scale_peak;
                }
                asm volatile("barrier.cta.sync 1, 256;" ::: "memory");
                float less = 1.f;
                if constexpr (L::BYTES) {
                    const float now = fmaxf(fmaxf(misc->scale_peak[0], misc->scale_peak[1]), LEAST_UNIT);
                    if (now > unit) {
                        const float to = __uint_as_float((__float_as_uint(now) + 0x007FFFFFu) & 0xFF800000u);         // a power of two
                        less = unit / to;
                        unit = to;
                    }
                }
                if (busy) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (real[k]) {
                            const float to = fmaxf(most[k], fmaxf(peaks[head[k]], peaks[GROUP + head[k]]));
                            const float keep = to == -INFINITY ? 1.f : exp2f(most[k] - to);
                            most[k] = to;
                            total[k] *= keep;
                            if (half == 0 && quad == 0) reinterpret_cast<float*>(shared + L::AT_ALPHA)[head[k]] = keep * less;
                        }
                }
                asm volatile("barrier.cta.sync 1, 256;" ::: "memory");
            }
            const uint32_t tile = base + L::AT_TILES + b * L::TILE_BYTES;
            auto last_read = [&] { if (j > 0) wait(bars + FREE + 8 * ((j - 1) % L::BUFFERS), (j - 1) / L::BUFFERS & 1u, misc); };
            if (busy) {
                float w[2][8];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == 1 && !two) continue;
                    const float from = most[k] == -INFINITY ? 0.f : most[k];
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        w[k][c] = exp2f(x[k][c] - from);
                        total[k] += w[k][c];
                    }
                }
                if constexpr (L::BYTES) {
                    const float inverse = 1.f / unit;
                    __half2 pair[2][4];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) if (k == 0 || two) pair[k][c] = __floats2half2_rn(w[k][2 * c] * ROOM, w[k][2 * c + 1] * ROOM);
                    last_read();
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const uint32_t piece = g < 3 ? base + L::AT_P + g * PIECE : tile + 4 * PIECE;
                        __half2 ratio[4];
#pragma unroll
                        for (int c = 0; c < 4; ++c) ratio[c] = __floats2half2_rn(scale[g][2 * c] * inverse, scale[g][2 * c + 1] * inverse);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if (k == 1 && !two) continue;
#pragma unroll
                            for (int c = 0; c < 4; c += 2) {
                                // Neighbouring lanes swap, so that each has four rows in a line: of columns 8 c or 8 (c + 1)
                                const uint32_t u = split(__hmul2(pair[k][c], ratio[c])), v = split(__hmul2(pair[k][c + 1], ratio[c + 1]));
                                const bool odd = lane & 1u;
                                const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? u : v, 1);
                                const uint32_t front = odd ? got : u, back = odd ? v : got;
                                const uint32_t key = 32u * half + 8u * (c + odd) + 4u * (quad / 2u);
                                if (real[k]) {
                                    put4(place_of(piece, head[k], key / 16u) + key % 16u, __byte_perm(front, back, 0x5410));
                                    put4(place_of(piece, head[k], 4u + key / 16u) + key % 16u, __byte_perm(front, back, 0x7632));
                                }
                            }
                        }
                    }
                } else {
                    uint32_t packed[2][4];
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) if (k == 0 || two) packed[k][c] = bf16_pair(w[k][2 * c], w[k][2 * c + 1]);
                    last_read();
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (real[k])
#pragma unroll
                            for (uint32_t c = 0; c < 4; ++c) put4(place_of(base + L::AT_P, head[k], 4u * half + c) + quad * 4u, packed[k][c]);
                    __syncwarp();
                }
            } else if (any) {
                last_read();
            }
            if (any && j > 0) {
                tmem_after_sync();
                const float* alpha = reinterpret_cast<const float*>(shared + L::AT_ALPHA);
                for (uint32_t part = 2 * half; part < 2 * half + 2; ++part)
                    for (uint32_t c = 0; c < columns; c += 16) {
                        float o[16];
                        tmem_load_32x16(lanes + COL_OUT + 64 * part + c, o);
                        tmem_loaded();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] *= alpha[c + i];
                        tmem_store_32x16(lanes + COL_OUT + 64 * part + c, o);
                    }
                tmem_stored();
            }
            fence_for_matrix_unit();
            tmem_before_sync();
            arrive(bars + WEIGHTS, lane);
        }
        // (the places' bytes are free: every warp that reads them is through with the last tile)
        asm volatile("barrier.cta.sync 1, 256;" ::: "memory");
        if (busy) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                total[k] += __shfl_xor_sync(0xffffffffu, total[k], 1);
                total[k] += __shfl_xor_sync(0xffffffffu, total[k], 2);
                if (real[k] && quad == 0) {
                    if (half == 0) reinterpret_cast<float*>(shared + L::AT_MOST)[head[k]] = most[k];
                    reinterpret_cast<float*>(shared + L::AT_SUM)[half * GROUP + head[k]] = total[k];
                }
            }
        }
        if (threadIdx.x == 0) misc->unit = L::BYTES ? unit / ROOM : 1.f;
    } else if (warp < SOFTMAX_WARPS + ROW_WARPS) {
        // ---- rows: a warp has 16 of a tile's, a lane every fourth 16-byte unit of two of them ----
        const uint32_t line = (warp - SOFTMAX_WARPS) * 16u + lane % 8u, sub = lane / 8u;
        const uint8_t* rows = p.buffer + (uint64_t)(p.mapped ? p.table_id[table] : table) * p.table_stride;
        int32_t begin = INT32_MIN, end = INT32_MAX;
        if (p.spans) { begin = p.spans[2 * item]; end = p.spans[2 * item + 1]; }
        // The slots (and ids) of a tile's lines, asked for two tiles ahead; where their rows are, once they are there.
        struct Places { int32_t slot[2], id[2]; };
        auto places_of = [&](uint32_t j) -> Places {
            Places to = {{-1, -1}, {0, 0}};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint64_t k = (uint64_t)(rank + j * p.cluster) * TILE + line + 8u * i;
                if (j < tiles && k < p.topk) {
                    to.slot[i] = __ldg(slots + k);
                    if (ids) to.id[i] = __ldg(ids + k);
                }
            }
            return to;
        };
        auto row_of = [&](int32_t slot, int32_t id) -> const uint8_t* {
            if (slot < 0 || (p.spans && (id < begin || id >= end))) return nullptr;
            if ((uint32_t)slot >= p.rows) { if (p.status) atomicOr(p.status, ST_BAD_SLOT); return nullptr; }
            return rows + (uint64_t)slot * p.row_stride;
        };
        auto put_place = [&](uint32_t b, int i, const uint8_t* row, int32_t id) {
            if (sub == 0) reinterpret_cast<float2*>(shared + L::AT_PLACES)[b * TILE + line + 8u * i] = make_float2(row ? 1.f : 0.f, __int_as_float(id));
        };
        if constexpr (FORMAT == AVSG_ROW_FP4) {
            NibbleRow part[2];
            const uint8_t* row[2];
            Places here = places_of(0), next = places_of(1);
#pragma unroll
            for (int i = 0; i < 2; ++i) { row[i] = row_of(here.slot[i], here.id[i]); get_nibbles(part[i], row[i], sub); }
            for (uint32_t j = 0; j < tiles; ++j) {
                const uint32_t b = j % L::BUFFERS;
                if (j >= L::BUFFERS && !wait(bars + FREE + 8 * b, (j / L::BUFFERS - 1) & 1u, misc)) break;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float4 unit = put_nibbles(part[i], base + L::AT_TILES + b * L::TILE_BYTES, line + 8u * i, sub);
                    if (sub == 0) reinterpret_cast<float4*>(shared + L::AT_SCALES)[b * TILE + line + 8u * i] = row[i] ? unit : make_float4(0.f, 0.f, 0.f, 0.f);
                    put_place(b, i, row[i], here.id[i]);
                }
                fence_for_matrix_unit();
                arrive(bars + FULL + 8 * b, lane);
                here = next;
                next = places_of(j + 2);
#pragma unroll
                for (int i = 0; i < 2; ++i) { row[i] = row_of(here.slot[i], here.id[i]); get_nibbles(part[i], row[i], sub); }
            }
        } else {
            constexpr uint32_t UNITS = FORMAT == AVSG_ROW_BF16 ? 16 : 8;         // a lane's units of a latent
            uint32_t there = 0;                                                  // tiles announced
            auto announce = [&](uint32_t tile) {
                fence_for_matrix_unit();
                arrive(bars + FULL + 8 * (tile % L::BUFFERS), lane);
            };
            Places here = places_of(0), next = places_of(1);
            for (uint32_t j = 0; j < tiles; ++j) {
                const uint32_t b = j % L::BUFFERS, tile = base + L::AT_TILES + b * L::TILE_BYTES;
                if (j >= L::BUFFERS) {
                    const uint32_t bar = bars + FREE + 8 * b, parity = (j / L::BUFFERS - 1) & 1u;
                    if (there < j && !__all_sync(0xffffffffu, barrier_is_done(bar, parity))) {
                        copies_wait<0>();                                        // time to spare: all that is under way is announced first
                        while (there < j) announce(there++);
                    }
                    if (!wait(bar, parity, misc)) break;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint8_t* row = row_of(here.slot[i], here.id[i]);
                    const uint8_t* from = row ? row : p.buffer;                  // (a masked row's bytes are zeros, nothing is read)
                    const uint32_t at = line + 8u * i;
#pragma unroll
                    for (uint32_t u = 0; u < UNITS; ++u) {
                        const uint32_t unit = 4 * u + sub;
                        copy16(place_of(tile + unit / 8u * PIECE, at, unit % 8u), from + 16 * unit, !row);
                    }
#pragma unroll
                    for (uint32_t u = 0; u < 2; ++u)
                        copy16(place_of(tile + L::BODY * PIECE, at, 4 * u + sub), from + row_bytes_of(FORMAT) - 2 * ROPE + 16 * (4 * u + sub), !row);
                    if (FORMAT == AVSG_ROW_FP8 && sub == 0) copy16(base + L::AT_SCALES + 16 * (b * TILE + at), from + LATENT, !row);
                    put_place(b, i, row, here.id[i]);
                }
                copies_close();
                here = next;
                next = places_of(j + 2);
                if (there < j) {                                                 // the tile before this one is announced when it is there
                    copies_wait<1>();
                    while (there < j) announce(there++);
                }
            }
            copies_wait<0>();
            if (!misc->failed) while (there < tiles) announce(there++);
        }
    } else {
        // ---- products ----
        constexpr Product TYPE = L::BYTES ? Product::E4M3 : Product::BF16;
        constexpr uint32_t S_SHAPE = product_shape(TYPE, L::BYTES ? 128 : 64, TILE, false), ROPE_SHAPE = product_shape(Product::BF16, 64, TILE, false);
        const uint32_t out_shape = product_shape(TYPE, 128, columns, true);
        const uint32_t query = operand(base + L::AT_Q, 16), query_rope = operand(base + L::AT_Q_ROPE, 16);
        auto score = [&](uint32_t sum, uint32_t j, uint32_t g) {
            const uint32_t to = tmem + COL_S + 64 * (sum % SLOTS), tile = operand(base + L::AT_TILES + j % L::BUFFERS * L::TILE_BYTES, 16);
            if constexpr (L::BYTES) {
                if (g < 4) {
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) multiply<TYPE>(to, query + (g * L::QUERY_PIECE + 32 * i) / 16, tile + (g * PIECE + 32 * i) / 16, S_SHAPE, i > 0);
                    products_done(bars + SUM_FULL + 8 * (sum % SLOTS));
                    return;
                }
            } else {
#pragma unroll
                for (uint32_t i = 0; i < 4 * L::BODY; ++i)
                    multiply<TYPE>(to, query + (i / 4 * PIECE + i % 4 * 32) / 16, tile + (i / 4 * PIECE + i % 4 * 32) / 16, S_SHAPE, i > 0);
            }
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) multiply<Product::BF16>(to, query_rope + 2 * i, tile + (L::BODY * PIECE + 32 * i) / 16, ROPE_SHAPE, !L::BYTES || i > 0);
            products_done(bars + SUM_FULL + 8 * (sum % SLOTS));
        };
        auto add = [&](uint32_t j) {
            const uint32_t tile = base + L::AT_TILES + j % L::BUFFERS * L::TILE_BYTES, rows = operand(tile, PIECE);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
                const uint32_t part = i / 4, k = i % 4, to = tmem + COL_OUT + 64 * part;
                if constexpr (L::BYTES)                    // both halves of the weights by the same rows
                    multiply<TYPE>(to, rows + (part * PIECE + k % 2 * 4096) / 16, operand(part < 3 ? base + L::AT_P + part * PIECE : tile + 4 * PIECE, 16) + 2 * k,
                                   out_shape, j + k > 0);
                else
                    multiply<TYPE>(to, rows + (part * 2 * PIECE + k * 2048) / 16, operand(base + L::AT_P, 16) + 2 * k, out_shape, j + k > 0);
            }
            products_done(bars + FREE + 8 * (j % L::BUFFERS));
        };
        if (tiles && wait(bars + QUERIES, 0, misc)) {
            uint32_t sum = 0, g = 0, scored = 0, added = 0;
            long long idle = clock64();
            while (added < tiles) {
                bool weights = added < scored || (added == scored && g > 0), next = scored < tiles;
                if (weights) weights = barrier_is_done(bars + WEIGHTS, added & 1u);
                if (next) next = (g > 0 || barrier_is_done(bars + FULL + 8 * (scored % L::BUFFERS), scored / L::BUFFERS & 1u)) &&
                                 (sum < SLOTS || barrier_is_done(bars + SUM_FREE + 8 * (sum % SLOTS), (sum / SLOTS - 1) & 1u));
                if (__all_sync(0xffffffffu, weights)) {
                    tmem_after_sync();
                    if (one_lane()) add(added);
                    __syncwarp();
                    ++added;
                } else if (__all_sync(0xffffffffu, next)) {
                    tmem_after_sync();
                    if (one_lane()) score(sum, scored, g);
                    __syncwarp();
                    ++sum;
                    if (++g == L::SUMS) { g = 0; ++scored; }
                } else {
                    if (__any_sync(0xffffffffu, reinterpret_cast<volatile Misc*>(misc)->failed || clock64() - idle > WAIT_CLOCKS)) { misc->failed = 1; break; }
                    continue;
                }
                idle = clock64();
            }
        }
    }

    // ---- the block's sums to shared memory, and the cluster's blocks' together ----
    __syncwarp();
    if (tiles) wait(bars + FREE + 8 * ((tiles - 1) % L::BUFFERS), (tiles - 1) / L::BUFFERS & 1u, misc);
    tmem_after_sync();
    if (warp < SOFTMAX_WARPS && tiles) {
        float* out = reinterpret_cast<float*>(shared + L::AT_OUT);
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
    if (warp == WARPS - 1) {
        if (misc->failed) __nanosleep(100000);                  // (products that nobody waits for any more)
        __syncwarp();
        tmem_after_sync();
        tmem_free(tmem, COLUMNS);
    }
    if (p.cluster > 1) cluster_sync();
    float* share = reinterpret_cast<float*>(shared + L::AT_SHARE);
    if (threadIdx.x < heads) {
        const uint32_t h = threadIdx.x, at_most = base + L::AT_MOST + 4 * h, at_sum = base + L::AT_SUM + 4 * h;
        float most = -INFINITY, total = 0.f;
        for (uint32_t c = 0; c < p.cluster; ++c) most = fmaxf(most, load_float(in_block(at_most, c)));
        const float from = most == -INFINITY ? 0.f : most;
        for (uint32_t c = 0; c < p.cluster; ++c) {
            const float sum = load_float(in_block(at_sum, c)) + load_float(in_block(at_sum + 4 * GROUP, c));
            const float weight = exp2f(load_float(in_block(at_most, c)) - from);
            total += sum * weight;
            share[c * GROUP + h] = sum == 0.f ? 0.f : weight * load_float(in_block(base + L::AT_MISC + offsetof(Misc, unit), c));
        }
        for (uint32_t c = 0; c < p.cluster; ++c) share[c * GROUP + h] = total == 0.f ? 0.f : share[c * GROUP + h] / total;
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
                const uint32_t at = in_block(base + L::AT_OUT + (h * LATENT + 8 * d) * 4u, c);
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
    c.gridDim = dim3(blocks); c.blockDim = dim3(THREADS); c.dynamicSmemBytes = SHARED_MOST; c.stream = stream;
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
            if ((e = cudaFuncSetAttribute(attend_kernel(f, s), cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED_MOST)) != cudaSuccess) return e;
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
