// avsg_attend on the matrix unit: a block (or a cluster of them) per query and group of up to 64 heads.
//
// For 64 selected rows at a time ("tile"), S = Q K^T (64 heads x 64 rows, 576 steps), softmax weights P with a running maximum, and
// O^T += V^T P^T (512 numbers x heads, 64 steps).  A row is gathered, made 16-bit numbers and laid out in shared memory ONCE, and serves
// both products: as K with lines along the sum, as V^T with lines along its rows, which the unit reads from the same bytes.  O is kept
// transposed, so that its 512 numbers fill all 128 lanes four times over, and heads, of which there may be few, are the free dimension.
//
// bf16 rows are multiplied as they are, with bf16 weights.  4-bit codes times their scales are exact as fp16, in units of a power of two of the
// row's, which goes onto score and weight.  e4m3 rows have a scale for every 128 numbers.  A score is computed from the codes as they are
// (e4m3 x e4m3, a query being two e4m3 numbers: its bf16 has 8 significant bits, two of 4 hold them, down to 2^-17 of the head's largest
// number), in four sums, onto which the scales go in 32 bits; values are the codes times their scales as fp16, made from the tile's codes beside
// the first product, with one weight to a row.  (From fp16 rows scores are 4e-4 off; unscaled fp16 rows are exact for both products, but take four
// sets of weights, one after another through the room that is left: 143 us where this took 125 at the time.)  Other queries become fp16 in units of
// a power of two of the head's (exact: bf16 has 8 bits, fp16 11), weights fp16 in units of the largest row's.  The rotated 64 numbers are bf16 on
// both sides and have a sum of their own.  Sums, maxima and totals are 32 bits throughout; what is rounded is said here.
//
// Warps: first those of softmax, by quarters of the heads and shares of a tile's rows; then those of the rows, eight rows each, which gather (and
// convert) them; the last one issues the products, whichever of the next tile's S and the last one's O can be next.  Softmax of e4m3 rows, which
// adds five sums up, has 16 warps (8: 98 us where 16 take 95, and 62 for 55 with capped scores); the others' 8 (16 for bf16: 18.3 us for 17.1; every warp
// more takes registers from all).
//
// A query's rows are split over a cluster's blocks where queries are few, tile by tile in turn; the blocks' sums are joined through
// distributed shared memory in a fixed order (same results on every run, no workspace).
//
// What bounds it: per tile and block the chain rows - scores - softmax - weights - sums, of which two tiles are under way (shared memory has room
// for two), about 4700 clocks; the matrix unit alone needs 1700 to 2000, shared memory's bandwidth (both products read their operands from
// there: a 64 x 64 product of 16 numbers takes 34 clocks, all of its bandwidth) 2200 to 3000.  Around it 9000 clocks until the first scores (queries,
// rows from DRAM) and 4000 to 6000 behind the last.  Device times: 32 requests, two tokens, 128 heads, 2048 of 8192 e4m3 rows 94 us (387
// TFLOP/s); 16 heads, 4-bit rows 46; one request, two tokens, 128 heads, bf16 rows 17; one token, 16 heads, 256 rows 11.
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
constexpr uint32_t PIECE = 64 * 128;                        // 64 lines of 64 numbers
constexpr uint32_t BODY = LATENT / 64;                      // pieces of 64 16-bit numbers a line
constexpr uint32_t SLOTS = 2;                               // steps of S under way in TMEM, one or two sums each

// What differs between the formats, and how shared memory is laid out (bytes).
template <uint32_t FORMAT>
struct Layout {
    static constexpr bool HALF = FORMAT != AVSG_ROW_BF16;                       // fp16 weights and values
    static constexpr bool CODES = FORMAT == AVSG_ROW_FP8;                       // scores from e4m3 codes
    static constexpr uint32_t SOFTMAX_WARPS = CODES ? 16 : 8, SHARES = SOFTMAX_WARPS / 4, EACH = TILE / SHARES;        // rows of a tile to each
    static constexpr uint32_t ROW_WARPS = 8, WARPS = SOFTMAX_WARPS + ROW_WARPS + 1, THREADS = 32 * WARPS;
    static constexpr uint32_t STEPS = CODES ? 3 : 1;                            // of a tile's S: two latent sums, two, the rotated one; or all at once
    static constexpr uint32_t PARTS = CODES ? 3 : 2;                            // in which its products are issued
    static constexpr uint32_t ROPE_PIECE = CODES ? BODY / 2 : BODY;             // of a tile: the rotated numbers (behind 128 or 64 numbers a line)
    static constexpr uint32_t TILE_BYTES = (ROPE_PIECE + 1) * PIECE;
    // (queries: 8 pieces, of high and low halves in turn for codes, and the rotated one's.)  Weights have a place of their own beside codes,
    // which are overwritten as soon as scores are there; else they take that of the tile's rotated numbers, read by then.
    static constexpr uint32_t AT_Q = 0, AT_TILES = (BODY + 1) * PIECE, AT_VALUES = AT_TILES + 2 * TILE_BYTES, AT_WEIGHTS = AT_VALUES + (CODES ? BODY * PIECE : 0);
    static constexpr uint32_t AT_SCALES = AT_WEIGHTS + (CODES ? PIECE : 0), AT_UNITS = AT_SCALES + (CODES ? 2 * 4 * TILE * 4 : 0);
    // (units of the tiles' rows are powers of two, by their exponents; 16 bits of who is seen)
    static constexpr uint32_t AT_SEEN = AT_UNITS + 2 * TILE, AT_TOPS = AT_SEEN + 16, TOPS = 8, AT_ALPHA = AT_TOPS + 2 * TOPS * 4;
    static constexpr uint32_t AT_PEAK = AT_ALPHA + GROUP * 4, AT_BARS = AT_PEAK + GROUP * 4, AT_MISC = AT_BARS + 16 * 8, TOTAL = AT_MISC + 128;
    static constexpr uint32_t AT_UNIT = AT_ALPHA;                               // the queries' units, until the softmax warps have read them
    // once all products are through: O in 32 bits [heads][512], each head's maximum, sum, unit and their quotient; the running maxima and the sums of each share of a tile's rows
    static constexpr uint32_t AT_OUT = AT_TILES, AT_STATE = AT_OUT + GROUP * LATENT * 4, AT_MOST = AT_STATE + GROUP * 16, AT_SUM = AT_MOST + GROUP * 4;
    static_assert(AT_SUM + SHARES * GROUP * 4 <= AT_SCALES && TOTAL <= 232448, "");
};
constexpr uint32_t SHARED_MOST = Layout<AVSG_ROW_FP8>::TOTAL, MAX_WARPS = 25;

// Barriers, by their place: half of a tile laid out (two of two tiles); tile read (2); step of S there, read (2 each); weights there (2); values
// there; queries there; codes read by the matrix unit (2).
constexpr uint32_t FULL = 0, FREE = 32, SUM_FULL = 48, SUM_FREE = 64, WEIGHTS = 80, VALUES = 96, QUERIES = 104, CODES_READ = 112;

// TMEM columns: O^T in four parts of 128 numbers, then the sums S.
constexpr uint32_t COL_OUT = 0, COL_S = 256, COLUMNS = 512;

constexpr float LOG2E = 1.4426950408889634f;
// The maximum that weights refer to lags behind by up to LAZY (log2), so that O is rescaled seldom.  fp16 weights are whole to 2^-25 then, the
// largest being 1 to 2^15.  (2^4 to 2^15: 6% slower with scores that spread over 2^+-12.)  bf16 has the range for more, but O has to hold weights
// times values: bf16 weights are in units of BF16_UNIT, the largest being 2^-15 to 2^15, so that 2048 values may be of 2^101.  (1 to 2^15: 3.5% slower
// with one request; 1 to 2^60: 0.5% faster, but values of 2^95 overflowed.)
template <uint32_t FORMAT> constexpr float LAZY = Layout<FORMAT>::HALF ? 15.f : 30.f;
constexpr float BF16_UNIT = 32768.f;
constexpr uint32_t LEAST_UNIT = 27u << 23;                  // 2^-100: no row's unit is smaller, so that ratios of units stay finite
constexpr long long WAIT_CLOCKS = 1ll << 29;                // about 0.3 s: longer than any wait that ends

struct Misc {
    uint32_t tmem, failed;
    int32_t last[MAX_WARPS];
    float unit;                         // what O's weights are multiples of
};
static_assert(sizeof(Misc) <= 128, "");

// Waits, bounded: false (and the block's other waits end too) if nothing came.  All lanes of a warp look together, in one instruction: 20
// clocks where the phase is over.  (One lane looking for the others: 400, coming together again.)
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile Misc* misc)
{
    if (barrier_wait(bar, parity)) return true;
    const long long start = clock64();
    while (true) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i) if (barrier_wait(bar, parity)) return true;
        if (misc->failed || clock64() - start > WAIT_CLOCKS) { misc->failed = 1; return false; }
    }
}

// A warp's lanes have done their part.
__device__ __forceinline__ void arrive(uint32_t bar, uint32_t lane)
{
    __syncwarp();
    if (lane == 0) barrier_arrive(bar);
}

// The bits of a float as an integer of the same order, and back.
__device__ __forceinline__ int in_order(int bits) { return bits ^ (bits >> 31 & 0x7FFFFFFF); }

__device__ __forceinline__ uint4 zeros() { return make_uint4(0u, 0u, 0u, 0u); }

__device__ __forceinline__ uint32_t place_of(uint32_t piece, uint32_t line, uint32_t unit) { return piece + line * 128u + ((unit ^ (line & 7u)) << 4); }

__device__ __forceinline__ void put16(uint32_t at, uint4 v)
{
    asm volatile("st.shared::cta.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void put4(uint32_t at, uint32_t v) { asm volatile("st.shared::cta.b32 [%0], %1;" :: "r"(at), "r"(v) : "memory"); }

__device__ __forceinline__ uint32_t bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }

__device__ __forceinline__ uint32_t bf16_pair(float a, float b)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// What a lane of a row warp has of eight rows in 4 bits: 16 bytes each of the codes' first and second half of row lane / 8 and of the one 4
// further on; of the rotated numbers likewise; all scales of row lane % 8 (lanes 0-7).  (Eight lanes read 128 bytes of a row side by side:
// eight rows' 16 bytes would be eight lookups of the cache for one, which bound the kernel.)
struct RowPart { uint4 body[2][2], rope[2], scales; };

// (masked: zeros, so that nothing of it reaches a sum)
__device__ __forceinline__ uint4 unit_at(const uint8_t* row, uint32_t unit) { return row ? __ldg(reinterpret_cast<const uint4*>(row) + unit) : zeros(); }

// The unit that a 4-bit row's numbers are in: 2^-13 of its largest scale, so that they reach 6 x 8192 = 49152.
__device__ __forceinline__ uint32_t nibble_unit(uint4 scales)
{
    uint32_t most = __vmaxu4(__vmaxu4(scales.x, scales.y), __vmaxu4(scales.z, scales.w));
    most = __vmaxu4(most, most >> 16);
    most = max(most & 255u, most >> 8 & 255u);
    return (uint32_t)max((int)most - 13, (int)(LEAST_UNIT >> 23));
}

// Lays the lane's 16 bytes of half c of row i (of those above) out as fp16 in line `line` of a tile: 32 numbers go to four units of a piece, in
// another order for each two lanes, so that the eight lanes of a store's phase, which have one line, share no bank.  unit and scales are of that row.
__device__ __forceinline__ void put_codes(uint4 body, int c, int unit, uint32_t scales, uint32_t tile, uint32_t line, uint32_t lane)
{
    const uint32_t turn = lane / 2u & 3u, piece = tile + (4u * c + turn) * PIECE;
    uint32_t w[4] = {body.x, body.y, body.z, body.w};
    if (turn & 1u) { const uint32_t x = w[0]; w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = x; }
    if (turn & 2u) { uint32_t x = w[0]; w[0] = w[2]; w[2] = x; x = w[1]; w[1] = w[3]; w[3] = x; }
    {
        const uint32_t e = scales >> (8u * (lane & 3u)) & 255u;
        const int power = (int)e - unit;                                        // scale / unit is 2^power, power <= 13
        if (power >= -13 && e != 255u) {
            // The upper bytes of 0, .5, 1, 1.5 and 2, 3, 4, 6 times 2^power as fp16 (the lower are zero), looked up by a code's last three bits, four
            // codes at a time; signs beside.  (By a conversion and a product for two codes: 46.4 us for 46.0.)
            const uint32_t small = 0x3E3C3800u + (uint32_t)(4 * power) * 0x01010100u, large = 0x46444240u + (uint32_t)(4 * power) * 0x01010101u;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t even = w[u] << 4;
                const uint32_t a = __byte_perm(small, large, w[u] & 0x7777u) | (__byte_perm(even, w[u], 0xD9C8) & 0x80808080u);
                const uint32_t b = __byte_perm(small, large, w[u] >> 16 & 0x7777u) | (__byte_perm(even, w[u], 0xFBEA) & 0x80808080u);
                put16(place_of(piece, line, 4u * (lane & 1u) + (turn + u & 3u)),
                      make_uint4(__byte_perm(a, 0, 0x1404), __byte_perm(a, 0, 0x3424), __byte_perm(b, 0, 0x1404), __byte_perm(b, 0, 0x3424)));
            }
        } else {                                                                // below fp16's full digits, or no number
            const uint32_t one = e == 255u ? 0x7E00u : power > -25 ? 1u << (power + 24) : 0u, ratio = one | one << 16;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = bits(__hmul2(e2m1_pair(w[u] >> (8 * j) & 255u), *reinterpret_cast<const __half2*>(&ratio)));
                put16(place_of(piece, line, 4u * (lane & 1u) + (turn + u & 3u)), make_uint4(x[0], x[1], x[2], x[3]));
            }
        }
    }
}

// The unit that an e4m3 row's values are in: the power of two at or above its largest scale, / 128, so that they reach 448 x 128 = 57344.
__device__ __forceinline__ uint32_t code_unit(const float (&s)[4])
{
    uint32_t most = LEAST_UNIT + (7u << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(s[i]) & 0x7FFFFFFFu);
    return most < 0x7F800000u ? ((most + 0x007FFFFFu) & 0xFF800000u) - (7u << 23) : most;
}

// Two numbers up to 448 as e4m3, and what that leaves of them as e4m3 again, in the lower 16 bits each.
__device__ __forceinline__ void split(__half2 x, uint32_t& high, uint32_t& low)
{
    high = __nv_cvt_halfraw2_to_fp8x2(__half2_raw(x), __NV_SATFINITE, __NV_E4M3);
    low = __nv_cvt_halfraw2_to_fp8x2(__half2_raw(__hsub2(x, __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)high, __NV_E4M3)))), __NV_SATFINITE, __NV_E4M3);
}

// cap x tanh(x / cap) for a score in log2.  tanh(y) / y is a polynomial in y^2 where |y| < 0.6 (off by 2^-23 of itself; coefficients of the
// least largest relative error, by reweighted least squares), so that a score far below its cap keeps its digits, and comes from exp2 beyond:
// either is within 2^-20 of the result.  per_cap: 1 / cap in these units, in two factors, since the cap may be any number from 2^-126 on.
__device__ __forceinline__ float capped(float x, float cap, const float (&per_cap)[2])
{
    const float y = x * per_cap[0] * per_cap[1], u = y * y;
    const float near = x * (1.f + u * (-0.333325982f + u * (0.133131161f + u * (-0.0522118062f + u * 0.0156126339f))));
    const float far = cap * (1.f - 2.f / (1.f + exp2f(y * (2.f * LOG2E)))) * LOG2E;
    return fabsf(y) < 0.6f ? near : far;
}

__device__ __forceinline__ float logarithm(float most, float total) { return total == 0.f ? -INFINITY : (most + log2f(total)) * 0.6931471805599453f; }

// The sums of a cluster's C blocks, joined: a warp takes a head, or half or a quarter of one, tasks going to the blocks in turn; lanes 0 .. C - 1
// have the head's numbers of a block each.  What is far away is asked for at once, eight float4 a lane: the time of a task is that of one look.
template <uint32_t C, uint32_t WARPS>
__device__ __forceinline__ void join(uint32_t at_state, uint32_t at_out, uint32_t heads, uint32_t rank, uint32_t warp, uint32_t lane, uint8_t* out, uint64_t stride, float* lse)
{
    constexpr uint32_t UNITS = 8 / C, TASKS = 4 / UNITS;                        // of 32 float4; of a head
    for (uint32_t t = warp * C + rank; t < heads * TASKS; t += WARPS * C) {
        const uint32_t h = t / TASKS, first = t % TASKS * UNITS * 32u + lane;
        const float4 its = lane < C ? load_float4(in_block(at_state + 16 * h, lane)) : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        float4 v[C][UNITS];
#pragma unroll
        for (uint32_t c = 0; c < C; ++c)
#pragma unroll
            for (uint32_t u = 0; u < UNITS; ++u) v[c][u] = load_float4(in_block(at_out + 16 * (h * (LATENT / 4) + first + 32 * u), c));
        float most = its.x;
#pragma unroll
        for (int m = 1; m < (int)C; m *= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, m));
        const float share = its.y == 0.f ? 0.f : exp2f(its.x - (most == -INFINITY ? 0.f : most));
        float total = its.y * share;
#pragma unroll
        for (int m = 1; m < (int)C; m *= 2) total += __shfl_xor_sync(0xffffffffu, total, m);
        const float mine = total == 0.f ? 0.f : share * its.z / total;
        if (lse && first == 0) lse[h] = logarithm(most, total);
        float w[C];
#pragma unroll
        for (uint32_t c = 0; c < C; ++c) w[c] = __shfl_sync(0xffffffffu, mine, (int)c);
#pragma unroll
        for (uint32_t u = 0; u < UNITS; ++u) {
            float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t c = 0; c < C; ++c)
                if (w[c] != 0.f) { x[0] += w[c] * v[c][u].x; x[1] += w[c] * v[c][u].y; x[2] += w[c] * v[c][u].z; x[3] += w[c] * v[c][u].w; }      // (without rows there are no sums)
            *reinterpret_cast<uint2*>(out + h * stride + 8 * (first + 32 * u)) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
        }
    }
}

}  // namespace

template <uint32_t FORMAT, bool SHAPED>
__global__ void __launch_bounds__(Layout<FORMAT>::THREADS, 1) avsg_attend_kernel(const __grid_constant__ AttendParams p)
{
    using L = Layout<FORMAT>;
    constexpr uint32_t SOFTMAX_WARPS = L::SOFTMAX_WARPS, ROW_WARPS = L::ROW_WARPS, WARPS = L::WARPS, THREADS = L::THREADS, SHARES = L::SHARES;
    static_assert(WARPS <= MAX_WARPS, "");
    extern __shared__ __align__(1024) uint8_t shared[];
    const uint32_t base = shared_address(shared), bars = base + L::AT_BARS;
    Misc* misc = reinterpret_cast<Misc*>(shared + L::AT_MISC);
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

    const uint32_t rank = blockIdx.x % p.cluster, work = blockIdx.x / p.cluster;
    const uint32_t group = work % p.groups, item = work / p.groups;
    const uint32_t table = item / p.n_tokens, token = item - table * p.n_tokens;
    const uint32_t first_head = group * p.group_heads, heads = min(p.group_heads, p.heads - first_head);
    const uint32_t columns = (heads + 15u) & ~15u;
    // Head h is line 16 (h / in_quarter) + h % in_quarter of S: a quarter of TMEM's lanes, and SHARES softmax warps, have in_quarter heads.
    const uint32_t in_quarter = (heads + 3u) / 4u, quarters = (heads + in_quarter - 1u) / in_quarter;
    const int32_t* slots = p.slots + (uint64_t)item * p.topk;
    const int32_t* ids = p.ids ? p.ids + (uint64_t)item * p.topk : nullptr;

    // Queries are asked for first: warp w has heads w, w + WARPS, ...
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
                q[i][0] = __ldg(reinterpret_cast<const uint4*>(at) + (L::CODES ? 2u * lane : lane));
                q[i][1] = __ldg(reinterpret_cast<const uint4*>(at) + (L::CODES ? 2u * lane + 1u : lane + 32u));
                qa[i] = reinterpret_cast<const __nv_bfloat16*>(at)[LATENT + first];
                qb[i] = reinterpret_cast<const __nv_bfloat16*>(at)[LATENT + second];
            }
        }
    }
    // A row warp's first slots too: lane l speaks for line l % 8 of its warp's eight.
    const uint32_t sub = lane / 8u, group_warp = (warp - SOFTMAX_WARPS) & 7u, line = group_warp * 8u + lane % 8u;
    const uint8_t* rows = p.buffer + (uint64_t)(p.mapped ? p.table_id[table] : table) * p.table_stride;
    int32_t begin = INT32_MIN, end = INT32_MAX;
    struct Place { int32_t slot, id; };
    auto place = [&](uint32_t j) -> Place {                 // the slot (and id) of tile j's line
        Place to = {-1, 0};
        const uint64_t k = (uint64_t)(rank + j * p.cluster) * TILE + line;
        if (k < p.topk) {
            to.slot = __ldg(slots + k);
            if (p.spans) to.id = __ldg(ids + k);
        }
        return to;
    };
    auto row_of = [&](Place to) -> const uint8_t* {         // where its row is
        if (to.slot < 0 || (p.spans && (to.id < begin || to.id >= end))) return nullptr;
        if ((uint32_t)to.slot >= p.rows) { if (p.status) atomicOr(p.status, ST_BAD_SLOT); return nullptr; }
        return rows + (uint64_t)to.slot * p.row_stride;
    };
    Place here = {-1, 0}, next = {-1, 0};                   // of the next tile whose rows are asked for, and the one behind
    if (warp >= SOFTMAX_WARPS && warp < SOFTMAX_WARPS + ROW_WARPS) {
        if (p.spans) { begin = p.spans[2 * item]; end = p.spans[2 * item + 1]; }
        here = place(0);
        next = place(1);
    }
    if (warp == WARPS - 1) {
        if (lane == 0) {
            misc->failed = 0;
            for (uint32_t i = 0; i < 4; ++i) barrier_init(bars + FULL + 8 * i, 8);
            for (uint32_t i = 0; i < 2; ++i) {
                barrier_init(bars + FREE + 8 * i, 1);
                barrier_init(bars + SUM_FULL + 8 * i, 1);
                barrier_init(bars + SUM_FREE + 8 * i, SHARES * quarters);
                barrier_init(bars + WEIGHTS + 8 * i, SOFTMAX_WARPS);
            }
            barrier_init(bars + VALUES, 8);
            for (uint32_t i = 0; i < 2; ++i) barrier_init(bars + CODES_READ + 8 * i, 1);
            barrier_init(bars + QUERIES, WARPS);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        tmem_alloc(base + L::AT_MISC, COLUMNS);
    }
    // The selection's last position: what is behind it (padding) costs nothing.
    int32_t last = -1;
    for (uint32_t k = threadIdx.x; k < p.topk; k += THREADS) if (slots[k] >= 0) last = (int32_t)k;
    last = __reduce_max_sync(0xffffffffu, last);
    if (lane == 0) misc->last[warp] = last;
    if (threadIdx.x < GROUP) reinterpret_cast<int*>(shared + L::AT_PEAK)[threadIdx.x] = in_order(__float_as_int(-INFINITY));
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&misc->tmem);
#pragma unroll
    for (uint32_t w = 0; w < WARPS; ++w) last = max(last, misc->last[w]);
    const uint32_t all_tiles = (uint32_t)(last + 1 + (int32_t)TILE - 1) / TILE;
    const uint32_t tiles = all_tiles > rank ? (all_tiles - rank + p.cluster - 1) / p.cluster : 0u;       // rank, rank + cluster, ...

    const uint8_t* row = nullptr;                           // of lane % 8 of a warp's eight
    auto row_at = [&](const uint8_t* row, uint32_t from) {
        return reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(row), (int)from));
    };
    float4 scales = make_float4(0.f, 0.f, 0.f, 0.f);        // (e4m3 rows, lanes 0-7)
    // The rows of tile j, copied as they are.  A masked row's bytes are zeros, nothing is read.
    auto fetch = [&](uint32_t j) {
        const uint32_t tile = base + L::AT_TILES + (j & 1u) * L::TILE_BYTES;
        row = row_of(here);
        here = next;
        next = j + 2 < tiles ? place(j + 2) : Place{-1, 0};
        // Eight lanes copy 128 bytes of a row side by side.  (Eight rows' 16 bytes: eight lookups of the cache for one, which bound the kernel.)
        const uint8_t* from[2] = {row_at(row, lane / 8u), row_at(row, 4u + lane / 8u)};
        if (L::CODES && lane < 8u) scales = row ? __ldg(reinterpret_cast<const float4*>(row + LATENT)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (uint32_t u = 0; u <= L::ROPE_PIECE; ++u)
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
                copy16(place_of(tile + u * PIECE, group_warp * 8u + 4u * i + lane / 8u, lane % 8u),
                       (from[i] ? from[i] : p.buffer) + (u < L::ROPE_PIECE ? 128 * u : row_bytes_of(FORMAT) - 2 * ROPE) + 16u * (lane % 8u), !from[i]);
        copies_close();
    };
    if (warp >= SOFTMAX_WARPS && warp < SOFTMAX_WARPS + ROW_WARPS && tiles) {
        if constexpr (FORMAT == AVSG_ROW_FP4) {             // (registers are for queries now)
            if (here.slot >= 0 && (uint32_t)here.slot < p.rows) asm volatile("prefetch.global.L2 [%0];" :: "l"(rows + (uint64_t)here.slot * p.row_stride + min(128u * sub, 399u)));
        } else {
            fetch(0);
        }
    }

    // ---- queries ----
    {
        float cosine = 1.f, sine = 0.f;
        if (p.rope.on) rotation(p.rope, lane, p.positions[item], cosine, sine);
#pragma unroll
        for (uint32_t i = 0; i < MINE; ++i) {
            const uint32_t h = warp + i * WARPS, quarter = h / in_quarter, line = 16u * quarter + h - quarter * in_quarter;
            if (h >= heads) break;
            float a = __bfloat162float(qa[i]), b = __bfloat162float(qb[i]);
            if (p.rope.on) {
                const float turned = a * cosine - b * sine;
                b = a * sine + b * cosine;
                a = turned;
            }
            auto put_bf16 = [&](uint32_t d, float v) {
                *reinterpret_cast<__nv_bfloat16*>(shared + place_of(L::AT_Q + BODY * PIECE, line, d >> 3) + (d & 7u) * 2u) = __float2bfloat16_rn(v);
            };
            put_bf16(first, a);
            put_bf16(second, b);
            uint32_t w[8] = {q[i][0].x, q[i][0].y, q[i][0].z, q[i][0].w, q[i][1].x, q[i][1].y, q[i][1].z, q[i][1].w};
            if constexpr (L::HALF) {
                uint32_t most = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) most = max(most, max(w[j] << 16 & 0x7FFF0000u, w[j] & 0x7FFF0000u));
                most = __reduce_max_sync(0xffffffffu, most);
                // the largest becomes 2^TO or more, below twice that
                constexpr uint32_t TO = L::CODES ? 7u : 13u;
                const uint32_t e = max(most >> 23, TO + 1u);
                const float inverse = __uint_as_float((254u + TO - e) << 23);
                if (lane == 0) reinterpret_cast<float*>(shared + L::AT_UNIT)[h] = __uint_as_float(most >= 0x7F800000u ? 0x7FC00000u : (e - TO) << 23);
                __half2 x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = __floats2half2_rn(__uint_as_float(w[j] << 16) * inverse, __uint_as_float(w[j] & 0xFFFF0000u) * inverse);
                if constexpr (L::CODES) {
                    uint32_t high[4], low[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t h0, h1, l0, l1;
                        split(x[2 * j], h0, l0);
                        split(x[2 * j + 1], h1, l1);
                        high[j] = __byte_perm(h0, h1, 0x5410);
                        low[j] = __byte_perm(l0, l1, 0x5410);
                    }
                    const uint32_t piece = base + L::AT_Q + (lane / 8u) * 2u * PIECE;
                    put16(place_of(piece, line, lane % 8u), make_uint4(high[0], high[1], high[2], high[3]));
                    put16(place_of(piece + PIECE, line, lane % 8u), make_uint4(low[0], low[1], low[2], low[3]));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = bits(x[j]);
                }
            }
            if constexpr (!L::CODES) {
                put16(place_of(base + L::AT_Q + (lane / 8u) * PIECE, line, lane % 8u), make_uint4(w[0], w[1], w[2], w[3]));
                put16(place_of(base + L::AT_Q + (lane / 8u + 4u) * PIECE, line, lane % 8u), make_uint4(w[4], w[5], w[6], w[7]));
            }
        }
        fence_for_matrix_unit();
        arrive(bars + QUERIES, lane);
    }

    if (warp < SOFTMAX_WARPS) {
        // ---- softmax: a thread has COUNT rows' scores of two heads, lines r and r + 8 of its quarter ----
        constexpr int COUNT = L::EACH / 4;
        const uint32_t quarter = warp & 3u, share = warp >> 2, quad = lane & 3u;
        const bool busy = quarter < quarters, two = in_quarter > 8u;               // (not two: nobody has a second head)
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
                factor[k] = L::HALF ? reinterpret_cast<const float*>(shared + L::AT_UNIT)[head[k]] * to_log2 : to_log2;
                if (SHAPED && p.slopes) slope[k] = p.slopes[first_head + head[k]] * LOG2E;
            }
        }
        const int32_t position = SHAPED && p.slopes ? p.positions[item] : 0;
        float most[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f}, unit = __uint_as_float(LEAST_UNIT);
        const uint32_t lanes = tmem + (quarter * 32u << 16), row = L::EACH * share + 2u * quad;       // (this thread's rows: 8 c + i, i = 0, 1, from there)
        auto outgrown = [](float peak, float most) { return peak > most + LAZY<FORMAT> || (most == -INFINITY && peak > -INFINITY); };
        auto meet = [] { asm volatile("barrier.cta.sync 1, %0;" :: "n"(32 * SOFTMAX_WARPS) : "memory"); };
        auto pair_at = [&](uint32_t at, uint32_t c) { return *reinterpret_cast<const float2*>(shared + at + 4u * (row + 8u * c)); };
        auto unit_of = [&](uint32_t j, uint32_t c) {
            const uint32_t two = *reinterpret_cast<const uint16_t*>(shared + L::AT_UNITS + TILE * (j & 1u) + row + 8u * c);
            return make_float2(__uint_as_float((two & 255u) << 23), __uint_as_float(two >> 8 << 23));
        };
        auto scale_of = [&](uint32_t j, uint32_t g, uint32_t c) { return pair_at(L::AT_SCALES + 4u * TILE * (4u * (j & 1u) + g), c); };
        float x[2][COUNT];                                    // a tile's scores (log2), complete after its last step
        // Step g of tile j: a sum or two from TMEM.
        auto take = [&](uint32_t j, uint32_t g) {
            if (!busy || j >= tiles) return;
            const uint32_t step = j * L::STEPS + g, at = lanes + COL_S + 128 * (step % SLOTS) + L::EACH * share;
            wait(bars + SUM_FULL + 8 * (step % SLOTS), step / SLOTS & 1u, misc);
            __syncwarp();
            tmem_after_sync();
            float s[2 * COUNT], t[2 * COUNT];
            tmem_load_scores(at, s);
            if (FORMAT == AVSG_ROW_FP4 || (FORMAT == AVSG_ROW_FP8 && g < 2)) tmem_load_scores(at + 64, t);
            float2 u[COUNT / 2], v[COUNT / 2];
#pragma unroll
            for (int c = 0; c < COUNT / 2; ++c) {
                if (L::CODES && g < 2) { u[c] = scale_of(j, 2 * g, c); v[c] = scale_of(j, 2 * g + 1, c); }
                if (FORMAT == AVSG_ROW_FP4) u[c] = unit_of(j, c);
            }
            tmem_loaded();
            tmem_before_sync();
            arrive(bars + SUM_FREE + 8 * (step % SLOTS), lane);
#pragma unroll
            for (int c = 0; c < COUNT / 2; ++c)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == 1 && !two) continue;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float a = s[4 * c + 2 * k + i], d = t[4 * c + 2 * k + i];
                        float& to = x[k][2 * c + i];
                        if (FORMAT == AVSG_ROW_BF16) to = a * to_log2;
                        else if (FORMAT == AVSG_ROW_FP4) to = a * (factor[k] * (i ? u[c].y : u[c].x)) + d * to_log2;
                        else if (g == 0) to = a * (i ? u[c].y : u[c].x) + d * (i ? v[c].y : v[c].x);
                        else if (g == 1) to += a * (i ? u[c].y : u[c].x) + d * (i ? v[c].y : v[c].x);
                        else to = to * factor[k] + a * to_log2;
                    }
                }
        };
        int32_t id[COUNT];                                     // of this thread's rows, where scores have a bias by distance
        auto ask_ids = [&](uint32_t j) {
            if (SHAPED && busy && p.slopes)
#pragma unroll
                for (int c = 0; c < COUNT; ++c) {
                    const uint64_t at = (uint64_t)(rank + j * p.cluster) * TILE + row + 8 * (c / 2) + c % 2;
                    id[c] = at < p.topk ? __ldg(ids + at) : 0;
                }
        };
        ask_ids(0);
#pragma unroll
        for (uint32_t g = 0; g < L::STEPS; ++g) take(0, g);
        for (uint32_t j = 0; j < tiles; ++j) {              // (also after a wait that failed: the warps meet at a barrier)
            const uint32_t b = j & 1u;
            bool behind = false;
            float peak[2] = {-INFINITY, -INFINITY};
            if (busy) {
                if constexpr (SHAPED) {
#pragma unroll
                    for (int c = 0; c < COUNT; ++c) {
                        const float away = p.slopes ? (float)(id[c] - position) : 0.f;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            if (k == 1 && !two) continue;
                            if (p.softcap > 0.f) x[k][c] = capped(x[k][c], p.softcap, p.per_cap);
                            if (p.slopes) x[k][c] += slope[k] * away;
                        }
                    }
                }
                const uint32_t seen = (COUNT == 8 ? *reinterpret_cast<const uint32_t*>(shared + L::AT_SEEN + 8 * b + 4 * share)
                                                  : *reinterpret_cast<const uint16_t*>(shared + L::AT_SEEN + 8 * b + 2 * share)) >> (2u * quad);
                constexpr uint32_t ALL = COUNT == 8 ? 0x03030303u : 0x0303u;
                if ((seen & ALL) != ALL) {  // masked ones among this thread's rows
#pragma unroll
                    for (int c = 0; c < COUNT; ++c)
                        if (!(seen >> (8 * (c / 2) + c % 2) & 1u)) x[0][c] = x[1][c] = -INFINITY;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == 1 && !two) continue;
#pragma unroll
                    for (int c = 0; c < COUNT; ++c) peak[k] = fmaxf(peak[k], x[k][c]);
                    behind |= real[k] && outgrown(peak[k], most[k]);
                }
                if (L::HALF) behind |= reinterpret_cast<const float*>(shared + L::AT_TOPS)[b * L::TOPS + lane % L::TOPS] > unit;
            }
            // Weights would grow beyond their range: the references move, and O is brought to the new ones before it is added to.
            int any;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tbarrier.cta.red.or.pred p, 1, %2, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
                         : "=r"(any) : "r"((int)behind), "n"(32 * SOFTMAX_WARPS) : "memory");
            if (any) {
                int* peaks = reinterpret_cast<int*>(shared + L::AT_PEAK);
                if (busy)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        peak[k] = fmaxf(peak[k], __shfl_xor_sync(0xffffffffu, peak[k], 1));
                        peak[k] = fmaxf(peak[k], __shfl_xor_sync(0xffffffffu, peak[k], 2));
                        if (real[k] && quad == 0) atomicMax(peaks + head[k], in_order(__float_as_int(peak[k])));
                    }
                float less = 1.f, keep[2] = {1.f, 1.f};
                if (L::HALF) {
                    float now = 0.f;
#pragma unroll
                    for (uint32_t w = 0; w < L::TOPS; ++w) now = fmaxf(now, reinterpret_cast<const float*>(shared + L::AT_TOPS)[b * L::TOPS + w]);
                    if (now > unit) {                       // (powers of two, both)
                        const float to = now * 8.f;                             // (with room, so that the next larger row moves nothing)
                        less = unit / to;
                        unit = to;
                    }
                }
                meet();
                if (busy)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        if (real[k]) {
                            const float to = __int_as_float(in_order(peaks[head[k]]));
                            if (outgrown(to, most[k])) {
                                keep[k] = exp2f(most[k] - to);
                                most[k] = to;
                                total[k] *= keep[k];
                            }
                            if (share == 0 && quad == 0) reinterpret_cast<float*>(shared + L::AT_ALPHA)[head[k]] = keep[k] * less;
                        }
                meet();
                if (busy && share == 0 && quad == 0)        // (for the next time, which everybody meets before)
#pragma unroll
                    for (int k = 0; k < 2; ++k) if (real[k]) peaks[head[k]] = in_order(__float_as_int(-INFINITY));
                if (j > 0) {
                    wait(bars + FREE + 8 * (b ^ 1u), (j - 1) >> 1 & 1u, misc);
                    __syncwarp();
                    tmem_after_sync();
                    const float* alpha = reinterpret_cast<const float*>(shared + L::AT_ALPHA);
                    // 16 heads at a time, those of which one moved
                    const uint32_t low = __ballot_sync(0xffffffffu, lane < heads && alpha[lane] != 1.f);
                    const uint32_t high = __ballot_sync(0xffffffffu, lane + 32u < heads && alpha[lane + 32u] != 1.f);
                    for (uint32_t part = share; part < 4u; part += SHARES)
                        for (uint32_t c = 0; c < columns; c += 16) {
                            if (((c < 32u ? low : high) >> (c % 32u) & 0xFFFFu) == 0) continue;
                            float o[16];
                            tmem_load_32x16(lanes + COL_OUT + 64 * part + c, o);
                            tmem_loaded();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] *= alpha[c + i];
                            tmem_store_32x16(lanes + COL_OUT + 64 * part + c, o);
                        }
                    tmem_stored();
                }
            }
            uint32_t pair[2][COUNT / 2];                            // weights, two neighbouring rows' to a word
            if (busy) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (k == 1 && !two) continue;
                    const float from = (most[k] == -INFINITY ? 0.f : most[k]);
#pragma unroll
                    for (int c = 0; c < COUNT / 2; ++c) {
                        const float v = exp2f(x[k][2 * c] - from), w = exp2f(x[k][2 * c + 1] - from);
                        total[k] += v + w;
                        pair[k][c] = L::HALF ? bits(__floats2half2_rn(v, w)) : bf16_pair(v * (1.f / BF16_UNIT), w * (1.f / BF16_UNIT));
                    }
                }
            }
            // The next tile's first sums, already: their place in TMEM is wanted.  (94 us; 100 where they are taken after the weights are out.)
            if (L::CODES) take(j + 1, 0);
            if (busy) {
                const float inverse = 1.f / unit;
                const uint32_t piece = base + (L::CODES ? L::AT_WEIGHTS : L::AT_TILES + b * L::TILE_BYTES + L::ROPE_PIECE * PIECE);
                if (L::HALF)
#pragma unroll
                    for (int c = 0; c < COUNT / 2; ++c) {
                        const float2 u = unit_of(j, c);
                        const __half2 ratio = __floats2half2_rn(u.x * inverse, u.y * inverse);
#pragma unroll
                        for (int k = 0; k < 2; ++k) if (k == 0 || two) pair[k][c] = bits(__hmul2(*reinterpret_cast<const __half2*>(&pair[k][c]), ratio));
                    }
                if (L::CODES && j > 0) wait(bars + FREE + 8 * (b ^ 1u), (j - 1) >> 1 & 1u, misc);              // (the last ones are read)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (real[k])
#pragma unroll
                        for (int c = 0; c < COUNT / 2; ++c) put4(place_of(piece, head[k], COUNT / 2 * share + c) + quad * 4u, pair[k][c]);
            }
            fence_for_matrix_unit();
            tmem_before_sync();
            arrive(bars + WEIGHTS + 8 * b, lane);
            ask_ids(j + 1);
            if (!L::CODES) take(j + 1, 0);
#pragma unroll
            for (uint32_t g = 1; g < L::STEPS; ++g) take(j + 1, g);
        }
        if (tiles) wait(bars + FREE + 8 * ((tiles - 1) & 1u), (tiles - 1) >> 1 & 1u, misc);       // (the tiles' place is free then)
        meet();
        if (busy) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                total[k] += __shfl_xor_sync(0xffffffffu, total[k], 1);
                total[k] += __shfl_xor_sync(0xffffffffu, total[k], 2);
                if (real[k] && quad == 0) {
                    if (share == 0) reinterpret_cast<float*>(shared + L::AT_MOST)[head[k]] = most[k];
                    reinterpret_cast<float*>(shared + L::AT_SUM)[share * GROUP + head[k]] = total[k];
                }
            }
        }
        if (threadIdx.x == 0) misc->unit = L::HALF ? unit : BF16_UNIT;
    } else if (warp < SOFTMAX_WARPS + ROW_WARPS) {
        // ---- rows ----
        // (lanes 0-7 speak for eight rows)
        auto put_seen = [&](uint32_t b, uint32_t eight, const uint8_t* row) {
            const uint32_t seen = __ballot_sync(0xffffffffu, row != nullptr);
            if (lane == 0) shared[L::AT_SEEN + 8 * b + eight] = (uint8_t)seen;
        };
        auto announce = [&](uint32_t b, uint32_t half) {
            fence_for_matrix_unit();
            arrive(bars + FULL + 16 * b + 8 * half, lane);
        };
        auto put_top = [&](uint32_t b, float top) {
            top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));                // (not negative; a NaN, too)
            if (lane == 0) reinterpret_cast<float*>(shared + L::AT_TOPS)[b * L::TOPS + group_warp] = top;
        };
        auto passed = [&](uint32_t bar, uint32_t j) { return __all_sync(0xffffffffu, wait(bars + bar + 8 * (j & 1u), j >> 1 & 1u, misc)); };    // of tile j
        uint8_t* units = shared + L::AT_UNITS + line;
        if constexpr (FORMAT == AVSG_ROW_FP4) {
            // A tile's numbers are in registers; as soon as some are laid out the next tile's are asked for.
            RowPart part;
            const uint8_t* from[2];
            auto advance = [&](uint32_t j) {                // tile j's rows, whose places are known by now
                row = row_of(here);
                here = next;
                next = j + 2 < tiles ? place(j + 2) : Place{-1, 0};
                for (int i = 0; i < 2; ++i) from[i] = row_at(row, 4u * i + lane / 8u);
                part.scales = unit_at(lane < 8u ? row : nullptr, 16);
            };
            auto ask = [&](int c, int i) { part.body[c][i] = unit_at(from[i], 8u * c + lane % 8u); };
            auto ask_rope = [&](int i) { part.rope[i] = unit_at(from[i], 17u + lane % 8u); };
            if (tiles) {
                advance(0);
#pragma unroll
                for (int c = 0; c < 2; ++c) { ask(c, 0); ask(c, 1); }
                ask_rope(0); ask_rope(1);
            }
            for (uint32_t j = 0; j < tiles; ++j) {
                const uint32_t b = j & 1u, tile = base + L::AT_TILES + b * L::TILE_BYTES;
                const uint4 scales = part.scales;
                const uint32_t unit = nibble_unit(scales), seen = __ballot_sync(0xffffffffu, row != nullptr);
                const uint32_t top = __reduce_max_sync(0xffffffffu, lane < 8u && row ? unit : 0u);
                advance(j + 1);                             // (beyond the last tile: nothing)
                if (j >= 2 && !passed(FREE, j - 2)) break;
                if (lane == 0) {
                    shared[L::AT_SEEN + 8 * b + group_warp] = (uint8_t)seen;
                    reinterpret_cast<float*>(shared + L::AT_TOPS)[b * L::TOPS + group_warp] = __uint_as_float(top << 23);
                }
                if (lane < 8u) units[b * TILE] = (uint8_t)(seen >> lane & 1u ? unit : 0u);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    // (codes 32 U .. have scale U: this lane's U is 8 c + lane % 8)
                    const uint32_t low = c ? scales.z : scales.x, high = c ? scales.w : scales.y;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int line = 4 * i + (int)(lane / 8u);
                        const uint32_t s0 = __shfl_sync(0xffffffffu, low, line), s1 = __shfl_sync(0xffffffffu, high, line);
                        const int its_unit = (int)__shfl_sync(0xffffffffu, unit, line);
                        put_codes(part.body[c][i], c, its_unit, lane & 4u ? s1 : s0, tile, group_warp * 8u + line, lane);
                        ask(c, i);
                    }
                    if (c == 1)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            put16(place_of(tile + L::ROPE_PIECE * PIECE, group_warp * 8u + 4u * i + lane / 8u, lane % 8u), part.rope[i]);
                            ask_rope(i);
                        }
                    announce(b, c);
                }
            }
        } else if constexpr (L::CODES) {
            // Codes are copied as they are, a tile ahead; each warp makes values of its own eight rows', which nobody else has to wait for.
            __half2 ratio[4];                               // of scales and unit
            auto show = [&](uint32_t j) {                   // tile j is there: what softmax wants to know of its rows, then the matrix unit may begin
                const uint32_t b = j & 1u;
                const float s[4] = {__shfl_sync(0xffffffffu, scales.x, lane % 8u), __shfl_sync(0xffffffffu, scales.y, lane % 8u),
                                    __shfl_sync(0xffffffffu, scales.z, lane % 8u), __shfl_sync(0xffffffffu, scales.w, lane % 8u)};
                const uint32_t unit = s[0] != 0.f || s[1] != 0.f || s[2] != 0.f || s[3] != 0.f ? code_unit(s) : 0u;
                const float inverse = __uint_as_float((254u << 23) - (unit & 0x7F800000u));
#pragma unroll
                for (int g = 0; g < 4; ++g)                 // (NaN where one is no number)
                    ratio[g] = __half2half2(__float2half_rn(unit < 0x7F800000u ? s[g] * inverse : __uint_as_float(0x7FC00000u)));
                reinterpret_cast<float*>(shared + L::AT_SCALES)[(4 * b + sub) * TILE + line] = sub == 0 ? s[0] : sub == 1 ? s[1] : sub == 2 ? s[2] : s[3];
                if (sub == 0) units[b * TILE] = (uint8_t)(unit >> 23);
                put_top(b, __uint_as_float(unit));
                put_seen(b, group_warp, row);
                announce(b, 0);
            };
            if (tiles) {
                copies_wait<0>();
                show(0);
            }
            for (uint32_t j = 0; j < tiles; ++j) {
                __half2 now[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) now[g] = ratio[g];
                if (j + 1 < tiles) {                        // into the other place, as soon as the scores of the tile there are through
                    if (j >= 1 && !passed(CODES_READ, j - 1)) break;
                    fetch(j + 1);
                    copies_wait<0>();
                    if (j >= 1 && !passed(WEIGHTS, j - 1)) break;                // (who reads the scales of the tile before is through)
                    show(j + 1);
                }
                if (j >= 1 && !passed(FREE, j - 1)) break;
                __syncwarp();                               // (all lanes' copies are there)
                const uint32_t tile = base + L::AT_TILES + (j & 1u) * L::TILE_BYTES;
#pragma unroll
                for (uint32_t u = 0; u < 8; u += 4) {       // numbers 64 u + 16 sub ..
                    uint32_t w[4][4];
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i)
                        asm volatile("ld.shared::cta.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i][0]), "=r"(w[i][1]), "=r"(w[i][2]), "=r"(w[i][3])
                                     : "r"(place_of(tile + (u + i) / 2u * PIECE, line, (u + i) % 2u * 4u + sub)));
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        uint32_t x[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            x[k] = bits(__hmul2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i][k / 2] >> (k % 2 * 16)), __NV_E4M3)), now[(u + i) / 2]));
                        put16(place_of(base + L::AT_VALUES + (u + i) * PIECE, line, 2 * sub), make_uint4(x[0], x[1], x[2], x[3]));
                        put16(place_of(base + L::AT_VALUES + (u + i) * PIECE, line, 2 * sub + 1), make_uint4(x[4], x[5], x[6], x[7]));
                    }
                }
                fence_for_matrix_unit();
                arrive(bars + VALUES, lane);
            }
        } else {
            uint32_t there = 0;                                                  // tiles announced
            auto announce_both = [&](uint32_t tile) { announce(tile & 1u, 0); announce(tile & 1u, 1); };
            if (tiles) put_seen(0, group_warp, row);
            for (uint32_t j = 1; j < tiles; ++j) {
                const uint32_t b = j & 1u;
                if (j >= 2) {
                    const uint32_t bar = bars + FREE + 8 * b, parity = (j - 2) >> 1 & 1u;
                    if (there < j && !__all_sync(0xffffffffu, barrier_done(bar, parity))) {
                        copies_wait<0>();                                        // time to spare: all that is under way is announced first
                        while (there < j) announce_both(there++);
                    }
                    if (!__all_sync(0xffffffffu, wait(bar, parity, misc))) break;
                }
                fetch(j);
                put_seen(b, group_warp, row);
                if (there < j) {                                                 // the tile before this one is announced when it is there
                    copies_wait<1>();
                    while (there < j) announce_both(there++);
                }
            }
            copies_wait<0>();
            if (!misc->failed) while (there < tiles) announce_both(there++);
        }
        copies_wait<0>();
    } else {
        // ---- products ----
        constexpr Product TYPE = L::HALF ? Product::FP16 : Product::BF16, S_TYPE = L::CODES ? Product::E4M3 : TYPE;
        constexpr uint32_t S_SHAPE = product_shape(S_TYPE, 64, TILE, false), ROPE_SHAPE = product_shape(Product::BF16, 64, TILE, false);
        const uint32_t out_shape = product_shape(TYPE, 128, columns, true);
        const uint32_t query = operand(base + L::AT_Q, 16);
        // Part `part` of tile j's S: pieces 0-3 are there with the first half of the tile, the others and the rotated one with the second.
        auto score = [&](uint32_t step, uint32_t j, uint32_t part) {
            const uint32_t to = tmem + COL_S + 128 * (step % SLOTS), tile = operand(base + L::AT_TILES + (j & 1u) * L::TILE_BYTES, 16);
            if (part < 2) {
                const uint32_t q = query + part * (4 * PIECE / 16), rows = tile + part * ((L::CODES ? 2 : 4) * PIECE / 16);
#pragma unroll
                for (uint32_t i = 0; i < 16; ++i) {
                    const uint32_t at = (i / 4 * PIECE + i % 4 * 32) / 16;
                    // codes: two sums of 128 numbers each, both halves of the queries by the same rows; else one of all 512
                    if constexpr (L::CODES) multiply<S_TYPE>(to + i / 8 * 64, q + at, rows + (i / 8 * PIECE + i % 4 * 32) / 16, S_SHAPE, i % 8 > 0);
                    else multiply<S_TYPE>(to, q + at, rows + at, S_SHAPE, part + i > 0);
                }
            }
            if (part == L::PARTS - 1) {
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    multiply<Product::BF16>(to + (FORMAT == AVSG_ROW_FP4 ? 64 : 0), query + (BODY * PIECE + 32 * i) / 16, tile + (L::ROPE_PIECE * PIECE + 32 * i) / 16,
                                            ROPE_SHAPE, FORMAT == AVSG_ROW_BF16 || i > 0);
            }
            if (L::CODES || part == L::PARTS - 1) products_done(bars + SUM_FULL + 8 * (step % SLOTS));
            if (L::CODES && part == L::PARTS - 1) products_done(bars + CODES_READ + 8 * (j & 1u));
        };
        auto add = [&](uint32_t j) {
            const uint32_t tile = base + L::AT_TILES + (j & 1u) * L::TILE_BYTES;
            const uint32_t rows = operand(L::CODES ? base + L::AT_VALUES : tile, PIECE), weights = operand(L::CODES ? base + L::AT_WEIGHTS : tile + L::ROPE_PIECE * PIECE, 16);
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) {
                const uint32_t part = i / 4, k = i % 4;
                multiply<TYPE>(tmem + COL_OUT + 64 * part, rows + (part * 2 * PIECE + k * 2048) / 16, weights + 2 * k, out_shape, j + k > 0);
            }
            products_done(bars + FREE + 8 * (j & 1u));
        };
        if (tiles && one_lane() && wait(bars + QUERIES, 0, misc)) {
            uint32_t scored = 0, part = 0, added = 0;           // tiles, parts of the next one, tiles
            uint32_t looks = 0;                                 // without success
            long long idle = 0;
            while (added < tiles) {
                const uint32_t step = L::STEPS > 1 ? scored * L::STEPS + part : scored;
                if (barrier_done(bars + WEIGHTS + 8 * (added & 1u), added >> 1 & 1u) && (!L::CODES || barrier_done(bars + VALUES, added & 1u))) {
                    tmem_after_sync();
                    add(added++);
                    looks = 0;
                } else if (scored < tiles && barrier_done(bars + FULL + 16 * (scored & 1u) + (part && !L::CODES ? 8 : 0), scored >> 1 & 1u) &&
                           (step < SLOTS || (L::STEPS == 1 && part > 0) || barrier_done(bars + SUM_FREE + 8 * (step % SLOTS), (step / SLOTS - 1) & 1u))) {
                    tmem_after_sync();
                    score(step, scored, part);
                    if (++part == L::PARTS) { part = 0; ++scored; }
                    looks = 0;
                } else if ((++looks & 255u) == 0) {
                    if (looks == 256u) idle = clock64();
                    else if (reinterpret_cast<volatile Misc*>(misc)->failed || clock64() - idle > WAIT_CLOCKS) { misc->failed = 1; break; }
                }
            }
        }
    }

    // ---- the block's sums to shared memory, and the cluster's blocks' together ----
    __syncwarp();
    tmem_after_sync();
    if (warp < SOFTMAX_WARPS && tiles) {                        // (who have waited for the last product)
        float* out = reinterpret_cast<float*>(shared + L::AT_OUT);
        const uint32_t quarter = warp & 3u;
        for (uint32_t part = warp / 4u; part < 4u; part += SHARES)
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
    // A head's maximum, sum and unit in this block, and the unit's share in the sum.
    if (threadIdx.x < heads) {
        const float* sums = reinterpret_cast<const float*>(shared + L::AT_SUM) + threadIdx.x;
        float sum = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < SHARES; ++i) sum += sums[i * GROUP];
        reinterpret_cast<float4*>(shared + L::AT_STATE)[threadIdx.x] = make_float4(reinterpret_cast<const float*>(shared + L::AT_MOST)[threadIdx.x], sum, misc->unit, sum == 0.f ? 0.f : misc->unit / sum);
    }
    if (p.cluster > 1) cluster_sync();
    else __syncthreads();
    uint8_t* out = p.out + table * p.out_stride[0] + token * p.out_stride[1] + first_head * p.out_stride[2];
    float* lse = p.lse ? p.lse + (uint64_t)item * p.heads + first_head : nullptr;
    if (!misc->failed) {
        if (p.cluster == 1) {
            const float4* from = reinterpret_cast<const float4*>(shared + L::AT_OUT);
            const float4* state = reinterpret_cast<const float4*>(shared + L::AT_STATE);
            if (lse && threadIdx.x < heads) lse[threadIdx.x] = logarithm(state[threadIdx.x].x, state[threadIdx.x].y);
#pragma unroll 4
            for (uint32_t u = threadIdx.x; u < heads * (LATENT / 4); u += THREADS) {
                const uint32_t h = u / (LATENT / 4), d = u % (LATENT / 4);
                const float w = state[h].w;
                const float4 v = w == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : from[u];                  // (without rows there are no sums)
                *reinterpret_cast<uint2*>(out + h * p.out_stride[2] + 8 * d) = make_uint2(bf16_pair(w * v.x, w * v.y), bf16_pair(w * v.z, w * v.w));
            }
        } else {
            if (p.cluster == 2) join<2, WARPS>(base + L::AT_STATE, base + L::AT_OUT, heads, rank, warp, lane, out, p.out_stride[2], lse);
            else if (p.cluster == 4) join<4, WARPS>(base + L::AT_STATE, base + L::AT_OUT, heads, rank, warp, lane, out, p.out_stride[2], lse);
            else join<8, WARPS>(base + L::AT_STATE, base + L::AT_OUT, heads, rank, warp, lane, out, p.out_stride[2], lse);
        }
    } else if (threadIdx.x == 0 && p.status) {
        atomicOr(p.status, ST_WAIT_TIMEOUT);
    }
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

// Clusters of 1, 2, 4, 8 blocks that a device runs at once (blocks of a cluster share a GPC), as found by attend_prepare().
constexpr int MAX_DEVICES = 64;
std::atomic<int> g_active[MAX_DEVICES][4];

constexpr uint32_t threads_of(uint32_t format)
{
    return format == AVSG_ROW_FP8 ? Layout<AVSG_ROW_FP8>::THREADS : format == AVSG_ROW_FP4 ? Layout<AVSG_ROW_FP4>::THREADS : Layout<AVSG_ROW_BF16>::THREADS;
}

cudaLaunchConfig_t config(uint32_t format, uint32_t blocks, uint32_t cluster, cudaLaunchAttribute* attr, cudaStream_t stream)
{
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3(blocks); c.blockDim = dim3(threads_of(format)); c.dynamicSmemBytes = SHARED_MOST; c.stream = stream;
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
    for (int i = 0; i < 4; ++i) {
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t c = config(AVSG_ROW_FP8, 1u << i, 1u << i, &attr, nullptr);
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, attend_kernel(AVSG_ROW_FP8, false), &c) != cudaSuccess) { cudaGetLastError(); n = 0; }
        g_active[device][i] = n;
    }
    return cudaSuccess;
}

cudaError_t launch_attend(AttendParams& p, uint32_t format, cudaStream_t stream)
{
    // Blocks of a query: its rows over a cluster's, its heads in groups; as many as find room at once.  First the rows, a tile or more to
    // a block: 17 us for 62 with one request of 128 heads and bf16 rows, 46 for 79 with 64 queries of 4-bit rows, but 56 and 94 with two and four times
    // the blocks that fit.  Then smaller groups of heads, down to 16, although each gathers the rows again (a block's sums travel between a cluster's
    // blocks, heads x 2 KB): 17 us for 20 with that one request.
    const uint32_t least = (p.heads + GROUP - 1) / GROUP, tiles = (p.topk + TILE - 1) / TILE;
    const uint64_t queries = (uint64_t)p.n * p.n_tokens;
    int device = -1;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    uint32_t log = 0;
    if (device >= 0 && device < MAX_DEVICES)
        for (log = 3; log > 0; --log) if (queries * least <= (uint64_t)g_active[device][log] && tiles >= 1u << log) break;
    p.cluster = 1u << log;
    p.groups = least;
    while (device >= 0 && device < MAX_DEVICES && p.heads > 16u * p.groups && queries * p.groups * 2 <= (uint64_t)g_active[device][log]) p.groups *= 2;
    p.group_heads = (p.heads + p.groups - 1) / p.groups;
    p.groups = (p.heads + p.group_heads - 1) / p.group_heads;
    const uint64_t work = queries * p.groups;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t c = config(format, (uint32_t)(work * p.cluster), p.cluster, &attr, stream);
    void* args[] = {&p};
    return cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(attend_kernel(format, p.softcap > 0.f || p.slopes)), args);
}

}  // namespace avsg
