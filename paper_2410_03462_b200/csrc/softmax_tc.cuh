// What the tensor-core kernels of softmax attention share: boxes of rows by the copy engine, which tiles a block visits, scores from raw products.
#pragma once

#include "softmax.cuh"
#include "tc_common.cuh"

namespace grf_softmax_tc {

using namespace grf_tc;

constexpr int BT = 128;                 // queries, and keys, of a tile
constexpr int32_t MOST_WITH_DOCS = 1 << 20;     // tokens, with documents: the tiles' bits of more do not fit beside d = 128
constexpr uint32_t HALF = BT * 128;     // bytes of 64 columns of a tile: rows of 128 bytes, swizzled over a row

// A box of 64 columns and BT rows of (columns, tokens, heads, sequences), by one elected lane of a converged warp.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int32_t col, int32_t row, int32_t head, int32_t batch, uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];\n\t}"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(col), "r"(row), "r"(head), "r"(batch), "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_elected(uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "@q mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar) : "memory");
}

// A tile as the operand whose rows are the product's rows or columns (K-major): 32 bytes along a row per step of 16, HALF per 64.
__device__ __forceinline__ uint64_t rows_operand(uint32_t base) { return swizzled_desc(base, 16, 1024, 2); }
// A tile as the right operand summed over its rows (MN-major): 64 columns every HALF bytes, eight rows every 1024; 2048 per step of 16 rows.
__device__ __forceinline__ uint64_t columns_operand(uint32_t base) { return swizzled_desc(base, HALF, 1024, 2); }
__device__ __forceinline__ uint32_t lo32(uint64_t x) { return (uint32_t)x; }
__device__ __forceinline__ uint32_t hi32(uint64_t x) { return (uint32_t)(x >> 32); }

// D[128][128] = A B^T over d columns (rounded up to 16), both operands rows in shared memory.
template <int DP>
__device__ __forceinline__ void product_over_columns(uint32_t acc, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, int32_t steps)
{
    constexpr uint32_t idesc = instr_desc(BT, false, false);
#pragma unroll
    for (int y = 0; y < DP / 16; ++y) {
        if (y < steps) {
            const uint32_t at = (uint32_t)(y / 4) * (HALF / 16) + (uint32_t)(y % 4) * 2;
            if (y == 0) mma_bf16_ss_halves<false>(acc, a_lo + at, a_hi, b_lo + at, b_hi, idesc);
            else mma_bf16_ss_halves<true>(acc, a_lo + at, a_hi, b_lo + at, b_hi, idesc);
        }
    }
}
// acc[128][DP] (+)= A[128][128] B[128][DP]: A in tensor memory (bf16 pairs), B's rows in shared memory.
template <int DP>
__device__ __forceinline__ void product_over_rows(uint32_t acc, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t accumulate)
{
    constexpr uint32_t idesc = instr_desc(DP, false, true);
#pragma unroll
    for (int y = 0; y < BT / 16; ++y) mma_bf16_ts_halves(acc, a_tmem + y * 8, b_lo + y * (2048 / 16), b_hi, idesc, y > 0 ? 1u : accumulate);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 2^x of two values by multiply-adds, for some of a tile's values, as the pipe of ex2 (a warp in eight cycles) bounds a softmax: x = i + f with i the
// nearest integer (a sum with 1.5 * 2^23 rounds to it), 2^f by a cubic whose largest relative error over -1/2 .. 1/2 is least, constant term 1
// (measured 1.0e-4: a fortieth of what rounding to bf16 takes), and i added to the exponent.  x <= 127 - 1/2; what is below -127, -infinity with it,
// becomes 0.  NaN becomes 0: callers let it reach a row by its maximum.
__device__ __forceinline__ void ex2_by_fma(uint64_t x, float& y0, float& y1)
{
    constexpr float MAGIC = 12582912.0f;
    float x0, x1;
    unpack2(x, x0, x1);
    x = pack2(fmaxf(x0, -127.0f), fmaxf(x1, -127.0f));
    const uint64_t r = add2(x, pack2(MAGIC, MAGIC)), f = fma2(add2(r, pack2(-MAGIC, -MAGIC)), pack2(-1.0f, -1.0f), x);
    uint64_t q = fma2(f, pack2(0.055008933f, 0.055008933f), pack2(0.24221097f, 0.24221097f));
    q = fma2(q, f, pack2(0.69328290f, 0.69328290f));
    q = fma2(q, f, pack2(1.0f, 1.0f));
    float r0, r1, q0, q1;
    unpack2(r, r0, r1);
    unpack2(q, q0, q1);
    y0 = __uint_as_float(__float_as_uint(q0) + (__float_as_uint(r0) << 23));
    y1 = __uint_as_float(__float_as_uint(q1) + (__float_as_uint(r1) << 23));
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// tanh within 2e-7 (absolute): 1 - 2 / (1 + e^2y).
__device__ __forceinline__ float tanh_any(float y)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + ex2(y * (2.0f * GRF_LOG2E))));
    return fmaf(-2.0f, r, 1.0f);
}
// Every value of a thread becomes tanh(by * value).  Where |by * value| <= 1 in the whole warp, which caps are chosen for, by a polynomial: y P(y^2) with
// P of degree 5, interpolating tanh(sqrt w) / sqrt w at the Chebyshev points of 0 .. 1, is within 5.2e-7 of tanh (measured over the range) and
// takes eight packed multiply-adds a pair, where the exponential and the reciprocal of tanh_any take 32 cycles of the pipe that the softmax's own
// exponentials need (8 each).
template <int N> __device__ __forceinline__ void capped(uint32_t (&v)[N][16], float by)
{
    const uint64_t by2 = pack2(by, by);
    float most[2] = {0.0f, 0.0f};
#pragma unroll
    for (int y = 0; y < N; ++y)
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const uint64_t x = mul2(pack2(v[y][e], v[y][e + 1]), by2);
            float x0, x1;
            unpack2(x, x0, x1);
            v[y][e] = __float_as_uint(x0);
            v[y][e + 1] = __float_as_uint(x1);
            most[e >> 1 & 1] = max3(most[e >> 1 & 1], fabsf(x0), fabsf(x1));
        }
    if (__all_sync(0xffffffffu, fmaxf(most[0], most[1]) <= 1.0f)) {        // (max passes over NaN, which stays NaN either way)
#pragma unroll
        for (int y = 0; y < N; ++y)
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const uint64_t x = pack2(v[y][e], v[y][e + 1]), w = mul2(x, x);
                uint64_t t = fma2(w, pack2(-0.0030582291f, -0.0030582291f), pack2(0.016720856f, 0.016720856f));
                t = fma2(t, w, pack2(-0.051585987f, -0.051585987f));
                t = fma2(t, w, pack2(0.13280721f, 0.13280721f));
                t = fma2(t, w, pack2(-0.33328950f, -0.33328950f));
                t = fma2(t, w, pack2(0.99999940f, 0.99999940f));
                t = mul2(t, x);
                float x0, x1;
                unpack2(t, x0, x1);
                v[y][e] = __float_as_uint(x0);
                v[y][e + 1] = __float_as_uint(x1);
            }
    } else {
#pragma unroll
        for (int y = 0; y < N; ++y)
#pragma unroll
            for (int e = 0; e < 16; ++e) v[y][e] = __float_as_uint(tanh_any(__uint_as_float(v[y][e])));
    }
}

__device__ __forceinline__ int32_t uniform(int32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// Documents of two blocks: the same one throughout.
__device__ __forceinline__ bool one_document(const int4& q, const int4& k) { return q.x == q.y && k.x == k.y && q.x == k.x && (q.z | k.z) == 0; }
// Bits of a block's tiles, in shared memory; only with documents, as otherwise the tiles follow from positions alone.
__device__ __forceinline__ bool bit(const uint32_t* w, int32_t t) { return w[t >> 5] >> (t & 31) & 1u; }

}  // namespace grf_softmax_tc

// [B][heads][tokens][d] bf16 by strides (0: that axis is not stepped along): boxes of 64 columns and 128 rows, swizzled.
bool grf_make_token_box_map(CUtensorMap* map, const void* base, const int64_t (&stride)[3], int32_t batch, int32_t heads, int32_t tokens, int32_t d);
