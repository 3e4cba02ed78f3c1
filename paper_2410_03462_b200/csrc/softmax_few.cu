// Softmax attention of a few queries per sequence (new tokens against a cache): the keys are split over CTAs and warps, and K and V are
// read straight into registers, once for every block of rows.
//
// The rows of one key head are its group's heads times n_q queries, in blocks of 16 (bf16) or 4 (fp32).  A warp goes over every fourth
// 16-key (fp32: 8-key) tile of its CTA's stretch with running maxima and sums; warps join in shared memory, CTAs of a sequence and head
// in a cluster of up to eight through distributed shared memory, more than eight through the workspace and a second launch.
//
// bf16: S^T = K Q^T and O^T = V^T P^T by m16n8k16 products, keys or value columns as the 16 rows, so that a group of up to eight rows costs one
// instruction.  A thread loads 16 bytes of a key: eight consecutive values where the fragment wants four pairs eight apart.  A product over d
// does not depend on its order, so Q is loaded in the same order; value fragments are 8 x 8 blocks transposed in registers, which
// permutes the columns of O^T in the same known way.  No shared memory is filled, and a tile's loads are under way while the one before
// is multiplied.  P is rounded to bf16 for its product (by 2^-8 relative at most, as the outputs are; l sums it unrounded).
// fp32: a thread holds a quarter of a key's dimensions and adds in plain arithmetic; four rows, whose sums fit in registers up to d = 64 (d = 96
// spills 96 bytes a thread, d = 128 444).
//
// What bounds bf16 is the memory: 64 sequences x 32 heads (8 of keys) of up to 8192 keys, d = 128, 248 .. 260 us on several cards, 5.4 .. 5.2 TB/s; eight
// times as many CTAs as SMs, as lengths are uneven (four and sixteen times: no better).  One sequence of 1000 keys takes 8 us, latency from end to end.
// fp32: latency and instructions, at 1.7 warps a scheduler (issue slots 20 % busy), and more than four rows read the keys again.
#include <cooperative_groups.h>

#include "softmax.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int MAX_CLUSTER = 8;
constexpr int BF16_ROWS = 16, F32_ROWS = 4;

struct few_shape {
    int32_t rows, row_blocks, splits;       // rows = group * Nq; block x: split x % splits of unit x / splits
    float* part;                            // [unit][split][ROWS][DP + 2]: sums, then maximum and total; NULL: joined in the cluster
};

__device__ __forceinline__ uint4 load16(const void* p)
{
    uint4 v;
    asm("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// both halves: 0 in the place of an infinity or NaN
__device__ __forceinline__ uint32_t only_finite(uint32_t x, bool& found)
{
    uint32_t keep = 0xffffffffu;
    if ((x & 0x7f80u) == 0x7f80u) keep &= 0xffff0000u;
    if ((x & 0x7f800000u) == 0x7f800000u) keep &= 0x0000ffffu;
    found |= keep != 0xffffffffu;
    return x & keep;
}

__device__ __forceinline__ float unless_finite(float x) { return fabsf(x) <= 3.4028235e38f ? 0.0f : x; }

// A row of the block: head and query, what it sees.
struct few_row {
    int32_t h, i, pos, doc;
    bool in;
    __device__ __forceinline__ void set(const grf_softmax_params& p, const grf_sight& sight, const int32_t* qdoc, int32_t kvh, int32_t r, int32_t rows)
    {
        in = r < rows;
        h = kvh * p.group + (in ? r / p.Nq : 0);
        i = in ? r % p.Nq : 0;
        pos = sight.position(i);
        doc = qdoc && in ? qdoc[i] : -1;
    }
    __device__ __forceinline__ bool sees(const grf_sight& sight, const int32_t* kdoc, int32_t j) const
    {
        return in && sight.sees(pos, j) && (!kdoc || (doc >= 0 && kdoc[j] == doc));
    }
};

__device__ __forceinline__ float capped2(const grf_softmax_params& p, float x)
{
    return p.cap > 0.0f ? p.cap * GRF_LOG2E * tanhf(x * (p.scale / p.cap)) : x * (p.scale * GRF_LOG2E);
}

template <int ROWS, int DP> struct FewShared {
    float o[WARPS][ROWS][DP], m[WARPS][ROWS], l[WARPS][ROWS];
    float co[ROWS][DP], cm[ROWS], cl[ROWS];
};

template <typename T>
__device__ __forceinline__ void store_out(const grf_softmax_params& p, int32_t b, int32_t kvh, int32_t r, int c, float o, float m, float l)
{
    const int32_t h = kvh * p.group + r / p.Nq, i = r % p.Nq;
    if (c < p.d) {
        const float x = l == 0.0f ? 0.0f : o / l;
        const T y = grf_from_float<T>(x);
        (reinterpret_cast<T*>(p.out_w) + b * p.os[0] + h * p.os[1] + (int64_t)i * p.os[2])[c] = y;
        if (p.rest_w) p.rest_w[(((int64_t)b * p.H + h) * p.Nq + i) * p.d + c] = grf_rest(x, y);
    }
    if (c == 0 && p.lse_w) p.lse_w[((int64_t)b * p.H + h) * p.Nq + i] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * GRF_LN2;
}

// Weight of a part with maximum m beside the maximum top of all parts (a part without a key weighs nothing).
__device__ __forceinline__ float weight(float m, float top) { return m == -CUDART_INF_F ? 0.0f : exp2f(m - top); }

// The warps' results joined, then the CTAs'.
template <typename T, int ROWS, int DP>
__device__ __forceinline__ void join(FewShared<ROWS, DP>& sh, const grf_softmax_params& p, const few_shape& f, int32_t b, int32_t kvh, int32_t r0)
{
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * DP; x += THREADS) {
        const int r = x / DP, c = x % DP;
        float top = -CUDART_INF_F;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) top = fmaxf(top, sh.m[w][r]);
        float o = 0.0f, l = 0.0f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            // (a row of NaN scores has NaN sums beside a maximum that is not NaN)
            const float a = weight(sh.m[w][r], top);
            const bool empty = sh.m[w][r] == -CUDART_INF_F && sh.l[w][r] == 0.0f;
            o += empty ? 0.0f : a * sh.o[w][r][c] + (sh.l[w][r] != sh.l[w][r] ? CUDART_NAN_F : 0.0f);
            l += empty ? 0.0f : a * sh.l[w][r] + (sh.l[w][r] != sh.l[w][r] ? CUDART_NAN_F : 0.0f);
        }
        sh.co[r][c] = o;
        if (c == 0) { sh.cm[r] = top; sh.cl[r] = l; }
    }
    if (f.part) {
        __syncthreads();
        float* at = f.part + (int64_t)blockIdx.x * (ROWS * (DP + 2));
        for (int x = threadIdx.x; x < ROWS * DP; x += THREADS) at[x] = (&sh.co[0][0])[x];
        for (int x = threadIdx.x; x < ROWS; x += THREADS) { at[ROWS * DP + x] = sh.cm[x]; at[ROWS * DP + ROWS + x] = sh.cl[x]; }
        return;
    }
    if (f.splits == 1) {
        __syncthreads();
        for (int x = threadIdx.x; x < ROWS * DP; x += THREADS)
            if (r0 + x / DP < f.rows) store_out<T>(p, b, kvh, r0 + x / DP, x % DP, sh.co[x / DP][x % DP], sh.cm[x / DP], sh.cl[x / DP]);
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    cluster.sync();
    const int S = f.splits;
    for (int x = (int)cluster.block_rank() * THREADS + threadIdx.x; x < ROWS * DP; x += S * THREADS) {
        const int r = x / DP, c = x % DP;
        if (r0 + r >= f.rows) continue;
        float top = -CUDART_INF_F, o = 0.0f, l = 0.0f, m[MAX_CLUSTER], part_l[MAX_CLUSTER], part_o[MAX_CLUSTER];
#pragma unroll
        for (int s = 0; s < MAX_CLUSTER; ++s) {
            m[s] = -CUDART_INF_F;
            part_l[s] = part_o[s] = 0.0f;
            if (s < S) {
                m[s] = *cluster.map_shared_rank(&sh.cm[r], s);
                part_l[s] = *cluster.map_shared_rank(&sh.cl[r], s);
                part_o[s] = *cluster.map_shared_rank(&sh.co[r][c], s);
            }
            top = fmaxf(top, m[s]);
        }
#pragma unroll
        for (int s = 0; s < MAX_CLUSTER; ++s) {
            const float a = weight(m[s], top), bad = part_l[s] != part_l[s] ? CUDART_NAN_F : 0.0f;
            o += a * part_o[s] + bad;
            l += a * part_l[s] + bad;
        }
        store_out<T>(p, b, kvh, r0 + r, c, o, top, l);
    }
    cluster.sync();                                             // nobody's shared memory goes while it is read
}

template <int DG, int NB>
__global__ void __launch_bounds__(THREADS) softmax_few_bf16_kernel(const __grid_constant__ grf_softmax_params p, const few_shape f)
{
    constexpr int DP = 32 * DG, ROWS = 8 * NB;
    extern __shared__ __align__(16) unsigned char smem[];
    FewShared<ROWS, DP>& sh = *reinterpret_cast<FewShared<ROWS, DP>*>(smem);
    __shared__ grf_buckets bucket;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int32_t unit = blockIdx.x / f.splits, split = blockIdx.x % f.splits, b = unit / (p.KV * f.row_blocks), kvh = unit / f.row_blocks % p.KV, r0 = unit % f.row_blocks * ROWS;
    const grf_sight sight(p, b);
    const int32_t *qdoc = sight.docs ? p.q_doc + (int64_t)b * p.Nq : nullptr, *kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    const __nv_bfloat16* K = reinterpret_cast<const __nv_bfloat16*>(p.k) + b * p.ks[0] + kvh * p.ks[1] + 8 * t;
    const __nv_bfloat16* V = reinterpret_cast<const __nv_bfloat16*>(p.v) + b * p.vs[0] + kvh * p.vs[1] + 8 * t;
    const int32_t end = sight.end(p.Nq), tiles = (end + 15) / 16;
    const int32_t t0 = (int32_t)((int64_t)tiles * split / f.splits), t1 = (int32_t)((int64_t)tiles * (split + 1) / f.splits);
    // a tile that all rows see whole: the first row's position decides, as later queries see more
    const int32_t whole = sight.docs ? 0 : sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(sight.position(0) + 1, sight.prefix));

    uint4 kr[2][DG], vr[2][DG];
    auto load = [&](uint4 (&x)[2][DG], const __nv_bfloat16* base, int64_t stride, int32_t tile) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const int32_t j = tile * 16 + 8 * y + g;
#pragma unroll
            for (int c = 0; c < DG; ++c) x[y][c] = tile < t1 && j < end && 32 * c + 8 * t < p.d ? load16(base + (int64_t)j * stride + 32 * c) : make_uint4(0, 0, 0, 0);
        }
    };
    load(kr, K, p.ks[2], t0 + warp);
    load(vr, V, p.vs[2], t0 + warp);
    bucket.fill(p);
    __syncthreads();
    // Q as the right operand: row g of a block of eight, in the order of the keys' dimensions
    uint4 q[NB][DG];
    few_row row[NB][2];
    float m[NB][2], l[NB][2], o[NB][DG][2][4];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int32_t r = r0 + 8 * n + g;
        const bool in = r < f.rows;
        const __nv_bfloat16* Q = reinterpret_cast<const __nv_bfloat16*>(p.q) + b * p.qs[0] + (int64_t)(kvh * p.group + (in ? r / p.Nq : 0)) * p.qs[1] +
                                 (int64_t)(in ? r % p.Nq : 0) * p.qs[2] + 8 * t;
#pragma unroll
        for (int c = 0; c < DG; ++c) q[n][c] = in && 32 * c + 8 * t < p.d ? load16(Q + 32 * c) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            row[n][e].set(p, sight, qdoc, kvh, r0 + 8 * n + 2 * t + e, f.rows);
            m[n][e] = -CUDART_INF_F;
            l[n][e] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < DG; ++c)
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][c][y][e] = 0.0f;
    }
    bool bad = false;
    for (int32_t tile = t0 + warp; tile < t1; tile += WARPS) {
        float s[NB][4];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
#pragma unroll
            for (int c = 0; c < DG; ++c) {
                mma16816(s[n], kr[0][c].x, kr[1][c].x, kr[0][c].y, kr[1][c].y, q[n][c].x, q[n][c].y);
                mma16816(s[n], kr[0][c].z, kr[1][c].z, kr[0][c].w, kr[1][c].w, q[n][c].z, q[n][c].w);
            }
        }
        load(kr, K, p.ks[2], tile + WARPS);
        const bool partial = tile * 16 + 16 > whole;
        uint32_t pw[NB][2];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            // s[n][2 y + e]: key 8 y + g, row 2 t + e
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int32_t j = tile * 16 + 8 * y + g;
                    float x = capped2(p, s[n][2 * y + e]);
                    if (p.bias != GRF_BIAS_NONE) x += grf_bias2<__nv_bfloat16>(p, bucket, row[n][e].h, j - row[n][e].pos);
                    if (partial && !row[n][e].sees(sight, kdoc, j)) x = -CUDART_INF_F;
                    s[n][2 * y + e] = x;
                }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = fmaxf(m[n][e], fmaxf(s[n][e], s[n][2 + e]));
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
                const float base = top == -CUDART_INF_F ? 0.0f : top, alpha = exp2f(m[n][e] - base);
                m[n][e] = top;
                s[n][e] = exp2f(s[n][e] - base);
                s[n][2 + e] = exp2f(s[n][2 + e] - base);
                l[n][e] = l[n][e] * alpha + (s[n][e] + s[n][2 + e]);            // this thread's keys only, joined at the end
                if (__any_sync(0xffffffffu, alpha != 1.0f)) {
#pragma unroll
                    for (int c = 0; c < DG; ++c)
#pragma unroll
                        for (int y = 0; y < 2; ++y) { o[n][c][y][e] *= alpha; o[n][c][y][2 + e] *= alpha; }
                }
            }
            // P^T as the right operand: keys 2 t, 2 t + 1 of row g
            pw[n][0] = transposed(pack_bf16(s[n][0], s[n][1]));
            pw[n][1] = transposed(pack_bf16(s[n][2], s[n][3]));
        }
        if (partial) {
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int c = 0; c < DG; ++c) {
                    vr[y][c].x = only_finite(vr[y][c].x, bad);
                    vr[y][c].y = only_finite(vr[y][c].y, bad);
                    vr[y][c].z = only_finite(vr[y][c].z, bad);
                    vr[y][c].w = only_finite(vr[y][c].w, bad);
                }
        }
#pragma unroll
        for (int c = 0; c < DG; ++c) {
            const uint32_t a0 = transposed(vr[0][c].x), a1 = transposed(vr[0][c].y), a2 = transposed(vr[1][c].x), a3 = transposed(vr[1][c].y);
            const uint32_t b0 = transposed(vr[0][c].z), b1 = transposed(vr[0][c].w), b2 = transposed(vr[1][c].z), b3 = transposed(vr[1][c].w);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                mma16816(o[n][c][0], a0, a1, a2, a3, pw[n][0], pw[n][1]);
                mma16816(o[n][c][1], b0, b1, b2, b3, pw[n][0], pw[n][1]);
            }
        }
        load(vr, V, p.vs[2], tile + WARPS);
    }
    // o[n][c][y][2 z + e]: column 32 c + 8 (g / 2) + 4 y + 2 z + g % 2 of row 8 n + 2 t + e
    if (__any_sync(0xffffffffu, bad)) {
        // values that are not finite, left out of tiles that not every row sees whole, go to the rows that see them
        for (int32_t tile = t0 + warp; tile < t1; tile += WARPS)
            for (int32_t j = tile * 16; j < min(tile * 16 + 16, end); ++j) {
                if (tile * 16 + 16 <= whole) continue;
#pragma unroll
                for (int c = 0; c < DG; ++c)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int col = 32 * c + 8 * (g >> 1) + 2 * x + (g & 1);
                        if (col >= p.d) continue;
                        const float v = __bfloat162float(V[(int64_t)j * p.vs[2] + col - 8 * t]);
                        if (fabsf(v) <= 3.4028235e38f) continue;
#pragma unroll
                        for (int n = 0; n < NB; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (row[n][e].sees(sight, kdoc, j)) o[n][c][x >> 1][2 * (x & 1) + e] += v;
                    }
            }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * t + e;
#pragma unroll
            for (int y = 4; y < 32; y <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], y);
#pragma unroll
            for (int c = 0; c < DG; ++c)
#pragma unroll
                for (int x = 0; x < 4; ++x) sh.o[warp][r][32 * c + 8 * (g >> 1) + 2 * x + (g & 1)] = o[n][c][x >> 1][2 * (x & 1) + e];
            if (g == 0) { sh.m[warp][r] = m[n][e]; sh.l[warp][r] = l[n][e]; }
        }
    join<__nv_bfloat16, ROWS, DP>(sh, p, f, b, kvh, r0);
}

// fp32: thread (g, t) holds dimensions 16 c + 4 t .. + 3 of key g of a tile of eight.  Every g has running maxima and sums of its own, so nothing
// is exchanged but a score's four parts; U tiles at a time, whose chains overlap.
template <int DG, int ROWS>
__global__ void __launch_bounds__(THREADS) softmax_few_f32_kernel(const __grid_constant__ grf_softmax_params p, const few_shape f)
{
    constexpr int DP = 32 * DG, NC = 2 * DG, U = DG <= 2 ? 2 : 1;
    extern __shared__ __align__(16) unsigned char smem[];
    FewShared<ROWS, DP>& sh = *reinterpret_cast<FewShared<ROWS, DP>*>(smem);
    __shared__ grf_buckets bucket;
    __shared__ float4 q[ROWS][DP / 4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int32_t unit = blockIdx.x / f.splits, split = blockIdx.x % f.splits, b = unit / (p.KV * f.row_blocks), kvh = unit / f.row_blocks % p.KV, r0 = unit % f.row_blocks * ROWS;
    const grf_sight sight(p, b);
    const int32_t *qdoc = sight.docs ? p.q_doc + (int64_t)b * p.Nq : nullptr, *kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    const float* K = reinterpret_cast<const float*>(p.k) + b * p.ks[0] + kvh * p.ks[1] + 4 * t;
    const float* V = reinterpret_cast<const float*>(p.v) + b * p.vs[0] + kvh * p.vs[1] + 4 * t;
    const int32_t end = sight.end(p.Nq), tiles = (end + 7) / 8;
    const int32_t t0 = (int32_t)((int64_t)tiles * split / f.splits), t1 = (int32_t)((int64_t)tiles * (split + 1) / f.splits);
    const int32_t whole = sight.docs ? 0 : sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(sight.position(0) + 1, sight.prefix));

    float4 kr[U][NC], vr[U][NC];
    auto load = [&](float4 (&x)[U][NC], const float* base, int64_t stride, int32_t tile) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t j = (tile + u) * 8 + g;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint4 w = tile + u < t1 && j < end && 16 * c + 4 * t < p.d ? load16(base + (int64_t)j * stride + 16 * c) : make_uint4(0, 0, 0, 0);
                x[u][c] = make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w));
            }
        }
    };
    load(kr, K, p.ks[2], t0 + warp * U);
    load(vr, V, p.vs[2], t0 + warp * U);
    bucket.fill(p);
    for (int x = threadIdx.x; x < ROWS * (DP / 4); x += THREADS) {
        const int r = x / (DP / 4), c = x % (DP / 4);
        few_row w;
        w.set(p, sight, qdoc, kvh, r0 + r, f.rows);
        q[r][c] = w.in && 4 * c < p.d ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.q) + b * p.qs[0] + w.h * p.qs[1] + (int64_t)w.i * p.qs[2] + 4 * c)
                                       : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    __syncthreads();
    few_row row[ROWS];
    float m[ROWS], l[ROWS], slope2[ROWS];
    float4 o[ROWS][NC];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        row[r].set(p, sight, qdoc, kvh, r0 + r, f.rows);
        slope2[r] = p.bias == GRF_BIAS_SLOPES ? -grf_slope2(p, row[r].h) : 0.0f;
        m[r] = -CUDART_INF_F;
        l[r] = 0.0f;
#pragma unroll
        for (int c = 0; c < NC; ++c) o[r][c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    bool bad = false;
    auto clean = [&](float& x) {
        if (!(fabsf(x) <= 3.4028235e38f)) { x = 0.0f; bad = true; }
    };
    for (int32_t tile = t0 + warp * U; tile < t1; tile += WARPS * U) {
        float x[U][ROWS];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float a0 = 0.0f, a1 = 0.0f;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const float4 y = q[r][4 * c + t];
                    a0 = fmaf(kr[u][c].x, y.x, fmaf(kr[u][c].y, y.y, a0));
                    a1 = fmaf(kr[u][c].z, y.z, fmaf(kr[u][c].w, y.w, a1));
                }
                x[u][r] = a0 + a1;
            }
        load(kr, K, p.ks[2], tile + WARPS * U);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) x[u][r] += __shfl_xor_sync(0xffffffffu, x[u][r], 1);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) x[u][r] += __shfl_xor_sync(0xffffffffu, x[u][r], 2);
        bool grow = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t j = (tile + u) * 8 + g;
            const bool partial = (tile + u) * 8 + 8 > whole;
            if (partial) {
#pragma unroll
                for (int c = 0; c < NC; ++c) { clean(vr[u][c].x); clean(vr[u][c].y); clean(vr[u][c].z); clean(vr[u][c].w); }
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float y = capped2(p, x[u][r]);
                if (p.bias == GRF_BIAS_SLOPES) y = fmaf(slope2[r], fabsf((float)(j - row[r].pos)), y);
                if (p.bias == GRF_BIAS_BUCKETS) y += grf_bias2<float>(p, bucket, row[r].h, j - row[r].pos);
                if (tile + u >= t1 || (partial && !row[r].sees(sight, kdoc, j))) y = -CUDART_INF_F;
                x[u][r] = y;
                grow |= y > m[r] + 8.0f;
            }
        }
        // a new maximum only where it matters (see the tensor-core kernels), or for the first key
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float top = m[r];
#pragma unroll
                for (int u = 0; u < U; ++u) top = fmaxf(top, x[u][r]);
                const float alpha = m[r] == -CUDART_INF_F ? 0.0f : exp2f(m[r] - top);
                m[r] = top;
                l[r] *= alpha;
#pragma unroll
                for (int c = 0; c < NC; ++c) { o[r][c].x *= alpha; o[r][c].y *= alpha; o[r][c].z *= alpha; o[r][c].w *= alpha; }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float w = exp2f(x[u][r] - (m[r] == -CUDART_INF_F ? 0.0f : m[r]));
                l[r] += w;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    o[r][c].x = fmaf(w, vr[u][c].x, o[r][c].x); o[r][c].y = fmaf(w, vr[u][c].y, o[r][c].y);
                    o[r][c].z = fmaf(w, vr[u][c].z, o[r][c].z); o[r][c].w = fmaf(w, vr[u][c].w, o[r][c].w);
                }
            }
        load(vr, V, p.vs[2], tile + WARPS * U);
    }
    if (__any_sync(0xffffffffu, bad)) {
        for (int32_t tile0 = t0 + warp * U; tile0 < t1; tile0 += WARPS * U)
            for (int32_t tile = tile0; tile < min(tile0 + U, t1); ++tile) {
                const int32_t j = tile * 8 + g;
                if (tile * 8 + 8 <= whole || j >= end) continue;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (16 * c + 4 * t >= p.d) continue;
                    const float* v = V + (int64_t)j * p.vs[2] + 16 * c;
                    const float4 add = make_float4(unless_finite(v[0]), unless_finite(v[1]), unless_finite(v[2]), unless_finite(v[3]));
#pragma unroll
                    for (int r = 0; r < ROWS; ++r)
                        if (row[r].sees(sight, kdoc, j)) { o[r][c].x += add.x; o[r][c].y += add.y; o[r][c].z += add.z; o[r][c].w += add.w; }
                }
            }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        float top = m[r];
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
        // (a lane without a key has zeros, or NaN beside a maximum that is not one)
        const float a = m[r] == -CUDART_INF_F ? 1.0f : exp2f(m[r] - top);
        l[r] *= a;
#pragma unroll
        for (int y = 4; y < 32; y <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], y);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            float v[4] = {o[r][c].x * a, o[r][c].y * a, o[r][c].z * a, o[r][c].w * a};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) v[e] += __shfl_xor_sync(0xffffffffu, v[e], y);
            }
            if (g == 0) *reinterpret_cast<float4*>(&sh.o[warp][r][16 * c + 4 * t]) = make_float4(v[0], v[1], v[2], v[3]);
        }
        if (lane == 0) { sh.m[warp][r] = top; sh.l[warp][r] = l[r]; }
    }
    join<float, ROWS, DP>(sh, p, f, b, kvh, r0);
}

template <typename T, int ROWS, int DP>
__global__ void __launch_bounds__(THREADS) softmax_few_join_kernel(const __grid_constant__ grf_softmax_params p, const few_shape f)
{
    const int32_t unit = blockIdx.x, b = unit / (p.KV * f.row_blocks), kvh = unit / f.row_blocks % p.KV, r0 = unit % f.row_blocks * ROWS;
    const float* at = f.part + (int64_t)unit * f.splits * (ROWS * (DP + 2));
    for (int x = threadIdx.x; x < ROWS * DP; x += THREADS) {
        const int r = x / DP;
        if (r0 + r >= f.rows) continue;
        float top = -CUDART_INF_F, o = 0.0f, l = 0.0f;
        for (int s = 0; s < f.splits; ++s) top = fmaxf(top, at[(int64_t)s * (ROWS * (DP + 2)) + ROWS * DP + r]);
        for (int s = 0; s < f.splits; ++s) {
            const float* part = at + (int64_t)s * (ROWS * (DP + 2));
            const float a = weight(part[ROWS * DP + r], top), pl = part[ROWS * DP + ROWS + r], bad = pl != pl ? CUDART_NAN_F : 0.0f;
            o += a * part[x] + bad;
            l += a * pl + bad;
        }
        store_out<T>(p, b, kvh, r0 + r, x % DP, o, top, l);
    }
}

int row_block(int32_t rows, int dtype)
{
    if (dtype == GRF_DTYPE_BF16) return rows <= 8 ? 8 : BF16_ROWS;
    return rows == 1 ? 1 : rows == 2 ? 2 : F32_ROWS;
}

few_shape shape_of(const grf_ctx* ctx, const grf_softmax_params& p, int dtype)
{
    few_shape f;
    f.rows = p.group * p.Nq;
    f.row_blocks = grf_ceil_div(f.rows, row_block(f.rows, dtype));
    f.part = nullptr;
    // as many CTAs as keep the memory busy, of 128 keys or more; more than a cluster's only where its CTAs would have over 1024
    const int64_t units = (int64_t)p.B * p.KV * f.row_blocks;
    int64_t s = (8 * (int64_t)ctx->sm_count + units - 1) / units;
    const int64_t most = (p.Nk + 127) / 128;
    if (s > most) s = most;
    if (s > MAX_CLUSTER && p.Nk <= MAX_CLUSTER * 1024) s = MAX_CLUSTER;
    f.splits = (int32_t)s;
    return f;
}

size_t part_floats(const few_shape& f, const grf_softmax_params& p, int dtype)
{
    if (f.splits <= MAX_CLUSTER) return 0;
    const int dp = (p.d + 31) / 32 * 32;
    return (size_t)p.B * p.KV * f.row_blocks * f.splits * row_block(f.rows, dtype) * (dp + 2);
}

template <typename T, int ROWS, int DP, typename Kernel>
int launch(grf_ctx* ctx, Kernel kernel, const grf_softmax_params& p, const few_shape& f)
{
    const size_t smem = sizeof(FewShared<ROWS, DP>);
    if (smem > 32 * 1024) GRF_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    const unsigned units = (unsigned)(p.B * p.KV * f.row_blocks);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(units * f.splits);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = f.part ? 1 : (unsigned)f.splits;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    grf_softmax_scope scope(ctx, "grf:softmax_few", f.part ? 2 : 1);
    GRF_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p, f));
    if (f.part) softmax_few_join_kernel<T, ROWS, DP><<<units, THREADS, 0, ctx->stream>>>(p, f);
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}

template <int DG> int launch_dim(grf_ctx* ctx, const grf_softmax_params& p, const few_shape& f, int dtype)
{
    constexpr int DP = 32 * DG;
    const int rows = row_block(f.rows, dtype);
    if (dtype == GRF_DTYPE_BF16)
        return rows == 8 ? launch<__nv_bfloat16, 8, DP>(ctx, softmax_few_bf16_kernel<DG, 1>, p, f)
                         : launch<__nv_bfloat16, 16, DP>(ctx, softmax_few_bf16_kernel<DG, 2>, p, f);
    return rows == 1 ? launch<float, 1, DP>(ctx, softmax_few_f32_kernel<DG, 1>, p, f)
         : rows == 2 ? launch<float, 2, DP>(ctx, softmax_few_f32_kernel<DG, 2>, p, f)
                     : launch<float, F32_ROWS, DP>(ctx, softmax_few_f32_kernel<DG, F32_ROWS>, p, f);
}

}  // namespace

size_t grf_softmax_few_workspace(const grf_ctx* ctx, const grf_softmax_params& p, int dtype)
{
    return part_floats(shape_of(ctx, p, dtype), p, dtype) * sizeof(float);
}

int grf_softmax_few(grf_ctx* ctx, const grf_softmax_params& p, int dtype, void* workspace)
{
    few_shape f = shape_of(ctx, p, dtype);
    if (part_floats(f, p, dtype) > 0) f.part = (float*)workspace;
    if (p.d <= 32) return launch_dim<1>(ctx, p, f, dtype);
    if (p.d <= 64) return launch_dim<2>(ctx, p, f, dtype);
    if (p.d <= 96) return launch_dim<3>(ctx, p, f, dtype);
    return launch_dim<4>(ctx, p, f, dtype);
}
