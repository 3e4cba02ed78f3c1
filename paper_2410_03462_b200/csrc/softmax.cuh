// What the kernels of softmax attention over ordered tokens share: the call's parameters, which tiles a query block sees, the distance bias.
#pragma once

#include <math_constants.h>

#include "grf_internal.cuh"

struct grf_softmax_params {
    int32_t B, H, KV, group, Nq, Nk, d;     // group = H / KV
    float scale, cap;
    int32_t order, bias, n_first, two_sided;
    int32_t first[GRF_MAX_BUCKETS];
    const float* slopes;
    const void* table;
    const int32_t *k_len, *q_start, *prefix, *q_doc, *k_doc;
    const int4 *q_range, *k_range;          // documents of blocks of `range_block` tokens: smallest, largest, whether one is negative
    int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];
    const void *q, *k, *v, *dout;
    const void *out, *rest;                 // read by the backward pass
    void* out_w;
    float* lse_w;
    __nv_bfloat16* rest_w;                  // [B][H][Nq][d]
    const float* lse;
    const float* dsum;                      // D_i of the backward pass, [B][H][Nq]
    void *dq, *dk, *dv;
    float* dtable_part;                     // per (sequence, head, query block): sums by bucket, or NULL
    int* error_word;
};

__host__ __device__ static inline int grf_softmax_columns(const grf_softmax_params& p) { return p.n_first * (1 + p.two_sided); }

// Largest magnitude that a bias keeps once it is in units of log 2 (a type's lowest value, times log2(e), would be -infinity).
#define GRF_BIAS_MOST 3.0e38f
#define GRF_LOG2E 1.4426950408889634f
#define GRF_LN2 0.6931471805599453f

// Buckets of distances, in shared memory: parameters indexed by a thread's own distance are read one address at a time.
struct grf_buckets {
    static constexpr int NEAR = 1024;
    int32_t first[GRF_MAX_BUCKETS];
    unsigned char near[NEAR];               // of distances below NEAR, where the last bucket starts there
    __device__ __forceinline__ int32_t searched(const grf_softmax_params& p, int32_t n) const
    {
        int lo = 0, hi = p.n_first;         // the last y with first[y] <= n
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= n) lo = mid;
            else hi = mid;
        }
        return lo;
    }
    // by the whole block; a barrier of the block follows
    __device__ __forceinline__ void fill(const grf_softmax_params& p)
    {
        if (p.bias != GRF_BIAS_BUCKETS) return;
        for (int x = threadIdx.x; x < p.n_first; x += blockDim.x) first[x] = p.first[x];
        __syncthreads();
        const int32_t far = p.first[p.n_first - 1];
        if (far < NEAR)
            for (int x = threadIdx.x; x <= far; x += blockDim.x) near[x] = (unsigned char)searched(p, x);
    }
    __device__ __forceinline__ int32_t operator()(const grf_softmax_params& p, int32_t delta) const
    {
        const int32_t n = p.two_sided ? abs(delta) : max(-delta, 0), far = p.first[p.n_first - 1];
        const int32_t y = far < NEAR ? near[min(n, far)] : searched(p, n);
        return p.two_sided && delta > 0 ? y + p.n_first : y;
    }
};

__device__ __forceinline__ float grf_to_float(float x) { return x; }
__device__ __forceinline__ float grf_to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T grf_from_float(float x);
template <> __device__ __forceinline__ float grf_from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 grf_from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// What rounding took from an output of storage type T, for rest_w.
template <typename T> __device__ __forceinline__ __nv_bfloat16 grf_rest(float x, T stored)
{
    const float r = x - grf_to_float(stored);
    return __float2bfloat16_rn(r == r ? r : 0.0f);              // (an infinity or NaN has none)
}

// The slope of head h in units of log 2: finite where the slope is (an infinity would make NaN of distance 0).
__device__ __forceinline__ float grf_slope2(const grf_softmax_params& p, int32_t h)
{
    const float a = p.slopes[h], a2 = a * GRF_LOG2E;
    return fabsf(a) <= 3.4028235e38f ? fminf(fmaxf(a2, -3.4028235e38f), 3.4028235e38f) : a2;
}

// The bias of relative position delta for head h, in units of log 2.
template <typename T>
__device__ __forceinline__ float grf_bias2(const grf_softmax_params& p, const grf_buckets& bucket, int32_t h, int32_t delta)
{
    float b;
    if (p.bias == GRF_BIAS_SLOPES) b = -p.slopes[h] * fabsf((float)delta);
    else b = grf_to_float(reinterpret_cast<const T*>(p.table)[(size_t)h * grf_softmax_columns(p) + bucket(p, delta)]);
    // an infinity and NaN stay what they are
    const float b2 = b * GRF_LOG2E;
    return fabsf(b) <= 3.4028235e38f ? fminf(fmaxf(b2, -GRF_BIAS_MOST), GRF_BIAS_MOST) : b2;
}

// bins[b] += v of every lane, by one converged warp and in a fixed order: equal b lie in neighbouring lanes (buckets follow each other along
// diagonals), so a scan within runs leaves a run's sum in its last lane.  b < 0: nothing to add.
__device__ __forceinline__ void grf_add_runs(float* bins, int32_t b, float v)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const float u = __shfl_up_sync(0xffffffffu, v, o);
        const int32_t c = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o && c == b) v += u;
    }
    const int32_t next = __shfl_down_sync(0xffffffffu, b, 1);
    if (b >= 0 && (lane == 31 || next != b)) bins[b] += v;
    __syncwarp();
}

// What a sequence's queries see.
struct grf_sight {
    int32_t start, len, prefix, order;      // prefix: keys before it are seen whatever the order
    bool docs;
    __device__ __forceinline__ grf_sight(const grf_softmax_params& p, int32_t b)
    {
        start = p.q_start ? p.q_start[b] : p.Nk - p.Nq;
        len = p.k_len ? min(max(p.k_len[b], 0), p.Nk) : p.Nk;
        order = p.order;
        prefix = order == GRF_ORDER_PREFIX ? p.prefix[b] : 0;
        docs = p.q_doc != nullptr;
    }
    // position of query i; saturates, so that no start overflows
    __device__ __forceinline__ int32_t position(int32_t i) const
    {
        const int64_t x = (int64_t)start + i;
        return (int32_t)(x < -(1 << 30) ? -(1 << 30) : x > (1 << 30) ? (1 << 30) : x);
    }
    // without documents
    __device__ __forceinline__ bool sees(int32_t pos, int32_t j) const
    {
        return j < len && (order == GRF_ORDER_FULL || j <= pos || j < prefix);
    }
    // one past the last key that queries i0 .. i1 - 1 can see
    __device__ __forceinline__ int32_t end(int32_t i1) const
    {
        if (order == GRF_ORDER_FULL) return len;
        const int32_t e = max(position(i1 - 1) + 1, prefix);
        return max(min(e, len), 0);
    }
    // queries i0 .. i1 - 1 against keys j0 .. j1 - 1: 0 nothing to see, 1 some of it, 2 all of it.  qr, kr: the documents of blocks
    // that hold them (used only with documents)
    __device__ __forceinline__ int tile(int32_t i0, int32_t i1, int32_t j0, int32_t j1, const int4& qr, const int4& kr) const
    {
        if (j0 >= end(i1)) return 0;
        int what = j1 <= len && (order == GRF_ORDER_FULL || j1 - 1 <= position(i0) || j1 <= prefix) ? 2 : 1;
        if (docs) {
            if (qr.x > kr.y || kr.x > qr.y) return 0;
            if (qr.x != qr.y || kr.x != kr.y || (qr.z | kr.z) != 0) what = 1;
        }
        return what;
    }
};

// softmax_alu.cu: plain-ALU kernels, fp32 and bf16 (the latter when the context's tensor cores are off)
int grf_softmax_alu_forward(grf_ctx* ctx, const grf_softmax_params& p, int dtype);
int grf_softmax_alu_backward(grf_ctx* ctx, const grf_softmax_params& p, int dtype);
// softmax_tc.cu, softmax_tc_grad.cu: bf16 on the tensor cores; documents' ranges over blocks of 128.  1 (nothing launched) where no tensor map
// can be made of the operands
int grf_softmax_tc_forward(grf_ctx* ctx, const grf_softmax_params& p);
int grf_softmax_tc_backward(grf_ctx* ctx, const grf_softmax_params& p);
// softmax_few.cu: few queries, keys split over CTAs
#define GRF_FEW_QUERIES 16
size_t grf_softmax_few_workspace(const grf_ctx* ctx, const grf_softmax_params& p, int dtype);
int grf_softmax_few(grf_ctx* ctx, const grf_softmax_params& p, int dtype, void* workspace);
// Counts launches and names them in a profiler's timeline.
struct grf_softmax_scope {
    grf_softmax_scope(grf_ctx* ctx, const char* name, int launches = 1);
    ~grf_softmax_scope();
};
