// Softmax attention over ordered tokens: entry points, checks of arguments, and the small kernels around the attention itself.
#include <cmath>
#include <cstring>

#include <nvtx3/nvToolsExt.h>

#include "packed.cuh"
#include "softmax.cuh"

grf_softmax_scope::grf_softmax_scope(grf_ctx* ctx, const char* name, int launches)
{
    nvtxRangePushA(name);
    ctx->launches += launches;
}
grf_softmax_scope::~grf_softmax_scope() { nvtxRangePop(); }

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
size_t elem(int dtype) { return dtype == GRF_DTYPE_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// A warp per block of `block` tokens: the smallest and largest document (INT32_MAX, -1 where there is none), and whether a token has none.
__global__ void __launch_bounds__(128) document_ranges_kernel(const int32_t* __restrict__ doc, int4* __restrict__ range, int32_t tokens, int32_t block, int32_t blocks,
                                                              int64_t count)
{
    const int64_t x = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (x >= count) return;
    const int32_t lane = threadIdx.x & 31;
    const int64_t b = x / blocks;
    const int32_t from = (int32_t)(x % blocks) * block, to = min(from + block, tokens);
    int32_t lo = INT32_MAX, hi = -1, none = 0;
    for (int32_t i = from + lane; i < to; i += 32) {
        const int32_t y = doc[b * tokens + i];
        if (y < 0) none = 1;
        else { lo = min(lo, y); hi = max(hi, y); }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    none = __reduce_max_sync(0xffffffffu, none);
    if (lane == 0) range[x] = make_int4(lo, hi, none, 0);
}

// D_i = dout_i . (out_i + rest_i): LANES lanes a row, 16 bytes each.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) output_products_kernel(const __grid_constant__ grf_softmax_params p, float* __restrict__ dsum)
{
    constexpr int CH = 16 / (int)sizeof(T);
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES, rows = (int64_t)p.B * p.H * p.Nq;
    const int c = threadIdx.x % LANES * CH;
    float sum = 0.0f;
    if (row < rows && c < p.d) {
        const int32_t i = (int32_t)(row % p.Nq), h = (int32_t)(row / p.Nq % p.H), b = (int32_t)(row / p.Nq / p.H);
        const uint4 x = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.out) + b * p.os[0] + h * p.os[1] + i * p.os[2] + c);
        const uint4 y = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.dout) + b * p.dos[0] + h * p.dos[1] + i * p.dos[2] + c);
        const T *u = reinterpret_cast<const T*>(&x), *v = reinterpret_cast<const T*>(&y);
#pragma unroll
        for (int e = 0; e < CH; ++e) sum = fmaf(grf_to_float(u[e]), grf_to_float(v[e]), sum);
        if (p.rest) {
            const uint4 z = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.rest) + row * p.d + c);
            const T* w = reinterpret_cast<const T*>(&z);
#pragma unroll
            for (int e = 0; e < CH; ++e) sum = fmaf(grf_to_float(w[e]), grf_to_float(v[e]), sum);
        }
    }
#pragma unroll
    for (int y = 1; y < LANES; y <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
    if (row < rows && threadIdx.x % LANES == 0) dsum[row] = sum;
}

// dst[h][y] = sum over outer and x of part[outer][h][x][y], in a fixed order.
template <typename T>
__global__ void __launch_bounds__(256) bucket_sums_kernel(const float* __restrict__ part, T* __restrict__ dst, int32_t outer, int32_t heads, int32_t count, int32_t columns)
{
    __shared__ float sums[8];
    const int32_t y = blockIdx.x, h = blockIdx.y;
    const int64_t all = (int64_t)outer * count;
    float sum = 0.0f;
    for (int64_t x = threadIdx.x; x < all; x += 256) sum += part[((x / count * heads + h) * count + x % count) * columns + y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) sum += sums[w];
        dst[(int64_t)h * columns + y] = grf_from_float<T>(sum);
    }
}

int first_ok(int32_t n, const int32_t* first)
{
    if (n < 1 || n > GRF_MAX_BUCKETS || !first || first[0] != 0) return GRF_ERR_INVALID;
    for (int32_t y = 1; y < n; ++y)
        if (first[y] <= first[y - 1]) return GRF_ERR_INVALID;
    return first[n - 1] <= (1 << 29) ? GRF_OK : GRF_ERR_INVALID;   // relative positions are kept within +-2^30
}

// Strides of one array (a triple of zeros: contiguous), checked; zero where the extent is 1, so that it is never used.
int strides(int64_t (&to)[3], const int64_t (&from)[3], int32_t batch, int32_t heads, int32_t tokens, int32_t dim, size_t e, bool written)
{
    const int64_t extent[3] = {batch, heads, tokens};
    if (from[0] == 0 && from[1] == 0 && from[2] == 0) {
        to[2] = dim; to[1] = (int64_t)tokens * dim; to[0] = to[1] * heads;
    } else {
        for (int x = 0; x < 3; ++x) {
            to[x] = 0;
            if (extent[x] == 1) continue;
            if (from[x] < 0 || from[x] * (int64_t)e % 16 != 0 || from[x] > ((int64_t)1 << 36)) return GRF_ERR_INVALID;
            to[x] = from[x];
        }
        if (written) {
            // no two places alike: sorted by stride, each stride passes the extent of what is inside it
            int order[3] = {0, 1, 2};
            for (int x = 0; x < 3; ++x)
                for (int y = x + 1; y < 3; ++y)
                    if (to[order[y]] < to[order[x]]) { const int z = order[x]; order[x] = order[y]; order[y] = z; }
            int64_t inside = dim;
            for (int x = 0; x < 3; ++x) {
                if (extent[order[x]] == 1) continue;
                if (to[order[x]] < inside) return GRF_ERR_INVALID;
                inside = to[order[x]] * (extent[order[x]] - 1) + inside;
            }
        }
    }
    for (int x = 0; x < 3; ++x)
        if (extent[x] == 1) to[x] = 0;
    return GRF_OK;
}

int read_desc(grf_softmax_params* p, const grf_softmax_desc* s, bool backward)
{
    if (s->batch <= 0 || s->heads <= 0 || s->kv_heads <= 0 || s->n_q <= 0 || s->n_k <= 0 || s->heads % s->kv_heads != 0) return GRF_ERR_INVALID;
    if (s->dim < 8 || s->dim > 128 || s->dim % 8 != 0 || (s->dtype != GRF_DTYPE_F32 && s->dtype != GRF_DTYPE_BF16)) return GRF_ERR_INVALID;
    if (!std::isfinite(s->scale * GRF_LOG2E) || !std::isfinite(s->cap * GRF_LOG2E) || s->cap < 0.0f) return GRF_ERR_INVALID;
    if (s->cap > 0.0f && !std::isfinite(s->scale / s->cap)) return GRF_ERR_INVALID;         // (0 times these would be NaN)
    if (s->order < GRF_ORDER_FULL || s->order > GRF_ORDER_PREFIX || s->bias < GRF_BIAS_NONE || s->bias > GRF_BIAS_BUCKETS) return GRF_ERR_INVALID;
    if ((s->order == GRF_ORDER_PREFIX) != (s->prefix != nullptr) || (s->q_doc != nullptr) != (s->k_doc != nullptr)) return GRF_ERR_INVALID;
    if ((s->bias == GRF_BIAS_SLOPES) != (s->slopes != nullptr) || (s->bias == GRF_BIAS_BUCKETS) != (s->table != nullptr)) return GRF_ERR_INVALID;
    if (s->bias == GRF_BIAS_BUCKETS && ((s->two_sided & ~1) != 0 || first_ok(s->n_buckets, s->first) != GRF_OK)) return GRF_ERR_INVALID;
    const size_t e = elem(s->dtype);
    memset(p, 0, sizeof *p);
    GRF_TRY(strides(p->qs, s->q_stride, s->batch, s->heads, s->n_q, s->dim, e, false));
    GRF_TRY(strides(p->ks, s->k_stride, s->batch, s->kv_heads, s->n_k, s->dim, e, false));
    GRF_TRY(strides(p->vs, s->v_stride, s->batch, s->kv_heads, s->n_k, s->dim, e, false));
    GRF_TRY(strides(p->os, s->out_stride, s->batch, s->heads, s->n_q, s->dim, e, true));
    if (backward) {
        GRF_TRY(strides(p->dos, s->dout_stride, s->batch, s->heads, s->n_q, s->dim, e, false));
        GRF_TRY(strides(p->dqs, s->dq_stride, s->batch, s->heads, s->n_q, s->dim, e, true));
        GRF_TRY(strides(p->dks, s->dk_stride, s->batch, s->kv_heads, s->n_k, s->dim, e, true));
        GRF_TRY(strides(p->dvs, s->dv_stride, s->batch, s->kv_heads, s->n_k, s->dim, e, true));
    }
    if (s->n_q > GRF_MAX_TOKENS || s->n_k > GRF_MAX_TOKENS || (int64_t)s->batch * s->heads > 65535) return GRF_ERR_TOO_LARGE;
    p->B = s->batch; p->H = s->heads; p->KV = s->kv_heads; p->group = s->heads / s->kv_heads;
    p->Nq = s->n_q; p->Nk = s->n_k; p->d = s->dim;
    p->scale = s->scale; p->cap = s->cap; p->order = s->order; p->bias = s->bias;
    if (s->bias == GRF_BIAS_BUCKETS) {
        p->n_first = s->n_buckets; p->two_sided = s->two_sided;
        memcpy(p->first, s->first, sizeof(int32_t) * s->n_buckets);
    }
    p->slopes = s->slopes; p->table = s->table; p->k_len = s->k_len; p->q_start = s->q_start; p->prefix = s->prefix;
    p->q_doc = s->q_doc; p->k_doc = s->k_doc;
    return GRF_OK;
}

// (bf16's few-query kernel multiplies on the tensor cores)
bool by_few(const grf_ctx* ctx, const grf_softmax_params& p, int dtype) { return p.Nq <= GRF_FEW_QUERIES && (dtype == GRF_DTYPE_F32 || ctx->use_tensor_cores); }

// Places inside the workspace.
struct room {
    size_t bytes = 0;
    size_t take(size_t n) { const size_t at = bytes; bytes += align256(n); return at; }
};

constexpr int RANGE_BLOCK = 64;         // the smallest block that a route takes: sizes of the workspace

struct doc_room {
    size_t q = 0, k = 0;
    doc_room(room& r, const grf_softmax_params& p)
    {
        if (!p.q_doc) return;
        q = r.take(sizeof(int4) * (size_t)p.B * grf_ceil_div(p.Nq, RANGE_BLOCK));
        k = r.take(sizeof(int4) * (size_t)p.B * grf_ceil_div(p.Nk, RANGE_BLOCK));
    }
    int fill(grf_ctx* ctx, grf_softmax_params& p, char* ws, int32_t block) const
    {
        if (!p.q_doc) return GRF_OK;
        const int32_t q_blocks = grf_ceil_div(p.Nq, block), k_blocks = grf_ceil_div(p.Nk, block);
        p.q_range = (const int4*)(ws + q);
        p.k_range = (const int4*)(ws + k);
        const bool same = p.q_doc == p.k_doc && p.Nq == p.Nk;
        if (same) p.k_range = p.q_range;
        grf_softmax_scope scope(ctx, "grf:document_ranges", same ? 1 : 2);
        const int64_t nq = (int64_t)p.B * q_blocks, nk = (int64_t)p.B * k_blocks;
        document_ranges_kernel<<<grf_ceil_div(nq, 4), 128, 0, ctx->stream>>>(p.q_doc, (int4*)(ws + q), p.Nq, block, q_blocks, nq);
        if (!same) document_ranges_kernel<<<grf_ceil_div(nk, 4), 128, 0, ctx->stream>>>(p.k_doc, (int4*)(ws + k), p.Nk, block, k_blocks, nk);
        return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
    }
};

size_t forward_bytes(const grf_ctx* ctx, const grf_softmax_params& p, int dtype)
{
    if (by_few(ctx, p, dtype)) return grf_softmax_few_workspace(ctx, p, dtype);
    room r;
    doc_room docs(r, p);
    return r.bytes;
}

struct backward_room : room {
    doc_room docs;
    size_t dsum, table;
    explicit backward_room(const grf_softmax_params& p) : docs(*this, p)
    {
        dsum = take(sizeof(float) * (size_t)p.B * p.H * p.Nq);
        table = take(p.bias == GRF_BIAS_BUCKETS ? sizeof(float) * (size_t)p.B * p.H * grf_ceil_div(p.Nq, RANGE_BLOCK) * grf_softmax_columns(p) : 0);
    }
};

template <typename T, int LANES> void output_products(grf_ctx* ctx, const grf_softmax_params& p, float* dsum)
{
    const int64_t threads = (int64_t)p.B * p.H * p.Nq * LANES;
    output_products_kernel<T, LANES><<<grf_ceil_div(threads, 256), 256, 0, ctx->stream>>>(p, dsum);
}

}  // namespace

extern "C" int grf_relative_buckets(int32_t n_buckets, int32_t max_distance, int32_t* first)
{
    if (!first || n_buckets < 2 || n_buckets > GRF_MAX_BUCKETS) return GRF_ERR_INVALID;
    const int32_t h = n_buckets / 2, L = n_buckets - h;
    if (max_distance <= h || max_distance > (1 << 24)) return GRF_ERR_INVALID;
    for (int32_t y = 0; y < h; ++y) first[y] = y;
    // n^L against max_distance^y h^(L - y): numbers of up to 24 * 32 bits, in 32-bit digits
    constexpr int DIGITS = 26;
    auto power = [](uint32_t (&x)[DIGITS], uint32_t base, int32_t times) {
        for (int32_t t = 0; t < times; ++t) {
            uint64_t carry = 0;
            for (int i = 0; i < DIGITS; ++i) { carry += (uint64_t)x[i] * base; x[i] = (uint32_t)carry; carry >>= 32; }
        }
    };
    for (int32_t y = 0; y < L; ++y) {
        uint32_t want[DIGITS] = {1};
        power(want, (uint32_t)max_distance, y);
        power(want, (uint32_t)h, L - y);
        int32_t lo = h, hi = max_distance;                      // the smallest n with n^L >= want lies in lo .. hi
        while (lo < hi) {
            const int32_t mid = lo + (hi - lo) / 2;
            uint32_t have[DIGITS] = {1};
            power(have, (uint32_t)mid, L);
            int c = 0;
            for (int i = DIGITS - 1; i >= 0 && c == 0; --i) c = have[i] < want[i] ? -1 : have[i] > want[i] ? 1 : 0;
            if (c >= 0) hi = mid;
            else lo = mid + 1;
        }
        first[h + y] = lo > first[h + y - 1] ? lo : first[h + y - 1] + 1;
    }
    return GRF_OK;
}

extern "C" size_t grf_softmax_attn_workspace_bytes(const grf_ctx* ctx, const grf_softmax_desc* desc, int backward)
{
    grf_softmax_params p;
    if (!ctx || !desc) return 0;
    if (read_desc(&p, desc, backward != 0) != GRF_OK) return 0;
    return backward ? backward_room(p).bytes : forward_bytes(ctx, p, desc->dtype);
}

extern "C" int grf_softmax_attn(grf_ctx* ctx, const grf_softmax_desc* desc, const void* Q, const void* K, const void* V, void* out, float* lse,
                                void* rest, void* workspace, size_t workspace_bytes)
{
    if (!ctx || !desc || !Q || !K || !V || !out) return GRF_ERR_INVALID;
    grf_softmax_params p;
    GRF_TRY(read_desc(&p, desc, false));
    if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(out, 16) || !aligned(rest, 16) || !aligned(workspace, 256)) return GRF_ERR_INVALID;
    if (rest && desc->dtype != GRF_DTYPE_BF16) return GRF_ERR_INVALID;
    const size_t need = forward_bytes(ctx, p, desc->dtype);
    if (need > 0 && !workspace) return GRF_ERR_INVALID;
    if (need > workspace_bytes) return GRF_ERR_WORKSPACE;
    GRF_CUDA_TRY(cudaSetDevice(ctx->device));
    p.q = Q; p.k = K; p.v = V; p.out_w = out; p.lse_w = lse; p.rest_w = (__nv_bfloat16*)rest;
    p.error_word = ctx->error_word;
    if (by_few(ctx, p, desc->dtype)) return grf_softmax_few(ctx, p, desc->dtype, workspace);
    room r;
    const doc_room docs(r, p);
    if (desc->dtype == GRF_DTYPE_BF16 && ctx->use_tensor_cores) {
        GRF_TRY(docs.fill(ctx, p, (char*)workspace, 128));
        const int rc = grf_softmax_tc_forward(ctx, p);
        if (rc <= 0) return rc;
    }
    GRF_TRY(docs.fill(ctx, p, (char*)workspace, 64));
    return grf_softmax_alu_forward(ctx, p, desc->dtype);
}

extern "C" int grf_softmax_attn_backward(grf_ctx* ctx, const grf_softmax_desc* desc, const void* Q, const void* K, const void* V, const void* out,
                                         const float* lse, const void* rest, const void* dout, void* dQ, void* dK, void* dV, void* dtable, void* workspace,
                                         size_t workspace_bytes)
{
    if (!ctx || !desc || !Q || !K || !V || !out || !lse || !dout || !dQ || !dK || !dV) return GRF_ERR_INVALID;
    grf_softmax_params p;
    GRF_TRY(read_desc(&p, desc, true));
    if (dtable && p.bias != GRF_BIAS_BUCKETS) return GRF_ERR_INVALID;
    if (rest && desc->dtype != GRF_DTYPE_BF16) return GRF_ERR_INVALID;
    for (const void* x : {Q, K, V, out, rest, dout, (const void*)dQ, (const void*)dK, (const void*)dV})
        if (!aligned(x, 16)) return GRF_ERR_INVALID;
    if (!workspace || !aligned(workspace, 256)) return GRF_ERR_INVALID;
    const backward_room r(p);
    if (r.bytes > workspace_bytes) return GRF_ERR_WORKSPACE;
    GRF_CUDA_TRY(cudaSetDevice(ctx->device));
    char* ws = (char*)workspace;
    p.q = Q; p.k = K; p.v = V; p.out = out; p.rest = rest; p.lse = lse; p.dout = dout; p.dq = dQ; p.dk = dK; p.dv = dV;
    p.dsum = (const float*)(ws + r.dsum);
    p.dtable_part = dtable ? (float*)(ws + r.table) : nullptr;
    p.error_word = ctx->error_word;
    {
        grf_softmax_scope scope(ctx, "grf:output_products");
        const int lanes = (int)(p.d * elem(desc->dtype) / 16);
        float* dsum = (float*)(ws + r.dsum);
        if (desc->dtype == GRF_DTYPE_F32) {
            if (lanes <= 8) output_products<float, 8>(ctx, p, dsum);
            else if (lanes <= 16) output_products<float, 16>(ctx, p, dsum);
            else output_products<float, 32>(ctx, p, dsum);
        } else {
            if (lanes <= 4) output_products<__nv_bfloat16, 4>(ctx, p, dsum);
            else if (lanes <= 8) output_products<__nv_bfloat16, 8>(ctx, p, dsum);
            else output_products<__nv_bfloat16, 16>(ctx, p, dsum);
        }
    }
    int rc = 1, block = 128;
    if (desc->dtype == GRF_DTYPE_BF16 && ctx->use_tensor_cores) {
        GRF_TRY(r.docs.fill(ctx, p, ws, block));
        rc = grf_softmax_tc_backward(ctx, p);
    }
    if (rc > 0) {
        block = 64;
        GRF_TRY(r.docs.fill(ctx, p, ws, block));
        rc = grf_softmax_alu_backward(ctx, p, desc->dtype);
    }
    GRF_TRY(rc);
    if (dtable) {
        const int32_t q_blocks = grf_ceil_div(p.Nq, block);
        grf_softmax_scope scope(ctx, "grf:bucket_sums");
        const dim3 grid(grf_softmax_columns(p), p.H);
        if (desc->dtype == GRF_DTYPE_F32) bucket_sums_kernel<float><<<grid, 256, 0, ctx->stream>>>(p.dtable_part, (float*)dtable, p.B, p.H, q_blocks, grf_softmax_columns(p));
        else bucket_sums_kernel<__nv_bfloat16><<<grid, 256, 0, ctx->stream>>>(p.dtable_part, (__nv_bfloat16*)dtable, p.B, p.H, q_blocks, grf_softmax_columns(p));
    }
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}

// ------------------------------------------------------------------------------------------------ the bias by itself
//
// Both directions are bound by the matrix's bytes.  A warp takes a row at a time: beyond the distance F at which the last bucket starts there is
// one value to either side, so only the places within F of the diagonal take a look-up (in shared memory, or a search where F >= BIAS_NEAR),
// and the others are written, or added up, 16 bytes at a time.
namespace {

constexpr int BIAS_NEAR = 2048, BIAS_THREADS = 256;

struct bias_shape {
    int32_t heads, n_q, n_k, start, n_first, two_sided, near;   // near: whether distances are looked up
    int32_t strips;
    int32_t first[GRF_MAX_BUCKETS];
    __host__ __device__ int32_t columns() const { return n_first * (1 + two_sided); }
};

// column of the table for a relative position (|delta| < 2^31: starts are kept within +-2^30)
__device__ __forceinline__ int32_t column_of(const bias_shape& s, int32_t delta)
{
    const int32_t n = s.two_sided ? abs(delta) : max(-delta, 0);
    int lo = 0, hi = s.n_first;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.first[mid] <= n) lo = mid;
        else hi = mid;
    }
    return s.two_sided && delta > 0 ? lo + s.n_first : lo;
}
// columns of the distances -F .. F, if they are looked up
__device__ __forceinline__ void load_near(const bias_shape& s, int32_t F, unsigned char* near)
{
    if (s.near)
        for (int x = threadIdx.x; x <= 2 * F; x += BIAS_THREADS) near[x] = (unsigned char)column_of(s, x - F);
}
__device__ __forceinline__ int32_t column_at(const bias_shape& s, int32_t F, const unsigned char* near, int32_t delta)
{
    return s.near ? near[min(max(delta + F, 0), 2 * F)] : column_of(s, delta);
}
// A row's three stretches: [0, left) lies beyond F before the diagonal, [right, n_k) beyond it behind.
struct bias_row {
    int32_t left, right, delta0;            // delta0: relative position of the row's first place
    __device__ __forceinline__ bias_row(const bias_shape& s, int32_t F, int32_t i)
    {
        delta0 = -s.start - i;
        left = min(max(1 - F - delta0, 0), s.n_k);
        right = min(max((s.two_sided ? max(F, 1) : 0) - delta0, left), s.n_k);
    }
};
// A stretch from .. to - 1 of a row of T as whole 16-byte pieces and what lies before the first and behind the last border.
template <typename T> struct stretch {
    static constexpr int CH = 16 / (int)sizeof(T);
    int32_t from, to, first, count, last;
    __device__ __forceinline__ stretch(const T* row, int32_t from_, int32_t to_) : from(from_), to(max(from_, to_))
    {
        const int32_t ahead = (int32_t)((0u - (uint32_t)(uintptr_t)(row + from) / (uint32_t)sizeof(T)) & (uint32_t)(CH - 1));
        first = min(from + ahead, to);
        count = (to - first) / CH;
        last = first + count * CH;
    }
    // the place beside the pieces that this lane has, or -1 (fewer than 16 before, and behind)
    __device__ __forceinline__ int32_t beside(int lane) const
    {
        return lane < 16 ? (lane < first - from ? from + lane : -1) : (lane - 16 < to - last ? last + lane - 16 : -1);
    }
};

template <typename T>
__global__ void __launch_bounds__(BIAS_THREADS) relative_rows_kernel(const __grid_constant__ bias_shape s, const T* __restrict__ table, T* __restrict__ rows)
{
    constexpr int CH = 16 / (int)sizeof(T);
    __shared__ unsigned char near[2 * BIAS_NEAR];
    __shared__ T value[2 * GRF_MAX_BUCKETS];
    const int32_t h = blockIdx.y, F = s.first[s.n_first - 1], lane = threadIdx.x & 31;
    load_near(s, F, near);
    for (int x = threadIdx.x; x < s.columns(); x += BIAS_THREADS) value[x] = table[(int64_t)h * s.columns() + x];
    __syncthreads();
    const T outer[2] = {value[s.n_first - 1], value[s.two_sided ? 2 * s.n_first - 1 : 0]};
    uint4 whole[2];
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        T v[CH];
#pragma unroll
        for (int e = 0; e < CH; ++e) v[e] = outer[y];
        memcpy(&whole[y], v, 16);
    }
    for (int32_t i = blockIdx.x * (BIAS_THREADS / 32) + (threadIdx.x >> 5); i < s.n_q; i += s.strips * (BIAS_THREADS / 32)) {
        T* row = rows + ((int64_t)h * s.n_q + i) * s.n_k;
        const bias_row r(s, F, i);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            const stretch<T> w(row, y ? r.right : 0, y ? s.n_k : r.left);
            if (w.beside(lane) >= 0) row[w.beside(lane)] = outer[y];
            for (int32_t x = lane; x < w.count; x += 32) *reinterpret_cast<uint4*>(row + w.first + x * CH) = whole[y];
        }
        for (int32_t j = r.left + lane; j < r.right; j += 32) row[j] = value[column_at(s, F, near, r.delta0 + j)];
    }
}

// Every lane of a warp meets the same relative positions in every row: 1 - F + 32 y + lane, y < NEAR.  Their sums are registers; only where the band is
// wider (F > 16 NEAR) are the others added into bins that every thread has for itself in shared memory.
constexpr int NEAR = 8;

template <typename T>
__global__ void __launch_bounds__(BIAS_THREADS) relative_sums_kernel(const __grid_constant__ bias_shape s, int32_t batch, const T* __restrict__ drows, float* __restrict__ part)
{
    constexpr int CH = 16 / (int)sizeof(T), FAR_AHEAD = 2, WARPS = BIAS_THREADS / 32;
    extern __shared__ float bins[];                             // [column][thread], where the band is wide
    __shared__ unsigned char near[2 * BIAS_NEAR];
    __shared__ float diagonals[WARPS][32 * NEAR], outer[WARPS][2];
    const int32_t h = blockIdx.y, columns = s.columns(), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, F = s.first[s.n_first - 1];
    const bool wide = F > 16 * NEAR;
    load_near(s, F, near);
    if (wide)
        for (int x = tid; x < columns * BIAS_THREADS; x += BIAS_THREADS) bins[x] = 0.0f;
    __syncthreads();
    float band[NEAR];
#pragma unroll
    for (int y = 0; y < NEAR; ++y) band[y] = 0.0f;
    uint64_t far[2] = {0ull, 0ull};                             // two sums each
    auto add_piece = [&](uint64_t& sum, const uint4& u) {
        if constexpr (sizeof(T) == 2) {
            sum = add2(sum, pack2(u.x << 16, u.x & 0xffff0000u));
            sum = add2(sum, pack2(u.y << 16, u.y & 0xffff0000u));
            sum = add2(sum, pack2(u.z << 16, u.z & 0xffff0000u));
            sum = add2(sum, pack2(u.w << 16, u.w & 0xffff0000u));
        } else {
            sum = add2(sum, pack2(u.x, u.y));
            sum = add2(sum, pack2(u.z, u.w));
        }
    };
    const int32_t step = s.strips * WARPS;
    int32_t b = 0, i = blockIdx.x * WARPS + warp;
    for (;; i += step) {
        while (i >= s.n_q && b < batch) { i -= s.n_q; ++b; }
        if (b >= batch) break;
        const T* row = drows + (((int64_t)b * s.heads + h) * s.n_q + i) * s.n_k;
        const bias_row r(s, F, i);
        const stretch<T> side[2] = {stretch<T>(row, 0, r.left), stretch<T>(row, r.right, s.n_k)};
        // everything of the row that fits is under way before the first of it is used
        uint4 w[2][FAR_AHEAD];
        T v[NEAR], e[2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const uint4* at = reinterpret_cast<const uint4*>(row + side[z].first);
#pragma unroll
            for (int y = 0; y < FAR_AHEAD; ++y) w[z][y] = lane + 32 * y < side[z].count ? __ldcs(at + lane + 32 * y) : make_uint4(0, 0, 0, 0);
            const int32_t beside = side[z].beside(lane);
            e[z] = beside >= 0 ? row[beside] : grf_from_float<T>(0.0f);
        }
        const int32_t j0 = 1 - F - r.delta0 + lane;             // may lie before the row
#pragma unroll
        for (int y = 0; y < NEAR; ++y) v[y] = j0 + 32 * y >= r.left && j0 + 32 * y < r.right ? row[j0 + 32 * y] : grf_from_float<T>(0.0f);
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            const uint4* at = reinterpret_cast<const uint4*>(row + side[z].first);
#pragma unroll
            for (int y = 0; y < FAR_AHEAD; ++y) add_piece(far[z], w[z][y]);
            for (int32_t y = lane + 32 * FAR_AHEAD; y < side[z].count; y += 32) add_piece(far[z], __ldcs(at + y));
            far[z] = add2(far[z], pack2(grf_to_float(e[z]), 0.0f));
        }
#pragma unroll
        for (int y = 0; y < NEAR; ++y) band[y] += grf_to_float(v[y]);
        if (wide)
            for (int32_t j = max(j0 - lane + 32 * NEAR, r.left) + lane; j < r.right; j += 32)
                bins[column_at(s, F, near, r.delta0 + j) * BIAS_THREADS + tid] += grf_to_float(row[j]);
    }
#pragma unroll
    for (int y = 0; y < NEAR; ++y) diagonals[warp][32 * y + lane] = band[y];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        float x0, x1;
        unpack2(far[z], x0, x1);
        x0 += x1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) x0 += __shfl_xor_sync(0xffffffffu, x0, o);
        if (lane == 0) outer[warp][z] = x0;
    }
    __syncthreads();
    // one sum per diagonal, then per column, in order
    float sum = 0.0f;
#pragma unroll
    for (int x = 0; x < WARPS; ++x) sum += diagonals[x][tid];
    __syncthreads();
    diagonals[0][tid] = sum;
    __syncthreads();
    for (int y = warp; y < columns; y += WARPS) {
        float total = 0.0f;
        for (int x = lane; x < 32 * NEAR; x += 32)
            if (x < 2 * F - 1 && column_at(s, F, near, 1 - F + x) == y) total += diagonals[0][x];
        if (wide)
            for (int x = lane; x < BIAS_THREADS; x += 32) total += bins[y * BIAS_THREADS + x];
        if (lane < WARPS) total += (y == s.n_first - 1 ? outer[lane][0] : 0.0f) + (y == (s.two_sided ? 2 * s.n_first - 1 : 0) ? outer[lane][1] : 0.0f);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        if (lane == 0) part[((int64_t)h * s.strips + blockIdx.x) * columns + y] = total;
    }
}

int read_bias(bias_shape* s, int32_t heads, int32_t n_q, int32_t n_k, int32_t q_start, int32_t n_buckets, int two_sided, const int32_t* first, int dtype)
{
    if (heads <= 0 || n_q <= 0 || n_k <= 0 || (two_sided & ~1) != 0 || (dtype != GRF_DTYPE_F32 && dtype != GRF_DTYPE_BF16)) return GRF_ERR_INVALID;
    GRF_TRY(first_ok(n_buckets, first));
    if (n_q > GRF_MAX_TOKENS || n_k > GRF_MAX_TOKENS || heads > 65535) return GRF_ERR_TOO_LARGE;
    memset(s, 0, sizeof *s);
    s->heads = heads; s->n_q = n_q; s->n_k = n_k;
    s->start = q_start < -(1 << 30) ? -(1 << 30) : q_start > (1 << 30) ? 1 << 30 : q_start;      // (no bucket starts beyond 2^29)
    s->n_first = n_buckets; s->two_sided = two_sided;
    memcpy(s->first, first, sizeof(int32_t) * n_buckets);
    s->near = first[n_buckets - 1] < BIAS_NEAR;
    return GRF_OK;
}

// CTAs of one head: enough to fill the device, of eight rows or more
int32_t bias_strips(int32_t heads, int32_t n_q, int32_t most)
{
    const int32_t by_size = (n_q + 7) / 8, by_heads = most > heads ? most / heads : 1;     // (no more than are resident at once)
    return by_size < by_heads ? by_size : by_heads;
}

constexpr int32_t ROW_CTAS = 1184, SUM_CTAS = 592;

template <typename T> int bias_rows(grf_ctx* ctx, const bias_shape& s, const void* table, void* rows)
{
    grf_softmax_scope scope(ctx, "grf:relative_rows");
    relative_rows_kernel<T><<<dim3(s.strips, s.heads), BIAS_THREADS, 0, ctx->stream>>>(s, (const T*)table, (T*)rows);
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}
template <typename T> int bias_sums(grf_ctx* ctx, const bias_shape& s, int32_t batch, const void* drows, void* dtable, float* part)
{
    const size_t smem = s.first[s.n_first - 1] > 16 * NEAR ? sizeof(float) * (size_t)s.columns() * BIAS_THREADS : 0;
    // (the most of any call: the attribute is the whole process's, and another thread may set it between here and the launch)
    if (smem > 0) GRF_CUDA_TRY(cudaFuncSetAttribute(relative_sums_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(float) * 2 * GRF_MAX_BUCKETS * BIAS_THREADS));
    grf_softmax_scope scope(ctx, "grf:relative_sums", 2);
    relative_sums_kernel<T><<<dim3(s.strips, s.heads), BIAS_THREADS, smem, ctx->stream>>>(s, batch, (const T*)drows, part);
    bucket_sums_kernel<T><<<dim3(s.columns(), s.heads), 256, 0, ctx->stream>>>(part, (T*)dtable, 1, s.heads, s.strips, s.columns());
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}

}  // namespace

extern "C" int grf_relative_bias(grf_ctx* ctx, int32_t heads, int32_t n_q, int32_t n_k, int32_t q_start, int32_t n_buckets, int two_sided,
                                 const int32_t* first, int dtype, const void* table, void* rows)
{
    if (!ctx || !table || !rows || !aligned(rows, 16)) return GRF_ERR_INVALID;
    bias_shape s;
    GRF_TRY(read_bias(&s, heads, n_q, n_k, q_start, n_buckets, two_sided, first, dtype));
    s.strips = bias_strips(heads, n_q, ROW_CTAS);
    GRF_CUDA_TRY(cudaSetDevice(ctx->device));
    return dtype == GRF_DTYPE_F32 ? bias_rows<float>(ctx, s, table, rows) : bias_rows<__nv_bfloat16>(ctx, s, table, rows);
}

extern "C" size_t grf_relative_bias_workspace_bytes(int32_t heads, int32_t n_q, int32_t n_k, int32_t n_buckets, int two_sided)
{
    if (heads <= 0 || n_q <= 0 || n_k <= 0 || n_buckets < 1 || n_buckets > GRF_MAX_BUCKETS || (two_sided & ~1) != 0) return 0;
    return align256(sizeof(float) * (size_t)heads * bias_strips(heads, n_q, SUM_CTAS) * n_buckets * (1 + two_sided));
}

extern "C" int grf_relative_bias_backward(grf_ctx* ctx, int32_t batch, int32_t heads, int32_t n_q, int32_t n_k, int32_t q_start,
                                          int32_t n_buckets, int two_sided, const int32_t* first, int dtype, const void* drows, void* dtable,
                                          void* workspace, size_t workspace_bytes)
{
    if (!ctx || batch <= 0 || !drows || !dtable || !aligned(drows, 16)) return GRF_ERR_INVALID;
    bias_shape s;
    GRF_TRY(read_bias(&s, heads, n_q, n_k, q_start, n_buckets, two_sided, first, dtype));
    if (!workspace || !aligned(workspace, 256)) return GRF_ERR_INVALID;
    if (workspace_bytes < grf_relative_bias_workspace_bytes(heads, n_q, n_k, n_buckets, two_sided)) return GRF_ERR_WORKSPACE;
    s.strips = bias_strips(heads, n_q, SUM_CTAS);
    GRF_CUDA_TRY(cudaSetDevice(ctx->device));
    return dtype == GRF_DTYPE_F32 ? bias_sums<float>(ctx, s, batch, drows, dtable, (float*)workspace)
                                  : bias_sums<__nv_bfloat16>(ctx, s, batch, drows, dtable, (float*)workspace);
}
