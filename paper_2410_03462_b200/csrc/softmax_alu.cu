// Softmax attention over ordered tokens and its gradients in plain fp32 arithmetic: what serves fp32, and bf16 when the context keeps off
// the tensor cores.
//
// Forward: a CTA has 64 queries of one head and goes over the keys in tiles of 64 with the running maximum and sum of each row
// (s in units of log 2): m' = max(m, max s), l' = l 2^(m - m') + sum 2^(s - m'), O' = O 2^(m - m') + P V, out = O / l.
// Backward, in two kernels so that nothing is added atomically: a CTA of 64 queries recomputes P = 2^(s - lse) and dS = P (dP - D) tile by
// tile for dQ (and the sums of dS along the tile's diagonals for the bias table); a CTA of 64 keys does the same over the queries of
// all heads that share it for dK and dV.
//
// 256 threads hold 4 x 4 scores each; operands lie in shared memory as rows with four words of padding, read 16 bytes at a time: two reads
// for sixteen multiply-adds.  What bounds it is latency: two CTAs of eight warps fit an SM (d <= 64, where the next tile's loads wait in registers as
// well) and issue in 31 % of the cycles (forward, d = 32; 26 % with d = 64, gradients 21 %), waiting at a tile's barriers (1.7 .. 4.0 cycles per instruction),
// for shared memory (1.6 .. 1.9) and for memory (0.8 .. 2.9): about 12 TFLOP/s of visible work on 3 x 5 heads x 1003.  Products run over 32, 64 or 128
// dimensions, so others pay for the next of these.
#include <cooperative_groups.h>

#include "packed.cuh"
#include "softmax.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int BT = 64;                  // queries, and keys, of a tile
constexpr int THREADS = 256;
constexpr int PS = BT + 4;              // row of a score tile

// Tiles of a block's other side are dealt out to the CTAs of a cluster, which add what they have through distributed shared memory: one CTA per block
// leaves too few warps per SM on all but the largest calls, and with causal order the longest block decides.  (us, one CTA a block
// / clusters: training, 2 x 4 heads x 1531, causal with documents 484 / 347, forward 3 x 5 heads x 1003 with a prefix 112 / 94.)
struct alu_split { int32_t splits; };

template <int DP> struct Alu {
    static constexpr int ROW = DP + 4;
    static constexpr int TILE = BT * ROW;
    static constexpr int W = DP / 16 < 4 ? DP / 16 : 4;        // neighbouring output columns of a thread
    static constexpr int NC = DP / 16 / W;                      // and groups of them, 16 W apart
};

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.4028235e38f; }

// A chunk of a row as floats.  clean: what is not finite becomes 0, and *some (or NULL) 1; true if there was any.
template <typename T> __device__ __forceinline__ bool to_floats(float (&v)[16 / sizeof(T)], const uint4& w, bool clean, int* some)
{
    const T* t = reinterpret_cast<const T*>(&w);
    bool found = false;
#pragma unroll
    for (int e = 0; e < 16 / (int)sizeof(T); ++e) {
        v[e] = grf_to_float(t[e]);
        if (clean && !finite(v[e])) {
            v[e] = 0.0f;
            found = true;
            if (some) *some = 1;
        }
    }
    return found;
}
// bad[r]: whether any lane of row r has found something (PER lanes a row, all of the warp here)
template <int PER> __device__ __forceinline__ void mark_row(int* bad, int r, bool found)
{
    const uint32_t who = __ballot_sync(0xffffffffu, found), lane = threadIdx.x & 31u;
    if (lane % PER == 0) bad[r] = (who >> lane & (0xffffffffu >> (32 - PER))) != 0u;
}

// Rows r0 .. r0 + 63 of [tokens][d] as floats: zeros behind `rows`, behind d, and for tokens whose document is negative.  clean: what is not
// finite becomes 0 too; true if this thread has found any, bad (or NULL) says in which rows there is some, *some (or NULL) becomes 1 then.
template <typename T, int DP>
__device__ __forceinline__ bool load_rows(float* tile, const T* base, int64_t stride, int32_t r0, int32_t rows, int32_t d, const int32_t* doc,
                                          bool clean, int* bad, int* some = nullptr)
{
    constexpr int CH = 16 / (int)sizeof(T), PER = DP / CH;
    static_assert(BT * PER % THREADS == 0 && 32 % PER == 0, "rows are whole warps' business");
    bool any = false;
    for (int x = threadIdx.x; x < BT * PER; x += THREADS) {
        const int r = x / PER, c = x % PER * CH;
        float v[CH];
        bool found = false;
#pragma unroll
        for (int e = 0; e < CH; ++e) v[e] = 0.0f;
        if (r0 + r < rows && c < d && (!doc || doc[r0 + r] >= 0)) {
            found = to_floats<T>(v, *reinterpret_cast<const uint4*>(base + (int64_t)(r0 + r) * stride + c), clean, some);
        }
        if (bad) mark_row<PER>(bad, r, found);
        any |= found;
#pragma unroll
        for (int e = 0; e < CH; e += 4) *reinterpret_cast<float4*>(tile + r * Alu<DP>::ROW + c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
    return any;
}

// The same in two steps, so that a tile's loads are under way while the one before is computed (d <= 64: they fit in registers).
template <typename T, int DP> struct rows_ahead {
    static constexpr int CH = 16 / (int)sizeof(T), PER = DP / CH, N = BT * PER / THREADS;
    static_assert(BT * PER % THREADS == 0, "no thread is left out");
    uint4 w[N];
    __device__ __forceinline__ void fetch(const T* base, int64_t stride, int32_t r0, int32_t rows, int32_t d, const int32_t* doc)
    {
#pragma unroll
        for (int y = 0; y < N; ++y) {
            const int x = threadIdx.x + y * THREADS, r = x / PER, c = x % PER * CH;
            w[y] = r0 + r < rows && c < d && (!doc || doc[r0 + r] >= 0) ? *reinterpret_cast<const uint4*>(base + (int64_t)(r0 + r) * stride + c)
                                                                                          : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ bool store(float* tile, bool clean, int* bad, int* some = nullptr) const
    {
        bool any = false;
#pragma unroll
        for (int y = 0; y < N; ++y) {
            const int x = threadIdx.x + y * THREADS, r = x / PER, c = x % PER * CH;
            float v[CH];
            const bool found = to_floats<T>(v, w[y], clean, some);
            if (bad) mark_row<PER>(bad, r, found);
            any |= found;
#pragma unroll
            for (int e = 0; e < CH; e += 4) *reinterpret_cast<float4*>(tile + r * Alu<DP>::ROW + c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        }
        return any;
    }
};

// acc[r][c] = sum over d of a[4 ty + r][.] b[tx + 16 c][.], even and odd d by themselves: packed multiply-adds on values as they are read
template <int DP>
__device__ __forceinline__ void products(float (&acc)[4][4], const float* a, const float* b, int ty, int tx)
{
    constexpr int ROW = Alu<DP>::ROW;
    uint64_t sum[4][4];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[r][c] = 0ull;
#pragma unroll 4
    for (int k = 0; k < DP; k += 4) {
        ulonglong2 x[4], y[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = *reinterpret_cast<const ulonglong2*>(a + (4 * ty + r) * ROW + k);
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = *reinterpret_cast<const ulonglong2*>(b + (tx + 16 * c) * ROW + k);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[r][c] = fma2(x[r].y, y[c].y, fma2(x[r].x, y[c].x, sum[r][c]));
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float lo, hi;
            unpack2(sum[r][c], lo, hi);
            acc[r][c] = lo + hi;
        }
}

template <int W> __device__ __forceinline__ void load_w(float (&v)[W], const float* at)
{
    if constexpr (W == 4) {
        const float4 x = *reinterpret_cast<const float4*>(at);
        v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else {
        const float2 x = *reinterpret_cast<const float2*>(at);
        v[0] = x.x; v[1] = x.y;
    }
}

// acc[r][.] += sum over x of w[x][4 ty + r] rows[x][this thread's columns]
template <int DP>
__device__ __forceinline__ void accumulate(float (&acc)[4][DP / 16], const float* w, const float* rows, int ty, int tx)
{
    using A = Alu<DP>;
    uint64_t sum[4][DP / 32];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) sum[r][c] = pack2(acc[r][2 * c], acc[r][2 * c + 1]);
#pragma unroll 4
    for (int x = 0; x < BT; ++x) {
        const float4 p = *reinterpret_cast<const float4*>(w + x * PS + 4 * ty);
        const uint64_t pr[4] = {pack2(p.x, p.x), pack2(p.y, p.y), pack2(p.z, p.z), pack2(p.w, p.w)};
#pragma unroll
        for (int g = 0; g < A::NC; ++g) {
            float v[A::W];
            load_w<A::W>(v, rows + x * A::ROW + A::W * tx + 16 * A::W * g);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int e = 0; e < A::W; e += 2) sum[r][(g * A::W + e) / 2] = fma2(pr[r], pack2(v[e], v[e + 1]), sum[r][(g * A::W + e) / 2]);
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < DP / 32; ++c) unpack2(sum[r][c], acc[r][2 * c], acc[r][2 * c + 1]);
}

template <typename T, int DP>
__device__ __forceinline__ void store_row(T* dst, const float (&v)[DP / 16], int tx, int32_t d)
{
    using A = Alu<DP>;
#pragma unroll
    for (int g = 0; g < A::NC; ++g) {
        const int c = A::W * tx + 16 * A::W * g;
        if (c < d) {
#pragma unroll
            for (int e = 0; e < A::W; ++e) dst[c + e] = grf_from_float<T>(v[g * A::W + e]);
        }
    }
}

// Where a row of a head lies; heads of keys and values: h / group.
template <typename T> __device__ __forceinline__ const T* at_head(const void* base, const int64_t (&s)[3], int32_t b, int32_t h)
{
    return reinterpret_cast<const T*>(base) + b * s[0] + h * s[1];
}
template <typename T> __device__ __forceinline__ T* at_head_w(void* base, const int64_t (&s)[3], int32_t b, int32_t h)
{
    return reinterpret_cast<T*>(base) + b * s[0] + h * s[1];
}

__device__ __forceinline__ int4 all_docs() { return make_int4(0, 0, 0, 0); }

// Bias of every diagonal of a tile, index (j - j0) - (i - i0) + BT - 1.
template <typename T> __device__ __forceinline__ void load_bias(float* lut, const grf_softmax_params& p, const grf_buckets& bucket, int32_t h, int32_t j0, int32_t pos0)
{
    if (p.bias == GRF_BIAS_NONE) return;
    for (int x = threadIdx.x; x < 2 * BT - 1; x += THREADS) lut[x] = grf_bias2<T>(p, bucket, h, j0 - pos0 + x - (BT - 1));
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, DP <= 64 ? 2 : 1) softmax_alu_forward_kernel(const __grid_constant__ grf_softmax_params p, const alu_split f)
{
    using A = Alu<DP>;
    extern __shared__ float smem[];
    float *qs = smem, *ks = qs + A::TILE, *vs = ks + A::TILE, *pt = vs + A::TILE;
    __shared__ float lut[2 * BT];
    __shared__ grf_buckets bucket;
    __shared__ int bad;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    bucket.fill(p);
    const int32_t b = blockIdx.y / p.H, h = blockIdx.y % p.H, kvh = h / p.group, qblocks = gridDim.x / f.splits;
    const int32_t i0 = (qblocks - 1 - (int32_t)blockIdx.x / f.splits) * BT, rank = blockIdx.x % f.splits;
    const grf_sight sight(p, b);
    const int32_t *qdoc = sight.docs ? p.q_doc + (int64_t)b * p.Nq : nullptr, *kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    const int32_t kblocks = (p.Nk + BT - 1) / BT, i1 = min(i0 + BT, p.Nq);
    const int4 qr = sight.docs ? p.q_range[(int64_t)b * qblocks + i0 / BT] : all_docs();
    const T *K = at_head<T>(p.k, p.ks, b, kvh), *V = at_head<T>(p.v, p.vs, b, kvh);
    if (tid == 0) bad = 0;
    load_rows<T, DP>(qs, at_head<T>(p.q, p.qs, b, h), p.qs[2], i0, p.Nq, p.d, nullptr, false, nullptr);
    float o[4][DP / 16], m[4], l[4];
    int32_t doc[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        m[r] = -CUDART_INF_F;
        l[r] = 0.0f;
        doc[r] = qdoc && i0 + 4 * ty + r < p.Nq ? qdoc[i0 + 4 * ty + r] : -1;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) o[r][c] = 0.0f;
    }
    const float to2 = p.scale * GRF_LOG2E, cap2 = p.cap * GRF_LOG2E, by_cap = p.cap > 0.0f ? p.scale / p.cap : 0.0f;
    const int32_t end = sight.end(i1);
    constexpr bool AHEAD = DP <= 64;
    rows_ahead<T, AHEAD ? DP : 32> ka, va;
    auto what_of = [&](int32_t j) { return sight.tile(i0, i1, j, j + BT, qr, sight.docs ? __ldg(p.k_range + (int64_t)b * kblocks + j / BT) : all_docs()); };
    auto seen_from = [&](int32_t j) {
        while (j < end && what_of(j) == 0) j += f.splits * BT;
        return j;
    };
    auto fetch = [&](int32_t j) {
        if constexpr (AHEAD)
            if (j < end) {
                ka.fetch(K, p.ks[2], j, sight.len, p.d, kdoc);
                va.fetch(V, p.vs[2], j, sight.len, p.d, kdoc);
            }
    };
    int32_t j_next = seen_from(rank * BT);
    fetch(j_next);
    for (int32_t j0 = j_next; j0 < end; j0 = j_next) {
        const int what = what_of(j0);
        j_next = seen_from(j0 + f.splits * BT);
        __syncthreads();
        if constexpr (AHEAD) {
            ka.store(ks, false, nullptr);
            va.store(vs, what == 1, nullptr, &bad);
            fetch(j_next);
        } else {
            load_rows<T, DP>(ks, K, p.ks[2], j0, sight.len, p.d, kdoc, false, nullptr);
            load_rows<T, DP>(vs, V, p.vs[2], j0, sight.len, p.d, kdoc, what == 1, nullptr, &bad);
        }
        load_bias<T>(lut, p, bucket, h, j0, sight.position(i0));
        __syncthreads();
        float s[4][4];
        products<DP>(s, qs, ks, ty, tx);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 4 * ty + r;
            float top = m[r];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = tx + 16 * c;
                float x = p.cap > 0.0f ? cap2 * tanhf(s[r][c] * by_cap) : s[r][c] * to2;
                if (p.bias != GRF_BIAS_NONE) x += lut[j - i + BT - 1];
                if (what == 1) {
                    const bool seen = sight.sees(sight.position(i0 + i), j0 + j) && (!kdoc || (doc[r] >= 0 && kdoc[j0 + j] == doc[r]));
                    if (!seen) x = -CUDART_INF_F;
                }
                s[r][c] = x;
                top = fmaxf(top, x);
            }
#pragma unroll
            for (int y = 1; y < 16; y <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, y));
            const float base = top == -CUDART_INF_F ? 0.0f : top, alpha = exp2f(m[r] - base);
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                s[r][c] = exp2f(s[r][c] - base);
                sum += s[r][c];
            }
#pragma unroll
            for (int y = 1; y < 16; y <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
            l[r] = l[r] * alpha + sum;
            m[r] = top;
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) o[r][c] *= alpha;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<float4*>(pt + (tx + 16 * c) * PS + 4 * ty) = make_float4(s[0][c], s[1][c], s[2][c], s[3][c]);
        __syncthreads();
        accumulate<DP>(o, pt, vs, ty, tx);
    }
    __syncthreads();
    // Values that are not finite, in tiles that not every query sees whole, were left out above: they go to the queries that see them.
    if (bad) {
        for (int32_t j = 0; j < end; ++j) {
            const int32_t j0 = j & ~(BT - 1);
            const int what = sight.tile(i0, i1, j0, j0 + BT, qr, sight.docs ? p.k_range[(int64_t)b * kblocks + j0 / BT] : all_docs());
            if (what != 1 || j0 / BT % f.splits != rank) { j = j0 + BT - 1; continue; }
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                const int col = c / A::W * 16 * A::W + A::W * tx + c % A::W;
                if (col >= p.d) continue;
                const float v = grf_to_float(V[(int64_t)j * p.vs[2] + col]);
                if (finite(v)) continue;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (sight.sees(sight.position(i0 + 4 * ty + r), j) && (!kdoc || (doc[r] >= 0 && kdoc[j] == doc[r]))) o[r][c] += v;
            }
        }
    }
    if (f.splits > 1) {
        // maxima, sums and outputs of all parts, in order; every CTA joins a share of the rows
        float *os = ks, *ms = pt, *ls = pt + BT;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            store_row<float, DP>(os + (4 * ty + r) * DP, o[r], tx, DP);
            if (tx == 0) { ms[4 * ty + r] = m[r]; ls[4 * ty + r] = l[r]; }
        }
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        const int r0 = BT * rank / f.splits, r1 = BT * (rank + 1) / f.splits;
        for (int x = tid; x < (r1 - r0) * DP; x += THREADS) {
            const int r = r0 + x / DP, c = x % DP;
            const int32_t i = i0 + r;
            if (i >= p.Nq || c >= p.d) continue;
            float top = -CUDART_INF_F, sum = 0.0f, total = 0.0f;
            for (int y = 0; y < f.splits; ++y) top = fmaxf(top, *cluster.map_shared_rank(ms + r, y));
            for (int y = 0; y < f.splits; ++y) {
                const float my = *cluster.map_shared_rank(ms + r, y), ly = *cluster.map_shared_rank(ls + r, y), oy = *cluster.map_shared_rank(os + r * DP + c, y);
                // (a part without a key weighs nothing; NaN scores leave NaN sums beside a maximum that is not one)
                const float w = my == -CUDART_INF_F ? 0.0f : exp2f(my - top), bad = ly != ly ? CUDART_NAN_F : 0.0f;
                total += w * ly + bad;
                sum += w * oy + bad;
            }
            const float y = total == 0.0f ? 0.0f : sum / total;
            const T z = grf_from_float<T>(y);
            (at_head_w<T>(p.out_w, p.os, b, h) + (int64_t)i * p.os[2])[c] = z;
            const int64_t row = ((int64_t)b * p.H + h) * p.Nq + i;
            if (p.rest_w) p.rest_w[row * p.d + c] = grf_rest(y, z);
            if (p.lse_w && c == 0) p.lse_w[row] = total == 0.0f ? -CUDART_INF_F : (top + log2f(total)) * GRF_LN2;
        }
        cluster.sync();
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int32_t i = i0 + 4 * ty + r;
        if (i >= p.Nq) continue;
        const float inv = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) o[r][c] = l[r] == 0.0f ? 0.0f : o[r][c] * inv;
        store_row<T, DP>(at_head_w<T>(p.out_w, p.os, b, h) + (int64_t)i * p.os[2], o[r], tx, p.d);
        if (p.rest_w) {
#pragma unroll
            for (int c = 0; c < DP / 16; ++c) {
                const int col = c / A::W * 16 * A::W + A::W * tx + c % A::W;
                if (col < p.d) p.rest_w[(((int64_t)b * p.H + h) * p.Nq + i) * p.d + col] = grf_rest(o[r][c], grf_from_float<T>(o[r][c]));
            }
        }
        if (p.lse_w && tx == 0)
            p.lse_w[((int64_t)b * p.H + h) * p.Nq + i] = l[r] == 0.0f ? -CUDART_INF_F : (m[r] + log2f(l[r])) * GRF_LN2;
    }
}

// This CTA's share of a block's rows, [BT][DP] summed over the cluster in order.
template <typename T, int DP>
__device__ __forceinline__ void add_parts(cg::cluster_group& cluster, float* mine, int splits, int rank, T* dst, int64_t stride, int32_t rows, int32_t d, float by)
{
    const int r0 = BT * rank / splits, r1 = BT * (rank + 1) / splits;
    for (int x = threadIdx.x; x < (r1 - r0) * DP; x += THREADS) {
        const int r = r0 + x / DP, c = x % DP;
        if (r >= rows || c >= d) continue;
        float sum = 0.0f;
        for (int y = 0; y < splits; ++y) sum += *cluster.map_shared_rank(mine + r * DP + c, y);
        dst[(int64_t)r * stride + c] = grf_from_float<T>(sum * by);
    }
}

// P and dS of one tile from its products: on entry s = q.k and dp = dout.v; on return s = P, dp = dX (dS through the cap), ds = dS.
struct alu_row { float lse2, dsum; int32_t doc, pos; bool any; };
template <typename T>
__device__ __forceinline__ alu_row load_alu_row(const grf_softmax_params& p, const grf_sight& sight, const int32_t* qdoc, int32_t b, int32_t h, int32_t i)
{
    alu_row w;
    const bool in = i < p.Nq;
    const int64_t x = ((int64_t)b * p.H + h) * p.Nq + i;
    const float lse = in ? p.lse[x] : -CUDART_INF_F;
    w.any = !(fabsf(lse) > 1.0e30f);
    w.lse2 = lse * GRF_LOG2E;
    w.dsum = in ? p.dsum[x] : 0.0f;
    w.doc = qdoc && in ? qdoc[i] : -1;
    w.pos = sight.position(i);
    return w;
}
__device__ __forceinline__ void score_gradient(const grf_softmax_params& p, const grf_sight& sight, const alu_row& w, const int32_t* kdoc, int what,
                                               int32_t j, float bias2, bool spoilt, float& s, float& dp, float& ds)
{
    float t = 0.0f, x;
    if (p.cap > 0.0f) { t = tanhf(s * (p.scale / p.cap)); x = p.cap * GRF_LOG2E * t; }
    else x = s * (p.scale * GRF_LOG2E);
    x += bias2;
    bool seen = w.any;
    if (what == 1) seen = seen && sight.sees(w.pos, j) && (!kdoc || (w.doc >= 0 && kdoc[j] == w.doc));
    s = seen ? exp2f(x - w.lse2) : 0.0f;
    ds = seen ? s * (dp - w.dsum) : 0.0f;
    dp = p.cap > 0.0f ? (seen ? ds * (1.0f - t * t) : 0.0f) : ds;
    // a row of dout that is not finite was left out of the products (0 times it, where it is not seen or has no scores, would be NaN)
    if (seen && !finite(w.dsum)) s = CUDART_NAN_F;
    // and so was a row of q or k that is not: its scores are not those that the row has
    if (seen && spoilt) s = dp = ds = CUDART_NAN_F;
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, DP <= 64 ? 2 : 1) softmax_alu_dq_kernel(const __grid_constant__ grf_softmax_params p, const alu_split f)
{
    using A = Alu<DP>;
    extern __shared__ float smem[];
    float *qs = smem, *gs = qs + A::TILE, *ks = gs + A::TILE, *vs = ks + A::TILE, *xt = vs + A::TILE, *st = xt + BT * PS;
    __shared__ grf_buckets bucket;
    __shared__ int bad_key[BT];
    __shared__ float lut[2 * BT], bins[4][2 * GRF_MAX_BUCKETS];   // sums by bucket, of diagonals 32 w .. 32 w + 31 of each tile
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    bucket.fill(p);
    const int32_t b = blockIdx.y / p.H, h = blockIdx.y % p.H, kvh = h / p.group, qblocks = gridDim.x / f.splits;
    const int32_t i0 = (qblocks - 1 - (int32_t)blockIdx.x / f.splits) * BT, rank = blockIdx.x % f.splits;
    const grf_sight sight(p, b);
    const int32_t *qdoc = sight.docs ? p.q_doc + (int64_t)b * p.Nq : nullptr, *kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    const int32_t kblocks = (p.Nk + BT - 1) / BT, i1 = min(i0 + BT, p.Nq), columns = grf_softmax_columns(p);
    const int4 qr = sight.docs ? p.q_range[(int64_t)b * qblocks + i0 / BT] : all_docs();
    const T *K = at_head<T>(p.k, p.ks, b, kvh), *V = at_head<T>(p.v, p.vs, b, kvh);
    load_rows<T, DP>(qs, at_head<T>(p.q, p.qs, b, h), p.qs[2], i0, p.Nq, p.d, nullptr, false, nullptr);
    load_rows<T, DP>(gs, at_head<T>(p.dout, p.dos, b, h), p.dos[2], i0, p.Nq, p.d, nullptr, false, nullptr);
    alu_row row[4];
    float dq[4][DP / 16];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        row[r] = load_alu_row<T>(p, sight, qdoc, b, h, i0 + 4 * ty + r);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) dq[r][c] = 0.0f;
    }
    for (int x = tid; x < 4 * 2 * GRF_MAX_BUCKETS; x += THREADS) (&bins[0][0])[x] = 0.0f;
    const int32_t end = sight.end(i1);
    constexpr bool AHEAD = DP <= 64;
    rows_ahead<T, AHEAD ? DP : 32> ka, va;
    auto what_of = [&](int32_t j) { return sight.tile(i0, i1, j, j + BT, qr, sight.docs ? __ldg(p.k_range + (int64_t)b * kblocks + j / BT) : all_docs()); };
    auto seen_from = [&](int32_t j) {
        while (j < end && what_of(j) == 0) j += f.splits * BT;
        return j;
    };
    auto fetch = [&](int32_t j) {
        if constexpr (AHEAD)
            if (j < end) {
                ka.fetch(K, p.ks[2], j, sight.len, p.d, kdoc);
                va.fetch(V, p.vs[2], j, sight.len, p.d, kdoc);
            }
    };
    int32_t j_next = seen_from(rank * BT);
    fetch(j_next);
    for (int32_t j0 = j_next; j0 < end; j0 = j_next) {
        const int what = what_of(j0);
        j_next = seen_from(j0 + f.splits * BT);
        bool found;
        __syncthreads();
        if constexpr (AHEAD) {
            found = ka.store(ks, true, bad_key);
            va.store(vs, false, nullptr);
            fetch(j_next);
        } else {
            found = load_rows<T, DP>(ks, K, p.ks[2], j0, sight.len, p.d, kdoc, true, bad_key);
            load_rows<T, DP>(vs, V, p.vs[2], j0, sight.len, p.d, kdoc, false, nullptr);
        }
        load_bias<T>(lut, p, bucket, h, j0, sight.position(i0));
        const bool any_bad = __syncthreads_or(found);
        float s[4][4], dp[4][4];
        products<DP>(s, qs, ks, ty, tx);
        products<DP>(dp, gs, vs, ty, tx);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int i = 4 * ty + r, j = tx + 16 * c;
                float ds;
                score_gradient(p, sight, row[r], kdoc, what, j0 + j, p.bias != GRF_BIAS_NONE ? lut[j - i + BT - 1] : 0.0f, any_bad && bad_key[j], s[r][c], dp[r][c], ds);
                if (p.dtable_part) st[i * PS + j] = ds;
            }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            *reinterpret_cast<float4*>(xt + (tx + 16 * c) * PS + 4 * ty) = make_float4(dp[0][c], dp[1][c], dp[2][c], dp[3][c]);
        __syncthreads();
        accumulate<DP>(dq, xt, ks, ty, tx);
        if (p.dtable_part) {
            if (tid < 2 * BT) {
                float sum = 0.0f;
                const int delta = tid - (BT - 1);               // j - i
                for (int i = max(0, -delta); i < min(BT, BT - delta); ++i) sum += st[i * PS + i + delta];
                grf_add_runs(bins[tid >> 5], tid < 2 * BT - 1 ? bucket(p, j0 - sight.position(i0) + delta) : -1, sum);
            }
        }
    }
    __syncthreads();
    float* part = p.dtable_part ? p.dtable_part + ((int64_t)blockIdx.y * qblocks + i0 / BT) * columns : nullptr;
    if (f.splits > 1) {
#pragma unroll
        for (int r = 0; r < 4; ++r) store_row<float, DP>(ks + (4 * ty + r) * DP, dq[r], tx, DP);
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        if (part && rank == 0 && tid < columns) {
            float sum = 0.0f;
            for (int y = 0; y < f.splits; ++y)
                for (int w = 0; w < 4; ++w) sum += *cluster.map_shared_rank(&bins[w][tid], y);
            part[tid] = sum;
        }
        add_parts<T, DP>(cluster, ks, f.splits, rank, at_head_w<T>(p.dq, p.dqs, b, h) + (int64_t)i0 * p.dqs[2], p.dqs[2], p.Nq - i0, p.d, p.scale);
        cluster.sync();
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int32_t i = i0 + 4 * ty + r;
        if (i >= p.Nq) continue;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) dq[r][c] *= p.scale;
        store_row<T, DP>(at_head_w<T>(p.dq, p.dqs, b, h) + (int64_t)i * p.dqs[2], dq[r], tx, p.d);
    }
    if (part && tid < columns) part[tid] = (bins[0][tid] + bins[1][tid]) + (bins[2][tid] + bins[3][tid]);
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS, DP <= 64 ? 2 : 1) softmax_alu_dkv_kernel(const __grid_constant__ grf_softmax_params p, const alu_split f)
{
    using A = Alu<DP>;
    extern __shared__ float smem[];
    float *qs = smem, *gs = qs + A::TILE, *ks = gs + A::TILE, *vs = ks + A::TILE, *ps = vs + A::TILE, *xs = ps + BT * PS;
    __shared__ int bad_query[BT];
    __shared__ float lut[2 * BT];
    __shared__ grf_buckets bucket;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
    bucket.fill(p);
    const int32_t b = blockIdx.y / p.KV, kvh = blockIdx.y % p.KV, j0 = (int32_t)blockIdx.x / f.splits * BT, j1 = j0 + BT, rank = blockIdx.x % f.splits;
    const grf_sight sight(p, b);
    const int32_t *qdoc = sight.docs ? p.q_doc + (int64_t)b * p.Nq : nullptr, *kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    const int32_t qblocks = (p.Nq + BT - 1) / BT;
    const int4 kr = sight.docs ? p.k_range[(int64_t)b * (gridDim.x / f.splits) + j0 / BT] : all_docs();
    load_rows<T, DP>(ks, at_head<T>(p.k, p.ks, b, kvh), p.ks[2], j0, sight.len, p.d, kdoc, false, nullptr);
    load_rows<T, DP>(vs, at_head<T>(p.v, p.vs, b, kvh), p.vs[2], j0, sight.len, p.d, kdoc, false, nullptr);
    float dk[4][DP / 16], dv[4][DP / 16];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) dk[r][c] = dv[r][c] = 0.0f;
    constexpr bool AHEAD = DP <= 64;
    rows_ahead<T, AHEAD ? DP : 32> qa, ga;
    const int32_t all = p.group * qblocks;
    auto what_of = [&](int32_t x) {
        const int32_t i = x % qblocks * BT;
        return sight.tile(i, min(i + BT, p.Nq), j0, j1, sight.docs ? __ldg(p.q_range + (int64_t)b * qblocks + i / BT) : all_docs(), kr);
    };
    auto seen_from = [&](int32_t x) {
        while (x < all && what_of(x) == 0) x += f.splits;
        return x;
    };
    auto fetch = [&](int32_t x) {
        if constexpr (AHEAD)
            if (x < all) {
                const int32_t h = kvh * p.group + x / qblocks, i = x % qblocks * BT;
                qa.fetch(at_head<T>(p.q, p.qs, b, h), p.qs[2], i, p.Nq, p.d, qdoc);
                ga.fetch(at_head<T>(p.dout, p.dos, b, h), p.dos[2], i, p.Nq, p.d, qdoc);
            }
    };
    int32_t x_next = seen_from(rank);
    fetch(x_next);
    for (int32_t x = x_next; x < all; x = x_next) {
        const int32_t h = kvh * p.group + x / qblocks, i0 = x % qblocks * BT;
        const int what = what_of(x);
        x_next = seen_from(x + f.splits);
        bool found;
        __syncthreads();
        if constexpr (AHEAD) {
            found = qa.store(qs, true, bad_query);
            ga.store(gs, true, nullptr);
            fetch(x_next);
        } else {
            found = load_rows<T, DP>(qs, at_head<T>(p.q, p.qs, b, h), p.qs[2], i0, p.Nq, p.d, qdoc, true, bad_query);
            load_rows<T, DP>(gs, at_head<T>(p.dout, p.dos, b, h), p.dos[2], i0, p.Nq, p.d, qdoc, true, nullptr);
        }
        load_bias<T>(lut, p, bucket, h, j0, sight.position(i0));
        const bool any_bad = __syncthreads_or(found);
        float s[4][4], dp[4][4];
        products<DP>(s, qs, ks, ty, tx);
        products<DP>(dp, gs, vs, ty, tx);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int i = 4 * ty + r;
            const alu_row w = load_alu_row<T>(p, sight, qdoc, b, h, i0 + i);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int j = tx + 16 * c;
                float ds;
                score_gradient(p, sight, w, kdoc, what, j0 + j, p.bias != GRF_BIAS_NONE ? lut[j - i + BT - 1] : 0.0f, any_bad && bad_query[i], s[r][c], dp[r][c], ds);
                ps[i * PS + j] = s[r][c];
                xs[i * PS + j] = dp[r][c];
            }
        }
        __syncthreads();
        accumulate<DP>(dv, ps, gs, ty, tx);
        accumulate<DP>(dk, xs, qs, ty, tx);
    }
    if (f.splits > 1) {
        __syncthreads();
        float *dks = qs, *dvs = ks;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            store_row<float, DP>(dks + (4 * ty + r) * DP, dk[r], tx, DP);
            store_row<float, DP>(dvs + (4 * ty + r) * DP, dv[r], tx, DP);
        }
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        add_parts<T, DP>(cluster, dks, f.splits, rank, at_head_w<T>(p.dk, p.dks, b, kvh) + (int64_t)j0 * p.dks[2], p.dks[2], p.Nk - j0, p.d, p.scale);
        add_parts<T, DP>(cluster, dvs, f.splits, rank, at_head_w<T>(p.dv, p.dvs, b, kvh) + (int64_t)j0 * p.dvs[2], p.dvs[2], p.Nk - j0, p.d, 1.0f);
        cluster.sync();
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int32_t j = j0 + 4 * ty + r;
        if (j >= p.Nk) continue;
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) dk[r][c] *= p.scale;
        store_row<T, DP>(at_head_w<T>(p.dk, p.dks, b, kvh) + (int64_t)j * p.dks[2], dk[r], tx, p.d);
        store_row<T, DP>(at_head_w<T>(p.dv, p.dvs, b, kvh) + (int64_t)j * p.dvs[2], dv[r], tx, p.d);
    }
}

// one CTA per block, or a cluster of up to eight where the blocks fill the device less than four times over and every CTA gets two tiles or more
alu_split split_of(const grf_ctx* ctx, int64_t blocks, int64_t tiles)
{
    alu_split f = {1};
    while (f.splits < 8 && blocks * f.splits < 4 * ctx->sm_count && tiles >= 2 * (f.splits + 1)) ++f.splits;
    return f;
}

template <typename Kernel> int launch(grf_ctx* ctx, Kernel kernel, const grf_softmax_params& p, int32_t blocks, int32_t heads, int64_t tiles, size_t smem)
{
    GRF_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    const alu_split f = split_of(ctx, (int64_t)blocks * heads, tiles);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks * f.splits, heads);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)f.splits;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    GRF_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, p, f));
    return GRF_OK;
}

template <typename T, int DP> int forward(grf_ctx* ctx, const grf_softmax_params& p)
{
    const int32_t qb = grf_ceil_div(p.Nq, BT), kb = grf_ceil_div(p.Nk, BT);
    grf_softmax_scope scope(ctx, "grf:softmax_attention");
    return launch(ctx, softmax_alu_forward_kernel<T, DP>, p, qb, p.B * p.H, kb, sizeof(float) * (3 * Alu<DP>::TILE + BT * PS));
}

template <typename T, int DP> int backward(grf_ctx* ctx, const grf_softmax_params& p)
{
    const int32_t qb = grf_ceil_div(p.Nq, BT), kb = grf_ceil_div(p.Nk, BT);
    const size_t smem = sizeof(float) * (4 * Alu<DP>::TILE + 2 * BT * PS);
    grf_softmax_scope scope(ctx, "grf:softmax_gradients", 2);
    GRF_TRY(launch(ctx, softmax_alu_dq_kernel<T, DP>, p, qb, p.B * p.H, kb, smem));
    return launch(ctx, softmax_alu_dkv_kernel<T, DP>, p, kb, p.B * p.KV, (int64_t)qb * p.group, smem);
}

}  // namespace

int grf_softmax_alu_forward(grf_ctx* ctx, const grf_softmax_params& p, int dtype)
{
    const bool wide = dtype == GRF_DTYPE_F32;
    if (p.d <= 32) return wide ? forward<float, 32>(ctx, p) : forward<__nv_bfloat16, 32>(ctx, p);
    if (p.d <= 64) return wide ? forward<float, 64>(ctx, p) : forward<__nv_bfloat16, 64>(ctx, p);
    return wide ? forward<float, 128>(ctx, p) : forward<__nv_bfloat16, 128>(ctx, p);
}

int grf_softmax_alu_backward(grf_ctx* ctx, const grf_softmax_params& p, int dtype)
{
    const bool wide = dtype == GRF_DTYPE_F32;
    if (p.d <= 32) return wide ? backward<float, 32>(ctx, p) : backward<__nv_bfloat16, 32>(ctx, p);
    if (p.d <= 64) return wide ? backward<float, 64>(ctx, p) : backward<__nv_bfloat16, 64>(ctx, p);
    return wide ? backward<float, 128>(ctx, p) : backward<__nv_bfloat16, 128>(ctx, p);
}
