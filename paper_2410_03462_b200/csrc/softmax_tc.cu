// Softmax attention over ordered tokens on the tensor cores (bf16): the forward pass.
//
// S = Q K^T of 128 queries and 128 keys comes out in tensor memory, a query per lane; a thread reads its query's 128 scores, keeps the
// running maximum m and sum l (in units of log 2), and writes P = 2^(s - m) back to tensor memory as bf16 pairs, where it is the left operand
// of O += P V.  O stays in tensor memory; it is rescaled only when a maximum grows by more than 2^8 (until then P <= 2^8, which costs no
// precision: bf16 has the same relative step everywhere and l is fp32), so almost never after the first tiles.
// A CTA has an SM to itself and works on two groups of 128 queries in turn with the tensor cores.  Two threads share a query, 64 columns
// each (they agree on the maximum through shared memory): with one thread a query, two warps per scheduler, the chain of a tile - load,
// maximum, exponentials, store - bounded the kernel (2 x 16 heads x 4096 causal and capped, d = 128: 272 us, with two 234 at that time, 247 with all that came since; d = 64: 207 and 182).
//   d > 64   P overwrites S
//   d <= 64  P has its own place, so the next S is made while P is
//   warps of the last warpgroup: copies of K and V (boxes by the copy engine), one issuing warp per group, and one that clears rows of V
//   which nobody sees (behind a length, of no document): 0 times an infinity there would reach every query of the tile.
// CTAs take block after block of queries; barriers, tensor memory and the pipeline of copies go on from one to the next.
// A value that some queries see and others do not, and that is not finite, does reach the others' accumulators: a row that ends up not finite
// has its columns summed again from what it does see (redo_row).
#include <type_traits>

#include "softmax_tc.cuh"

namespace {

using namespace grf_softmax_tc;

constexpr int QT = 2;                                           // groups of a CTA

// EXACT: P as the sum of two bf16 values, so that O has fp32 precision and D = dout . O of the backward pass, a difference of nearly equal terms
// where a row looks at few keys, loses nothing (dQ of the capped case: 2.8e-3 from 64 bits without, 2.4e-3 with, of which rounding dX and dQ to bf16 is all).  The second values take the rest of S's place.
template <int DP, bool EXACT> struct Fwd {
    static constexpr bool SEP = DP == 64 && !EXACT;             // P beside S
    static constexpr int NS = DP == 64 ? 3 : 2, QB = DP == 64 ? 2 : 1;     // stages of K and V; places for a group's queries
    static constexpr uint32_t TILE = HALF * (DP / 64);
    static constexpr uint32_t P_COL = SEP ? 256 : 0, P_STEP = SEP ? 64 : BT, O_COL = SEP ? 384 : 256;      // S: BT per group
    static constexpr size_t SMEM = 1024 + (size_t)TILE * (QT * QB + 2 * NS);    // then the tiles' bits
};
constexpr int SOFT = 8 * QT;                                    // warps that make P
constexpr int THREADS = 32 * (SOFT + 4);
constexpr int MORE = 104, LESS = 64;                            // registers: 4 * 104 + 64 = 5 * 96, the launch's

#define FMA_PAIRS(n) ((n) % 8 == 2 || (n) % 8 == 5)             // of a thread's 32 pairs of columns
constexpr int BIAS_NONE_SCALED = 3;     // no bias, scores scaled before anything else, every exponential by its own instruction

// What a block of queries sees.
struct forward_tiles {
    const uint32_t* bits;                                       // with documents: [seen, whole, one document] per group, then seen by any, then tiles with a token of no document
    bool docs;
    int32_t i0, tiles, words;
    int32_t last;                                               // one past the last key that any query of the sequence can see
    int32_t rows[QT], end[QT], whole[QT];                       // per group: whether it has queries, one past the last key seen, keys that all of them see
    __device__ __forceinline__ forward_tiles(const grf_softmax_params& p, const grf_sight& sight, const uint32_t* bits_, int32_t i0_) : bits(bits_), docs(sight.docs), i0(i0_)
    {
        last = sight.end(p.Nq);
        int32_t most = 0;
#pragma unroll
        for (int g = 0; g < QT; ++g) {
            const int32_t i = i0 + g * BT;
            rows[g] = i < p.Nq;
            end[g] = rows[g] ? sight.end(min(i + BT, p.Nq)) : 0;
            whole[g] = sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(sight.position(i) + 1, sight.prefix));
            most = max(most, end[g]);
        }
        tiles = (most + BT - 1) / BT;
        words = (tiles + 31) / 32;
    }
    // (chosen, not indexed: registers)
    static __device__ __forceinline__ int32_t of(const int32_t (&x)[QT], int g) { return g == 0 ? x[0] : x[QT - 1]; }
    // group g and tile t: 0 nothing to see, 1 some of it, 2 all of it
    __device__ __forceinline__ int what(int g, int32_t t) const
    {
        if (docs) return of(rows, g) && bit(bits + 3 * g * words, t) ? (bit(bits + (3 * g + 1) * words, t) ? 2 : 1) : 0;
        return t * BT >= of(end, g) ? 0 : t * BT + BT <= of(whole, g) ? 2 : 1;
    }
    // whether documents have to be compared in a tile
    __device__ __forceinline__ bool mixed(int g, int32_t t) const { return docs && !bit(bits + (3 * g + 2) * words, t); }
    // the first tile from t on that any group sees
    __device__ __forceinline__ int32_t next(int32_t t) const
    {
        if (!docs) return t;
        const uint32_t* any = bits + 3 * QT * words;
        while (t < tiles) {
            const uint32_t w = any[t >> 5] >> (t & 31);
            if (w) return min(t + __ffs(w) - 1, tiles);
            t = (t | 31) + 1;
        }
        return tiles;
    }
    __device__ __forceinline__ bool unclean(const grf_softmax_params& p, int32_t t) const
    {
        return (last < p.Nk && t * BT + BT > last) || (docs && bit(bits + (3 * QT + 1) * words, t));
    }
};

// The outputs of row i from the keys that it sees, where a value that it does not see may have spoilt them: the warp together, lanes take keys for
// the scores and four columns each for the sums.  Only columns that are not finite are replaced, and one whose sum is not finite either
// stays (the row sees such a value itself): with none left the row is done.  EXACT: the weights are not rounded.  steps: counted up now and then.
template <bool CAP, bool EXACT>
__device__ __noinline__ void redo_row(const grf_softmax_params& p, const grf_buckets& bucket, int32_t b, int32_t h, int32_t i, float m, float l, int32_t col0, int32_t col1,
                                      int* steps)
{
    const grf_sight sight(p, b);
    const int lane = threadIdx.x & 31, col = 4 * lane;
    const int32_t kvh = h / p.group, pos = sight.position(i), end = sight.end(i + 1);
    const __nv_bfloat16* Q = reinterpret_cast<const __nv_bfloat16*>(p.q) + b * p.qs[0] + h * p.qs[1] + (int64_t)i * p.qs[2];
    const __nv_bfloat16* K = reinterpret_cast<const __nv_bfloat16*>(p.k) + b * p.ks[0] + kvh * p.ks[1];
    const __nv_bfloat16* V = reinterpret_cast<const __nv_bfloat16*>(p.v) + b * p.vs[0] + kvh * p.vs[1] + col;
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out_w) + b * p.os[0] + h * p.os[1] + (int64_t)i * p.os[2] + col;
    const int32_t doc = sight.docs ? p.q_doc[(int64_t)b * p.Nq + i] : 0;
    const int32_t* kdoc = sight.docs ? p.k_doc + (int64_t)b * p.Nk : nullptr;
    float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    bool want[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) want[x] = col >= col0 && col < min(col1, p.d) && !(fabsf(__bfloat162float(out[x])) <= 3.4028235e38f);
    for (int32_t j0 = 0; j0 < end; j0 += 32) {
        const bool mine = want[0] || want[1] || want[2] || want[3];
        if (!__any_sync(0xffffffffu, mine)) return;
        if ((j0 & 1023) == 0 && lane == 0) atomicAdd(steps, 1);
        const int32_t j = j0 + lane;
        const bool seen = j < end && sight.sees(pos, j) && (!kdoc || (doc >= 0 && kdoc[j] == doc));
        const uint32_t who = __ballot_sync(0xffffffffu, seen);
        float w = 0.0f;
        if (seen) {
            // (loads first, here and below: most of this is their latency)
            for (int c0 = 0; c0 < p.d; c0 += 64) {
                uint4 k8[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) k8[x] = c0 + 8 * x < p.d ? *reinterpret_cast<const uint4*>(K + (int64_t)j * p.ks[2] + c0 + 8 * x) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const uint4 q8 = c0 + 8 * x < p.d ? *reinterpret_cast<const uint4*>(Q + c0 + 8 * x) : make_uint4(0, 0, 0, 0);
                    const uint32_t kw[4] = {k8[x].x, k8[x].y, k8[x].z, k8[x].w}, qw[4] = {q8.x, q8.y, q8.z, q8.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w = fmaf(__uint_as_float(qw[e] & 0xffff0000u), __uint_as_float(kw[e] & 0xffff0000u), fmaf(__uint_as_float(qw[e] << 16), __uint_as_float(kw[e] << 16), w));
                }
            }
            w = CAP ? p.cap * GRF_LOG2E * tanh_any(w * (p.scale / p.cap)) : w * (p.scale * GRF_LOG2E);
            if (p.bias != GRF_BIAS_NONE) w += grf_bias2<__nv_bfloat16>(p, bucket, h, j - pos);
            w = ex2(w - m);
            if (!EXACT) w = __bfloat162float(__float2bfloat16_rn(w));
        }
#pragma unroll 1
        for (int y0 = 0; y0 < 32; y0 += 16) {
            uint2 v[16];
#pragma unroll
            for (int y = 0; y < 16; ++y) v[y] = mine && (who >> (y0 + y) & 1u) ? *reinterpret_cast<const uint2*>(V + (int64_t)(j0 + y0 + y) * p.vs[2]) : make_uint2(0, 0);
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                const float wy = __shfl_sync(0xffffffffu, w, y0 + y);
                o[0] = fmaf(wy, __uint_as_float(v[y].x << 16), o[0]);
                o[1] = fmaf(wy, __uint_as_float(v[y].x & 0xffff0000u), o[1]);
                o[2] = fmaf(wy, __uint_as_float(v[y].y << 16), o[2]);
                o[3] = fmaf(wy, __uint_as_float(v[y].y & 0xffff0000u), o[3]);
            }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) want[x] = want[x] && fabsf(o[x]) <= 3.4028235e38f;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        if (!want[x]) continue;
        const float y = o[x] * inv;
        out[x] = __float2bfloat16_rn(y);
        if (p.rest_w) p.rest_w[(((int64_t)b * p.H + h) * p.Nq + i) * p.d + col + x] = grf_rest(y, __float2bfloat16_rn(y));
    }
}

// A bounded wait whose time starts anew while rows are summed again (a block all of whose rows are takes 6 us a key with
// d = 64, 9.6 with d = 128: 2.5 s with 2^18 keys, where a wait alone gives up after 2): that is a loop over keys, so it ends, and `steps` with it.
__device__ __forceinline__ bool wait_beside(uint32_t bar, uint32_t parity, volatile int* abort_flag, volatile int* steps)
{
    long long t0 = 0;
    int last = 0;
    for (uint32_t it = 0;; ++it) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((it & 63u) == 63u) {
            if (*abort_flag) return false;
            const long long now = clock64();
            const int step = *steps;
            if (t0 == 0 || step != last) { t0 = now; last = step; }
            else if (now - t0 > WAIT_CYCLES) { *abort_flag = 1; return false; }
        }
    }
}

template <int DP, bool CAP, int BIAS, bool EXACT>
__global__ void __launch_bounds__(THREADS, 1)
softmax_tc_forward_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                          const __grid_constant__ CUtensorMap map_v, const __grid_constant__ grf_softmax_params p)
{
    using Sh = Fwd<DP, EXACT>;
    constexpr int NS = Sh::NS, QB = Sh::QB;
    // some exponentials by multiply-adds: at d > 64, where nothing else is done to the scores, 4096 causal keys 165 -> 161 us (and 4096 seen ones 353 ->
    // 345); with d = 64, caps or biases, whose own arithmetic fills that pipe, it costs up to a tenth
    constexpr bool FMA = DP == 128 && BIAS == GRF_BIAS_NONE && !CAP && !EXACT;
    constexpr bool PLAIN = BIAS == GRF_BIAS_NONE && !CAP;   // (a scale that is not positive, or lse wanted at d > 64: BIAS_NONE_SCALED)
    extern __shared__ unsigned char smem_dyn[];
    constexpr int PER_GROUP = 5 + 2 * QB;
    __shared__ __align__(8) unsigned long long bars[5 * NS + PER_GROUP * QT];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, redo_steps;
    __shared__ float lut[BIAS == GRF_BIAS_BUCKETS ? QT * 2 * 256 : 1];
    __shared__ float tops[2][SOFT * 32], sums[SOFT * 32];
    __shared__ __align__(16) int32_t doc_of[QT * 2 * BT];
    __shared__ grf_buckets bucket;
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem_dyn + (smem - smem_u32(smem_dyn)) + Sh::TILE * (QT * QB + 2 * NS));
    const uint32_t q_at = smem, k_at = q_at + QT * QB * Sh::TILE, v_at = k_at + NS * Sh::TILE, bar0 = smem_u32(bars);
    auto k_full = [&](int s) { return bar0 + 8u * s; };
    auto v_full = [&](int s) { return bar0 + 8u * (NS + s); };
    auto k_empty = [&](int s) { return bar0 + 8u * (2 * NS + s); };
    auto v_empty = [&](int s) { return bar0 + 8u * (3 * NS + s); };
    auto v_clean = [&](int s) { return bar0 + 8u * (4 * NS + s); };
    auto of_group = [&](int g, int what) { return bar0 + 8u * (5 * NS + PER_GROUP * g + what); };
    auto s_full = [&](int g) { return of_group(g, 0); };
    auto s_read = [&](int g) { return of_group(g, 1); };
    auto p_full = [&](int g) { return of_group(g, 2); };
    auto pv_done = [&](int g) { return of_group(g, 3); };
    auto o_read = [&](int g) { return of_group(g, 4); };
    auto q_full = [&](int g, int y) { return of_group(g, 5 + y); };
    auto q_empty = [&](int g, int y) { return of_group(g, 5 + QB + y); };

    // Blocks of queries, the longest rows first, dealt out to the CTAs forwards and backwards in turn, so that all get about the same.
    // (With documents every CTA has one block, whose bits are made below.)
    const int32_t heads = p.B * p.H, blocks = (p.Nq + QT * BT - 1) / (QT * BT);
    const uint32_t items = (uint32_t)heads * (uint32_t)blocks;  // (at most 65535 * 32768)
    auto item = [&](uint32_t round) { return round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x); };
    const uint32_t rounds = (items - 1) / gridDim.x + 1;
    auto bh_of = [&](uint32_t x) { return (int32_t)(x % (uint32_t)heads); };
    auto i0_of = [&](uint32_t x) { return (blocks - 1 - (int32_t)(x / (uint32_t)heads)) * (QT * BT); };
    constexpr int COPY = SOFT, ISSUE = SOFT + 1, CLEAN = SOFT + 3;

    if (tid == 0) {
        abort_flag = redo_steps = 0;
        for (int s = 0; s < NS; ++s) {
            mbar_init(k_full(s), 1); mbar_init(v_full(s), 1); mbar_init(v_clean(s), 1);
            mbar_init(k_empty(s), QT); mbar_init(v_empty(s), QT + 1);
        }
        for (int g = 0; g < QT; ++g) {
            mbar_init(s_full(g), 1); mbar_init(pv_done(g), 1);
            mbar_init(s_read(g), 8); mbar_init(p_full(g), 8); mbar_init(o_read(g), 8);
            for (int y = 0; y < QB; ++y) { mbar_init(q_full(g, y), 1); mbar_init(q_empty(g, y), 1); }
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == COPY) tmem_alloc(&tmem_slot, 512u);
    if (BIAS == GRF_BIAS_BUCKETS) bucket.fill(p);
    if (p.q_doc) {
        const int32_t b = bh_of(blockIdx.x) / p.H, i0 = i0_of(blockIdx.x);
        const grf_sight sight(p, b);
        const forward_tiles T(p, sight, bits, i0);
        const int32_t tiles = T.tiles;
        const int32_t kblocks = (p.Nk + BT - 1) / BT, qblocks = (p.Nq + BT - 1) / BT;
        for (int32_t w = warp; w < T.words; w += THREADS / 32) {
            const int32_t t = w * 32 + lane;
            const int4 kr = t < tiles ? p.k_range[(int64_t)b * kblocks + t] : make_int4(INT32_MAX, -1, 0, 0);
            uint32_t any = 0u;
            for (int g = 0; g < QT; ++g) {
                int what = 0;
                bool same = true;
                if (t < tiles && T.of(T.rows, g)) {
                    const int4 qr = p.q_range[(int64_t)b * qblocks + (i0 + g * BT) / BT];
                    what = sight.tile((i0 + g * BT), min((i0 + g * BT) + BT, p.Nq), t * BT, t * BT + BT, qr, kr);
                    same = one_document(qr, kr);
                }
                const uint32_t seen = __ballot_sync(0xffffffffu, what != 0), whole = __ballot_sync(0xffffffffu, what == 2), one = __ballot_sync(0xffffffffu, same);
                any |= seen;
                if (lane == 0) { bits[3 * g * T.words + w] = seen; bits[(3 * g + 1) * T.words + w] = whole; bits[(3 * g + 2) * T.words + w] = one; }
            }
            const uint32_t hole = __ballot_sync(0xffffffffu, kr.z != 0);
            if (lane == 0) { bits[3 * QT * T.words + w] = any; bits[(3 * QT + 1) * T.words + w] = hole; }
        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = (uint32_t)uniform((int32_t)tmem_slot);
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_beside(bar, parity, &abort_flag, &redo_steps)) != 0; };

    if (warp >= SOFT) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LESS));
        if (warp == COPY) {
            // ------------------------------------------------------------ copies
            bool ok = true;
            int32_t n = 0, qn[QT] = {};
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t x = item(round);
                if (x >= items) break;
                const int32_t bh = bh_of(x), b = bh / p.H, h = bh % p.H, kvh = h / p.group, i0 = i0_of(x);
                const grf_sight sight(p, b);
                const forward_tiles T(p, sight, bits, i0);
                const int32_t tiles = T.tiles;
                const int32_t kb = p.ks[0] ? b : 0, kh = p.ks[1] ? kvh : 0, vb = p.vs[0] ? b : 0, vh = p.vs[1] ? kvh : 0;
                const int32_t t0 = T.next(0);
                for (int32_t t = t0; t < tiles && ok; t = T.next(t + 1), ++n) {
                    const int s = n % NS;
                    const uint32_t before = (uint32_t)(n / NS - 1) & 1u;
                    if (n >= NS && !(ok = wait(k_empty(s), before))) break;
                    expect_tx_elected(k_full(s), Sh::TILE);
                    for (int y = 0; y < DP / 64; ++y) load_box(k_at + s * Sh::TILE + y * HALF, &map_k, 64 * y, t * BT, kh, kb, k_full(s));
                    if (t == t0) {
#pragma unroll
                        for (int g = 0; g < QT; ++g) {
                            if (!T.of(T.rows, g)) continue;
                            const int y = qn[g] % QB;
                            if (qn[g] >= QB && !wait(q_empty(g, y), (uint32_t)(qn[g] / QB - 1) & 1u)) { ok = false; break; }
                            expect_tx_elected(q_full(g, y), Sh::TILE);
                            for (int z = 0; z < DP / 64; ++z)
                                load_box(q_at + (g * QB + y) * Sh::TILE + z * HALF, &map_q, 64 * z, (i0 + g * BT), p.qs[1] ? h : 0, p.qs[0] ? b : 0, q_full(g, y));
                            ++qn[g];
                        }
                    }
                    if (!ok || (n >= NS && !(ok = wait(v_empty(s), before)))) break;
                    expect_tx_elected(v_full(s), Sh::TILE);
                    for (int y = 0; y < DP / 64; ++y) load_box(v_at + s * Sh::TILE + y * HALF, &map_v, 64 * y, t * BT, vh, vb, v_full(s));
                }
            }
            // after an abort nobody may have waited for the last copies: they end before the CTA does
            if (!ok || *(volatile int*)&abort_flag) {
                for (int32_t x = max(0, n - NS); x <= n; ++x) {
                    mbar_drain(k_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                    mbar_drain(v_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                }
#pragma unroll
                for (int g = 0; g < QT; ++g)
                    for (int32_t x = max(0, qn[g] - QB); x < qn[g]; ++x) mbar_drain(q_full(g, x % QB), (uint32_t)(x / QB) & 1u, 20000000ll);
            }
        } else if (warp >= ISSUE && warp < ISSUE + QT) {
            // ------------------------------------------------------------ products of one group
            const int g = warp - ISSUE;
            const int32_t steps = (p.d + 15) / 16;
            const uint64_t q_op = rows_operand(q_at + g * QB * Sh::TILE), k_op = rows_operand(k_at), v_op = columns_operand(v_at);
            const uint32_t scores = tmem + g * BT, probs = tmem + Sh::P_COL + g * Sh::P_STEP, acc = tmem + Sh::O_COL + g * DP;
            bool ok = true;
            int32_t n = 0, made = 0, used = 0, qn = 0, outs = 0;        // tiles, S and P of this group, its queries, its outputs
            uint32_t cleaned = 0u;                              // parity of each stage's cleanings
            auto make_scores = [&](int32_t n_) {
                const int s = n_ % NS;
                if (Sh::SEP && made > 0 && !wait(s_read(g), (uint32_t)(made - 1) & 1u)) return false;
                if (!wait(k_full(s), (uint32_t)(n_ / NS) & 1u)) return false;
                fence_after_sync();
                product_over_columns<DP>(scores, lo32(q_op) + (qn % QB) * (Sh::TILE / 16), hi32(q_op), lo32(k_op) + s * (Sh::TILE / 16), hi32(k_op), steps);
                mma_commit(s_full(g));
                mma_commit(k_empty(s));
                ++made;
                return true;
            };
            auto values_ready = [&](const forward_tiles& T, int32_t t) {
                const int s = n % NS;
                if (!wait(v_full(s), (uint32_t)(n / NS) & 1u)) return false;
                if (T.unclean(p, t)) {
                    if (!wait(v_clean(s), cleaned >> s & 1u)) return false;
                    cleaned ^= 1u << s;
                }
                return true;
            };
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t x = item(round);
                if (x >= items) break;
                const int32_t b = bh_of(x) / p.H, i0 = i0_of(x);
                const grf_sight sight(p, b);
                const forward_tiles T(p, sight, bits, i0);
                const int32_t tiles = T.tiles;
                int32_t t = T.next(0), c = 0;
                const bool queries = t < tiles && T.of(T.rows, g);
                if (queries && !(ok = wait(q_full(g, qn % QB), (uint32_t)(qn / QB) & 1u))) break;
                bool ahead = false;                             // S of the present tile is already made
                for (; t < tiles && ok; ++n) {
                    const int s = n % NS;
                    const int32_t t_next = T.next(t + 1);
                    if (T.what(g, t) == 0) {
                        if (!(ok = wait(k_full(s), (uint32_t)(n / NS) & 1u))) break;
                        arrive_elected(k_empty(s));
                        if (!(ok = values_ready(T, t))) break;
                        arrive_elected(v_empty(s));
                        t = t_next;
                        continue;
                    }
                    if (!ahead && !(ok = make_scores(n))) break;
                    ahead = Sh::SEP && t_next < tiles && T.what(g, t_next) != 0;
                    if (ahead && !(ok = make_scores(n + 1))) break;
                    if (c == 0 && outs > 0 && !(ok = wait(o_read(g), (uint32_t)(outs - 1) & 1u))) break;
                    if (!(ok = wait(p_full(g), (uint32_t)used & 1u))) break;
                    if (!(ok = values_ready(T, t))) break;
                    fence_after_sync();
                    product_over_rows<DP>(acc, probs, lo32(v_op) + s * (Sh::TILE / 16), hi32(v_op), c > 0 ? 1u : 0u);
                    if (EXACT) product_over_rows<DP>(acc, probs + 64, lo32(v_op) + s * (Sh::TILE / 16), hi32(v_op), 1u);
                    mma_commit(v_empty(s));
                    mma_commit(pv_done(g));
                    ++c;
                    ++used;
                    t = t_next;
                }
                if (queries && ok) {
                    mma_commit(q_empty(g, qn % QB));
                    ++qn;
                }
                if (c > 0) ++outs;
            }
            if (!ok) {
                // products under way end before the CTA does (a barrier that nobody else needs any more)
                mma_commit(pv_done(g));
                mbar_drain(pv_done(g), (uint32_t)used & 1u, 20000000ll);
            }
        } else if (warp == CLEAN) {
            // ------------------------------------------------------------ rows of V that nobody sees
            int32_t n = 0;
            bool ok = true;
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t x = item(round);
                if (x >= items) break;
                const int32_t b = bh_of(x) / p.H, i0 = i0_of(x);
                const grf_sight sight(p, b);
                const forward_tiles T(p, sight, bits, i0);
                const int32_t tiles = T.tiles;
                for (int32_t t = T.next(0); t < tiles; t = T.next(t + 1), ++n) {
                    // (it waits for every tile, and holds the stage until then: a parity only tells a phase from the one before it)
                    const int s = n % NS;
                    if (!(ok = wait(v_full(s), (uint32_t)(n / NS) & 1u))) break;
                    if (T.unclean(p, t)) {
                        for (int r = lane; r < BT; r += 32) {
                            const int32_t j = t * BT + r;
                            if (j >= p.Nk || (j < T.last && !(sight.docs && p.k_doc[(int64_t)b * p.Nk + j] < 0))) continue;
                            for (int y = 0; y < DP / 64; ++y)
                                for (int z = 0; z < 8; ++z)
                                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_at + s * Sh::TILE + y * HALF + r * 128 + z * 16), "r"(0u) : "memory");
                        }
                        fence_async_smem();                     // the products read through the asynchronous proxy
                        __syncwarp();
                        arrive_elected(v_clean(s));
                    }
                    arrive_elected(v_empty(s));
                }
            }
        }
    } else {
        // ---------------------------------------------------------------- two threads per query
        // After a wait that gave up (the abort flag is up, every later wait returns at once) they go on to the end, as the barriers between them
        // count all of them.
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MORE));
        const int g = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane, c0 = half * 64;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_addr = tmem + g * BT + c0 + lanes, p_addr = tmem + Sh::P_COL + g * Sh::P_STEP + half * 32 + lanes,
                       o_addr = tmem + Sh::O_COL + g * DP + half * (DP / 2) + lanes;
        const float to2 = p.scale * GRF_LOG2E, by_cap = CAP ? p.scale / p.cap : 0.0f, cap2 = p.cap * GRF_LOG2E;
        auto with_other_half = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(1 + g * 4 + (warp & 3)) : "memory"); };
        auto with_group = [&]() { asm volatile("bar.sync %0, 256;" ::"r"(1 + 4 * QT + g) : "memory"); };
        int32_t done = 0, luts = 0;                             // tiles of this group, tiles with a bias per diagonal or documents
        for (uint32_t round = 0; round < rounds; ++round) {
            const uint32_t which = item(round);
            if (which >= items) break;
            const int32_t bh = bh_of(which), b = bh / p.H, h = bh % p.H, i0 = i0_of(which);
            const grf_sight sight(p, b);
            const forward_tiles T(p, sight, bits, i0);
            const int32_t tiles = T.tiles;
            const int32_t i = i0 + g * BT + r, pos = sight.position(i), pos0 = sight.position(i0 + g * BT);
            const int32_t limit = (sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(pos + 1, sight.prefix))) - c0;
            int32_t doc = sight.docs && i < p.Nq ? p.q_doc[(int64_t)b * p.Nq + i] : -1;
            if (doc < 0) doc = INT32_MIN;                       // (equal to no key's: these are -1 where they are negative)
            const float slope2 = BIAS == GRF_BIAS_SLOPES ? grf_slope2(p, h) : 0.0f;
            float m = -CUDART_INF_F;
            uint64_t sum2[2] = {0ull, 0ull};
            int32_t c = 0;
            for (int32_t t = T.next(0); t < tiles; t = T.next(t + 1)) {
                const int what = T.what(g, t);
                if (what == 0) continue;
                const int32_t j0 = t * BT;
                // the bias of this tile: one value, or one per diagonal; documents of its keys where they have to be compared
                float bias2 = 0.0f;
                bool diagonals = false;
                const bool mixed = what == 1 && T.mixed(g, t);
                const float* mine = lut;
                int32_t* docs = doc_of + (g * 2 + (luts & 1)) * BT;
                if (BIAS == GRF_BIAS_BUCKETS) {
                    diagonals = bucket(p, j0 - pos0 - (BT - 1)) != bucket(p, j0 + BT - 1 - pos0);
                    if (!diagonals) bias2 = grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0);
                }
                if (diagonals || mixed) {
                    if (BIAS == GRF_BIAS_BUCKETS && diagonals) {
                        float* at = lut + (g * 2 + (luts & 1)) * 256;
                        at[r + 128 * half] = grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0 + r + 128 * half - (BT - 1));
                        mine = at + (BT - 1 - r) + c0;
                    }
                    if (mixed && half == 0) docs[r] = j0 + r < p.Nk ? max(p.k_doc[(int64_t)b * p.Nk + j0 + r], -1) : -1;
                    with_group();
                    ++luts;
                }
                const int32_t to = limit - j0;
                wait(s_full(g), (uint32_t)done & 1u);
                fence_after_sync();
                uint32_t sv[4][16];
#pragma unroll
                for (int y = 0; y < 4; ++y) tmem_ld16_nowait(s_addr + 16 * y, sv[y]);
                tmem_ld_wait();
                if (Sh::SEP) {
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(s_read(g));
                }
                // scores in units of log 2 (PLAIN: still to be scaled, by a positive number)
                if (CAP) capped<4>(sv, by_cap);
                if (!PLAIN) {
                    const uint64_t by = CAP ? pack2(cap2, cap2) : pack2(to2, to2);
                    const float ahead = (float)(j0 + c0 - pos); // (exact, as are its sums, below 2^24; beyond, off by half a step as the distance itself)
                    // Where a half's last key is its 64 columns before the query, or more, the distance is a line from its first key; nearer its two parts would be
                    // far larger than their sum, and the score be rounded to their steps (slopes of 1e4: lse off by 3e-4, and gradients with it).
                    const bool line = BIAS == GRF_BIAS_SLOPES && __all_sync(0xffffffffu, j0 + c0 + 127 <= pos);
                    const float at0 = line ? slope2 * ahead : bias2;
                    const uint64_t at02 = pack2(at0, at0);
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const int col = 16 * y + e;
                            float x0, x1;
                            unpack2(fma2(pack2(sv[y][e], sv[y][e + 1]), by, at02), x0, x1);
                            if (BIAS == GRF_BIAS_SLOPES) {
                                if (line) {
                                    x0 = fmaf(slope2, (float)col, x0);
                                    x1 = fmaf(slope2, (float)(col + 1), x1);
                                } else {
                                    x0 = fmaf(-slope2, fabsf(ahead + (float)col), x0);
                                    x1 = fmaf(-slope2, fabsf(ahead + (float)(col + 1)), x1);
                                }
                            }
                            if (BIAS == GRF_BIAS_BUCKETS) {
                                if (diagonals) { x0 += mine[col]; x1 += mine[col + 1]; }
                            }
                            sv[y][e] = __float_as_uint(x0);
                            sv[y][e + 1] = __float_as_uint(x1);
                        }
                }
                if (what == 1) {
                    if (mixed) {
#pragma unroll
                        for (int y = 0; y < 4; ++y)
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const int4 d4 = *reinterpret_cast<const int4*>(docs + c0 + 16 * y + e);
                                if (!(16 * y + e < to && d4.x == doc)) sv[y][e] = 0xff800000u;
                                if (!(16 * y + e + 1 < to && d4.y == doc)) sv[y][e + 1] = 0xff800000u;
                                if (!(16 * y + e + 2 < to && d4.z == doc)) sv[y][e + 2] = 0xff800000u;
                                if (!(16 * y + e + 3 < to && d4.w == doc)) sv[y][e + 3] = 0xff800000u;
                            }
                    } else {
#pragma unroll
                        for (int y = 0; y < 4; ++y)
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                if (16 * y + e >= to) sv[y][e] = 0xff800000u;
                    }
                }
                // (four chains: one would take longer than the exponentials)
                float top4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int e = 0; e < 16; e += 2) top4[e >> 1 & 3] = max3_nan(top4[e >> 1 & 3], __uint_as_float(sv[y][e]), __uint_as_float(sv[y][e + 1]));
                float top = max_nan(max_nan(top4[0], top4[1]), max_nan(top4[2], top4[3]));
                tops[done & 1][tid] = top;
                with_other_half();                              // (by then the other half has read its S, which P may overwrite)
                top = max_nan(top, tops[done & 1][tid ^ 128]);
                if (PLAIN) top *= to2;
                // a new maximum only when it matters: 2^8 above the one in use (or the first)
                // (NaN grows too, and stays; an infinite score makes its row NaN, as infinity - infinity would)
                const bool grow = !(top <= m + 8.0f);
                if (top == CUDART_INF_F) top = CUDART_NAN_F;
                if (__any_sync(0xffffffffu, grow)) {
                    const float alpha = grow ? ex2(m - top) : 1.0f;
                    if (grow) m = top;
                    if (c > 0) {
                        wait(pv_done(g), (uint32_t)(done - 1) & 1u);
                        fence_after_sync();
                        const uint64_t a2 = pack2(alpha, alpha);
                        sum2[0] = mul2(sum2[0], a2);
                        sum2[1] = mul2(sum2[1], a2);
#pragma unroll 1
                        for (int y = 0; y < DP / 32; ++y) {
                            uint32_t o[16];
                            tmem_ld16(o_addr + 16 * y, o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tmem_st16(o_addr + 16 * y, o);
                        }
                    }
                }
                if (Sh::SEP && done > 0) {
                    wait(pv_done(g), (uint32_t)(done - 1) & 1u);
                    fence_after_sync();
                }
                const float base = m == -CUDART_INF_F ? 0.0f : m;
                const uint64_t minus = pack2(-base, -base), to22 = pack2(to2, to2);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    uint32_t w[16], u[EXACT ? 16 : 1];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int a = 2 * y + (e >> 3), z = (2 * e) & 15;
                        float x0, x1;
                        const uint64_t v = pack2(sv[a][z], sv[a][z + 1]);
                        unpack2(PLAIN ? fma2(v, to22, minus) : add2(v, minus), x0, x1);
                        if (FMA && FMA_PAIRS(16 * y + e)) ex2_by_fma(pack2(x0, x1), x0, x1);
                        else { x0 = ex2(x0); x1 = ex2(x1); }
                        sum2[e & 1] = add2(sum2[e & 1], pack2(x0, x1));
                        w[e] = pack_bf16(x0, x1);
                        if (EXACT) u[EXACT ? e : 0] = pack_bf16(x0 - __uint_as_float(w[e] << 16), x1 - __uint_as_float(w[e] & 0xffff0000u));
                    }
                    tmem_st16(p_addr + 16 * y, w);
                    if constexpr (EXACT) tmem_st16(p_addr + 64 + 16 * y, u);
                }
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(g));
                ++c;
                ++done;
            }
            if (c > 0) wait(pv_done(g), (uint32_t)(done - 1) & 1u);
            fence_after_sync();
            float l0, l1;
            unpack2(add2(sum2[0], sum2[1]), l0, l1);
            sums[tid] = l0 + l1;
            with_other_half();
            const float l = sums[tid & ~128] + sums[tid | 128], inv = l == 0.0f ? 0.0f : 1.0f / l;
            bool spoilt = false;
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out_w) + b * p.os[0] + h * p.os[1] + (int64_t)i * p.os[2];
            __nv_bfloat16* rest = p.rest_w ? p.rest_w + (((int64_t)b * p.H + h) * p.Nq + i) * p.d : nullptr;
            // (a loop: once a block, its instructions come from afar)
#pragma unroll 1
            for (int y = 0; y < DP / 32; ++y) {
                uint32_t o[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0u;
                if (c > 0) tmem_ld16(o_addr + 16 * y, o);
                if (c > 0 && y == DP / 32 - 1) {
                    // the accumulator may be written again
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(o_read(g));
                }
                if (i >= p.Nq) continue;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int col = half * (DP / 2) + 16 * y + 8 * z;
                    if (col >= p.d) continue;
                    uint32_t w[4], u[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // (no key seen: 0, whatever the accumulator holds)
                        const float x0 = l == 0.0f ? 0.0f : __uint_as_float(o[8 * z + 2 * e]) * inv, x1 = l == 0.0f ? 0.0f : __uint_as_float(o[8 * z + 2 * e + 1]) * inv;
                        spoilt |= !(fabsf(x0) + fabsf(x1) <= 3.4028235e38f);
                        w[e] = pack_bf16(x0, x1);
                        if (EXACT) {
                            const __nv_bfloat16 r0 = grf_rest(x0, __float2bfloat16_rn(x0)), r1 = grf_rest(x1, __float2bfloat16_rn(x1));
                            u[e] = pack_bf16(__bfloat162float(r0), __bfloat162float(r1));
                        }
                    }
                    *reinterpret_cast<uint4*>(out + col) = make_uint4(w[0], w[1], w[2], w[3]);
                    if (EXACT) *reinterpret_cast<uint4*>(rest + col) = make_uint4(u[0], u[1], u[2], u[3]);
                }
            }
            if (half == 0 && p.lse_w && i < p.Nq) p.lse_w[((int64_t)b * p.H + h) * p.Nq + i] = l == 0.0f ? -CUDART_INF_F : (m + log2f(l)) * GRF_LN2;
            // rows whose scores are finite but whose outputs are not: each half its own columns
            uint32_t again = __ballot_sync(0xffffffffu, spoilt && l <= 3.4028235e38f && fabsf(m) <= 3.4028235e38f);
            __syncwarp();
            while (again) {
                const int y = __ffs(again) - 1;
                again &= again - 1;
                redo_row<CAP, EXACT>(p, bucket, b, h, __shfl_sync(0xffffffffu, i, y), __shfl_sync(0xffffffffu, m, y), __shfl_sync(0xffffffffu, l, y), half * (DP / 2),
                                     (half + 1) * (DP / 2), &redo_steps);
            }
            with_other_half();                                  // (the sums are read: they may be written again)
        }
        fence_before_sync();
    }
    fence_before_sync();
    __syncthreads();
    if (warp == COPY) tmem_dealloc(tmem, 512u);
    if (tid == 0 && abort_flag) atomicExch(p.error_word, 1);
}

struct forward_maps { CUtensorMap q, k, v; };

template <int DP, bool CAP, int BIAS, bool EXACT> int launch(grf_ctx* ctx, const grf_softmax_params& p, const forward_maps& m)
{
    using Sh = Fwd<DP, EXACT>;
    const auto kernel = softmax_tc_forward_kernel<DP, CAP, BIAS, EXACT>;
    auto bits = [](int32_t tokens) { return 4 * (size_t)(3 * QT + 2) * (grf_ceil_div(tokens, BT) / 32 + 1); };
    const size_t smem = Sh::SMEM + (p.q_doc ? bits(p.Nk) : 0);
    // (the most of any call: the attribute is the whole process's, and another thread may set it between here and the launch)
    GRF_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(Sh::SMEM + bits(MOST_WITH_DOCS))));
    grf_softmax_scope scope(ctx, "grf:softmax_attention");
    // as many CTAs as the device holds at once, which take block after block; with documents a CTA per block
    const int64_t items = (int64_t)p.B * p.H * grf_ceil_div(p.Nq, QT * BT), room = ctx->sm_count;
    kernel<<<(unsigned)(p.q_doc || items < room ? items : room), THREADS, smem, ctx->stream>>>(m.q, m.k, m.v, p);
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}

template <int DP, bool EXACT, bool CAP> int by_bias(grf_ctx* ctx, const grf_softmax_params& p, const forward_maps& m)
{
    // (lse is a sum of fp32 exponentials: where it is wanted, none by multiply-adds)
    if constexpr (!CAP)
        if (p.bias == GRF_BIAS_NONE && (!(p.scale > 0.0f) || (DP == 128 && !EXACT && p.lse_w))) return launch<DP, CAP, BIAS_NONE_SCALED, EXACT>(ctx, p, m);
    return p.bias == GRF_BIAS_NONE ? launch<DP, CAP, GRF_BIAS_NONE, EXACT>(ctx, p, m)
         : p.bias == GRF_BIAS_SLOPES ? launch<DP, CAP, GRF_BIAS_SLOPES, EXACT>(ctx, p, m) : launch<DP, CAP, GRF_BIAS_BUCKETS, EXACT>(ctx, p, m);
}
template <int DP, bool EXACT> int by_cap(grf_ctx* ctx, const grf_softmax_params& p, const forward_maps& m)
{
    return p.cap > 0.0f ? by_bias<DP, EXACT, true>(ctx, p, m) : by_bias<DP, EXACT, false>(ctx, p, m);
}
template <int DP> int by_rest(grf_ctx* ctx, const grf_softmax_params& p, const forward_maps& m)
{
    return p.rest_w ? by_cap<DP, true>(ctx, p, m) : by_cap<DP, false>(ctx, p, m);
}

}  // namespace

int grf_softmax_tc_forward(grf_ctx* ctx, const grf_softmax_params& p)
{
    if (p.q_doc && p.Nk > MOST_WITH_DOCS) return 1;
    forward_maps m;
    if (!grf_make_token_box_map(&m.q, p.q, p.qs, p.B, p.H, p.Nq, p.d) || !grf_make_token_box_map(&m.k, p.k, p.ks, p.B, p.KV, p.Nk, p.d) ||
        !grf_make_token_box_map(&m.v, p.v, p.vs, p.B, p.KV, p.Nk, p.d)) return 1;
    return p.d <= 64 ? by_rest<64>(ctx, p, m) : by_rest<128>(ctx, p, m);
}
