// Softmax attention over ordered tokens on the tensor cores (bf16): gradients, in two kernels so that nothing is added atomically.
//
//   dQ     a CTA of 128 queries goes over the key tiles: S = Q K^T, dP = dout V^T (a query per lane of tensor memory), dS = P (dP - D), and
//          dQ += dX K with dX as bf16 pairs in tensor memory.  Where the bias table wants its gradient, dS is summed along diagonals by
//          shuffles (a lane hands its sum to the next lane, which adds the next column), and the diagonals by bucket
//   dK, dV a CTA of 128 keys goes over the query tiles of all heads that share it, transposed: S^T = K Q^T, dP^T = V dout^T (a key per lane), so
//          that P^T and dX^T are left operands where they are made: dV += P^T dout, dK += dX^T Q
// Seven products a tile where a single kernel would need five, but no tile of dQ travels through memory.  Four warpgroups share a tile, 32
// columns each, and work in turn with the products: while P of a tile is made the tensor cores finish the one before, while dS is made they
// make the next S.  Three warps copy, issue, and prepare: lse and D of the queries (dK, dV), and rows that nobody sees cleared (0 times an
// infinity there would reach a whole tile).  CTAs take block after block, as in the forward pass (64 x 12 heads x 196, with a CTA per block, which
// takes three microseconds before its first product: 246 us for both kernels and the products of the outputs; so: 194).
#include <cooperative_groups.h>

#include "softmax_tc.cuh"

namespace cg = cooperative_groups;

namespace {

using namespace grf_softmax_tc;

constexpr int THREADS = 640, WORKERS = 16;          // warps that make P and dS
constexpr int MORE = 104, LESS = 64;                // registers: 4 * 104 + 64 = 5 * 96
constexpr int W = 32;                               // columns of a worker
constexpr int COPY = WORKERS, ISSUE = WORKERS + 1, PREPARE = WORKERS + 2;

struct head_split { int32_t splits; };

template <int DP> struct Grad {
    // stages: a tile's place is free only once its last product is done, a tile's time before the next but one is wanted, and a copy takes
    // about as long: two stages leave it in the open (16 heads x 4096, d = 64: both kernels 414 us with two, 376 with four, which d = 128 has no room for)
    static constexpr int NS = DP == 64 ? 4 : 2;
    static constexpr int QB = DP == 64 ? 2 : 1;        // places for what a block keeps
    static constexpr uint32_t TILE = HALF * (DP / 64);
    static constexpr size_t SMEM = 1024 + (size_t)TILE * (2 * QB + 2 * NS);        // then the tiles' bits
};

// Tiles of the other side that a block sees, in order; with documents from bits in shared memory.
struct grad_tiles {
    const uint32_t* bits;               // seen, whole, tiles of one document
    int32_t first, tiles, words;
    bool docs;
    __device__ __forceinline__ int32_t next(int32_t t) const
    {
        if (!docs) return t;
        while (t < tiles) {
            const uint32_t w = bits[t >> 5] >> (t & 31);
            if (w) return min(t + __ffs(w) - 1, tiles);
            t = (t | 31) + 1;
        }
        return tiles;
    }
    __device__ __forceinline__ int32_t begin() const { return next(first); }
    __device__ __forceinline__ bool whole(int32_t t) const { return bit(bits + words, t); }
    __device__ __forceinline__ bool mixed(int32_t t) const { return docs && !bit(bits + 2 * words, t); }
};

constexpr float LARGEST = 1.0e30f;                  // of lse
// a pair's values where they are to stay, else 0
__device__ __forceinline__ void keep(uint64_t& x, bool first, bool second)
{
    float x0, x1;
    unpack2(x, x0, x1);
    x = pack2(first ? x0 : 0.0f, second ? x1 : 0.0f);
}
// dP, and the slope of the cap where there is one, are 0 where P is: a place that is not seen holds 0, whatever came out of the products there
template <bool CAP>
__device__ __forceinline__ void only_seen(uint32_t (&dp)[W / 16][16], uint64_t (&slope)[CAP ? W / 2 : 1], const uint64_t (&p)[W / 2])
{
#pragma unroll
    for (int e = 0; e < W; e += 2) {
        float p0, p1;
        unpack2(p[e / 2], p0, p1);
        if (p0 == 0.0f) dp[e / 16][e % 16] = 0u;
        if (p1 == 0.0f) dp[e / 16][e % 16 + 1] = 0u;
        if constexpr (CAP) keep(slope[e / 2], p0 != 0.0f, p1 != 0.0f);
    }
}
__device__ __forceinline__ void clear_row(uint32_t tile, int r, int halves)
{
    for (int y = 0; y < halves; ++y)
        for (int x = 0; x < 8; ++x) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + y * HALF + r * 128 + x * 16), "r"(0u) : "memory");
}
// Rows of a tile of bf16 that hold an infinity or NaN, by a warp: bit y of lanes 8 z .. 8 z + 7 is row 4 y + z.
template <int HALVES> __device__ __forceinline__ uint32_t not_finite(uint32_t tile, int lane)
{
    uint32_t rows = 0u;
#pragma unroll 4
    for (int y = 0; y < BT / 4; ++y)
#pragma unroll
        for (int x = 0; x < HALVES; ++x) {
            uint4 v;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(tile + x * HALF + y * 512 + lane * 16) : "memory");
            // (an exponent of ones carries into the sign)
            auto bad = [](uint32_t w) { return (w & 0x7f807f80u) + 0x00800080u; };
            if ((bad(v.x) | bad(v.y) | bad(v.z) | bad(v.w)) & 0x80008000u) rows |= 1u << y;
        }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) rows |= __shfl_xor_sync(0xffffffffu, rows, o);
    return rows;
}
// D[128][DP] (+)= A B: A's bf16 pairs in the first half of every worker's columns.
template <int DP>
__device__ __forceinline__ void product_of_parts(uint32_t acc, uint32_t a_tmem, uint32_t b_lo, uint32_t b_hi, uint32_t accumulate)
{
    constexpr uint32_t idesc = instr_desc(DP, false, true);
#pragma unroll
    for (int y = 0; y < BT / 16; ++y)
        mma_bf16_ts_halves(acc, a_tmem + (y / 2) * W + (y % 2) * 8, b_lo + y * (2048 / 16), b_hi, idesc, y > 0 ? 1u : accumulate);
}

template <int DP, bool CAP, int BIAS>
__global__ void __launch_bounds__(THREADS, 1)
softmax_tc_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_g, const __grid_constant__ grf_softmax_params p)
{
    using Sh = Grad<DP>;
    constexpr int NS = Sh::NS, QB = Sh::QB;
    constexpr int LUTS = BIAS == GRF_BIAS_BUCKETS ? 1 : 0;
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[5 * NS + 7 + 2 * QB];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ float lut[LUTS ? 2 * 256 : 1];
    __shared__ grf_buckets bucket;
    __shared__ __align__(16) int32_t doc_of[2 * BT];
    __shared__ float bins[LUTS ? WORKERS * 2 * GRF_MAX_BUCKETS : 1];
    __shared__ float diag[LUTS ? WORKERS * 64 : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem_dyn + (smem - smem_u32(smem_dyn)) + Sh::TILE * (2 * QB + 2 * NS));
    const uint32_t q_at = smem, g_at = q_at + QB * Sh::TILE, k_at = g_at + QB * Sh::TILE, v_at = k_at + NS * Sh::TILE, bar0 = smem_u32(bars);
    auto k_full = [&](int s) { return bar0 + 8u * s; };
    auto v_full = [&](int s) { return bar0 + 8u * (NS + s); };
    auto k_empty = [&](int s) { return bar0 + 8u * (2 * NS + s); };
    auto v_empty = [&](int s) { return bar0 + 8u * (3 * NS + s); };
    auto k_clean = [&](int s) { return bar0 + 8u * (4 * NS + s); };
    const uint32_t one = bar0 + 8u * (5 * NS);
    const uint32_t s_full0 = one, dp_full = one + 16, ds_full = one + 24, dq_done = one + 32, acc_read = one + 40, drain = one + 48;
    auto rows_full = [&](int y) { return one + 56 + 8u * y; };
    auto rows_empty = [&](int y) { return one + 56 + 8u * (QB + y); };

    // Blocks of queries dealt out as in the forward pass; with documents a CTA per block, whose bits are made below.
    const int32_t heads = p.B * p.H, blocks = (p.Nq + BT - 1) / BT;
    const uint32_t items = (uint32_t)heads * (uint32_t)blocks, rounds = (items - 1) / gridDim.x + 1;
    auto item = [&](uint32_t round) { return round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x); };
    struct block_of {
        int32_t b, h, kvh, qb, i0, last;
        grf_sight sight;
        grad_tiles T;
        __device__ __forceinline__ block_of(const grf_softmax_params& p, const uint32_t* bits, int32_t heads, int32_t blocks, uint32_t x)
            : b((int32_t)(x % (uint32_t)heads) / p.H), h((int32_t)(x % (uint32_t)heads) % p.H), kvh(h / p.group), qb(blocks - 1 - (int32_t)(x / (uint32_t)heads)),
              i0(qb * BT), sight(p, b)
        {
            const int32_t tiles = (sight.end(min(i0 + BT, p.Nq)) + BT - 1) / BT;
            T = grad_tiles{bits, 0, tiles, (tiles + 31) / 32, sight.docs};
            last = sight.end(p.Nq);
        }
        // a tile that may hold keys which nobody sees
        __device__ __forceinline__ bool unclean(const grf_softmax_params& p, int32_t t) const { return (last < p.Nk && t * BT + BT > last) || (T.docs && !T.whole(t)); }
    };

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < NS; ++s) {
            mbar_init(k_full(s), 1); mbar_init(v_full(s), 1); mbar_init(k_clean(s), 1);
            mbar_init(k_empty(s), 2); mbar_init(v_empty(s), 1);
        }
        mbar_init(s_full0, 1); mbar_init(s_full0 + 8, 1); mbar_init(dp_full, 1); mbar_init(ds_full, WORKERS);
        mbar_init(dq_done, 1); mbar_init(acc_read, WORKERS); mbar_init(drain, 1);
        for (int y = 0; y < QB; ++y) { mbar_init(rows_full(y), 1); mbar_init(rows_empty(y), 1); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == COPY) tmem_alloc(&tmem_slot, 512u);
    if (LUTS) bucket.fill(p);
    if (p.q_doc) {
        const block_of I(p, bits, heads, blocks, blockIdx.x);
        const grad_tiles& T = I.T;
        const int32_t b = I.b, tiles = T.tiles, i1 = min(I.i0 + BT, p.Nq);
        const int32_t kblocks = (p.Nk + BT - 1) / BT, qblocks = (p.Nq + BT - 1) / BT;
        const int4 qr = p.q_range[(int64_t)b * qblocks + I.qb];
        for (int32_t w = warp; w < T.words; w += THREADS / 32) {
            const int32_t t = w * 32 + lane;
            const int4 kr = t < tiles ? p.k_range[(int64_t)b * kblocks + t] : make_int4(INT32_MAX, -1, 0, 0);
            const int what = t < tiles ? I.sight.tile(I.i0, i1, t * BT, t * BT + BT, qr, kr) : 0;
            const uint32_t seen = __ballot_sync(0xffffffffu, what != 0), whole = __ballot_sync(0xffffffffu, what == 2),
                           one_doc = __ballot_sync(0xffffffffu, one_document(qr, kr));
            if (lane == 0) { bits[w] = seen; bits[T.words + w] = whole; bits[2 * T.words + w] = one_doc; }
        }
    }
    if (LUTS)
        for (int x = tid; x < WORKERS * 2 * GRF_MAX_BUCKETS; x += THREADS) bins[x] = 0.0f;
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = (uint32_t)uniform((int32_t)tmem_slot);
    const uint32_t dp_col = tmem + 256, acc = tmem + 384;
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, &abort_flag)) != 0; };

    if (warp >= WORKERS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LESS));
        if (warp == COPY) {
            bool ok = true;
            int32_t n = 0, kept = 0;
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                const block_of I(p, bits, heads, blocks, which);
                const grad_tiles& T = I.T;
                const int32_t kb = p.ks[0] ? I.b : 0, kh = p.ks[1] ? I.kvh : 0, vb = p.vs[0] ? I.b : 0, vh = p.vs[1] ? I.kvh : 0;
                for (int32_t t = T.begin(); t < T.tiles && ok; t = T.next(t + 1), ++n) {
                    const int s = n % NS;
                    const uint32_t before = (uint32_t)(n / NS - 1) & 1u;
                    if (n >= NS && !(ok = wait(k_empty(s), before) && wait(v_empty(s), before))) break;
                    expect_tx_elected(k_full(s), Sh::TILE);
                    expect_tx_elected(v_full(s), Sh::TILE);
                    for (int y = 0; y < DP / 64; ++y) {
                        load_box(k_at + s * Sh::TILE + y * HALF, &map_k, 64 * y, t * BT, kh, kb, k_full(s));
                        load_box(v_at + s * Sh::TILE + y * HALF, &map_v, 64 * y, t * BT, vh, vb, v_full(s));
                    }
                    if (t == T.begin()) {
                        const int y = kept % QB;
                        if (kept >= QB && !(ok = wait(rows_empty(y), (uint32_t)(kept / QB - 1) & 1u))) { ++n; break; }
                        expect_tx_elected(rows_full(y), 2 * Sh::TILE);
                        for (int z = 0; z < DP / 64; ++z) {
                            load_box(q_at + y * Sh::TILE + z * HALF, &map_q, 64 * z, I.i0, p.qs[1] ? I.h : 0, p.qs[0] ? I.b : 0, rows_full(y));
                            load_box(g_at + y * Sh::TILE + z * HALF, &map_g, 64 * z, I.i0, p.dos[1] ? I.h : 0, p.dos[0] ? I.b : 0, rows_full(y));
                        }
                        ++kept;
                    }
                }
            }
            if (!ok || *(volatile int*)&abort_flag) {
                for (int32_t x = max(0, n - NS); x < n; ++x) {
                    mbar_drain(k_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                    mbar_drain(v_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                }
                for (int32_t x = max(0, kept - QB); x < kept; ++x) mbar_drain(rows_full(x % QB), (uint32_t)(x / QB) & 1u, 20000000ll);
            }
        } else if (warp == ISSUE) {
            const int32_t steps = (p.d + 15) / 16;
            const uint64_t q_op = rows_operand(q_at), g_op = rows_operand(g_at), k_op = rows_operand(k_at), v_op = rows_operand(v_at), kc_op = columns_operand(k_at);
            uint32_t cleaned = 0u;
            bool ok = true;
            int32_t n = 0, kept = 0;                            // tiles, blocks that saw any
            auto make_scores = [&](int32_t n_) {
                const int s = n_ % NS;
                if (!wait(k_full(s), (uint32_t)(n_ / NS) & 1u)) return false;
                fence_after_sync();
                product_over_columns<DP>(tmem + (n_ & 1) * BT, lo32(q_op) + (kept % QB) * (Sh::TILE / 16), hi32(q_op), lo32(k_op) + s * (Sh::TILE / 16), hi32(k_op), steps);
                mma_commit(s_full0 + 8 * (n_ & 1));
                return true;
            };
            auto make_dp = [&](int32_t n_) {
                const int s = n_ % NS;
                if (!wait(v_full(s), (uint32_t)(n_ / NS) & 1u)) return false;
                fence_after_sync();
                product_over_columns<DP>(dp_col, lo32(g_op) + (kept % QB) * (Sh::TILE / 16), hi32(g_op), lo32(v_op) + s * (Sh::TILE / 16), hi32(v_op), steps);
                mma_commit(dp_full);
                mma_commit(v_empty(s));
                return true;
            };
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                const block_of I(p, bits, heads, blocks, which);
                const grad_tiles& T = I.T;
                int32_t t = T.begin();
                if (t >= T.tiles) continue;
                bool first = true;
                if (!(ok = wait(rows_full(kept % QB), (uint32_t)(kept / QB) & 1u) && make_scores(n) && make_dp(n))) break;
                for (; t < T.tiles && ok; ++n) {
                    const int s = n % NS;
                    const int32_t t_next = T.next(t + 1);
                    // (its place was read before the last tile's dS arrived)
                    if (t_next < T.tiles && !(ok = make_scores(n + 1))) break;
                    if (!(ok = wait(ds_full, (uint32_t)n & 1u))) break;
                    if (I.unclean(p, t)) {
                        if (!(ok = wait(k_clean(s), cleaned >> s & 1u))) break;
                        cleaned ^= 1u << s;
                    }
                    // (the accumulator is the last block's until it is read)
                    if (first && kept > 0 && !(ok = wait(acc_read, (uint32_t)(kept - 1) & 1u))) break;
                    fence_after_sync();
                    product_of_parts<DP>(acc, dp_col, lo32(kc_op) + s * (Sh::TILE / 16), hi32(kc_op), first ? 0u : 1u);
                    first = false;
                    mma_commit(k_empty(s));
                    if (t_next >= T.tiles) {
                        mma_commit(dq_done);
                        mma_commit(rows_empty(kept % QB));
                    } else ok = make_dp(n + 1);
                    t = t_next;
                }
                ++kept;
            }
            if (!ok) {
                mma_commit(drain);
                mbar_drain(drain, 0u, 20000000ll);
            }
        } else if (warp == PREPARE) {
            // rows of K that nobody sees, once they have come (dQ's product sums over rows; of S they make columns that are not looked at)
            int32_t n = 0;
            bool ok = true;
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                const block_of I(p, bits, heads, blocks, which);
                for (int32_t t = I.T.begin(); t < I.T.tiles; t = I.T.next(t + 1), ++n) {
                    const int s = n % NS;
                    if (!(ok = wait(k_full(s), (uint32_t)(n / NS) & 1u))) break;
                    if (I.unclean(p, t)) {
                        const int32_t* kdoc = I.sight.docs ? p.k_doc + (int64_t)I.b * p.Nk : nullptr;
                        for (int r = lane; r < BT; r += 32) {
                            const int32_t j = t * BT + r;
                            if (j < p.Nk && (j >= I.last || (kdoc && kdoc[j] < 0))) clear_row(k_at + s * Sh::TILE, r, DP / 64);
                        }
                        if (kdoc) {
                            // a key of a document that no query is of, or behind the last query of its document, is seen by nobody either: which
                            // ones these are takes a look at all queries, so only rows that hold an infinity or NaN are looked up, in this block
                            __syncwarp();
                            uint32_t rows = not_finite<DP / 64>(k_at + s * Sh::TILE, lane);
                            if (__any_sync(0xffffffffu, rows != 0u)) {
                                for (int x = 0; x < BT; ++x) {
                                    if (!(__shfl_sync(0xffffffffu, rows, 8 * (x & 3)) >> (x >> 2) & 1u)) continue;
                                    const int32_t j = t * BT + x;
                                    if (j >= p.Nk) break;
                                    const int32_t doc = kdoc[j];
                                    bool seen = false;
                                    for (int32_t i = I.i0 + lane; i < min(I.i0 + BT, p.Nq); i += 32)
                                        seen |= p.q_doc[(int64_t)I.b * p.Nq + i] == doc && I.sight.sees(I.sight.position(i), j);
                                    if (!__any_sync(0xffffffffu, seen) && lane == 0) clear_row(k_at + s * Sh::TILE, x, DP / 64);
                                }
                            }
                        }
                        fence_async_smem();
                        __syncwarp();
                        arrive_elected(k_clean(s));
                    }
                    arrive_elected(k_empty(s));
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MORE));
        // After a wait that gave up (the abort flag is up, every later wait returns at once) they go on to the end, as the barriers between them
        // count all of them.
        const int r = (warp & 3) * 32 + lane, part = warp >> 2, c0 = part * W;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const float to2 = p.scale * GRF_LOG2E, by_cap = CAP ? p.scale / p.cap : 0.0f, cap2 = p.cap * GRF_LOG2E;
        const bool sums = LUTS && p.dtable_part != nullptr;
        float* my_bins = bins + warp * 2 * GRF_MAX_BUCKETS;
        auto with_workers = [&]() { asm volatile("bar.sync 1, 512;" ::: "memory"); };
        int32_t n = 0, luts = 0, kept = 0;
        for (uint32_t round = 0; round < rounds; ++round) {
            const uint32_t which = item(round);
            if (which >= items) break;
            const block_of I(p, bits, heads, blocks, which);
            const grad_tiles& T = I.T;
            const grf_sight& sight = I.sight;
            const int32_t b = I.b, h = I.h, i0 = I.i0, tiles = T.tiles;
            const int32_t i = i0 + r, pos = sight.position(i), pos0 = sight.position(i0);
            const int32_t limit = sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(pos + 1, sight.prefix));
            const int32_t all_see = sight.order == GRF_ORDER_FULL ? sight.len : min(sight.len, max(pos0 + 1, sight.prefix));       // keys before it: the whole block
            int32_t doc = sight.docs && i < p.Nq ? p.q_doc[(int64_t)b * p.Nq + i] : -1;
            if (doc < 0) doc = INT32_MIN;                           // (equal to no key's: these are -1 where they are negative)
            const int64_t row = ((int64_t)b * p.H + h) * p.Nq + i;
            const float lse = i < p.Nq ? p.lse[row] : -CUDART_INF_F, dsum = i < p.Nq ? p.dsum[row] : 0.0f;
            const bool any = !(fabsf(lse) > LARGEST);               // a row without a key, or one whose scores tell nothing any more: P = 0
            const bool empties = __any_sync(0xffffffffu, !any);
            const float minus_lse = any ? -lse * GRF_LOG2E : -CUDART_INF_F;
            const float slope2 = BIAS == GRF_BIAS_SLOPES ? grf_slope2(p, h) : 0.0f;
            float far_sum = 0.0f;                                   // of dS in tiles of one bucket, until the bucket changes
            int32_t far_bucket = -1;
            auto flush = [&]() {
                float x = far_sum;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
                if (far_bucket >= 0 && lane == 0) my_bins[far_bucket] += x;
                far_sum = 0.0f;
                __syncwarp();
            };
            bool some = false;
            for (int32_t t = T.begin(); t < tiles; t = T.next(t + 1)) {
                const int32_t j0 = t * BT;
                const bool partial = sight.docs ? !T.whole(t) : j0 + BT > all_see;
                float bias2 = 0.0f;
                bool diagonals = false;
                int32_t bucket0 = 0;
                const float* mine = lut;
                const bool mixed = partial && T.mixed(t);           // documents have to be compared
                int32_t* docs = doc_of + (luts & 1) * BT;
                if (LUTS) {
                    bucket0 = bucket(p, j0 - pos0 - (BT - 1));
                    diagonals = bucket0 != bucket(p, j0 + BT - 1 - pos0);
                    if (!diagonals) bias2 = grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0);
                }
                if (diagonals || mixed) {
                    if (LUTS && diagonals) {
                        float* at = lut + (luts & 1) * 256;
                        if (tid < 256) at[tid] = tid < 2 * BT - 1 ? grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0 + tid - (BT - 1)) : 0.0f;
                        mine = at + (BT - 1 - r) + c0;
                    }
                    if (mixed && tid < BT) docs[tid] = j0 + tid < p.Nk ? max(p.k_doc[(int64_t)b * p.Nk + j0 + tid], -1) : -1;
                    with_workers();
                    ++luts;
                }
                // (branches that the compiler is to keep: without the barrier inside it runs a whole tile's masks under a predicate, a third of all instructions)
                const bool careful = partial || empties;
                const int32_t to = any ? limit - j0 - c0 : 0;
                wait(s_full0 + 8 * (n & 1), (uint32_t)(n >> 1) & 1u);
                fence_after_sync();
                uint64_t x[W / 2], slope[CAP ? W / 2 : 1];          // P, then dS; t^2 - 1 of the cap
                {
                    uint32_t sv[W / 16][16];
#pragma unroll
                    for (int y = 0; y < W / 16; ++y) tmem_ld16_nowait(tmem + (n & 1) * BT + c0 + 16 * y + lanes, sv[y]);
                    tmem_ld_wait();
                    if (CAP) capped<W / 16>(sv, by_cap);
                    const float ahead = (float)(j0 + c0 - pos);
                    const bool line = BIAS == GRF_BIAS_SLOPES && __all_sync(0xffffffffu, j0 + c0 + 2 * W - 1 <= pos);    // (as in the forward pass)
                    const float at0 = minus_lse + (BIAS == GRF_BIAS_SLOPES ? (line ? slope2 * ahead : 0.0f) : bias2);
                    const uint64_t by = CAP ? pack2(cap2, cap2) : pack2(to2, to2), at02 = pack2(at0, at0);
#pragma unroll
                    for (int e = 0; e < W; e += 2) {
                        const uint64_t v = pack2(sv[e / 16][e % 16], sv[e / 16][e % 16 + 1]);
                        if (CAP) slope[CAP ? e / 2 : 0] = fma2(v, v, pack2(-1.0f, -1.0f));
                        float x0, x1;
                        unpack2(fma2(v, by, at02), x0, x1);
                        if (BIAS == GRF_BIAS_SLOPES) {
                            if (line) { x0 = fmaf(slope2, (float)e, x0); x1 = fmaf(slope2, (float)(e + 1), x1); }
                            else { x0 = fmaf(-slope2, fabsf(ahead + (float)e), x0); x1 = fmaf(-slope2, fabsf(ahead + (float)(e + 1)), x1); }
                        }
                        if (LUTS) { if (diagonals) { x0 += mine[e]; x1 += mine[e + 1]; } }
                        x[e / 2] = pack2(ex2(x0), ex2(x1));
                    }
                }
                if (careful) {
                    __syncwarp();
                    if (mixed) {
                        __syncwarp();
#pragma unroll
                        for (int e = 0; e < W; e += 4) {
                            const int4 d4 = *reinterpret_cast<const int4*>(docs + c0 + e);
                            keep(x[e / 2], e < to && d4.x == doc, e + 1 < to && d4.y == doc);
                            keep(x[e / 2 + 1], e + 2 < to && d4.z == doc, e + 3 < to && d4.w == doc);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < W; e += 2) keep(x[e / 2], e < to, e + 1 < to);
                    }
                }
                wait(dp_full, (uint32_t)n & 1u);
                fence_after_sync();
                {
                    uint32_t dv[W / 16][16];
#pragma unroll
                    for (int y = 0; y < W / 16; ++y) tmem_ld16_nowait(dp_col + c0 + 16 * y + lanes, dv[y]);
                    tmem_ld_wait();
                    if (careful) {
                        __syncwarp();
                        only_seen<CAP>(dv, slope, x);
                    }
                    const uint64_t minus_d = pack2(any ? -dsum : 0.0f, any ? -dsum : 0.0f);
#pragma unroll
                    for (int e = 0; e < W; e += 2) x[e / 2] = mul2(x[e / 2], add2(pack2(dv[e / 16][e % 16], dv[e / 16][e % 16 + 1]), minus_d));
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float y0, y1;
                        unpack2(CAP ? mul2(x[e], slope[CAP ? e : 0]) : x[e], y0, y1);
                        w[e] = pack_bf16(y0, y1);
                    }
                    tmem_st16(dp_col + c0 + lanes, w);
                }
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_full);
                ++n;
                some = true;
                if (sums) {
                    if (!diagonals) {
                        if (bucket0 != far_bucket) { flush(); far_bucket = bucket0; }
                        uint64_t y[2] = {x[0], x[1]};
#pragma unroll
                        for (int e = 2; e < W / 2; ++e) y[e & 1] = add2(y[e & 1], x[e]);
                        float y0, y1;
                        unpack2(add2(y[0], y[1]), y0, y1);
                        far_sum += y0 + y1;
                    } else {
                        // diagonal e - lane is complete in lane 31 after column e; those that end at the last column are in the other lanes
                        float a = 0.0f;
                        float* at = diag + warp * 64;
#pragma unroll
                        for (int e = 0; e < W; ++e) {
                            const float up = __shfl_up_sync(0xffffffffu, a, 1);
                            float y0, y1;
                            unpack2(x[e / 2], y0, y1);
                            a = (e & 1 ? y1 : y0) + (lane > 0 ? up : 0.0f);
                            if (lane == 31) at[e] = a;
                        }
                        if (lane < 31) at[W + 30 - lane] = a;       // diagonal 31 - lane; place x holds diagonal x - 31
                        __syncwarp();
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int d = lane + 32 * z;
                            grf_add_runs(my_bins, d < 63 ? bucket(p, j0 + c0 + d - 31 - sight.position(i0 + (warp & 3) * 32)) : -1, d < 63 ? at[d] : 0.0f);
                        }
                        __syncwarp();
                    }
                }
            }
            if (sums) flush();
            if (some) wait(dq_done, (uint32_t)kept & 1u);
            fence_after_sync();
            {
                const float by = CAP ? -p.scale : p.scale;           // (slope of the cap with its sign turned)
                __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.dq) + b * p.dqs[0] + h * p.dqs[1] + (int64_t)i * p.dqs[2];
#pragma unroll 1
                for (int y = 0; y < DP / 64; ++y) {
                    const int col = part * (DP / 4) + 16 * y;
                    uint32_t o[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0u;
                    if (some) tmem_ld16(acc + col + lanes, o);
                    if (i >= p.Nq) continue;
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        if (col + 8 * z >= p.d) continue;
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = any ? pack_bf16(__uint_as_float(o[8 * z + 2 * e]) * by, __uint_as_float(o[8 * z + 2 * e + 1]) * by) : 0u;
                        *reinterpret_cast<uint4*>(dst + col + 8 * z) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (some) {
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_read);
                ++kept;
            }
            if (sums) {
                with_workers();
                if (tid < grf_softmax_columns(p)) {
                    float sum = 0.0f;
                    for (int w = 0; w < WORKERS; ++w) {
                        sum += bins[w * 2 * GRF_MAX_BUCKETS + tid];
                        bins[w * 2 * GRF_MAX_BUCKETS + tid] = 0.0f;
                    }
                    p.dtable_part[(((int64_t)b * p.H + h) * blocks + I.qb) * grf_softmax_columns(p) + tid] = sum;
                }
                with_workers();
            }
        }
        fence_before_sync();
    }
    fence_before_sync();
    __syncthreads();
    if (warp == COPY) tmem_dealloc(tmem, 512u);
    if (tid == 0 && abort_flag) atomicExch(p.error_word, 1);
}

template <int DP, bool CAP, int BIAS>
__global__ void __launch_bounds__(THREADS, 1)
softmax_tc_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ CUtensorMap map_g, const __grid_constant__ grf_softmax_params p, const head_split f)
{
    using Sh = Grad<DP>;
    constexpr int NS = Sh::NS, QB = Sh::QB;
    constexpr int LUTS = BIAS == GRF_BIAS_BUCKETS ? 1 : 0;
    constexpr int SUM_ROW = DP + 4;
    extern __shared__ unsigned char smem_dyn[];
    __shared__ __align__(8) unsigned long long bars[4 * NS + 7 + 2 * QB];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    __shared__ float lut[LUTS ? 2 * 256 : 1];
    __shared__ grf_buckets bucket;
    __shared__ __align__(16) float info[NS][2][BT];             // -lse (in units of log 2; -infinity where P = 0) and -D of a tile's queries
    __shared__ __align__(16) int32_t info_doc[NS][BT];
    const int tid = threadIdx.x, lane = tid & 31, warp = uniform(tid >> 5);
    const uint32_t smem = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    uint32_t* bits = reinterpret_cast<uint32_t*>(smem_dyn + (smem - smem_u32(smem_dyn)) + Sh::TILE * (2 * QB + 2 * NS));
    const uint32_t k_at = smem, v_at = k_at + QB * Sh::TILE, q_at = v_at + QB * Sh::TILE, g_at = q_at + NS * Sh::TILE, bar0 = smem_u32(bars);
    auto q_full = [&](int s) { return bar0 + 8u * s; };
    auto g_full = [&](int s) { return bar0 + 8u * (NS + s); };
    auto empty = [&](int s) { return bar0 + 8u * (2 * NS + s); };
    auto ready = [&](int s) { return bar0 + 8u * (3 * NS + s); };
    const uint32_t one = bar0 + 8u * (4 * NS);
    const uint32_t s_full = one, dp_full = one + 8, p_full = one + 16, ds_full = one + 24, acc_done = one + 32, acc_read = one + 40, drain = one + 48;
    auto keys_full = [&](int y) { return one + 56 + 8u * y; };
    auto keys_empty = [&](int y) { return one + 56 + 8u * (QB + y); };
    float* sums = reinterpret_cast<float*>(smem_dyn + (smem - smem_u32(smem_dyn)));       // [dV, dK][key][SUM_ROW], once the tiles are done with

    // Blocks of keys, those that most queries see first, dealt out forwards and backwards in turn.  With documents, and where the heads that share keys
    // are split over a cluster (CTA x: part x % splits of block x / splits), every CTA has one.
    const int32_t units = p.B * p.KV, kblocks = (p.Nk + BT - 1) / BT, qblocks = (p.Nq + BT - 1) / BT;
    const bool alone = f.splits > 1 || p.q_doc;
    const uint32_t items = (uint32_t)units * (uint32_t)kblocks, rounds = alone ? 1u : (items - 1) / gridDim.x + 1;
    auto item = [&](uint32_t round) {
        return alone ? blockIdx.x / (uint32_t)f.splits : round * gridDim.x + ((round & 1) ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    };
    struct block_of {
        int32_t b, kvh, kb, j0, h_first, h_end;
        grf_sight sight;
        grad_tiles T;
        bool some;
        __device__ __forceinline__ block_of(const grf_softmax_params& p, const uint32_t* bits, int32_t units, int32_t qblocks, int splits, uint32_t x)
            : b((int32_t)(x % (uint32_t)units) / p.KV), kvh((int32_t)(x % (uint32_t)units) % p.KV), kb((int32_t)(x / (uint32_t)units)), j0(kb * BT), sight(p, b)
        {
            const int32_t part = (int32_t)blockIdx.x % splits;
            h_first = kvh * p.group + p.group * part / splits;
            h_end = kvh * p.group + p.group * (part + 1) / splits;
            // the first query that sees a key of the block, were there no documents
            int32_t first = 0;
            if (sight.order != GRF_ORDER_FULL && j0 >= sight.prefix) {
                const int64_t y = (int64_t)j0 - sight.start;
                first = y <= 0 ? 0 : y >= p.Nq ? qblocks : (int32_t)y / BT;
            }
            if (j0 >= sight.len) first = qblocks;
            T = grad_tiles{bits, first, qblocks, (qblocks + 31) / 32, sight.docs};
        }
        // (once the bits are there)
        __device__ __forceinline__ void look() { some = T.begin() < T.tiles; }
        // the block's tiles, head after head: true while there is one, with t and h advanced to it
        __device__ __forceinline__ bool step(int32_t& t, int32_t& h) const
        {
            t = T.next(t + 1);
            if (t >= T.tiles) {
                if (++h >= h_end) return false;
                t = T.begin();
            }
            return true;
        }
    };

    if (tid == 0) {
        abort_flag = 0;
        for (int s = 0; s < NS; ++s) { mbar_init(q_full(s), 1); mbar_init(g_full(s), 1); mbar_init(empty(s), 1); mbar_init(ready(s), 1); }
        for (int y = 0; y < QB; ++y) { mbar_init(keys_full(y), 1); mbar_init(keys_empty(y), 1); }
        mbar_init(s_full, 1); mbar_init(dp_full, 1); mbar_init(p_full, WORKERS); mbar_init(ds_full, WORKERS);
        mbar_init(acc_done, 1); mbar_init(acc_read, WORKERS); mbar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == COPY) tmem_alloc(&tmem_slot, 512u);
    if (LUTS) bucket.fill(p);
    if (p.q_doc) {
        const block_of I(p, bits, units, qblocks, f.splits, item(0));
        const grad_tiles& T = I.T;
        const int32_t b = I.b, first = T.first, j0 = I.j0;
        const grf_sight& sight = I.sight;
        const int4 kr = p.k_range[(int64_t)b * kblocks + I.kb];
        for (int32_t w = warp; w < T.words; w += THREADS / 32) {
            const int32_t t = w * 32 + lane;
            const bool in = t >= first && t < qblocks;
            const int4 qr = in ? p.q_range[(int64_t)b * qblocks + t] : make_int4(INT32_MAX, -1, 0, 0);
            const int what = in ? sight.tile(t * BT, min(t * BT + BT, p.Nq), j0, j0 + BT, qr, kr) : 0;
            const uint32_t seen = __ballot_sync(0xffffffffu, what != 0), whole = __ballot_sync(0xffffffffu, what == 2),
                           one_doc = __ballot_sync(0xffffffffu, one_document(qr, kr));
            if (lane == 0) { bits[w] = seen; bits[T.words + w] = whole; bits[2 * T.words + w] = one_doc; }
        }
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = (uint32_t)uniform((int32_t)tmem_slot);
    const uint32_t s_col = tmem, dp_col = tmem + 128, dv_acc = tmem + 256, dk_acc = tmem + 256 + DP;
    auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, &abort_flag)) != 0; };

    if (warp >= WORKERS) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LESS));
        if (warp == COPY) {
            bool ok = true;
            int32_t n = 0, kept = 0;
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                block_of I(p, bits, units, qblocks, f.splits, which);
                I.look();
                if (!I.some) continue;
                int32_t t = I.T.begin(), h = I.h_first;
                bool first = true;
                do {
                    const int s = n % NS;
                    if (n >= NS && !(ok = wait(empty(s), (uint32_t)(n / NS - 1) & 1u))) break;
                    expect_tx_elected(q_full(s), Sh::TILE);
                    expect_tx_elected(g_full(s), Sh::TILE);
                    for (int y = 0; y < DP / 64; ++y) {
                        load_box(q_at + s * Sh::TILE + y * HALF, &map_q, 64 * y, t * BT, p.qs[1] ? h : 0, p.qs[0] ? I.b : 0, q_full(s));
                        load_box(g_at + s * Sh::TILE + y * HALF, &map_g, 64 * y, t * BT, p.dos[1] ? h : 0, p.dos[0] ? I.b : 0, g_full(s));
                    }
                    ++n;
                    if (first) {
                        first = false;
                        const int y = kept % QB;
                        if (kept >= QB && !(ok = wait(keys_empty(y), (uint32_t)(kept / QB - 1) & 1u))) break;
                        expect_tx_elected(keys_full(y), 2 * Sh::TILE);
                        for (int z = 0; z < DP / 64; ++z) {
                            load_box(k_at + y * Sh::TILE + z * HALF, &map_k, 64 * z, I.j0, p.ks[1] ? I.kvh : 0, p.ks[0] ? I.b : 0, keys_full(y));
                            load_box(v_at + y * Sh::TILE + z * HALF, &map_v, 64 * z, I.j0, p.vs[1] ? I.kvh : 0, p.vs[0] ? I.b : 0, keys_full(y));
                        }
                        ++kept;
                    }
                } while (I.step(t, h));
            }
            if (!ok || *(volatile int*)&abort_flag) {
                for (int32_t x = max(0, n - NS); x < n; ++x) {
                    mbar_drain(q_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                    mbar_drain(g_full(x % NS), (uint32_t)(x / NS) & 1u, 20000000ll);
                }
                for (int32_t x = max(0, kept - QB); x < kept; ++x) mbar_drain(keys_full(x % QB), (uint32_t)(x / QB) & 1u, 20000000ll);
            }
        } else if (warp == ISSUE) {
            const int32_t steps = (p.d + 15) / 16;
            const uint64_t k_op = rows_operand(k_at), v_op = rows_operand(v_at), q_op = rows_operand(q_at), g_op = rows_operand(g_at), qc_op = columns_operand(q_at),
                           gc_op = columns_operand(g_at);
            bool ok = true;
            int32_t n = 0, kept = 0;                            // tiles, blocks that were seen
            auto make_scores = [&](int32_t n_) {
                const int s = n_ % NS;
                if (!wait(ready(s), (uint32_t)(n_ / NS) & 1u)) return false;    // (behind both copies)
                fence_after_sync();
                product_over_columns<DP>(s_col, lo32(k_op) + (kept % QB) * (Sh::TILE / 16), hi32(k_op), lo32(q_op) + s * (Sh::TILE / 16), hi32(q_op), steps);
                mma_commit(s_full);
                return true;
            };
            auto make_dp = [&](int32_t n_) {
                const int s = n_ % NS;
                product_over_columns<DP>(dp_col, lo32(v_op) + (kept % QB) * (Sh::TILE / 16), hi32(v_op), lo32(g_op) + s * (Sh::TILE / 16), hi32(g_op), steps);
                mma_commit(dp_full);
                return true;
            };
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                block_of I(p, bits, units, qblocks, f.splits, which);
                I.look();
                if (!I.some) continue;
                int32_t t = I.T.begin(), h = I.h_first;
                if (!(ok = wait(keys_full(kept % QB), (uint32_t)(kept / QB) & 1u) && make_scores(n) && make_dp(n))) break;
                bool more = true, first = true;
                for (; ok && more; ++n) {
                    const int s = n % NS;
                    more = I.step(t, h);
                    if (!(ok = wait(p_full, (uint32_t)n & 1u))) break;
                    // (the accumulators are the last block's until they are read)
                    if (first && kept > 0 && !(ok = wait(acc_read, (uint32_t)(kept - 1) & 1u))) break;
                    fence_after_sync();
                    product_of_parts<DP>(dv_acc, s_col, lo32(gc_op) + s * (Sh::TILE / 16), hi32(gc_op), first ? 0u : 1u);
                    if (more && !(ok = make_scores(n + 1))) break;
                    if (!(ok = wait(ds_full, (uint32_t)n & 1u))) break;
                    fence_after_sync();
                    product_of_parts<DP>(dk_acc, dp_col, lo32(qc_op) + s * (Sh::TILE / 16), hi32(qc_op), first ? 0u : 1u);
                    first = false;
                    mma_commit(empty(s));
                    if (!more) {
                        mma_commit(acc_done);
                        mma_commit(keys_empty(kept % QB));
                    } else ok = make_dp(n + 1);
                }
                ++kept;
            }
            if (!ok) {
                mma_commit(drain);
                mbar_drain(drain, 0u, 20000000ll);
            }
        } else if (warp == PREPARE) {
            // (the next tile's values travel while this one's copies do; a place is free when its copies have come, as these waited for it)
            int32_t n = 0;
            bool ok = true;
            for (uint32_t round = 0; round < rounds && ok; ++round) {
                const uint32_t which = item(round);
                if (which >= items) break;
                block_of I(p, bits, units, qblocks, f.splits, which);
                I.look();
                if (!I.some) continue;
                int32_t t = I.T.begin(), h = I.h_first;
                float lse[4], d[4];
                int32_t docs[4];
                auto fetch = [&]() {
                    const int64_t row = ((int64_t)I.b * p.H + h) * p.Nq + t * BT;
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int r = lane + 32 * y;
                        const bool in = t * BT + r < p.Nq;
                        lse[y] = in ? p.lse[row + r] : -CUDART_INF_F;
                        d[y] = in ? p.dsum[row + r] : 0.0f;
                        docs[y] = in && I.sight.docs ? max(p.q_doc[(int64_t)I.b * p.Nq + t * BT + r], -1) : -1;
                    }
                };
                fetch();
                bool more = true;
                while (more) {
                    const int s = n % NS;
                    if (!(ok = wait(q_full(s), (uint32_t)(n / NS) & 1u) && wait(g_full(s), (uint32_t)(n / NS) & 1u))) break;
                    uint32_t none[4];
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        const int r = lane + 32 * y;
                        const bool empty_row = fabsf(lse[y]) > LARGEST;
                        none[y] = __ballot_sync(0xffffffffu, t * BT + r < p.Nq && empty_row);
                        info[s][0][r] = empty_row ? -CUDART_INF_F : -lse[y] * GRF_LOG2E;
                        info[s][1][r] = empty_row ? 0.0f : -d[y];
                        if (I.sight.docs) info_doc[s][r] = docs[y];
                    }
                    if (none[0] | none[1] | none[2] | none[3]) {
                        // what rows of queries that see nothing hold does not matter: cleared, as 0 times it is summed below
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            if (none[y] >> lane & 1u) {
                                clear_row(q_at + s * Sh::TILE, lane + 32 * y, DP / 64);
                                clear_row(g_at + s * Sh::TILE, lane + 32 * y, DP / 64);
                            }
                        fence_async_smem();
                    }
                    __syncwarp();
                    arrive_elected(ready(s));
                    ++n;
                    more = I.step(t, h);
                    if (more) fetch();
                }
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(MORE));
        // (after a wait that gave up they go on, as in the other kernel)
        const int r = (warp & 3) * 32 + lane, part = warp >> 2, c0 = part * W;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const float to2 = p.scale * GRF_LOG2E, by_cap = CAP ? p.scale / p.cap : 0.0f, cap2 = p.cap * GRF_LOG2E;
        auto with_workers = [&]() { asm volatile("bar.sync 1, 512;" ::: "memory"); };
        int32_t n = 0, luts = 0, kept = 0;
        for (uint32_t round = 0; round < rounds; ++round) {
            const uint32_t which = item(round);
            if (which >= items) break;
            block_of I(p, bits, units, qblocks, f.splits, which);
            I.look();
            const grad_tiles& T = I.T;
            const grf_sight& sight = I.sight;
            const int32_t b = I.b, kvh = I.kvh, j0 = I.j0, j = j0 + r;
            int32_t doc = sight.docs && j < p.Nk ? p.k_doc[(int64_t)b * p.Nk + j] : -1;
            if (doc < 0) doc = INT32_MIN;                           // (equal to no query's: these are -1 where they are negative)
            const bool block_partial = j0 + BT > sight.len, ordered = sight.order != GRF_ORDER_FULL && j0 + BT > sight.prefix;
            if (I.some) {
                int32_t t = T.begin(), h = I.h_first;
                do {
                    const int s = n % NS;
                    const int32_t i0 = t * BT, pos0 = sight.position(i0);
                    const bool partial = sight.docs ? !T.whole(t) : block_partial || (ordered && pos0 < j0 + BT - 1);
                    // columns from `from` on see this key
                    // (none, where those that would are behind the last query: there P is 0 only if the key's scores are numbers)
                    int32_t from = j >= sight.len ? BT : sight.order == GRF_ORDER_FULL || j < sight.prefix ? 0 : min(max(j - pos0, 0), BT);
                    if (i0 + from >= p.Nq) from = BT;
                    const float slope2 = BIAS == GRF_BIAS_SLOPES ? grf_slope2(p, h) : 0.0f;
                    float bias2 = 0.0f;
                    bool diagonals = false;
                    const float* mine = lut;
                    if (LUTS) {
                        diagonals = bucket(p, j0 - pos0 - (BT - 1)) != bucket(p, j0 + BT - 1 - pos0);
                        if (diagonals) {
                            float* at = lut + (luts & 1) * 256;
                            if (tid < 256) at[tid] = tid < 2 * BT - 1 ? grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0 + tid - (BT - 1)) : 0.0f;
                            mine = at + (BT - 1 + r - c0);          // column e: mine[-e]
                            with_workers();
                            ++luts;
                        } else bias2 = grf_bias2<__nv_bfloat16>(p, bucket, h, j0 - pos0);
                    }
                    const int32_t since = from - c0;
                    wait(ready(s), (uint32_t)(n / NS) & 1u);
                    wait(s_full, (uint32_t)n & 1u);
                    fence_after_sync();
                    uint64_t x[W / 2], slope[CAP ? W / 2 : 1];      // P, then dS; t^2 - 1 of the cap
                    {
                        uint32_t sv[W / 16][16];
#pragma unroll
                        for (int y = 0; y < W / 16; ++y) tmem_ld16_nowait(s_col + c0 + 16 * y + lanes, sv[y]);
                        tmem_ld_wait();
                        if (CAP) capped<W / 16>(sv, by_cap);
                        const float ahead = (float)(j - pos0 - c0);
                        const uint64_t by = CAP ? pack2(cap2, cap2) : pack2(to2, to2), bias22 = pack2(bias2, bias2);
#pragma unroll
                        for (int e = 0; e < W; e += 2) {
                            const uint64_t v = pack2(sv[e / 16][e % 16], sv[e / 16][e % 16 + 1]);
                            if (CAP) slope[CAP ? e / 2 : 0] = fma2(v, v, pack2(-1.0f, -1.0f));
                            uint64_t at = *reinterpret_cast<const uint64_t*>(&info[s][0][c0 + e]);
                            if (LUTS) at = add2(at, bias22);
                            float x0, x1;
                            unpack2(fma2(v, by, at), x0, x1);
                            if (BIAS == GRF_BIAS_SLOPES) { x0 = fmaf(-slope2, fabsf(ahead - (float)e), x0); x1 = fmaf(-slope2, fabsf(ahead - (float)(e + 1)), x1); }
                            if (LUTS) { if (diagonals) { x0 += mine[-e]; x1 += mine[-e - 1]; } }
                            x[e / 2] = pack2(ex2(x0), ex2(x1));
                        }
                    }
                    if (partial) {
                        __syncwarp();
                        if (T.mixed(t)) {
                            __syncwarp();
#pragma unroll
                            for (int e = 0; e < W; e += 4) {
                                const int4 d4 = *reinterpret_cast<const int4*>(&info_doc[s][c0 + e]);
                                keep(x[e / 2], e >= since && d4.x == doc, e + 1 >= since && d4.y == doc);
                                keep(x[e / 2 + 1], e + 2 >= since && d4.z == doc, e + 3 >= since && d4.w == doc);
                            }
                        } else {
#pragma unroll
                            for (int e = 0; e < W; e += 2) keep(x[e / 2], e >= since, e + 1 >= since);
                        }
                    }
                    {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float y0, y1;
                            unpack2(x[e], y0, y1);
                            w[e] = pack_bf16(y0, y1);
                        }
                        tmem_st16(s_col + c0 + lanes, w);
                    }
                    tmem_st_wait();
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full);
                    wait(dp_full, (uint32_t)n & 1u);
                    fence_after_sync();
                    {
                        uint32_t dv[W / 16][16];
#pragma unroll
                        for (int y = 0; y < W / 16; ++y) tmem_ld16_nowait(dp_col + c0 + 16 * y + lanes, dv[y]);
                        tmem_ld_wait();
                        if (partial) {
                            __syncwarp();
                            only_seen<CAP>(dv, slope, x);
                        }
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < W; e += 2) {
                            const uint64_t minus_d = *reinterpret_cast<const uint64_t*>(&info[s][1][c0 + e]);
                            uint64_t d = mul2(x[e / 2], add2(pack2(dv[e / 16][e % 16], dv[e / 16][e % 16 + 1]), minus_d));
                            if (CAP) d = mul2(d, slope[CAP ? e / 2 : 0]);
                            float d0, d1;
                            unpack2(d, d0, d1);
                            w[e / 2] = pack_bf16(d0, d1);
                        }
                        tmem_st16(dp_col + c0 + lanes, w);
                    }
                    tmem_st_wait();
                    fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ds_full);
                    ++n;
                } while (I.step(t, h));
                wait(acc_done, (uint32_t)kept & 1u);
            }
            fence_after_sync();
            // the first two warpgroups have dV, half of its columns each, the others dK
            const bool is_dv = part < 2;
            const int col0 = (part & 1) * (DP / 2);
            const int64_t (&st)[3] = is_dv ? p.dvs : p.dks;
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(is_dv ? p.dv : p.dk) + b * st[0] + kvh * st[1] + (int64_t)j * st[2];
            const float by = is_dv ? 1.0f : CAP ? -p.scale : p.scale;       // (slope of the cap with its sign turned)
#pragma unroll 1
            for (int y = 0; y < DP / 32; ++y) {
                uint32_t o[16];
                const int col = col0 + 16 * y;
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0u;
                if (I.some) tmem_ld16((is_dv ? dv_acc : dk_acc) + col + lanes, o);
                if (f.splits > 1) {
                    // for the other CTAs of the cluster, where the tiles were
                    float4* at = reinterpret_cast<float4*>(sums + ((is_dv ? 0 : 1) * BT + r) * SUM_ROW + col);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        at[e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3]));
                    continue;
                }
                if (j >= p.Nk) continue;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    if (col + 8 * z >= p.d) continue;
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = pack_bf16(__uint_as_float(o[8 * z + 2 * e]) * by, __uint_as_float(o[8 * z + 2 * e + 1]) * by);
                    *reinterpret_cast<uint4*>(dst + col + 8 * z) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (I.some) {
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_read);
                ++kept;
            }
        }
        fence_before_sync();
    }
    fence_before_sync();
    __syncthreads();
    if (warp == COPY) tmem_dealloc(tmem, 512u);
    if (f.splits > 1) {
        // sums over the heads' CTAs, in order; every CTA has a share of the rows
        const block_of I(p, bits, units, qblocks, f.splits, item(0));
        const int32_t b = I.b, kvh = I.kvh, j0 = I.j0;
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
        constexpr int PIECES = DP / 8;
        const int rank = (int)cluster.block_rank(), r0 = BT * rank / f.splits, r1 = BT * (rank + 1) / f.splits;
        for (int x = tid; x < 2 * (r1 - r0) * PIECES; x += THREADS) {
            const int what = x / ((r1 - r0) * PIECES), r = r0 + x / PIECES % (r1 - r0), col = x % PIECES * 8;
            if (j0 + r >= p.Nk || col >= p.d) continue;
            float v[8] = {};
            for (int s = 0; s < f.splits; ++s) {
                const float4* at = reinterpret_cast<const float4*>(cluster.map_shared_rank(sums + (what * BT + r) * SUM_ROW + col, s));
                const float4 u = at[0], w = at[1];
                v[0] += u.x; v[1] += u.y; v[2] += u.z; v[3] += u.w;
                v[4] += w.x; v[5] += w.y; v[6] += w.z; v[7] += w.w;
            }
            const int64_t (&st)[3] = what == 0 ? p.dvs : p.dks;
            const float by = what == 0 ? 1.0f : CAP ? -p.scale : p.scale;
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(what == 0 ? p.dv : p.dk) + b * st[0] + kvh * st[1] + (int64_t)(j0 + r) * st[2] + col;
            *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(v[0] * by, v[1] * by), pack_bf16(v[2] * by, v[3] * by), pack_bf16(v[4] * by, v[5] * by),
                                                        pack_bf16(v[6] * by, v[7] * by));
        }
        cluster.sync();                                         // nobody's shared memory goes while it is read
    }
    if (tid == 0 && abort_flag) atomicExch(p.error_word, 1);
}

struct grad_maps { CUtensorMap q, k, v, g; };

template <int DP, bool CAP, int BIAS> int launch(grf_ctx* ctx, const grf_softmax_params& p, const grad_maps& m)
{
    using Sh = Grad<DP>;
    auto bits = [](int32_t tokens) { return 12 * (size_t)(grf_ceil_div(tokens, BT) / 32 + 1); };
    const size_t dq_smem = Sh::SMEM + (p.q_doc ? bits(p.Nk) : 0), dkv_smem = Sh::SMEM + (p.q_doc ? bits(p.Nq) : 0);
    // (the most of any call, as in the forward pass)
    constexpr auto most = cudaFuncAttributeMaxDynamicSharedMemorySize;
    GRF_CUDA_TRY(cudaFuncSetAttribute(softmax_tc_dq_kernel<DP, CAP, BIAS>, most, (int)(Sh::SMEM + bits(MOST_WITH_DOCS))));
    GRF_CUDA_TRY(cudaFuncSetAttribute(softmax_tc_dkv_kernel<DP, CAP, BIAS>, most, (int)(Sh::SMEM + bits(MOST_WITH_DOCS))));
    grf_softmax_scope scope(ctx, "grf:softmax_gradients", 2);
    // The heads that share a key head are split over a cluster's CTAs, which add their sums through distributed shared memory, where there are
    // too few blocks of keys to fill the device evenly (causal ones take 1 to Nq / 128 tiles a head).  16 heads, 4 of keys,
    // x 4096 causal: dK and dV 403 us by one CTA per block, training step 680 -> 552.
    head_split f = {1};
    const int64_t blocks = (int64_t)p.B * p.KV * grf_ceil_div(p.Nk, BT);
    while (f.splits < p.group && f.splits < 8 && blocks * f.splits < 4 * ctx->sm_count) ++f.splits;
    cudaLaunchConfig_t cfg = {};
    const int64_t q_blocks = (int64_t)p.B * p.H * grf_ceil_div(p.Nq, BT);
    cfg.gridDim = dim3((unsigned)(f.splits > 1 || p.q_doc || blocks < ctx->sm_count ? blocks * f.splits : ctx->sm_count));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = dkv_smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)f.splits;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    GRF_CUDA_TRY(cudaLaunchKernelEx(&cfg, softmax_tc_dkv_kernel<DP, CAP, BIAS>, m.q, m.k, m.v, m.g, p, f));
    softmax_tc_dq_kernel<DP, CAP, BIAS><<<(unsigned)(p.q_doc || q_blocks < ctx->sm_count ? q_blocks : ctx->sm_count), THREADS, dq_smem, ctx->stream>>>(m.q, m.k, m.v, m.g, p);
    return cudaGetLastError() == cudaSuccess ? GRF_OK : GRF_ERR_CUDA;
}

template <int DP> int choose(grf_ctx* ctx, const grf_softmax_params& p, const grad_maps& m)
{
    if (p.cap > 0.0f) {
        if (p.bias == GRF_BIAS_NONE) return launch<DP, true, GRF_BIAS_NONE>(ctx, p, m);
        if (p.bias == GRF_BIAS_SLOPES) return launch<DP, true, GRF_BIAS_SLOPES>(ctx, p, m);
        return launch<DP, true, GRF_BIAS_BUCKETS>(ctx, p, m);
    }
    if (p.bias == GRF_BIAS_NONE) return launch<DP, false, GRF_BIAS_NONE>(ctx, p, m);
    if (p.bias == GRF_BIAS_SLOPES) return launch<DP, false, GRF_BIAS_SLOPES>(ctx, p, m);
    return launch<DP, false, GRF_BIAS_BUCKETS>(ctx, p, m);
}

}  // namespace

int grf_softmax_tc_backward(grf_ctx* ctx, const grf_softmax_params& p)
{
    if (p.q_doc && (p.Nk > MOST_WITH_DOCS || p.Nq > MOST_WITH_DOCS)) return 1;
    grad_maps m;
    if (!grf_make_token_box_map(&m.q, p.q, p.qs, p.B, p.H, p.Nq, p.d) || !grf_make_token_box_map(&m.k, p.k, p.ks, p.B, p.KV, p.Nk, p.d) ||
        !grf_make_token_box_map(&m.v, p.v, p.vs, p.B, p.KV, p.Nk, p.d) || !grf_make_token_box_map(&m.g, p.dout, p.dos, p.B, p.H, p.Nq, p.d)) return 1;
    return p.d <= 64 ? choose<64>(ctx, p, m) : choose<128>(ctx, p, m);
}
