// Gradient of the token log-probabilities for sm_100a.  With z[t][v] = f hidden[t] . lm_head[v] (f: the inverse
// temperature) and p[t][v] = exp(z[t][v] - lse[t]):
//   d_z[t][v]    = f d_logprob[t] ([v == target[t]] - p[t][v])
//   d_hidden[t]  = sum_v d_z[t][v] lm_head[v],      d_lm_head[v] = sum_t d_z[t][v] hidden[t]
// Three matrix products of 2 T V H operations each, which is what bounds a call of more than some hundred rows: the logits
// are computed again (they were never stored), d_z leaves that product's epilogue as bf16 [rows of a chunk][T], and both
// gradients are products with it.  d_z is the one rounding on the way: every term of a gradient is off by 2^-8 of itself at
// most, rounded independently.  The target's term is mostly the largest by far, and its rounding would be one error for a whole row, so
// what it lost is kept (rho [T], fp32) and added to both gradients in fp32 before they are rounded.  Sums are fp32 in tensor memory.
//
// Tokens without a gradient (d_logprob 0: prompts, padding) take no part.  In calls of more than one row tile the others' rows are
// gathered first, and everything after goes by their number, which stays on the device: the persistent grids read it.
// In calls of one, whose launches are what they take, all rows go through: d_z is 0 for such tokens, and DZ leaves TABLE a copy of the hidden
// rows with zeros for theirs, whatever they hold.
//
// One kernel, launched for DZ and then for the gradients: persistent CTA pairs that walk units of one 256 x 256 output tile each: a TMA warp streams
// 64-wide slices of the contracted axis through a ring, an MMA warp issues M256 x N256 x K16 MMAs into one of two
// accumulators, eight epilogue warps take the other one out through shared memory and tiled TMA stores.  An operand whose
// contracted axis is not its contiguous one is read as it lies (MN-major descriptors): nothing is transposed.
//   DZ      A = lm_head (K-major), B = hidden (K-major)        rows: vocabulary, columns: tokens, contracted: H
//   TABLE   A = d_z (K-major),     B = hidden (N-major)        rows: vocabulary, columns: H,      contracted: tokens
//   HIDDEN  A = lm_head (M-major), B = d_z (N-major)           rows: H,          columns: tokens, contracted: vocabulary
// Tokens are columns wherever they are not contracted: an MMA has 256 rows whatever is in them, but as few as 32 columns where the
// last tile has no more (contracted, they end at a multiple of 16).  So d_z lies as [vocabulary][tokens] and the sums behind d_hidden as [H][tokens]; the fold turns them.
// HIDDEN has few tiles with a long contracted axis (4001 x 3584: 224 tiles, 2376 slices, for 74 pairs), so the tiles of the last,
// partial round are split along it, into parts that are summed in ascending order by lpb_fold_kernel; TABLE's many short units follow.  Vocabularies whose d_z
// exceeds the scratch are taken in chunks; the sums behind d_hidden then grow in fp32, one addition an element and chunk, in order.
#include <type_traits>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

namespace lpb {
constexpr int DZ = 0, TABLE = 1, HIDDEN = 2, BOTH = 3;        // what a launch does
constexpr int TILE = 256;                    // rows (of a pair) and columns of a unit
constexpr uint32_t OP_BYTES = 128 * 128;     // an operand's share of a stage: 128 rows or columns x 64 of the contracted axis
constexpr uint32_t STAGE_BYTES = 2 * OP_BYTES;
constexpr int STAGES = 5;
constexpr uint32_t STG_BYTES = 128 * 128;    // output staging: 128 rows x 128 bytes, two buffers for each group of epilogue warps
constexpr uint32_t OFF_STG = STAGES * STAGE_BYTES;
constexpr uint32_t OFF_BAR = OFF_STG + 4 * STG_BYTES;
constexpr uint32_t BYTES = OFF_BAR + 256;
constexpr uint32_t ALLOC = BYTES + 1024;     // (1792 bytes are left for what is declared in the kernel)
constexpr int BAND = 16;                     // DZ: token tiles whose hidden rows stay in L2 while lm_head streams by
constexpr int THREADS = 320;                 // warp 0 TMA, warp 1 MMA, warps 2..9 epilogue: two groups of four
constexpr int HITS = 32;                     // TABLE: targets that a warp's list holds
constexpr int PAIRS = 74;                    // CTA pairs of a B200, by which HIDDEN's tiles are cut on any device
constexpr int MOST_PARTS = 4 * PAIRS;        // HIDDEN: split tiles' parts, four rounds
}  // namespace lpb

// Adds a staged fp32 tile to global memory (bulk async group).
__device__ __forceinline__ void tma_add_2d(const CUtensorMap* m, uint32_t src, int c0, int c1) {
    asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(m)),
                 "r"(src), "r"(c0), "r"(c1)
                 : "memory");
}

// Pair MMA chain over a 64-wide slice, its four K16 steps SA and SB (in 16-byte units) apart: 2 in a K-major operand (32 bytes of
// a 128-byte row), 128 in an MN-major one (16 rows of 128 bytes).
template <int SA, int SB>
__device__ __forceinline__ void mma_ss_chain4_pair_steps(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p0, pt, e;\n\telect.sync _|e, 0xffffffff;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p0, %4, 0;\n\tsetp.eq.b32 pt, 0, 0;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p0;\n\t"
        "add.u64 da, %1, %5;\n\tadd.u64 db, %2, %8;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.u64 da, %1, %6;\n\tadd.u64 db, %2, %9;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.u64 da, %1, %7;\n\tadd.u64 db, %2, %10;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "}" ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "n"(SA), "n"(2 * SA), "n"(3 * SA), "n"(SB), "n"(2 * SB), "n"(3 * SB)
        : "memory");
}
// The same for the first `steps` (1..4) of the four.
template <int SA, int SB>
__device__ __forceinline__ void mma_ss_chain_pair_steps(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, int steps) {
    asm volatile(
        "{\n\t.reg .pred p0, pt, e, e1, e2, e3;\n\telect.sync _|e, 0xffffffff;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p0, %4, 0;\n\tsetp.eq.b32 pt, 0, 0;\n\t"
        "setp.gt.and.s32 e1, %11, 1, e;\n\tsetp.gt.and.s32 e2, %11, 2, e;\n\tsetp.gt.and.s32 e3, %11, 3, e;\n\t"
        "@e tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p0;\n\t"
        "add.u64 da, %1, %5;\n\tadd.u64 db, %2, %8;\n\t"
        "@e1 tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.u64 da, %1, %6;\n\tadd.u64 db, %2, %9;\n\t"
        "@e2 tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "add.u64 da, %1, %7;\n\tadd.u64 db, %2, %10;\n\t"
        "@e3 tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, pt;\n\t"
        "}" ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "n"(SA), "n"(2 * SA), "n"(3 * SA), "n"(SB), "n"(2 * SB), "n"(3 * SB), "r"(steps)
        : "memory");
}

// Arrives on a barrier of either CTA.  What it announces is that tensor memory has been read, which the tcgen05 fence before it orders: memory
// needs no ordering, and a release to the cluster waits for the CTA's stores (2000 clk of a unit's 4600 where the output bounds a call).
__device__ __forceinline__ void lpb_arrive(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// One warp of both CTAs: all of tensor memory, two 256-column accumulators.  Before the CTA's dependents are released.
constexpr uint32_t LPB_TMEM_COLS = 512;
__device__ __forceinline__ void lpb_take_tensor_memory(volatile uint32_t* slot) {
    tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(slot)), LPB_TMEM_COLS);
    tmem_relinquish_pair();
}

// What a launch has to do, by the number of rows that take part.
struct LpbShape {
    int rows;                    // tokens
    int tokens, words, channels; // tiles of 256 of the tokens, the chunk's vocabulary, H
    int whole, split;            // HIDDEN: tiles done whole, parts of each of the others
    int hidden_units, units;     // BOTH: HIDDEN's units come first
};
// The tiles of the last round of pairs, split so that the round costs least in slices, a unit's epilogue and first loads counting as
// six and a part's way through memory as a quarter.
__host__ __device__ inline int lpb_split_cost(int s, int rest, int slices) {
    return (rest * s + lpb::PAIRS - 1) / lpb::PAIRS * ((slices + s - 1) / s + 6) * 4 + rest * s;
}
// What the choice goes by: tiles of the last round for so many rows, slices of a whole chunk, parts at most (the last chunk, the
// shortest, has a slice for each).
struct LpbRest {
    int rest, slices, most;
};
__host__ __device__ inline LpbRest lpb_rest(const LogprobBwdParams& p, int rows) {
    LpbRest r;
    r.rest = (rows + lpb::TILE - 1) / lpb::TILE * ((p.H + lpb::TILE - 1) / lpb::TILE) % lpb::PAIRS;
    r.slices = ((p.chunk < p.V ? p.chunk : p.V) + 63) / 64;
    const int least = (p.V - (p.V - 1) / p.chunk * p.chunk + 63) / 64, room = lpb::MOST_PARTS / (r.rest > 1 ? r.rest : 1);
    r.most = least < room ? least : room;
    if (r.most > 64) r.most = 64;
    return r;
}
__device__ __forceinline__ LpbShape lpb_shape(const LogprobBwdParams& p, int kind) {
    using namespace lpb;
    LpbShape g;
    g.rows = p.count ? __ldcg(p.count) : static_cast<int>(p.T);
    g.tokens = (g.rows + TILE - 1) / TILE;
    g.words = (p.nv + TILE - 1) / TILE;
    g.channels = (p.H + TILE - 1) / TILE;
    const int tiles = g.tokens * g.channels, rest = tiles % PAIRS;
    g.whole = tiles - rest;
    g.split = p.count ? __ldcg(p.count + 1) : p.split;
    g.hidden_units = kind == HIDDEN || kind == BOTH ? g.whole + rest * g.split : 0;
    g.units = kind == DZ ? g.tokens * g.words : g.hidden_units + (kind == HIDDEN ? 0 : g.words * g.channels);
    return g;
}

struct LpbUnit {
    bool table;                  // TABLE's, of the gradients'
    int row, col, cols;          // of the output tile; its columns, 256 or fewer
    int k0, k1;                  // slices of 64 of the contracted axis
    int slot;                    // HIDDEN: part of a split tile (its place in the parts' buffer), -1: a whole tile
};
// Columns of a token tile, in steps of the pair MMA's 32.  (What its accumulator holds behind them is not used.)
__device__ __forceinline__ int lpb_cols(const LpbShape& g, int first) { return min(lpb::TILE, (g.rows - first + 31) / 32 * 32); }
template <int KIND>
__device__ __forceinline__ LpbUnit lpb_unit(const LogprobBwdParams& p, const LpbShape& g, int u) {
    using namespace lpb;
    LpbUnit x;
    x.slot = -1;
    x.k0 = 0;
    x.table = KIND == TABLE || (KIND == BOTH && u >= g.hidden_units);
    if (KIND == DZ) {
        // token tiles fastest inside a band, so that the pairs at work share a few steps of lm_head, and another one first for each
        // step: the narrow last tiles go to all pairs in turn
        const int per_band = BAND * g.words, band = u / per_band, rem = u - band * per_band;
        const int tiles = min(BAND, g.tokens - band * BAND), word = rem / tiles;
        x.row = word * TILE;
        x.col = (band * BAND + (rem + word) % tiles) * TILE;
        x.cols = lpb_cols(g, x.col);
        x.k1 = p.H / 64;
        return x;
    }
    if (x.table) {
        const int tile = u - g.hidden_units;
        x.row = tile / g.channels * TILE;
        x.col = tile % g.channels * TILE;
        x.cols = TILE;
        x.k1 = (g.rows + 63) / 64;
        return x;
    }
    const int slices = (p.nv + 63) / 64;
    int tile = u;
    x.k1 = slices;
    if (u >= g.whole) {
        const int rest = g.tokens * g.channels - g.whole, q = u - g.whole, part = q / rest;
        tile = g.whole + q % rest;
        x.k0 = static_cast<int>(static_cast<long long>(slices) * part / g.split);
        x.k1 = static_cast<int>(static_cast<long long>(slices) * (part + 1) / g.split);
        x.slot = q;
    }
    x.row = tile % g.channels * TILE;                      // (the last token tile's come last, mostly among the split ones)
    x.col = tile / g.channels * TILE;
    x.cols = lpb_cols(g, x.col);
    return x;
}

// TABLE: calls f(token, row) for the tokens whose target is one of a warp's 32 rows from `first` on, in ascending order; whole warp.
template <class F>
__device__ __forceinline__ void lpb_targets(const int32_t* target, int tokens, int first, int lane, F&& f) {
    for (int t0 = 0; t0 < tokens; t0 += 128) {
        unsigned row[4], any = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t0 + 32 * j + lane;
            row[j] = t < tokens ? static_cast<unsigned>(target[t] - first) : 32u;
            any |= row[j] < 32u;
        }
        if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            for (unsigned hit = __ballot_sync(0xffffffffu, row[j] < 32u); hit; hit &= hit - 1) {
                const int src = __ffs(hit) - 1;
                f(t0 + 32 * j + src, static_cast<int>(__shfl_sync(0xffffffffu, row[j], src)));
            }
    }
}
// v += a * N bf16 from x on (N a multiple of 8)
template <int N>
__device__ __forceinline__ void lpb_add_row(uint32_t (&v)[N], float a, const __nv_bfloat16* x) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(x + i);
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[i + 2 * j] = __float_as_uint(fmaf(a, __uint_as_float(w[j] << 16), __uint_as_float(v[i + 2 * j])));
            v[i + 2 * j + 1] = __float_as_uint(fmaf(a, __uint_as_float(w[j] & 0xffff0000u), __uint_as_float(v[i + 2 * j + 1])));
        }
    }
}

template <int KIND>
__global__ void __launch_bounds__(lpb::THREADS, 1) lpb_kernel(const __grid_constant__ LogprobBwdMaps maps, const __grid_constant__ LogprobBwdParams p) {
    using namespace lpb;
    constexpr bool GRADS = KIND != DZ, TABLES = KIND == TABLE || KIND == BOTH;
    const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
    const uint32_t rank = cluster_ctarank();     // 0 = the CTA that issues the pair's MMAs
    const int first = static_cast<int>(blockIdx.x >> 1), stride = static_cast<int>(gridDim.x >> 1);
    __shared__ LpbShape shape;
    __shared__ int hits[TABLES ? 8 : 1][TABLES ? HITS : 1];
    __shared__ __align__(16) float token_factor[2][GRADS ? 1 : 64], token_lse2[2][GRADS ? 1 : 64];
    __shared__ __align__(16) int token_target[2][GRADS ? 1 : 64];

    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_addr = smem_u32(smem_raw);
    const uint32_t pad = (1024u - (raw_addr & 1023u)) & 1023u;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sbase = raw_addr + pad;
    const uint32_t bar_full = sbase + OFF_BAR;               // STAGES barriers
    const uint32_t bar_empty = bar_full + 8 * STAGES;        // STAGES barriers
    const uint32_t bar_acc_full = bar_empty + 8 * STAGES;    // 2
    const uint32_t bar_acc_empty = bar_acc_full + 16;        // 2
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + OFF_BAR + 8 * (2 * STAGES + 4));
    volatile int* abort_word = reinterpret_cast<volatile int*>(smem + OFF_BAR + 8 * (2 * STAGES + 4) + 4);

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(bar_acc_full + 8 * b, 1);
            mbar_init(bar_acc_empty + 8 * b, 16);            // the epilogue warps of both CTAs
        }
        fence_barrier_init();
        tma_prefetch_desc(&maps.dz_k);
        tma_prefetch_desc(GRADS ? &maps.head_mn : &maps.head_k);
        tma_prefetch_desc(GRADS ? &maps.hidden_mn : &maps.hidden_k);
    }
    if (warp == 1) lpb_take_tensor_memory(tmem_slot);
    pdl_wait();
    if (tid == 0) {
        *abort_word = (*reinterpret_cast<volatile int*>(p.dev_status) & TIK_DEV_WAIT_EXPIRED) ? 1 : 0;
        shape = lpb_shape(p, KIND);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();            // the peer's barriers exist before anything signals them
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    const LpbShape g = shape;
    const uint32_t lead_full = mapa_cluster(bar_full, 0);
    const uint32_t lead_acc_empty = mapa_cluster(bar_acc_empty, 0);
    const uint32_t peer_empty = mapa_cluster(bar_empty, 1);
    const uint32_t peer_acc_full = mapa_cluster(bar_acc_full, 1);
    const int half = 128 * static_cast<int>(rank);

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        if (lane == 0) {
            uint32_t it = 0;
            for (int u = first; u < g.units; u += stride) {
                const LpbUnit x = lpb_unit<KIND>(p, g, u);
                // each CTA stages its own 128 rows of A and its half of B's columns (and what is behind them, up to 128); what lies outside
                // the tensors arrives as zeros
                const int a0 = x.row + half, b0 = x.col + x.cols / 2 * static_cast<int>(rank);
                for (int kb = x.k0; kb < x.k1; ++kb, ++it) {
                    if (*abort_word) break;      // a wait expired somewhere: stop issuing copies
                    const int s = it % STAGES;
                    const uint32_t use = it / STAGES, dst = sbase + s * STAGE_BYTES;
                    if (use > 0) mbar_wait(bar_empty + 8 * s, (use - 1) & 1, abort_word, p.dev_status);
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2 * STAGE_BYTES);   // both CTAs' bytes
                    const uint32_t bar = lead_full + 8 * s;
                    if (!GRADS) {
                        tma_load_2d_pair(dst, &maps.head_k, bar, kb * 64, p.v0 + a0);
                        tma_load_2d_pair(dst + OP_BYTES, &maps.hidden_k, bar, kb * 64, b0);
                    } else {
                        if (x.table) {
                            tma_load_2d_pair(dst, &maps.dz_k, bar, kb * 64, a0);
                        } else {
                            tma_load_2d_pair(dst, &maps.head_mn, bar, a0, p.v0 + kb * 64);
                            tma_load_2d_pair(dst + OP_BYTES / 2, &maps.head_mn, bar, a0 + 64, p.v0 + kb * 64);
                        }
                        const CUtensorMap* const b = x.table ? &maps.hidden_mn : &maps.dz_mn;
                        tma_load_2d_pair(dst + OP_BYTES, b, bar, b0, kb * 64);
                        tma_load_2d_pair(dst + OP_BYTES + OP_BYTES / 2, b, bar, b0 + 64, kb * 64);
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (rank == 0) {
            const uint32_t tmem_u = warp_uniform(tmem);
            uint32_t it = 0, acc = 0;
            for (int u = first; u < g.units; u += stride, ++acc) {
                const LpbUnit x = lpb_unit<KIND>(p, g, u);
                const int buf = acc & 1;
                const uint32_t use = acc >> 1;
                if (use > 0) mbar_wait_warp(bar_acc_empty + 8 * buf, (use - 1) & 1, abort_word, p.dev_status);
                tc_fence_after();
                for (int kb = x.k0; kb < x.k1; ++kb, ++it) {
                    if (*abort_word) break;
                    const int s = it % STAGES;
                    mbar_wait_warp(bar_full + 8 * s, (it / STAGES) & 1, abort_word, p.dev_status);
                    tc_fence_after();
                    const uint32_t a = sbase + s * STAGE_BYTES, b = a + OP_BYTES;
                    // MN-major: 64 columns of the axis per 128-byte row, the next 64 half an operand further
                    const uint32_t more = kb > x.k0 ? 1u : 0u, d = tmem_u + buf * TILE;
                    const uint32_t idesc = mma_idesc_bf16(256, KIND == TABLE ? TILE : x.cols, GRADS, KIND == HIDDEN || (KIND == BOTH && !x.table));
                    if (!GRADS)
                        mma_ss_chain4_pair_steps<2, 2>(d, smem_desc_sw128(a, 0, 1024), smem_desc_sw128(b, 0, 1024), idesc, more);
                    else if (x.table)
                        mma_ss_chain_pair_steps<2, 128>(d, smem_desc_sw128(a, 0, 1024), smem_desc_sw128(b, OP_BYTES / 2, 1024), idesc, more,
                                                        min(4, (g.rows - 64 * kb + 15) / 16));      // (no more than there are tokens)
                    else
                        mma_ss_chain4_pair_steps<128, 128>(d, smem_desc_sw128(a, OP_BYTES / 2, 1024), smem_desc_sw128(b, OP_BYTES / 2, 1024), idesc, more);
                    mma_commit_pair(bar_empty + 8 * s);
                    mma_commit_pair(peer_empty + 8 * s);
                }
                mma_commit_pair(bar_acc_full + 8 * buf);
                mma_commit_pair(peer_acc_full + 8 * buf);
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue (warps 2..9), thread per row
        // The two groups take the tile's 128-byte wide pieces in turns (d_lm_head of 64 rows, 1.1 GB: one group 298 us, two
        // and a buffer more each 286, and with a relaxed arrival 214).
        const int quarter = warp & 3, group = (warp - 2) >> 2;         // TMEM lane quarter of this warp
        const int row = quarter * 32 + lane;
        if (!GRADS && p.clean) {
            // 256 channels of a token a warp, while the first accumulator is being filled
            const int pieces = (p.H + 255) / 256, T = static_cast<int>(p.T);
            for (int i = static_cast<int>(blockIdx.x) * 8 + warp - 2; i < T * pieces; i += static_cast<int>(gridDim.x) * 8) {
                const int t = i / pieces, h = (i - t * pieces) * 256 + 8 * lane, target = p.target[t];
                const bool on = __fmul_rn(p.d_logprob[t], p.inv_temperature) != 0.0f && target >= 0 && target < p.V;
                const long long at = static_cast<long long>(t) * p.H + h;
                if (h < p.H) *reinterpret_cast<uint4*>(p.clean + at) = on ? *reinterpret_cast<const uint4*>(p.hidden + at) : make_uint4(0, 0, 0, 0);
            }
        }
        uint32_t acc = 0;
        const bool storer = (warp == 2 || warp == 6) && lane == 0;
        uint32_t piece = 0;
        // the group's buffer of the piece before last, when its store has finished reading
        auto stage = [&]() {
            if (storer) tma_store_wait_read1();
            named_bar_sync(1 + group, 128);
            return smem + OFF_STG + (2 * group + (piece++ & 1)) * STG_BYTES;
        };
        for (int u = first; u < g.units; u += stride, ++acc) {
            const LpbUnit x = lpb_unit<KIND>(p, g, u);
            const int buf = acc & 1, row0 = x.row + half;
            float c = 0.0f, lse2 = 0.0f;                   // DZ: what a token of the group's pieces has of its own, a token a thread;
            int target = -1;                               // one that takes no part has factor 0
            if (!GRADS) {
                const int k = tid & 127, r = x.col + 64 * (group + 2 * (k >> 6)) + (k & 63);
                if (r < g.rows) {
                    const int t = p.index ? p.index[r] : r;
                    target = p.target[t];
                    c = __fmul_rn(p.d_logprob[t], p.inv_temperature);
                    lse2 = __fmul_rn(p.lse[t], LOG2E_F);
                    if (c != 0.0f && (target < 0 || target >= p.V)) {      // no gradient
                        c = 0.0f;
                        atomicOr(p.dev_status, TIK_DEV_BAD_TARGET);
                    }
                }
            }
            int nhits = 0;                                 // tokens whose targets are this warp's rows
            unsigned mine = 0;                             // ... and this lane's, of those in the list
            const int first_row = p.v0 + row0 + quarter * 32;
            const bool table = TABLES && x.table;
            if (table) {
                lpb_targets(p.row_target, g.rows, first_row, lane, [&](int t, int r) {
                    if (nhits < HITS) {
                        if (lane == 0) hits[warp - 2][nhits] = t;
                        mine |= lane == r ? 1u << nhits : 0u;
                    }
                    ++nhits;
                    // its hidden row's part comes to L1 while the accumulator is being filled
                    if (lane < 4 && x.col + 64 * lane < p.H)
                        asm volatile("prefetch.global.L1 [%0];" ::"l"(p.rows + static_cast<long long>(t) * p.H + x.col + 64 * lane));
                });
                __syncwarp();
            }
            // what the targets' terms lost in rounding, added to columns col .. of the rows that they belong to
            auto add_lost = [&](auto& v, int col) {
                auto one = [&](int t) { lpb_add_row(v, p.rho[t], p.rows + static_cast<long long>(t) * p.H + col); };
                if (nhits <= HITS)
                    for (unsigned rest = mine; rest; rest &= rest - 1) one(hits[warp - 2][__ffs(rest) - 1]);
                else
                    lpb_targets(p.row_target, g.rows, first_row, lane, [&](int t, int r) {
                        if (lane == r) one(t);
                    });
                __syncwarp();
            };
            mbar_wait(bar_acc_full + 8 * buf, (acc >> 1) & 1, abort_word, p.dev_status);
            tc_fence_after();
            const uint32_t taddr = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * TILE;
            const bool f32_out = GRADS && (!table || p.table_fp32);
            if (!f32_out) {
                const int limit = !GRADS ? x.col + x.cols : p.H;           // (of a token tile all 64 columns of a piece, zeros behind the last)
                const int v_row = p.v0 + row0 + row;                       // DZ: this thread's word
                const float scale2 = !GRADS ? __fmul_rn(p.inv_temperature, LOG2E_F) : 0.0f;
#pragma unroll 1
                for (int q = group; q < TILE / 64; q += 2) {
                    if (x.col + 64 * q >= limit) break;    // uniform: columns past the output
                    uint32_t v[64];
                    tmem_ld32(taddr + 64 * q, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
                    tmem_ld32(taddr + 64 * q + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
                    tmem_wait_ld();
                    if (table && x.k1 == 0) {      // no token takes part: the accumulator was not written
#pragma unroll
                        for (int i = 0; i < 64; ++i) v[i] = 0u;
                    }
                    if (table && nhits > 0) add_lost(v, x.col + 64 * q);
                    if (!GRADS && (tid & 127) >> 6 == q >> 1) {            // (the last piece's have been read: the group met since)
                        token_factor[group][tid & 63] = c;
                        token_lse2[group][tid & 63] = lse2;
                        token_target[group][tid & 63] = target;
                    }
                    uint8_t* const stg = stage();
                    if (!GRADS) {
                        const bool word = v_row < p.V;                 // words past the vocabulary are read by HIDDEN
                        // Shared memory's bandwidth is what the MMAs live on: their targets are looked at one by one only where one of
                        // the piece's is a row of the warp's (2048 x 1536: 640 -> 610 us).
                        auto gradients = [&](auto targets) {
#pragma unroll
                            for (int i = 0; i < 64; ++i) {
                                const float f = token_factor[group][i], e = ex2_ftz(__fmaf_rn(__uint_as_float(v[i]), scale2, -token_lse2[group][i]));
                                const bool hit = targets.value && token_target[group][i] == v_row;
                                float d = __fmul_rn(f, (hit ? 1.0f : 0.0f) - e);
                                if (f == 0.0f || !word) d = 0.0f;      // a masked token has no gradient whatever its logits are
                                if (hit) p.rho[x.col + 64 * q + i] = __fsub_rn(d, __bfloat162float(__float2bfloat16_rn(d)));
                                v[i] = __float_as_uint(d);
                            }
                        };
                        const unsigned t0 = token_target[group][lane] - first_row, t1 = token_target[group][lane + 32] - first_row;
                        if (__any_sync(0xffffffffu, t0 < 32u || t1 < 32u)) gradients(std::true_type());
                        else gradients(std::false_type());
                    }
#pragma unroll
                    for (int c16 = 0; c16 < 8; ++c16) {
                        const uint4 val = make_uint4(
                            pack_bf16x2(__uint_as_float(v[8 * c16]), __uint_as_float(v[8 * c16 + 1])),
                            pack_bf16x2(__uint_as_float(v[8 * c16 + 2]), __uint_as_float(v[8 * c16 + 3])),
                            pack_bf16x2(__uint_as_float(v[8 * c16 + 4]), __uint_as_float(v[8 * c16 + 5])),
                            pack_bf16x2(__uint_as_float(v[8 * c16 + 6]), __uint_as_float(v[8 * c16 + 7])));
                        *reinterpret_cast<uint4*>(stg + row * 128 + ((c16 ^ (row & 7)) << 4)) = val;
                    }
                    fence_proxy_async_smem();
                    named_bar_sync(1 + group, 128);
                    if (storer) {
                        tma_store_2d(GRADS ? &maps.table_out : &maps.dz_k, smem_u32(stg), x.col + 64 * q, GRADS ? p.v0 + row0 : row0);
                        tma_store_commit();
                    }
                }
            } else {
#pragma unroll 1
                for (int q = group; q < TILE / 32; q += 2) {
                    if (table ? x.col + 32 * q >= p.H : 32 * q >= x.cols) break;
                    uint32_t v[32];
                    tmem_ld32(taddr + 32 * q, v);
                    tmem_wait_ld();
                    if (table && x.k1 == 0) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] = 0u;
                    }
                    if (table && nhits > 0) add_lost(v, x.col + 32 * q);
                    uint8_t* const stg = stage();
#pragma unroll
                    for (int c16 = 0; c16 < 8; ++c16)
                        *reinterpret_cast<uint4*>(stg + row * 128 + ((c16 ^ (row & 7)) << 4)) =
                            make_uint4(v[4 * c16], v[4 * c16 + 1], v[4 * c16 + 2], v[4 * c16 + 3]);
                    fence_proxy_async_smem();
                    named_bar_sync(1 + group, 128);
                    if (storer) {
                        const bool part = x.slot >= 0;
                        const CUtensorMap* to = table ? &maps.table_out : part ? &maps.part_out : &maps.sum_out;
                        const int c0 = (part ? 0 : x.col) + 32 * q, c1 = part ? x.slot * TILE + half : table ? p.v0 + row0 : row0;
                        if (table ? p.add_table : p.add_hidden) tma_add_2d(to, smem_u32(stg), c0, c1);
                        else tma_store_2d(to, smem_u32(stg), c0, c1);
                        tma_store_commit();
                    }
                }
            }
            // all TMEM reads of this accumulator are done: hand it back to the MMA warp
            tc_fence_before();
            __syncwarp();
            if (lane == 0) lpb_arrive(lead_acc_empty + 8 * buf);
        }
        if (storer) tma_store_wait_all();
    }

    if (*abort_word) {   // let copies and MMAs in flight finish before shared memory and TMEM are released
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 1000000ull) {
        }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();            // neither CTA leaves while the other may still touch it
    if (warp == 1) tmem_dealloc_pair(tmem, LPB_TMEM_COLS);
}

// d_hidden in bf16 from the whole tiles' sums and the others' parts, these in ascending order, and what the target's term lost; zeros
// for tokens that took no part.  The sums lie as [H][tokens]: a CTA turns 32 tokens x 32 channels in shared memory.  A thread adds the parts
// of four tokens at a channel, AT_ONCE of them on their way at a time, and writes four channels of a token.  (Rows of the result go by
// tokens that take part; the others' rows come last.)  256 x 256 with 32 parts 4.7 us with sixteen at a time, 7.5 with eight; 2048 x 1536 with six
// parts 19 with eight and four CTAs an SM, 28.6 with sixteen and two.
template <int AT_ONCE>
__global__ void __launch_bounds__(256, AT_ONCE == 16 ? 2 : 4) lpb_fold_kernel(const LogprobBwdParams p) {
    __shared__ float turn[32][33];
    pdl_wait();
    pdl_launch_dependents();
    const LpbShape g = lpb_shape(p, lpb::HIDDEN);
    const int tid = threadIdx.x, rest = g.tokens * g.channels - g.whole;
    const int bands = (p.H + 31) / 32;
    const long long blocks = static_cast<long long>((g.rows + 31) / 32) * bands;
    for (long long b = blockIdx.x; b < blocks; b += gridDim.x) {
        const int t0 = static_cast<int>(b / bands) * 32, h0 = static_cast<int>(b % bands) * 32;
        const int tile = t0 / lpb::TILE * g.channels + h0 / lpb::TILE;
        // what is written, and what it needs beside the sums
        const int r = tid / 8, h = tid % 8 * 4;
        uint2 w = make_uint2(0u, 0u);
        float lost = 0.0f;
        long long row = t0 + r;
        if (t0 + r < g.rows) {
            const int target = p.row_target[t0 + r];
            if (target >= 0 && target < p.V) {
                w = *reinterpret_cast<const uint2*>(p.head + static_cast<long long>(target) * p.H + h0 + h);
                lost = p.rho[t0 + r];
            }
            if (p.index) row = p.index[t0 + r];
        }
        {
            const int h = h0 + tid / 8, t = t0 + tid % 8 * 4;
            float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (tile < g.whole) {
                f = *reinterpret_cast<const float4*>(p.sum + static_cast<long long>(h) * p.ldt + t);
            } else {
                const float4* src = reinterpret_cast<const float4*>(
                    p.part + (static_cast<long long>(tile - g.whole) * lpb::TILE + h % lpb::TILE) * lpb::TILE + t % lpb::TILE);
                const long long next = static_cast<long long>(rest) * lpb::TILE * lpb::TILE / 4;
                for (int k = 0; k < g.split; k += AT_ONCE) {
                    float4 a[AT_ONCE];
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i)
                        a[i] = k + i < g.split ? __ldcg(src + i * next) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int i = 0; i < AT_ONCE; ++i) f.x += a[i].x, f.y += a[i].y, f.z += a[i].z, f.w += a[i].w;
                    src += AT_ONCE * next;
                }
            }
            __syncthreads();                               // (the last block has been read)
            float* const to = &turn[tid / 8][tid % 8 * 4];
            to[0] = f.x, to[1] = f.y, to[2] = f.z, to[3] = f.w;
        }
        __syncthreads();
        if (t0 + r < g.rows) {
            const float x0 = fmaf(lost, __uint_as_float(w.x << 16), turn[h][r]), x1 = fmaf(lost, __uint_as_float(w.x & 0xffff0000u), turn[h + 1][r]);
            const float x2 = fmaf(lost, __uint_as_float(w.y << 16), turn[h + 2][r]), x3 = fmaf(lost, __uint_as_float(w.y & 0xffff0000u), turn[h + 3][r]);
            *reinterpret_cast<uint2*>(p.d_hidden + row * p.H + h0 + h) = make_uint2(pack_bf16x2(x0, x1), pack_bf16x2(x2, x3));
        }
    }
    // the others' rows, a warp each
    if (!p.place) return;
    const int lane = tid & 31;
    for (long long row = static_cast<long long>(blockIdx.x) * 8 + (tid >> 5); row < p.T; row += static_cast<long long>(gridDim.x) * 8)
        if (p.place[row] < 0)
            for (int h = 8 * lane; h < p.H; h += 256) *reinterpret_cast<uint4*>(p.d_hidden + row * p.H + h) = make_uint4(0, 0, 0, 0);
}

// The tokens that take part, in order: index [rows] of theirs, their targets, and place [T], -1 for the others; the count.  One CTA:
// 4096 tokens a step (1.1 us), which is little beside what a step's products take.
constexpr int LPB_LIST_THREADS = 1024;
__global__ void __launch_bounds__(LPB_LIST_THREADS) lpb_list_kernel(const LogprobBwdParams p, int32_t* index, int32_t* target, int32_t* place,
                                                                    int32_t* count) {
    __shared__ int sums[LPB_LIST_THREADS / 32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    pdl_wait();
    pdl_launch_dependents();
    int total = 0;
    bool bad = false;
    for (long long base = 0; base < p.T; base += 4 * LPB_LIST_THREADS) {
        const long long first = base + 4 * tid;
        int tgt[4], n = 0;
        bool on[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            tgt[j] = -1;
            on[j] = first + j < p.T && p.d_logprob[first + j] != 0.0f;     // (NaN takes part)
            if (on[j]) {
                tgt[j] = p.target[first + j];
                if (tgt[j] < 0 || tgt[j] >= p.V) {
                    on[j] = false;
                    bad = true;
                }
            }
            n += on[j];
        }
        int before = n;                                    // of this warp's lanes up to this one
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, before, off);
            if (lane >= off) before += o;
        }
        if (lane == 31) sums[warp] = before;
        __syncthreads();
        int s = sums[lane];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, s, off);
            if (lane >= off) s += o;
        }
        int at = total + before - n + (warp ? __shfl_sync(0xffffffffu, s, warp - 1) : 0);
        total += __shfl_sync(0xffffffffu, s, 31);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (first + j < p.T) place[first + j] = on[j] ? at : -1;
            if (on[j]) {
                index[at] = static_cast<int32_t>(first + j);
                target[at++] = tgt[j];
            }
        }
        __syncthreads();
    }
    if (bad) atomicOr(p.dev_status, TIK_DEV_BAD_TARGET);
    if (warp == 0) {
        const LpbRest r = lpb_rest(p, total);
        int best = 1, cost = lpb_split_cost(1, r.rest, r.slices);
        for (int s = lane + 1; s <= r.most; s += 32) {
            const int c = lpb_split_cost(s, r.rest, r.slices);
            if (c < cost) best = s, cost = c;
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) {
            const int s = __shfl_xor_sync(0xffffffffu, best, off), c = __shfl_xor_sync(0xffffffffu, cost, off);
            if (c < cost || (c == cost && s < best)) best = s, cost = c;
        }
        if (lane == 0) {
            count[0] = total;
            count[1] = best;
        }
    }
}
// Their hidden rows, and zeros up to the next multiple of 64 (what TABLE multiplies d_z's zeros with).  A warp per row.
__global__ void __launch_bounds__(256) lpb_gather_kernel(const LogprobBwdParams p, const __nv_bfloat16* hidden, __nv_bfloat16* rows) {
    pdl_wait();
    pdl_launch_dependents();
    const int n = __ldcg(p.count), lane = threadIdx.x & 31, vecs = p.H / 8;
    const long long end = min(static_cast<long long>((n + 63) / 64) * 64, static_cast<long long>(p.T));
    for (long long r = static_cast<long long>(blockIdx.x) * 8 + (threadIdx.x >> 5); r < end; r += static_cast<long long>(gridDim.x) * 8) {
        uint4* to = reinterpret_cast<uint4*>(rows + r * p.H);
        if (r >= n) {
            for (int i = lane; i < vecs; i += 32) to[i] = make_uint4(0, 0, 0, 0);
            continue;
        }
        const uint4* from = reinterpret_cast<const uint4*>(hidden + static_cast<long long>(__ldcg(p.index + r)) * p.H);
#pragma unroll 4
        for (int i = lane; i < vecs; i += 32) to[i] = from[i];
    }
}

// How a call of T rows is cut: columns of a vocabulary chunk, as few chunks as keep d_z within 2 GiB (whole vocabularies up to 7000
// rows at V 152 064), of equal size; and its scratch.
LogprobBwdPlan logprob_bwd_plan(int64_t T, int H, int V) {
    constexpr int64_t pairs = lpb::PAIRS;
    LogprobBwdPlan g;
    g.ldt = static_cast<int>((T + 63) / 64 * 64);
    const int64_t steps = (V + 255) / 256;
    const int64_t most = std::max<int64_t>(1, (2ll << 30) / (g.ldt * 512ll));
    g.chunks = static_cast<int>((steps + most - 1) / most);
    g.chunk = static_cast<int>((steps + g.chunks - 1) / g.chunks * 256);
    g.chunks = (V + g.chunk - 1) / g.chunk;
    g.gather = T > lpb::TILE;
    const int64_t tiles = (T + 255) / 256 * ((H + 255) / 256);
    g.parts = static_cast<int>(std::min<int64_t>(lpb::MOST_PARTS, std::min(tiles, pairs) * std::min<int64_t>(64, (std::min(g.chunk, V) + 63) / 64)));
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t uT = static_cast<size_t>(T);
    size_t at = up(static_cast<size_t>(g.ldt) * g.chunk * 2);
    auto take = [&](size_t n) {
        const size_t here = at;
        at += up(n);
        return here;
    };
    g.sum_at = take(tiles >= pairs ? static_cast<size_t>(g.ldt) * H * 4 : 0);
    g.part_at = take(static_cast<size_t>(g.parts) * lpb::TILE * lpb::TILE * 4);
    g.rho_at = take(uT * 4);
    g.index_at = take(g.gather ? uT * 4 : 0);
    g.target_at = take(g.gather ? uT * 4 : 0);
    g.place_at = take(g.gather ? uT * 4 : 0);
    g.count_at = take(g.gather ? 8 : 0);
    g.rows_at = take(g.gather ? uT * H * 2 : 0);
    g.bytes = at;
    return g;
}

template <int KIND>
static cudaError_t launch_lpb(const LogprobBwdMaps& maps, const LogprobBwdParams& p, cudaStream_t stream) {
    auto kern = lpb_kernel<KIND>;
    static DeviceOnce configured;     // the opt-in belongs to the (function, device) pair
    cudaError_t e = configured.run([&]() {
        return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lpb::ALLOC));
    });
    if (e != cudaSuccess) return e;
    // no more pairs than there may be units
    const long long tokens = (p.T + 255) / 256, words = (p.nv + 255) / 256, channels = (p.H + 255) / 256;
    const long long units = KIND == lpb::DZ ? tokens * words : KIND == lpb::HIDDEN ? lpb::MOST_PARTS : words * channels + (KIND == lpb::BOTH ? lpb::MOST_PARTS : 0);
    return launch_pdl(kern, dim3(static_cast<unsigned>(2 * std::min<long long>(p.pairs, units))), lpb::THREADS, lpb::ALLOC, stream, 2, maps, p);
}

cudaError_t launch_logprob_bwd(const LogprobBwdMaps& m, LogprobBwdParams p, const LogprobBwdPlan& g, const void* hidden, bool add_table, int sm_count,
                               cudaStream_t stream) {
    p.chunk = g.chunk;
    p.ldt = g.ldt;
    p.pairs = std::max(1, sm_count / 2);
    cudaError_t e = cudaSuccess;
    if (!g.gather) {
        const LpbRest r = lpb_rest(p, static_cast<int>(p.T));
        p.split = 1;
        for (int s = 2; s <= r.most; ++s)
            if (lpb_split_cost(s, r.rest, r.slices) < lpb_split_cost(p.split, r.rest, r.slices)) p.split = s;
    } else {
        e = launch_pdl(lpb_list_kernel, dim3(1), LPB_LIST_THREADS, 0, stream, 1, p, const_cast<int32_t*>(p.index), const_cast<int32_t*>(p.row_target),
                       const_cast<int32_t*>(p.place), const_cast<int32_t*>(p.count));
        if (e != cudaSuccess) return e;
        e = launch_pdl(lpb_gather_kernel, dim3(static_cast<unsigned>(std::min<long long>((p.T + 7) / 8, 8ll * sm_count))), 256, 0, stream, 1, p,
                       static_cast<const __nv_bfloat16*>(hidden), const_cast<__nv_bfloat16*>(p.rows));
        if (e != cudaSuccess) return e;
    }
    for (int c = 0; c < g.chunks; ++c) {
        p.v0 = c * g.chunk;
        p.nv = std::min(g.chunk, p.V - p.v0);
        p.add_table = add_table;
        p.add_hidden = c > 0;
        e = launch_lpb<lpb::DZ>(m, p, stream);
        p.clean = nullptr;                                 // (once is enough)
        // Both gradients in one launch where d_lm_head is a few rounds of units and launches are what a call takes (256 x 256, vocabulary
        // 2048: 27.1 -> 21.5 us).  In long calls the pairs come to d_lm_head's units one after the other and no longer share their
        // operands in L2 (501 x 1536, vocabulary 151 936: 647 us apart, 659 together).
        const int words = (p.nv + 255) / 256, channels = (p.H + 255) / 256;
        const bool both = p.want_table && p.d_hidden && static_cast<long long>(words) * channels <= 4 * lpb::PAIRS;
        if (both && e == cudaSuccess) e = launch_lpb<lpb::BOTH>(m, p, stream);
        if (!both && p.want_table && e == cudaSuccess) e = launch_lpb<lpb::TABLE>(m, p, stream);
        if (!both && p.d_hidden && e == cudaSuccess) e = launch_lpb<lpb::HIDDEN>(m, p, stream);
        if (e != cudaSuccess) return e;
    }
    if (!p.d_hidden) return cudaSuccess;
    const long long blocks = (p.T + 31) / 32 * ((p.H + 31) / 32);
    // calls of a few CTAs wait for one part after the other, others for how much is on its way
    if (blocks <= 2ll * sm_count) return launch_pdl(lpb_fold_kernel<16>, dim3(static_cast<unsigned>(blocks)), 256, 0, stream, 1, p);
    return launch_pdl(lpb_fold_kernel<8>, dim3(static_cast<unsigned>(std::min<long long>(blocks, 8ll * sm_count))), 256, 0, stream, 1, p);
}

}  // namespace tik
