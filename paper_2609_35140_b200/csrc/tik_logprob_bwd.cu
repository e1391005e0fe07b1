// Gradient of the token log-probabilities for sm_100a.  With z[t][v] = f hidden[t] . lm_head[v] (f: the inverse
// temperature) and p[t][v] = exp(z[t][v] - lse[t]):
//   d_z[t][v]    = f d_logprob[t] ([v == target[t]] - p[t][v])
//   d_hidden[t]  = sum_v d_z[t][v] lm_head[v],      d_lm_head[v] = sum_t d_z[t][v] hidden[t]
// Three matrix products of 2 T V H operations each, which is what bounds a call of more than some hundred rows: the logits
// are computed again (they were never stored), d_z leaves that product's epilogue as bf16 [T][columns of a chunk], and both
// gradients are products with it.  d_z is the one rounding on the way: every term of a gradient is off by 2^-9 of itself at
// most, rounded independently, which is less in a sum of them than the sum's own rounding to bf16 at the end.  Sums
// are fp32 in tensor memory.
//
// One kernel for all three (KIND), persistent CTA pairs that walk units of one 256 x 256 output tile each: a TMA warp streams
// 64-wide slices of the contracted axis through a ring, an MMA warp issues M256 x N256 x K16 MMAs into one of two
// accumulators, four epilogue warps take the other one out through shared memory and tiled TMA stores.  An operand whose
// contracted axis is not its contiguous one is read as it lies (MN-major descriptors): nothing is transposed.
//   DZ      A = hidden (K-major),  B = lm_head (K-major)       rows: tokens,   columns: vocabulary, contracted: H
//   TABLE   A = d_z (M-major),     B = hidden (N-major)        rows: vocabulary, columns: H,        contracted: tokens
//   HIDDEN  A = d_z (K-major),     B = lm_head (N-major)       rows: tokens,   columns: H,          contracted: vocabulary
// HIDDEN has few tiles with a long contracted axis (4001 x 3584: 224 tiles, 2376 slices, for 74 pairs), so the tiles of the last,
// partial round are split along it, into parts that are summed in ascending order by lpb_fold_kernel.  Vocabularies whose d_z
// exceeds the scratch are taken in chunks; the sums behind d_hidden then grow in fp32, one addition an element and chunk, in order.
#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

namespace lpb {
constexpr int DZ = 0, TABLE = 1, HIDDEN = 2;
constexpr int TILE = 256;                    // rows (of a pair) and columns of a unit
constexpr uint32_t OP_BYTES = 128 * 128;     // an operand's share of a stage: 128 rows or columns x 64 of the contracted axis
constexpr uint32_t STAGE_BYTES = 2 * OP_BYTES;
constexpr int STAGES = 6;
constexpr uint32_t STG_BYTES = 128 * 128;    // output staging: 128 rows x 128 bytes, two buffers
constexpr uint32_t OFF_STG = STAGES * STAGE_BYTES;
constexpr uint32_t OFF_BAR = OFF_STG + 2 * STG_BYTES;
constexpr uint32_t BYTES = OFF_BAR + 256;
constexpr uint32_t ALLOC = BYTES + 1024;
constexpr int BAND = 16;                     // DZ: pairs of token tiles whose hidden rows stay in L2 while lm_head streams by
constexpr int THREADS = 192;                 // warp 0 TMA, warp 1 MMA, warps 2..5 epilogue
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

// One warp of both CTAs: all of tensor memory, two 256-column accumulators.  Before the CTA's dependents are released.
constexpr uint32_t LPB_TMEM_COLS = 512;
__device__ __forceinline__ void lpb_take_tensor_memory(volatile uint32_t* slot) {
    tmem_alloc_pair(smem_u32(const_cast<uint32_t*>(slot)), LPB_TMEM_COLS);
    tmem_relinquish_pair();
}

struct LpbUnit {
    int row, col;                // of the output tile
    int k0, k1;                  // slices of 64 of the contracted axis
    int slot;                    // HIDDEN: part of a split tile (its place in the parts' buffer), -1: a whole tile
};
template <int KIND>
__device__ __forceinline__ LpbUnit lpb_unit(const LogprobBwdParams& p, int u) {
    using namespace lpb;
    LpbUnit x;
    x.slot = -1;
    x.k0 = 0;
    if (KIND == DZ) {
        // token tiles fastest inside a band, so that the pairs at work share a few steps of lm_head
        const int per_band = BAND * p.col_tiles, band = u / per_band, rem = u - band * per_band;
        const int tiles = min(BAND, p.row_tiles - band * BAND);
        x.row = (band * BAND + rem % tiles) * TILE;
        x.col = rem / tiles * TILE;
        x.k1 = p.H / 64;
    } else if (KIND == TABLE) {
        x.row = u / p.col_tiles * TILE;
        x.col = u % p.col_tiles * TILE;
        x.k1 = static_cast<int>((p.T + 63) / 64);
    } else {
        const int slices = (p.nv + 63) / 64;
        int tile = u;
        x.k1 = slices;
        if (u >= p.whole) {
            const int rest = p.row_tiles * p.col_tiles - p.whole, q = u - p.whole, part = q / rest;
            tile = p.whole + q % rest;
            x.k0 = static_cast<int>(static_cast<long long>(slices) * part / p.split);
            x.k1 = static_cast<int>(static_cast<long long>(slices) * (part + 1) / p.split);
            x.slot = q;
        }
        x.row = tile / p.col_tiles * TILE;
        x.col = tile % p.col_tiles * TILE;
    }
    return x;
}

template <int KIND>
__global__ void __launch_bounds__(lpb::THREADS, 1)
lpb_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const __grid_constant__ CUtensorMap tmOut,
           const __grid_constant__ CUtensorMap tmPart, const LogprobBwdParams p) {
    using namespace lpb;
    constexpr bool A_MN = KIND == TABLE, B_MN = KIND != DZ;
    constexpr uint32_t IDESC = mma_idesc_bf16(256, TILE, B_MN, A_MN);
    const int tid = threadIdx.x, warp = warp_uniform(tid >> 5), lane = tid & 31;
    const uint32_t rank = cluster_ctarank();     // 0 = the CTA that issues the pair's MMAs
    const int first = static_cast<int>(blockIdx.x >> 1), stride = static_cast<int>(gridDim.x >> 1);

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
            mbar_init(bar_acc_empty + 8 * b, 256);           // the epilogue threads of both CTAs
        }
        fence_barrier_init();
        tma_prefetch_desc(&tmA);
        tma_prefetch_desc(&tmB);
        tma_prefetch_desc(&tmOut);
        if (KIND == HIDDEN) tma_prefetch_desc(&tmPart);
    }
    if (warp == 1) lpb_take_tensor_memory(tmem_slot);
    pdl_wait();
    if (tid == 0) *abort_word = (*reinterpret_cast<volatile int*>(p.dev_status) & TIK_DEV_WAIT_EXPIRED) ? 1 : 0;
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();            // the peer's barriers exist before anything signals them
    tc_fence_after();
    pdl_launch_dependents();
    const uint32_t tmem = *tmem_slot;
    const uint32_t lead_full = mapa_cluster(bar_full, 0);
    const uint32_t lead_acc_empty = mapa_cluster(bar_acc_empty, 0);
    const uint32_t peer_empty = mapa_cluster(bar_empty, 1);
    const uint32_t peer_acc_full = mapa_cluster(bar_acc_full, 1);
    const int half = 128 * static_cast<int>(rank);

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        if (lane == 0) {
            uint32_t it = 0;
            for (int u = first; u < p.nunit; u += stride) {
                const LpbUnit x = lpb_unit<KIND>(p, u);
                // each CTA stages its own 128 rows of A and its half of B; what lies outside the tensors arrives as zeros
                const int a0 = x.row + half, b0 = x.col + half;
                for (int kb = x.k0; kb < x.k1; ++kb, ++it) {
                    if (*abort_word) break;      // a wait expired somewhere: stop issuing copies
                    const int s = it % STAGES;
                    const uint32_t use = it / STAGES, dst = sbase + s * STAGE_BYTES;
                    if (use > 0) mbar_wait(bar_empty + 8 * s, (use - 1) & 1, abort_word, p.dev_status);
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, 2 * STAGE_BYTES);   // both CTAs' bytes
                    if (A_MN) {
                        tma_load_2d_pair(dst, &tmA, lead_full + 8 * s, a0, kb * 64);
                        tma_load_2d_pair(dst + OP_BYTES / 2, &tmA, lead_full + 8 * s, a0 + 64, kb * 64);
                    } else {
                        tma_load_2d_pair(dst, &tmA, lead_full + 8 * s, kb * 64, a0);
                    }
                    if (B_MN) {
                        const int k = kb * 64 + (KIND == HIDDEN ? p.v0 : 0);
                        tma_load_2d_pair(dst + OP_BYTES, &tmB, lead_full + 8 * s, b0, k);
                        tma_load_2d_pair(dst + OP_BYTES + OP_BYTES / 2, &tmB, lead_full + 8 * s, b0 + 64, k);
                    } else {
                        tma_load_2d_pair(dst + OP_BYTES, &tmB, lead_full + 8 * s, kb * 64, p.v0 + b0);
                    }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issuer
        if (rank == 0) {
            const uint32_t tmem_u = warp_uniform(tmem);
            uint32_t it = 0, acc = 0;
            for (int u = first; u < p.nunit; u += stride, ++acc) {
                const LpbUnit x = lpb_unit<KIND>(p, u);
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
                    mma_ss_chain4_pair_steps<A_MN ? 128 : 2, B_MN ? 128 : 2>(
                        tmem_u + buf * TILE, smem_desc_sw128(a, A_MN ? OP_BYTES / 2 : 0, 1024),
                        smem_desc_sw128(b, B_MN ? OP_BYTES / 2 : 0, 1024), IDESC, kb > x.k0 ? 1u : 0u);
                    mma_commit_pair(bar_empty + 8 * s);
                    mma_commit_pair(peer_empty + 8 * s);
                }
                mma_commit_pair(bar_acc_full + 8 * buf);
                mma_commit_pair(peer_acc_full + 8 * buf);
            }
        }
    } else {
        // ------------------------------------------------------------ epilogue (warps 2..5), thread per row
        const int quarter = warp & 3;                      // TMEM lane quarter of this warp
        const int row = quarter * 32 + lane;
        uint32_t piece = 0, acc = 0;
        const bool storer = warp == 2 && lane == 0;
        // a staging buffer that the store two pieces ago has finished reading
        auto stage = [&]() {
            if (storer) tma_store_wait_read1();
            named_bar_sync(1, 128);
            return smem + OFF_STG + (piece & 1) * STG_BYTES;
        };
        for (int u = first; u < p.nunit; u += stride, ++acc) {
            const LpbUnit x = lpb_unit<KIND>(p, u);
            const int buf = acc & 1, row0 = x.row + half;
            float c = 0.0f, lse2 = 0.0f;
            int target = -1;
            if (KIND == DZ) {
                const long long t = static_cast<long long>(row0) + row;
                if (t < p.T) {
                    target = p.target[t];
                    c = __fmul_rn(p.d_logprob[t], p.inv_temperature);
                    lse2 = __fmul_rn(p.lse[t], LOG2E_F);
                    if (target < 0 || target >= p.V) {     // no gradient
                        c = 0.0f;
                        atomicOr(p.dev_status, TIK_DEV_BAD_TARGET);
                    }
                    target -= p.v0 + x.col;                // column of this tile
                }
            }
            mbar_wait(bar_acc_full + 8 * buf, (acc >> 1) & 1, abort_word, p.dev_status);
            tc_fence_after();
            const uint32_t taddr = tmem + (static_cast<uint32_t>(quarter * 32) << 16) + buf * TILE;
            const bool f32_out = KIND == HIDDEN || (KIND == TABLE && p.table_fp32);
            if (!f32_out) {
                const int limit = KIND == DZ ? p.ldz : p.H;
                const float scale2 = KIND == DZ ? __fmul_rn(p.inv_temperature, LOG2E_F) : 0.0f;
#pragma unroll 1
                for (int q = 0; q < TILE / 64; ++q, ++piece) {
                    if (x.col + 64 * q >= limit) break;    // uniform: columns past the output
                    uint32_t v[64];
                    tmem_ld32(taddr + 64 * q, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
                    tmem_ld32(taddr + 64 * q + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
                    tmem_wait_ld();
                    if (KIND == DZ) {
                        const int valid = p.nv - x.col - 64 * q, hit = target - 64 * q;
#pragma unroll
                        for (int i = 0; i < 64; ++i) {
                            const float e = ex2_ftz(__fmaf_rn(__uint_as_float(v[i]), scale2, -lse2));
                            float d = __fmul_rn(c, (i == hit ? 1.0f : 0.0f) - e);
                            // a masked row has no gradient whatever its logits are; columns past the vocabulary are read by HIDDEN
                            if (c == 0.0f || i >= valid) d = 0.0f;
                            v[i] = __float_as_uint(d);
                        }
                    }
                    uint8_t* stg = stage();
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
                    named_bar_sync(1, 128);
                    if (storer) {
                        tma_store_2d(&tmOut, smem_u32(stg), x.col + 64 * q, KIND == TABLE ? p.v0 + row0 : row0);
                        tma_store_commit();
                    }
                }
            } else {
#pragma unroll 1
                for (int q = 0; q < TILE / 32; ++q, ++piece) {
                    if (x.col + 32 * q >= p.H) break;
                    uint32_t v[32];
                    tmem_ld32(taddr + 32 * q, v);
                    tmem_wait_ld();
                    uint8_t* stg = stage();
#pragma unroll
                    for (int c16 = 0; c16 < 8; ++c16)
                        *reinterpret_cast<uint4*>(stg + row * 128 + ((c16 ^ (row & 7)) << 4)) =
                            make_uint4(v[4 * c16], v[4 * c16 + 1], v[4 * c16 + 2], v[4 * c16 + 3]);
                    fence_proxy_async_smem();
                    named_bar_sync(1, 128);
                    if (storer) {
                        const bool part = KIND == HIDDEN && x.slot >= 0;
                        const CUtensorMap* to = part ? &tmPart : &tmOut;
                        const int c0 = (part ? 0 : x.col) + 32 * q, c1 = part ? x.slot * TILE + half : KIND == TABLE ? p.v0 + row0 : row0;
                        if (p.add) tma_add_2d(to, smem_u32(stg), c0, c1);
                        else tma_store_2d(to, smem_u32(stg), c0, c1);
                        tma_store_commit();
                    }
                }
            }
            // all TMEM reads of this accumulator are done: hand it back to the MMA warp
            tc_fence_before();
            mbar_arrive_cluster(lead_acc_empty + 8 * buf);
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

// d_hidden in bf16 from the whole tiles' sums and the others' parts, these in ascending order.  Thread per eight channels.
__global__ void __launch_bounds__(256) lpb_fold_kernel(const LogprobBwdParams p, int parts) {
    pdl_wait();
    pdl_launch_dependents();
    const int per_row = p.H / 8, rest = p.row_tiles * p.col_tiles - p.whole;
    const long long n = p.T * per_row;
    for (long long i = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; i < n; i += static_cast<long long>(gridDim.x) * 256) {
        const long long t = i / per_row;
        const int h = static_cast<int>(i - t * per_row) * 8;
        const int tile = static_cast<int>(t / lpb::TILE) * p.col_tiles + h / lpb::TILE;
        float f[8];
        if (tile < p.whole) {
            const float4* src = reinterpret_cast<const float4*>(p.sum + t * p.H + h);
            const float4 a = src[0], b = src[1];
            f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
        } else {
            const float4* src = reinterpret_cast<const float4*>(
                p.part + (static_cast<long long>(tile - p.whole) * lpb::TILE + t % lpb::TILE) * lpb::TILE + h % lpb::TILE);
            const long long next = static_cast<long long>(rest) * lpb::TILE * lpb::TILE / 4;
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = 0.0f;
#pragma unroll 4
            for (int s = 0; s < parts; ++s, src += next) {
                const float4 a = src[0], b = src[1];
                f[0] += a.x, f[1] += a.y, f[2] += a.z, f[3] += a.w, f[4] += b.x, f[5] += b.y, f[6] += b.z, f[7] += b.w;
            }
        }
        *reinterpret_cast<uint4*>(p.d_hidden + t * p.H + h) =
            make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
    }
}

// How a call of T rows is cut: columns of a vocabulary chunk, and for HIDDEN the tiles that are done whole, the others' parts.
//
// Chunks: as few as keep d_z within 2 GiB (whole vocabularies up to 7000 rows at V 152 064), of equal size.
// Parts: the tiles of the last round of pairs (74 on a B200), split so that the round costs least in slices, a unit's
// epilogue and first loads counting as six.
LogprobBwdPlan logprob_bwd_plan(int64_t T, int H, int V) {
    constexpr int64_t pairs = 74;
    LogprobBwdPlan g;
    const int64_t steps = (V + 255) / 256;
    const int64_t most = std::max<int64_t>(1, (2ll << 30) / (T * 512));
    g.chunks = static_cast<int>((steps + most - 1) / most);
    g.chunk = static_cast<int>((steps + g.chunks - 1) / g.chunks * 256);
    g.chunks = (V + g.chunk - 1) / g.chunk;
    const int64_t tiles = (T + 255) / 256 * ((H + 255) / 256);
    const int64_t rest = tiles % pairs;
    const int slices = (V - (g.chunks - 1) * g.chunk + 63) / 64;          // of the last chunk, the shortest: every part has some
    const int most_slices = (std::min(g.chunk, V) + 63) / 64;
    g.whole = static_cast<int>(tiles - rest);
    g.split = 1;
    double best = -1.0;
    for (int s = 1; rest > 0 && s <= 64 && s <= slices; ++s) {
        const double cost = static_cast<double>((rest * s + pairs - 1) / pairs) * ((most_slices + s - 1) / s + 6);
        if (best < 0.0 || cost < best) {
            best = cost;
            g.split = s;
        }
    }
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    g.dz_bytes = up(static_cast<size_t>(T) * g.chunk * 2);
    g.sum_bytes = g.whole > 0 ? up(static_cast<size_t>(T) * H * 4) : 0;
    g.part_bytes = static_cast<size_t>(rest) * g.split * lpb::TILE * lpb::TILE * 4;
    return g;
}

template <int KIND>
static cudaError_t launch_lpb(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmOut, const CUtensorMap& tmPart,
                              const LogprobBwdParams& p, cudaStream_t stream) {
    auto kern = lpb_kernel<KIND>;
    static DeviceOnce configured;     // the opt-in belongs to the (function, device) pair
    cudaError_t e = configured.run([&]() {
        return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lpb::ALLOC));
    });
    if (e != cudaSuccess) return e;
    const int pairs = std::max(1, p.sm_count / 2);
    return launch_pdl(kern, dim3(static_cast<unsigned>(2 * std::min(pairs, p.nunit))), lpb::THREADS, lpb::ALLOC, stream, 2, tmA, tmB,
                      tmOut, tmPart, p);
}

cudaError_t launch_logprob_bwd(const LogprobBwdMaps& m, LogprobBwdParams p, const LogprobBwdPlan& g, bool add_table, cudaStream_t stream) {
    const int token_tiles = static_cast<int>((p.T + 255) / 256), h_tiles = (p.H + 255) / 256;
    p.ldz = g.chunk;
    p.whole = g.whole;
    p.split = g.split;
    for (int c = 0; c < g.chunks; ++c) {
        p.v0 = c * g.chunk;
        p.nv = std::min(g.chunk, p.V - p.v0);
        const int v_tiles = (p.nv + 255) / 256;
        p.row_tiles = token_tiles;
        p.col_tiles = v_tiles;
        p.nunit = token_tiles * v_tiles;
        cudaError_t e = launch_lpb<lpb::DZ>(m.hidden_k, m.head_k, m.dz_out, m.dz_out, p, stream);
        if (e != cudaSuccess) return e;
        if (p.want_table) {
            p.row_tiles = v_tiles;
            p.col_tiles = h_tiles;
            p.nunit = v_tiles * h_tiles;
            p.add = add_table;
            e = launch_lpb<lpb::TABLE>(m.dz_mn, m.hidden_mn, m.table_out, m.table_out, p, stream);
            if (e != cudaSuccess) return e;
        }
        if (p.d_hidden) {
            p.row_tiles = token_tiles;
            p.col_tiles = h_tiles;
            p.nunit = g.whole + (token_tiles * h_tiles - g.whole) * g.split;
            p.add = c > 0;
            e = launch_lpb<lpb::HIDDEN>(m.dz_out, m.head_mn, m.sum_out, m.part_out, p, stream);
            if (e != cudaSuccess) return e;
        }
    }
    if (!p.d_hidden) return cudaSuccess;
    const long long n = p.T * (p.H / 8);
    return launch_pdl(lpb_fold_kernel, dim3(static_cast<unsigned>(std::min<long long>((n + 255) / 256, 8ll * p.sm_count))), 256, 0, stream, 1,
                      p, g.split);
}

}  // namespace tik
