// The step between two blocks of a layer -- norm after the block, gate, scaled residual sum, norm before the next block --
// and its gradient.
#include <cuda_bf16.h>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int BN_THREADS = 128;

// One CTA per row with the reduction shape of rmsnorm_kernel (NV 16-byte vectors per thread): without post norm and gate
// and with a scale of 1 the results are those of its residual form, bit for bit.
template <int NV>
__global__ void __launch_bounds__(BN_THREADS) block_norm_kernel(const BlockNormParams p) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long row = blockIdx.x;
    const int nvec = p.H / 8;
    const uint4* x = reinterpret_cast<const uint4*>(p.x) + row * nvec;
    const uint4* res = reinterpret_cast<const uint4*>(p.residual) + row * nvec;
    const uint4* wp = reinterpret_cast<const uint4*>(p.post_weight);
    const uint4* wn = reinterpret_cast<const uint4*>(p.weight);
    __shared__ float tot_x[4], tot_s[4];
    pdl_wait();
    pdl_launch_dependents();
    uint4 xv[NV], rv[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + BN_THREADS * j;
        if (v < nvec) {
            xv[j] = x[v];
            rv[j] = res[v];
        }
    }
    const float inv_h = 1.0f / static_cast<float>(p.H);
    const float gt = p.gate_kind == GATE_TOKEN ? __bfloat162float(p.gate[row]) : 1.0f;
    float inv_x = 1.0f;
    if (p.post_weight) {
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (tid + BN_THREADS * j < nvec) {
                float f[8];
                unpack8(xv[j], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) part = __fmaf_rn(f[e], f[e], part);
            }
        part = hn_warp_total(part);
        if (lane == 0) tot_x[warp] = part;
        __syncthreads();
        inv_x = prep_inv_rms(hn_block_total(tot_x), inv_h, p.eps);
    }
    float s[NV][8], part = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + BN_THREADS * j;
        if (v >= nvec) continue;
        float f[8], r[8];
        unpack8(xv[j], f);
        unpack8(rv[j], r);
        if (p.post_weight) {
            float w[8];
            unpack8(wp[v], w);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = prep_norm(f[e], inv_x, w[e]);
        }
        if (p.gate_kind == GATE_CHANNEL) {
            float g[8];
            unpack8(reinterpret_cast<const uint4*>(p.gate)[v], g);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(f[e], g[e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j][e] = __fadd_rn(r[e], __fmul_rn(__fmul_rn(f[e], gt), p.branch_scale));
        const uint4 packed = pack8(s[j]);
        reinterpret_cast<uint4*>(p.s)[row * nvec + v] = packed;
        unpack8(packed, s[j]);
#pragma unroll
        for (int e = 0; e < 8; ++e) part = __fmaf_rn(s[j][e], s[j][e], part);
    }
    if (!p.weight) return;
    part = hn_warp_total(part);
    if (lane == 0) tot_s[warp] = part;
    __syncthreads();
    const float inv_s = prep_inv_rms(hn_block_total(tot_s), inv_h, p.eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + BN_THREADS * j;
        if (v >= nvec) continue;
        float w[8], o[8];
        unpack8(wn[v], w);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = prep_norm(s[j][e], inv_s, w[e]);
        reinterpret_cast<uint4*>(p.y)[row * nvec + v] = pack8(o);
    }
}

// ---- gradient --------------------------------------------------------------------------------
// Per row of x, s, d_y and d_s two sums over the row have to be known before the next step: (x^2, s^2, d_y w s), which give G, and
// G x (post weight, gate), which gives d_x.  Six planes of T x H cross HBM once, which bounds the kernel.  Persistent CTAs take R
// rows at a time, so that barriers and reductions are paid for once and one row's chain passes under another's; rows arrive by
// bulk copies, a few ahead.  A thread has the same BN_NV x 8 columns of every row, so that the sums over tokens stay in its
// registers until the end; block_norm_fold_kernel adds up the CTAs'.
constexpr int BN_NV = 2;                                     // 16-byte vectors per thread
constexpr int BN_SM_WARPS = 16;                              // (four warps of 128 registers on each quarter of an SM)

struct BlockNormBwdShape {
    int rows, threads, ctas, slots, slot_bytes, factor_bytes;
    size_t smem;
};
struct BlockNormBwdSmem {                                    // at most 16 warps x 1 row or 8 warps x 2 rows
    unsigned long long full[8];
    float4 sums[2][16];                                      // [turn][warp, row]
    float dots[2][16];
    int abort_word;
};
constexpr int BN_RING = (sizeof(BlockNormBwdSmem) + 127) / 128 * 128;

// Sums over a warp of N values at a time (1, 2, 4 or 8): each step of the butterfly folds two values into one register while there
// are any, one half of the lanes going on with either.  Lane l ends with the total of value l / (32 / N).
template <int N>
__device__ __forceinline__ float bn_warp_sums(const float (&v)[N], int lane) {
    if constexpr (N == 1) {
        return hn_warp_total(v[0]);
    } else {
        float half[N / 2];
        const bool upper = lane & 16;
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            half[i] = (upper ? v[i + N / 2] : v[i]) + __shfl_xor_sync(0xffffffffu, upper ? v[i] : v[i + N / 2], 16);
        if constexpr (N >= 4) {
            const bool upper8 = lane & 8;
#pragma unroll
            for (int i = 0; i < N / 4; ++i)
                half[i] = (upper8 ? half[i + N / 4] : half[i]) + __shfl_xor_sync(0xffffffffu, upper8 ? half[i] : half[i + N / 4], 8);
        }
        if constexpr (N >= 8) {
            const bool upper4 = lane & 4;
            half[0] = (upper4 ? half[1] : half[0]) + __shfl_xor_sync(0xffffffffu, upper4 ? half[0] : half[1], 4);
        }
        float t = half[0];
#pragma unroll
        for (int off = 16 / N; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
        return t;
    }
}

template <int R>
__global__ void __launch_bounds__(512 / R, R) block_norm_bwd_kernel(const BlockNormParams p, const BlockNormBwdShape shape) {
    extern __shared__ __align__(128) unsigned char bn_smem[];
    BlockNormBwdSmem& sm = *reinterpret_cast<BlockNormBwdSmem*>(bn_smem);
    // branch_scale * post_weight * gate (per channel) of the columns in fp32; then the ring
    float4* const factors = reinterpret_cast<float4*>(bn_smem + BN_RING);
    unsigned char* const ring = bn_smem + BN_RING + shape.factor_bytes;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    const int nvec = p.H / 8, row_vecs = BN_NV * blockDim.x;                 // (a row in the ring is as wide as the threads' vectors)
    const float inv_h = 1.0f / static_cast<float>(p.H);
    const bool norm = p.weight != nullptr, post = p.post_weight != nullptr, branch = p.x != nullptr;
    // What is absent reads as zeros: planes that are not there, vectors behind the row.
    for (int i = tid; i < shape.slots * 4 * row_vecs; i += blockDim.x) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    if (tid == 0) {
        for (int i = 0; i < shape.slots; ++i) mbar_init(smem_u32(&sm.full[i]), 1);
        sm.abort_word = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const int planes = (norm ? 2 : 0) + (branch ? 1 : 0) + (p.d_s ? 1 : 0);
    // The CTA's q-th row is row q % R of its (q / R)-th group; planes of a slot: d_s, x, s, d_y.
    auto row_of = [&](long long q) { return R * (blockIdx.x + q / R * gridDim.x) + q % R; };
    auto request = [&](long long row, int slot) {
        if (row >= p.T) return;
        const uint32_t bar = smem_u32(&sm.full[slot]), to = smem_u32(ring + slot * shape.slot_bytes);
        mbar_expect_tx(bar, planes * p.H * 2);
        const __nv_bfloat16* src[4] = {p.d_s, p.x, norm ? p.s : nullptr, norm ? p.d_y : nullptr};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (src[i]) bulk_load(to + i * 16 * row_vecs, src[i] + row * p.H, p.H * 2, bar);
    };
    if (tid == 0)
        for (int q = 0; q < shape.slots; ++q) request(row_of(q), q);
    // A thread reads only what it wrote here.  [half vector][thread]: 16 bytes a thread and instruction.
    uint32_t w[BN_NV][4];
    F2 sum_w[BN_NV][4], sum_c[BN_NV][4];
#pragma unroll
    for (int j = 0; j < BN_NV; ++j) {
        const int v = tid + static_cast<int>(blockDim.x) * j;
        auto column = [&](const __nv_bfloat16* base, bool there, float (&to)[8]) {
            unpack8(there && v < nvec ? reinterpret_cast<const uint4*>(base)[v] : make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), to);
        };
        float f[8], g[8];
        column(p.post_weight, post, f);
        column(p.gate, p.gate_kind == GATE_CHANNEL, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = p.branch_scale * (f[e] * g[e]);
        factors[2 * j * blockDim.x + tid] = make_float4(f[0], f[1], f[2], f[3]);
        factors[(2 * j + 1) * blockDim.x + tid] = make_float4(f[4], f[5], f[6], f[7]);
        const uint4 wv = norm && v < nvec ? reinterpret_cast<const uint4*>(p.weight)[v] : make_uint4(0, 0, 0, 0);
        w[j][0] = wv.x, w[j][1] = wv.y, w[j][2] = wv.z, w[j][3] = wv.w;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum_w[j][e] = sum_c[j][e] = f2(0.0f);
    }
    int slot = 0, turn = 0;
    uint32_t parity = 0;
    long long q = 0;
    for (long long row0 = R * static_cast<long long>(blockIdx.x); row0 < p.T; row0 += R * static_cast<long long>(gridDim.x), q += R) {
        const uint4* at[R];
        int slots[R];
        float gt[R];
        bool there[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            there[r] = row0 + r < p.T;
            gt[r] = p.gate_kind == GATE_TOKEN && there[r] ? __bfloat162float(p.gate[row0 + r]) : 1.0f;
            slots[r] = slot;
            at[r] = reinterpret_cast<const uint4*>(ring + slot * shape.slot_bytes) + tid;
            if (there[r]) mbar_wait(smem_u32(&sm.full[slot]), parity, &sm.abort_word, p.dev_status);
            if (++slot == shape.slots) {
                slot = 0;
                parity ^= 1;
            }
            if (!there[r])                                   // a row behind the last one: zeros, which this thread alone reads
                for (int i = 0; i < 4 * BN_NV; ++i) const_cast<uint4*>(at[r])[i * blockDim.x] = make_uint4(0, 0, 0, 0);
        }
        // The rows stay in shared memory between the sums: registers are scarce.
        auto take = [&](int r, int plane, int j, uint32_t (&to)[4]) {
            const uint4 v = at[r][plane * row_vecs + blockDim.x * j];
            to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
        };
        float parts[4 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            F2 tx = f2(0.0f), ts = f2(0.0f), tq = f2(0.0f);
#pragma unroll
            for (int j = 0; j < BN_NV; ++j) {
                uint32_t x[4], s[4], dy[4];
                take(r, 1, j, x);
                take(r, 2, j, s);
                take(r, 3, j, dy);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const F2 xe = f2_bf16(x[e]), se = f2_bf16(s[e]);
                    tx = f2_fma(xe, xe, tx);
                    ts = f2_fma(se, se, ts);
                    tq = f2_fma(f2_mul(f2_bf16(dy[e]), f2_bf16(w[j][e])), se, tq);
                }
            }
            parts[4 * r] = f2_sum(tx), parts[4 * r + 1] = f2_sum(ts), parts[4 * r + 2] = f2_sum(tq), parts[4 * r + 3] = 0.0f;
        }
        const float part = bn_warp_sums(parts, lane);
        if ((lane & (8 / R - 1)) == 0) reinterpret_cast<float*>(sm.sums[turn] + warp * R)[lane / (8 / R)] = part;
        if (warps > 1) __syncthreads();
        else __syncwarp();
        float rx[R], ks[R];
        F2 rs2[R], ks2[R], c2[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float4 t = sm.sums[turn][r];
            for (int i = 1; i < warps; ++i) {
                const float4 more = sm.sums[turn][i * R + r];
                t.x += more.x, t.y += more.y, t.z += more.z;
            }
            const float rs = norm && there[r] ? rsqrtf(fmaf(t.y, inv_h, p.eps)) : 0.0f;
            rx[r] = post && there[r] ? rsqrtf(fmaf(t.x, inv_h, p.eps)) : 1.0f;
            ks[r] = -(rs * rs * rs * (t.z * inv_h));
            rs2[r] = f2(rs), ks2[r] = f2(ks[r]), c2[r] = f2(gt[r] * rx[r]);
        }
        uint32_t x[R][BN_NV][4];
        F2 Gf[R][BN_NV][4], td[R];                           // G times its factor
#pragma unroll
        for (int r = 0; r < R; ++r) td[r] = f2(0.0f);
#pragma unroll
        for (int j = 0; j < BN_NV; ++j) {
            const float4 f0 = factors[2 * j * blockDim.x + tid], f1 = factors[(2 * j + 1) * blockDim.x + tid];
            const F2 f[4] = {f2(f0.x, f0.y), f2(f0.z, f0.w), f2(f1.x, f1.y), f2(f1.z, f1.w)};
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint32_t ds[4], s[4], dy[4], out[4];
                take(r, 0, j, ds);
                take(r, 1, j, x[r][j]);
                take(r, 2, j, s);
                take(r, 3, j, dy);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const F2 xe = f2_bf16(x[r][j][e]), se = f2_bf16(s[e]), rdy = f2_mul(rs2[r], f2_bf16(dy[e]));
                    const F2 G = f2_fma(ks2[r], se, f2_fma(rdy, f2_bf16(w[j][e]), f2_bf16(ds[e])));
                    sum_w[j][e] = f2_fma(rdy, se, sum_w[j][e]);
                    sum_c[j][e] = f2_fma(f2_mul(G, xe), c2[r], sum_c[j][e]);
                    Gf[r][j][e] = f2_mul(G, f[e]);
                    td[r] = f2_fma(Gf[r][j][e], xe, td[r]);
                    float lo, hi;
                    f2_get(G, lo, hi);
                    out[e] = pack_bf16x2(lo, hi);
                }
                if (there[r] && tid + static_cast<int>(blockDim.x) * j < nvec)
                    reinterpret_cast<uint4*>(p.d_residual)[(row0 + r) * nvec + tid + blockDim.x * j] = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        float dots[R];
#pragma unroll
        for (int r = 0; r < R; ++r) dots[r] = f2_sum(td[r]);
        const float dot = bn_warp_sums(dots, lane);
        if ((lane & (32 / R - 1)) == 0) sm.dots[turn][warp * R + lane / (32 / R)] = dot;
        if (warps > 1) __syncthreads();
        else __syncwarp();
        // everybody is through with the rows: later ones take their slots
        if (tid == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) request(row_of(q + r + shape.slots), slots[r]);
        }
        if (branch) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float t = sm.dots[turn][r];
                for (int i = 1; i < warps; ++i) t += sm.dots[turn][i * R + r];
                if (p.gate_kind == GATE_TOKEN && there[r] && tid == 0) p.d_gate[row0 + r] = rx[r] * t;
                const F2 kx2 = f2(post ? -(gt[r] * rx[r] * rx[r] * rx[r] * (t * inv_h)) : 0.0f);
#pragma unroll
                for (int j = 0; j < BN_NV; ++j) {
                    uint32_t out[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float lo, hi;
                        f2_get(f2_fma(c2[r], Gf[r][j][e], f2_mul(kx2, f2_bf16(x[r][j][e]))), lo, hi);
                        out[e] = pack_bf16x2(lo, hi);
                    }
                    if (there[r] && tid + static_cast<int>(blockDim.x) * j < nvec)
                        reinterpret_cast<uint4*>(p.d_x)[(row0 + r) * nvec + tid + blockDim.x * j] = make_uint4(out[0], out[1], out[2], out[3]);
                }
            }
        }
        turn ^= 1;
    }
    auto keep = [&](int plane, const F2 (&sum)[BN_NV][4]) {
#pragma unroll
        for (int j = 0; j < BN_NV; ++j) {
            if (tid + static_cast<int>(blockDim.x) * j >= nvec) continue;
            float v[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) f2_get(sum[j][e], v[2 * e], v[2 * e + 1]);
            float4* to = reinterpret_cast<float4*>(p.part + (static_cast<long long>(plane) * gridDim.x + blockIdx.x) * p.H) + 2 * (tid + blockDim.x * j);
            to[0] = make_float4(v[0], v[1], v[2], v[3]);
            to[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    };
    if (norm) keep(0, sum_w);
    if (post || p.gate_kind == GATE_CHANNEL) keep(1, sum_c);
}

// Column sums over the CTAs of the gradient: warp w of a CTA adds up the sums of CTAs w, w + 16, ... of 128 columns, then the
// sixteen are added up.  blockIdx.y: 0 the weight's, 1 the post weight's and the gate's.
constexpr int BN_FOLD_WARPS = 16;
__global__ void __launch_bounds__(BN_FOLD_WARPS * 32) block_norm_fold_kernel(const BlockNormParams p, int ctas) {
    __shared__ float4 sums[BN_FOLD_WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;      // four columns a lane
    pdl_wait();
    pdl_launch_dependents();
    const bool there = blockIdx.y == 0 ? p.d_weight != nullptr : p.d_post_weight != nullptr || p.gate_kind == GATE_CHANNEL;
    if (!there) return;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (4 * c < p.H) {
        const float4* from = reinterpret_cast<const float4*>(p.part + static_cast<long long>(blockIdx.y) * ctas * p.H) + c;
#pragma unroll 8
        for (int i = warp; i < ctas; i += BN_FOLD_WARPS) {
            const float4 v = __ldcg(from + static_cast<long long>(i) * (p.H / 4));
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || 4 * c >= p.H) return;
#pragma unroll
    for (int i = 1; i < BN_FOLD_WARPS; ++i) {
        const float4 v = sums[i][lane];
        s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int h = 4 * c + e;
        if (blockIdx.y == 0) {
            p.d_weight[h] = v[e];
            continue;
        }
        const float g = p.gate_kind == GATE_CHANNEL ? __bfloat162float(p.gate[h]) : 1.0f;
        const float w = p.post_weight ? __bfloat162float(p.post_weight[h]) : 1.0f;
        if (p.d_post_weight) p.d_post_weight[h] = p.branch_scale * g * v[e];
        if (p.gate_kind == GATE_CHANNEL) p.d_gate[h] = p.branch_scale * w * v[e];
    }
}

// Threads for BN_NV vectors each, two rows at a time while those are at most eight warps; as many CTAs on an SM as their registers
// leave room for and as keep a row more than those in the ring, which fills shared memory.  (148 SMs: the number of CTAs decides
// the order of the sums over tokens, so it does not follow the device.)
static BlockNormBwdShape bwd_shape(int64_t T, int H) {
    BlockNormBwdShape s;
    s.threads = (H / 8 + 32 * BN_NV - 1) / (32 * BN_NV) * 32;
    s.rows = s.threads <= 256 ? 2 : 1;
    s.slot_bytes = 4 * 16 * BN_NV * s.threads;
    s.factor_bytes = 32 * BN_NV * s.threads;
    int per_sm = std::min(16, std::max(1, 32 * BN_SM_WARPS / s.threads));
    auto slots = [&]() { return (228 * 1024 / per_sm - 1024 - BN_RING - s.factor_bytes) / s.slot_bytes; };
    while (per_sm > 1 && slots() <= s.rows) --per_sm;
    s.ctas = static_cast<int>(std::min<int64_t>((T + s.rows - 1) / s.rows, 148ll * per_sm));
    s.slots = std::min(8, slots());
    s.smem = BN_RING + s.factor_bytes + static_cast<size_t>(s.slots) * s.slot_bytes;
    return s;
}
size_t block_norm_bwd_bytes(int64_t T, int H) { return static_cast<size_t>(bwd_shape(T, H).ctas) * 2 * H * sizeof(float); }

cudaError_t launch_block_norm(const BlockNormParams& p, cudaStream_t stream) {
    const int nv = (p.H / 8 + BN_THREADS - 1) / BN_THREADS;
    auto kern = nv <= 1 ? block_norm_kernel<1> : nv <= 2 ? block_norm_kernel<2> : nv <= 4 ? block_norm_kernel<4> : block_norm_kernel<8>;
    return launch_pdl(kern, dim3(static_cast<unsigned>(p.T)), BN_THREADS, 0, stream, 1, p);
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, cudaStream_t stream) {
    const BlockNormBwdShape shape = bwd_shape(p.T, p.H);
    if (shape.ctas > 0) {
        static DeviceOnce configured;
        cudaError_t e = configured.run([&]() {
            const cudaError_t e1 = cudaFuncSetAttribute(block_norm_bwd_kernel<1>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
            return e1 != cudaSuccess ? e1 : cudaFuncSetAttribute(block_norm_bwd_kernel<2>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
        });
        if (e != cudaSuccess) return e;
        auto kern = shape.rows == 2 ? block_norm_bwd_kernel<2> : block_norm_bwd_kernel<1>;
        e = launch_pdl(kern, dim3(shape.ctas), shape.threads, shape.smem, stream, 1, p, shape);
        if (e != cudaSuccess) return e;
    }
    if (!p.d_weight && !p.d_post_weight && p.gate_kind != GATE_CHANNEL) return cudaSuccess;
    return launch_pdl(block_norm_fold_kernel, dim3((p.H + 127) / 128, 2), BN_FOLD_WARPS * 32, 0, stream, 1, p, shape.ctas);
}

}  // namespace tik
