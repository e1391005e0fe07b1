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
// G x (post weight, gate), which gives d_x.  Six planes of T x H cross HBM once, which bounds the kernel; the arithmetic is
// ~20 operations an element, two-wide where it can be.  Persistent CTAs, several on an SM, so that one's sums across its warps
// pass under another's arithmetic; rows arrive by bulk copies, a few rows ahead.  A thread has the same BN_NV x 8 columns of
// every row, so that the sums over tokens stay in its registers until the end; block_norm_fold_kernel adds up the CTAs'.
constexpr int BN_NV = 2;                                     // 16-byte vectors per thread
constexpr int BN_MAX_THREADS = 512;

struct BlockNormBwdShape {
    int threads, ctas, stages, stage_bytes, row_bytes;
    size_t smem;
};
struct BlockNormBwdSmem {
    unsigned long long full[8];
    float4 sums[2][BN_MAX_THREADS / 32];
    float dots[2][BN_MAX_THREADS / 32];
    int abort_word;
};
constexpr size_t BN_RING = (sizeof(BlockNormBwdSmem) + 127) / 128 * 128;

__device__ __forceinline__ void bn_cta_sync(int warps) {
    if (warps == 1) __syncwarp();
    else __syncthreads();
}

template <int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) block_norm_bwd_kernel(const BlockNormParams p, const BlockNormBwdShape shape) {
    extern __shared__ __align__(128) unsigned char bn_smem[];
    BlockNormBwdSmem& sm = *reinterpret_cast<BlockNormBwdSmem*>(bn_smem);
    unsigned char* ring = bn_smem + BN_RING;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, warps = blockDim.x >> 5;
    const int nvec = p.H / 8;
    const float inv_h = 1.0f / static_cast<float>(p.H);
    if (tid == 0) {
        for (int i = 0; i < shape.stages; ++i) mbar_init(smem_u32(&sm.full[i]), 1);
        sm.abort_word = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const bool norm = p.weight != nullptr, post = p.post_weight != nullptr, branch = p.x != nullptr;
    const int planes = (norm ? 2 : 0) + (branch ? 1 : 0) + (p.d_s ? 1 : 0);
    // slots of a stage: d_s, x, s, d_y
    auto request = [&](long long row, int stage) {
        const uint32_t bar = smem_u32(&sm.full[stage]), to = smem_u32(ring + stage * shape.stage_bytes);
        mbar_expect_tx(bar, planes * p.H * 2);
        const __nv_bfloat16* src[4] = {p.d_s, p.x, norm ? p.s : nullptr, norm ? p.d_y : nullptr};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (src[i]) bulk_load(to + i * shape.row_bytes, src[i] + row * p.H, p.H * 2, bar);
    };
    if (tid == 0)
        for (int i = 0; i < shape.stages && blockIdx.x + static_cast<long long>(i) * gridDim.x < p.T; ++i)
            request(blockIdx.x + static_cast<long long>(i) * gridDim.x, i);
    // factors of this thread's columns: weight; branch_scale * post_weight * gate (per channel)
    uint32_t w[BN_NV][4];
    F2 f[BN_NV][4], sum_w[BN_NV][4], sum_c[BN_NV][4];
    bool in[BN_NV];
#pragma unroll
    for (int j = 0; j < BN_NV; ++j) {
        const int v = tid + static_cast<int>(blockDim.x) * j;
        in[j] = v < nvec;
        auto words = [&](const __nv_bfloat16* base, bool there) {
            return there && in[j] ? reinterpret_cast<const uint4*>(base)[v] : make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
        };
        const uint4 wv = words(p.weight, norm), pv = words(p.post_weight, post), gv = words(p.gate, p.gate_kind == GATE_CHANNEL);
        const uint32_t ww[4] = {wv.x, wv.y, wv.z, wv.w}, pw[4] = {pv.x, pv.y, pv.z, pv.w}, gw[4] = {gv.x, gv.y, gv.z, gv.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[j][e] = ww[e];
            f[j][e] = f2_mul(f2(p.branch_scale), f2_mul(f2_bf16(pw[e]), f2_bf16(gw[e])));
            sum_w[j][e] = sum_c[j][e] = f2(0.0f);
        }
    }
    int stage = 0, turn = 0;
    uint32_t parity = 0;
    for (long long row = blockIdx.x; row < p.T; row += gridDim.x) {
        const float gt = p.gate_kind == GATE_TOKEN ? __bfloat162float(p.gate[row]) : 1.0f;
        mbar_wait(smem_u32(&sm.full[stage]), parity, &sm.abort_word, p.dev_status);
        const unsigned char* at = ring + stage * shape.stage_bytes;
        uint32_t ds[BN_NV][4], x[BN_NV][4], s[BN_NV][4], dy[BN_NV][4];
        auto take = [&](int slot, bool there, uint32_t (&to)[BN_NV][4]) {
#pragma unroll
            for (int j = 0; j < BN_NV; ++j) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (there && in[j]) v = reinterpret_cast<const uint4*>(at + slot * shape.row_bytes)[tid + blockDim.x * j];
                to[j][0] = v.x, to[j][1] = v.y, to[j][2] = v.z, to[j][3] = v.w;
            }
        };
        take(0, p.d_s != nullptr, ds);
        take(1, branch, x);
        take(2, norm, s);
        take(3, norm, dy);
        F2 tx = f2(0.0f), ts = f2(0.0f), tq = f2(0.0f);
#pragma unroll
        for (int j = 0; j < BN_NV; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const F2 xe = f2_bf16(x[j][e]), se = f2_bf16(s[j][e]);
                tx = f2_fma(xe, xe, tx);
                ts = f2_fma(se, se, ts);
                tq = f2_fma(f2_mul(f2_bf16(dy[j][e]), se), f2_bf16(w[j][e]), tq);
            }
        float sx = hn_warp_total(f2_sum(tx)), ss = hn_warp_total(f2_sum(ts)), sq = hn_warp_total(f2_sum(tq));
        if (warps > 1) {
            if (lane == 0) sm.sums[turn][warp] = make_float4(sx, ss, sq, 0.0f);
            __syncthreads();
            const float4 first = sm.sums[turn][0];
            sx = first.x, ss = first.y, sq = first.z;
            for (int i = 1; i < warps; ++i) {
                const float4 t = sm.sums[turn][i];
                sx += t.x, ss += t.y, sq += t.z;
            }
        } else {
            __syncwarp();
        }
        // everybody has the row in registers: its stage takes a later row
        if (tid == 0 && row + static_cast<long long>(shape.stages) * gridDim.x < p.T) request(row + static_cast<long long>(shape.stages) * gridDim.x, stage);
        if (++stage == shape.stages) {
            stage = 0;
            parity ^= 1;
        }
        const float rs = norm ? prep_inv_rms(ss, inv_h, p.eps) : 0.0f, rx = post ? prep_inv_rms(sx, inv_h, p.eps) : 1.0f;
        const F2 rs2 = f2(rs), ks2 = f2(-(rs * rs * rs * (sq * inv_h))), c2 = f2(gt * rx);
        F2 G[BN_NV][4], td = f2(0.0f);
#pragma unroll
        for (int j = 0; j < BN_NV; ++j) {
            uint32_t out[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const F2 se = f2_bf16(s[j][e]), rdy = f2_mul(rs2, f2_bf16(dy[j][e]));
                G[j][e] = f2_fma(ks2, se, f2_fma(rdy, f2_bf16(w[j][e]), f2_bf16(ds[j][e])));
                sum_w[j][e] = f2_fma(rdy, se, sum_w[j][e]);
                const F2 gx = f2_mul(G[j][e], f2_bf16(x[j][e]));
                sum_c[j][e] = f2_fma(gx, c2, sum_c[j][e]);
                td = f2_fma(gx, f[j][e], td);
                float lo, hi;
                f2_get(G[j][e], lo, hi);
                out[e] = pack_bf16x2(lo, hi);
            }
            if (in[j]) reinterpret_cast<uint4*>(p.d_residual)[row * nvec + tid + blockDim.x * j] = make_uint4(out[0], out[1], out[2], out[3]);
        }
        if (branch) {
            float dot = 0.0f;
            if (post || p.gate_kind == GATE_TOKEN) {
                dot = hn_warp_total(f2_sum(td));
                if (warps > 1) {
                    if (lane == 0) sm.dots[turn][warp] = dot;
                    __syncthreads();
                    dot = sm.dots[turn][0];
                    for (int i = 1; i < warps; ++i) dot += sm.dots[turn][i];
                }
                if (p.gate_kind == GATE_TOKEN && tid == 0) p.d_gate[row] = rx * dot;
            }
            const F2 kx2 = f2(post ? -(gt * rx * rx * rx * (dot * inv_h)) : 0.0f);
#pragma unroll
            for (int j = 0; j < BN_NV; ++j) {
                uint32_t out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const F2 dn = f2_mul(c2, f2_mul(f[j][e], G[j][e]));
                    float lo, hi;
                    f2_get(post ? f2_fma(kx2, f2_bf16(x[j][e]), dn) : dn, lo, hi);
                    out[e] = pack_bf16x2(lo, hi);
                }
                if (in[j]) reinterpret_cast<uint4*>(p.d_x)[row * nvec + tid + blockDim.x * j] = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
        turn ^= 1;                               // (a row without the second sum has one barrier: the next one's sums go elsewhere)
    }
    auto keep = [&](int plane, const F2 (&sum)[BN_NV][4]) {
#pragma unroll
        for (int j = 0; j < BN_NV; ++j) {
            if (!in[j]) continue;
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

// Threads for BN_NV vectors each; as many CTAs as 128 registers a thread leave room for on an SM (148 of them: the number decides
// the order of the sums over tokens, so it does not follow the device); the ring fills shared memory, four rows at most.
static BlockNormBwdShape bwd_shape(int64_t T, int H) {
    BlockNormBwdShape s;
    s.threads = (H / 8 + 32 * BN_NV - 1) / (32 * BN_NV) * 32;
    const int per_sm = std::min(16, std::max(1, BN_MAX_THREADS / s.threads));
    s.ctas = static_cast<int>(std::min<int64_t>(T, 148ll * per_sm));
    s.row_bytes = (2 * H + 127) / 128 * 128;
    s.stage_bytes = 4 * s.row_bytes;
    const size_t room = (227u * 1024) / per_sm - 1024 - BN_RING;
    s.stages = static_cast<int>(std::max<size_t>(1, std::min<size_t>(4, room / s.stage_bytes)));
    s.smem = BN_RING + static_cast<size_t>(s.stages) * s.stage_bytes;
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
            const cudaError_t e1 = cudaFuncSetAttribute(block_norm_bwd_kernel<256, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024);
            return e1 != cudaSuccess ? e1 : cudaFuncSetAttribute(block_norm_bwd_kernel<BN_MAX_THREADS, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024);
        });
        if (e != cudaSuccess) return e;
        auto kern = shape.threads <= 256 ? block_norm_bwd_kernel<256, 2> : block_norm_bwd_kernel<BN_MAX_THREADS, 1>;
        e = launch_pdl(kern, dim3(shape.ctas), shape.threads, shape.smem, stream, 1, p, shape);
        if (e != cudaSuccess) return e;
    }
    if (!p.d_weight && !p.d_post_weight && p.gate_kind != GATE_CHANNEL) return cudaSuccess;
    return launch_pdl(block_norm_fold_kernel, dim3((p.H + 127) / 128, 2), BN_FOLD_WARPS * 32, 0, stream, 1, p, shape.ctas);
}

}  // namespace tik
