// The step between two blocks of a layer -- norm after the block, gate, scaled residual sum, norm before the next block --
// and its gradient.
#include <cuda_bf16.h>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int BN_THREADS = 128;
constexpr int BN_BWD_CTAS = 296;

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

// Sum of N values over a CTA of W warps, the same bits in every thread.  buf: W * N floats that the CTA's previous
// reduction does not use.
template <int N, int W>
__device__ __forceinline__ void bn_block_sum(float (&v)[N], float* buf, int warp, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = hn_warp_total(v[i]);
        if (lane == 0) buf[warp * N + i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = buf[i];
#pragma unroll
        for (int w = 1; w < W; ++w) t = __fadd_rn(t, buf[w * N + i]);
        v[i] = t;
    }
}

// Rows blockIdx.x, + gridDim.x, ... of the gradient; the sums over a CTA's rows stay in registers.
template <int THREADS, int NV>
__global__ void __launch_bounds__(THREADS) block_norm_bwd_kernel(const BlockNormParams p) {
    constexpr int W = THREADS / 32;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int nvec = p.H / 8;
    const float inv_h = 1.0f / static_cast<float>(p.H);
    __shared__ float red_a[2][W * 3], red_b[W];        // (without x a row has one reduction: red_a alternates)
    pdl_wait();
    pdl_launch_dependents();
    float sum_w[NV][8] = {}, sum_c[NV][8] = {};
    const uint4 zero = make_uint4(0, 0, 0, 0);
    auto at = [&](const __nv_bfloat16* base, long long row, int v) {
        return base && v < nvec ? reinterpret_cast<const uint4*>(base)[row * nvec + v] : zero;
    };
    int turn = 0;
    for (long long row = blockIdx.x; row < p.T; row += gridDim.x, turn ^= 1) {
        uint4 dyv[NV], dsv[NV], xv[NV], sv[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = tid + THREADS * j;
            dyv[j] = at(p.d_y, row, v);
            dsv[j] = at(p.d_s, row, v);
            xv[j] = at(p.x, row, v);
            sv[j] = p.weight ? at(p.s, row, v) : zero;
        }
        const float a = p.branch_scale * (p.gate_kind == GATE_TOKEN ? __bfloat162float(p.gate[row]) : 1.0f);
        float tot[3] = {};                         // x^2, s^2, q s
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[8], s[8], dy[8], w[8];
            unpack8(xv[j], x);
            unpack8(sv[j], s);
            unpack8(dyv[j], dy);
            unpack8(at(p.weight, 0, tid + THREADS * j), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                tot[0] = __fmaf_rn(x[e], x[e], tot[0]);
                tot[1] = __fmaf_rn(s[e], s[e], tot[1]);
                tot[2] = __fmaf_rn(dy[e] * w[e], s[e], tot[2]);
            }
        }
        bn_block_sum<3, W>(tot, red_a[turn], warp, lane);
        const float rx = prep_inv_rms(tot[0], inv_h, p.eps), rs = prep_inv_rms(tot[1], inv_h, p.eps);
        const float ks = p.weight ? rs * rs * rs * (tot[2] * inv_h) : 0.0f;
        float G[NV][8], dot[1] = {};               // G; sum of d_n o n (gate per channel: without the gate's gradient in mind)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = tid + THREADS * j;
            float x[8], s[8], dy[8], w[8], ds[8], wp[8], g[8];
            unpack8(xv[j], x);
            unpack8(sv[j], s);
            unpack8(dyv[j], dy);
            unpack8(dsv[j], ds);
            unpack8(at(p.weight, 0, v), w);
            unpack8(at(p.post_weight, 0, v), wp);
            if (p.gate_kind == GATE_CHANNEL) unpack8(at(p.gate, 0, v), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float t = ds[e];
                if (p.weight) {
                    t += rs * (dy[e] * w[e]) - ks * s[e];
                    sum_w[j][e] = __fmaf_rn(dy[e], s[e] * rs, sum_w[j][e]);
                }
                G[j][e] = t;
                const float gx = t * (p.post_weight ? x[e] * rx : x[e]);       // G o (x normalised, or x)
                sum_c[j][e] = __fmaf_rn(p.gate_kind == GATE_TOKEN ? __bfloat162float(p.gate[row]) : 1.0f, gx, sum_c[j][e]);
                dot[0] = __fmaf_rn(gx, (p.post_weight ? wp[e] : 1.0f) * (p.gate_kind == GATE_CHANNEL ? g[e] : 1.0f), dot[0]);
            }
        }
        if (p.x) bn_block_sum<1, W>(dot, red_b, warp, lane);
        if (p.gate_kind == GATE_TOKEN && tid == 0) p.d_gate[row] = p.branch_scale * dot[0];
        const float kx = rx * rx * (a * dot[0] * inv_h);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int v = tid + THREADS * j;
            if (v >= nvec) continue;
            reinterpret_cast<uint4*>(p.d_residual)[row * nvec + v] = pack8(G[j]);
            if (!p.x) continue;
            float x[8], wp[8], g[8], dx[8];
            unpack8(xv[j], x);
            unpack8(at(p.post_weight, 0, v), wp);
            if (p.gate_kind == GATE_CHANNEL) unpack8(at(p.gate, 0, v), g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float dn = a * (p.gate_kind == GATE_CHANNEL ? g[e] : 1.0f) * G[j][e];
                dx[e] = p.post_weight ? rx * (dn * wp[e]) - kx * x[e] : dn;
            }
            reinterpret_cast<uint4*>(p.d_x)[row * nvec + v] = pack8(dx);
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + THREADS * j;
        if (v >= nvec) continue;
        float4* to = reinterpret_cast<float4*>(p.part + (static_cast<long long>(blockIdx.x) * 2) * p.H) + 2 * v;
        to[0] = make_float4(sum_w[j][0], sum_w[j][1], sum_w[j][2], sum_w[j][3]);
        to[1] = make_float4(sum_w[j][4], sum_w[j][5], sum_w[j][6], sum_w[j][7]);
        to += p.H / 4;
        to[0] = make_float4(sum_c[j][0], sum_c[j][1], sum_c[j][2], sum_c[j][3]);
        to[1] = make_float4(sum_c[j][4], sum_c[j][5], sum_c[j][6], sum_c[j][7]);
    }
}

// Column sums over the CTAs of the gradient, in their order.
__global__ void __launch_bounds__(BN_THREADS) block_norm_fold_kernel(const BlockNormParams p, int ctas) {
    pdl_wait();
    pdl_launch_dependents();
    const int h = blockIdx.x * BN_THREADS + threadIdx.x;
    if (h >= p.H) return;
    float sum_w = 0.0f, sum_c = 0.0f;
    for (int i = 0; i < ctas; ++i) {
        sum_w = __fadd_rn(sum_w, p.part[(2ll * i) * p.H + h]);
        sum_c = __fadd_rn(sum_c, p.part[(2ll * i + 1) * p.H + h]);
    }
    const float g = p.gate_kind == GATE_CHANNEL ? __bfloat162float(p.gate[h]) : 1.0f;
    const float w = p.post_weight ? __bfloat162float(p.post_weight[h]) : 1.0f;
    if (p.d_weight) p.d_weight[h] = sum_w;
    if (p.d_post_weight) p.d_post_weight[h] = p.branch_scale * g * sum_c;
    if (p.gate_kind == GATE_CHANNEL) p.d_gate[h] = p.branch_scale * w * sum_c;
}

static int bwd_ctas(int64_t T) { return static_cast<int>(std::min<int64_t>(T, BN_BWD_CTAS)); }
size_t block_norm_bwd_bytes(int64_t T, int H) { return static_cast<size_t>(bwd_ctas(T)) * 2 * H * sizeof(float); }

cudaError_t launch_block_norm(const BlockNormParams& p, cudaStream_t stream) {
    const int nv = (p.H / 8 + BN_THREADS - 1) / BN_THREADS;
    auto kern = nv <= 1 ? block_norm_kernel<1> : nv <= 2 ? block_norm_kernel<2> : nv <= 4 ? block_norm_kernel<4> : block_norm_kernel<8>;
    return launch_pdl(kern, dim3(static_cast<unsigned>(p.T)), BN_THREADS, 0, stream, 1, p);
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, cudaStream_t stream) {
    const int ctas = bwd_ctas(p.T), nvec = p.H / 8;
    if (ctas > 0) {
        auto go = [&](auto kern, unsigned threads) { return launch_pdl(kern, dim3(ctas), threads, 0, stream, 1, p); };
        cudaError_t e = nvec <= 128 ? go(block_norm_bwd_kernel<128, 1>, 128) : nvec <= 256 ? go(block_norm_bwd_kernel<256, 1>, 256)
                      : nvec <= 512 ? go(block_norm_bwd_kernel<256, 2>, 256) : go(block_norm_bwd_kernel<512, 2>, 512);
        if (e != cudaSuccess) return e;
    }
    if (!p.d_weight && !p.d_post_weight && p.gate_kind != GATE_CHANNEL) return cudaSuccess;
    return launch_pdl(block_norm_fold_kernel, dim3((p.H + BN_THREADS - 1) / BN_THREADS), BN_THREADS, 0, stream, 1, p, ctas);
}

}  // namespace tik
