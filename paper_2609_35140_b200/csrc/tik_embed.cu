// Embedding lookup and its gradient by sorted tokens.
#include <cuda_bf16.h>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int EMB_THREADS = 256;

__device__ __forceinline__ uint4 scaled8(uint4 v, float scale) {
    float f[8];
    unpack8(v, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __fmul_rn(f[e], scale);
    return pack8(f);
}

// y[t] = scale * table[ids[t]]: one 16-byte vector per thread.
__global__ void __launch_bounds__(EMB_THREADS) embed_kernel(const EmbedParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int vpr = p.H / 8;
    const long long i = static_cast<long long>(blockIdx.x) * EMB_THREADS + threadIdx.x;
    if (i >= p.T * vpr) return;
    const long long t = i / vpr;
    const int c = static_cast<int>(i - t * vpr), id = p.ids[t];
    uint4 v = make_uint4(0, 0, 0, 0);
    if (id >= 0 && id < p.V) v = scaled8(reinterpret_cast<const uint4*>(p.table)[static_cast<long long>(id) * vpr + c], p.scale);
    else if (c == 0) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
    reinterpret_cast<uint4*>(p.y)[i] = v;
}

// Tokens by id, equal ids by position: a token's place is the number of tokens before it in that order.
__global__ void __launch_bounds__(EMB_THREADS) embed_rank_kernel(const EmbedParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int t = static_cast<int>(blockIdx.x) * EMB_THREADS + threadIdx.x, T = static_cast<int>(p.T);
    if (t >= T) return;
    auto key = [&](int i) {
        const int id = p.ids[i];
        return id >= 0 && id < p.V ? id : p.V;
    };
    const int mine = key(t);
    if (mine == p.V) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
    int place = 0;
    for (int i = 0; i < T; ++i) {
        const int k = key(i);
        place += k < mine || (k == mine && i < t);
    }
    p.sorted[place] = mine;
    p.order[place] = t;
}

// One CTA per table row: its tokens lie next to each other in the sorted list.
__global__ void __launch_bounds__(EMB_THREADS) embed_rows_kernel(const EmbedParams p) {
    pdl_wait();
    pdl_launch_dependents();
    const int v = blockIdx.x;
    auto lower = [&](int key) {
        int lo = 0, hi = static_cast<int>(p.T);
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (p.sorted[mid] < key) lo = mid + 1;
            else hi = mid;
        }
        return lo;
    };
    const int first = lower(v), last = lower(v + 1);
    if (first == last && p.accumulate) return;
    const int vpr = p.H / 8;
    for (int c = threadIdx.x; c < vpr; c += EMB_THREADS) {
        float sum[8] = {};
        for (int i = first; i < last; ++i) {
            float f[8];
            unpack8(reinterpret_cast<const uint4*>(p.d_y)[static_cast<long long>(p.order[i]) * vpr + c], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __fadd_rn(sum[e], f[e]);
        }
        const long long at = static_cast<long long>(v) * vpr + c;
        float old[8] = {};
        if (p.fp32) {
            float4* d = reinterpret_cast<float4*>(p.d_table) + 2 * at;
            if (p.accumulate) {
                const float4 a = d[0], b = d[1];
                old[0] = a.x, old[1] = a.y, old[2] = a.z, old[3] = a.w, old[4] = b.x, old[5] = b.y, old[6] = b.z, old[7] = b.w;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __fmaf_rn(p.scale, sum[e], old[e]);
            d[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            d[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
        } else {
            uint4* d = reinterpret_cast<uint4*>(p.d_table) + at;
            if (p.accumulate) unpack8(*d, old);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __fmaf_rn(p.scale, sum[e], old[e]);
            *d = pack8(sum);
        }
    }
}

size_t embed_bwd_bytes(int64_t T, int, int) { return static_cast<size_t>(T) * 8; }

cudaError_t launch_embed(const EmbedParams& p, cudaStream_t stream) {
    const long long n = p.T * (p.H / 8);
    return launch_pdl(embed_kernel, dim3(static_cast<unsigned>((n + EMB_THREADS - 1) / EMB_THREADS)), EMB_THREADS, 0, stream, 1, p);
}

cudaError_t launch_embed_bwd(EmbedParams& p, void* ws, cudaStream_t stream) {
    p.sorted = static_cast<int32_t*>(ws);
    p.order = p.sorted + p.T;
    if (p.T > 0) {
        const unsigned grid = static_cast<unsigned>((p.T + EMB_THREADS - 1) / EMB_THREADS);
        cudaError_t e = launch_pdl(embed_rank_kernel, dim3(grid), EMB_THREADS, 0, stream, 1, p);
        if (e != cudaSuccess) return e;
    }
    return launch_pdl(embed_rows_kernel, dim3(static_cast<unsigned>(p.V)), EMB_THREADS, 0, stream, 1, p);
}

}  // namespace tik
