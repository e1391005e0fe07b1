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

// ---- gradient --------------------------------------------------------------------------------
// Tokens are brought into the order of their ids, equal ids by position.  A run of one id is cut, from its start, into pieces of
// EMB_PIECE tokens; a piece's rows are added up in fp32 in ascending order, and where a run has several pieces their sums
// are added up by embed_fold_kernel.  So a table row's bits depend on its own tokens' gradients and their number alone.
// What begins at a place of the order is one record, written by the sort, so that nothing has to be counted or
// searched afterwards: {id, info, tokens of the run, token}, info = length of the piece (0: a place inside of one) and flags.
constexpr int EMB_PIECE = 32;
constexpr uint32_t EMB_LEN = 63, EMB_MANY = 64, EMB_HEAD = 128;      // a run of several pieces; the first place of a run

__device__ __forceinline__ uint4 emb_record(int key, int in_run, int run, int token) {
    uint32_t info = 0;
    if (in_run % EMB_PIECE == 0) {
        const int left = run - in_run;
        info = (left < EMB_PIECE ? left : EMB_PIECE) | (run > EMB_PIECE ? EMB_MANY : 0) | (in_run == 0 ? EMB_HEAD : 0);
    }
    return make_uint4(key, info, run, token);
}
// Row of `part` for a piece of a long run: whole pieces begin EMB_PIECE places apart, and between the shorter last pieces of
// two long runs lies a whole one, so place / EMB_PIECE numbers either kind without a clash.
__device__ __forceinline__ long long emb_slot(long long place, uint32_t len) {
    return 2 * (place / EMB_PIECE) + (len < EMB_PIECE ? 1 : 0);
}
__device__ __forceinline__ int emb_key(const EmbedParams& p, int id) { return id >= 0 && id < p.V ? id : p.V; }

// Calls of few tokens: a token's place is the number of tokens before it in the order, counted by comparing all pairs.
// Lanes are tokens; the warps of a CTA share the tokens that they are compared with.
constexpr int EMB_RANK_TOKENS = 4096;
constexpr int EMB_RANK_WARPS = 8;
__global__ void __launch_bounds__(EMB_RANK_WARPS * 32) embed_rank_kernel(const EmbedParams p) {
    __shared__ int count[EMB_RANK_WARPS][3][32];
    pdl_wait();
    pdl_launch_dependents();
    const int T = static_cast<int>(p.T), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.x * 32 + lane;
    const int mine = t < T ? emb_key(p, p.ids[t]) : -1;
    int less = 0, same = 0, same_before = 0;
    const int per = (T + EMB_RANK_WARPS - 1) / EMB_RANK_WARPS, to = min(T, per * (warp + 1));
#pragma unroll 8
    for (int i = per * warp; i < to; ++i) {
        const int k = emb_key(p, p.ids[i]);
        less += k < mine;
        same += k == mine;
        same_before += k == mine && i < t;
    }
    count[warp][0][lane] = less;
    count[warp][1][lane] = same;
    count[warp][2][lane] = same_before;
    __syncthreads();
    if (warp != 0 || t >= T) return;
    less = same = same_before = 0;
#pragma unroll
    for (int w = 0; w < EMB_RANK_WARPS; ++w) {
        less += count[w][0][lane];
        same += count[w][1][lane];
        same_before += count[w][2][lane];
    }
    const int at = less + same_before;
    p.order[at] = t;
    uint4 rec = emb_record(mine, same_before, same, t);
    if (mine == p.V) {
        atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
        rec.y = 0;
    }
    p.place[at] = rec;
}

// Other calls: a stable radix sort by one cluster of eight CTAs, whose 256 warps own consecutive stretches of the list.  Per
// digit: each warp counts its digits, the CTAs exchange their counts through distributed shared memory, and each
// warp moves its elements, in order, to where the elements before them end.
constexpr int EMB_CLUSTER = 8, EMB_SORT_THREADS = 1024, EMB_SORT_WARPS = EMB_SORT_THREADS / 32;
constexpr int EMB_BINS = 512;
constexpr size_t EMB_SORT_SMEM = (EMB_SORT_WARPS * EMB_BINS + EMB_BINS + 32) * sizeof(int);

__device__ __forceinline__ int ld_cluster_int(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
// first place of [0, n) whose key is >= key, found by a whole warp (keys ascending)
__device__ __forceinline__ int emb_lower_bound(const uint2* keys, int n, uint32_t key, int lane) {
    int lo = 0, hi = n;                      // keys before lo are < key, keys from hi on are not
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, probe = lo + step * (lane + 1) - 1;
        const unsigned below = __ballot_sync(0xffffffffu, probe < hi && __ldcg(&keys[probe]).x < key);
        const int c = __popc(below);
        hi = min(hi, lo + step * (c + 1) - 1);
        lo += step * c;
    }
    return lo;
}

__global__ void __launch_bounds__(EMB_SORT_THREADS) embed_sort_kernel(const EmbedParams p, int passes, int digit_bits) {
    extern __shared__ int emb_smem[];
    int* hist = emb_smem;                                        // [warps][bins]
    int* total = hist + EMB_SORT_WARPS * EMB_BINS;               // [bins] of this CTA
    int* warp_sum = total + EMB_BINS;
    const int T = static_cast<int>(p.T), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    pdl_wait();
    pdl_launch_dependents();
    const int bins = 1 << digit_bits;
    const int per = ((T + EMB_CLUSTER * EMB_SORT_WARPS - 1) / (EMB_CLUSTER * EMB_SORT_WARPS) + 31) / 32 * 32;
    const long long from = static_cast<long long>(per) * (rank * EMB_SORT_WARPS + warp);
    const int first = static_cast<int>(from < T ? from : T), last = static_cast<int>(from + per < T ? from + per : T);
    int* mine = hist + warp * EMB_BINS;
    for (int pass = 0; pass < passes; ++pass) {
        const uint2* src = p.keys[(pass + 1) & 1];               // pass 0 reads the ids
        uint2* dst = p.keys[pass & 1];
        const int shift = pass * digit_bits;
        auto element = [&](int i) { return pass == 0 ? make_uint2(emb_key(p, p.ids[i]), i) : __ldcg(&src[i]); };
        for (int i = lane; i < bins; i += 32) mine[i] = 0;
        __syncwarp();
        for (int i0 = first; i0 < last; i0 += 32) {
            const int i = i0 + lane;
            const unsigned here = __ballot_sync(0xffffffffu, i < last);
            if (i < last) {
                const int digit = (element(i).x >> shift) & (bins - 1);
                const unsigned peers = __match_any_sync(here, digit);
                if (lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
            }
            __syncwarp();
        }
        __syncthreads();
        int sum = 0;
        if (tid < bins) {                                        // a bin's counts -> counts of the warps before
#pragma unroll
            for (int w = 0; w < EMB_SORT_WARPS; ++w) {
                const int n = hist[w * EMB_BINS + tid];
                hist[w * EMB_BINS + tid] = sum;
                sum += n;
            }
            total[tid] = sum;
        }
        __syncwarp();
        cluster_sync_all();
        int before = 0, all = 0;                                 // of the CTAs before, of the cluster
        if (tid < bins) {
#pragma unroll
            for (uint32_t r = 0; r < EMB_CLUSTER; ++r) {
                const int n = ld_cluster_int(mapa_cluster(smem_u32(total + tid), r));
                before += r < rank ? n : 0;
                all += n;
            }
        }
        int scan = all;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int n = __shfl_up_sync(0xffffffffu, scan, off);
            if (lane >= off) scan += n;
        }
        if (lane == 31) warp_sum[warp] = scan;
        __syncthreads();
        int base = scan - all + before;
        for (int w = 0; w < warp; ++w) base += warp_sum[w];
        if (tid < bins) {
#pragma unroll
            for (int w = 0; w < EMB_SORT_WARPS; ++w) hist[w * EMB_BINS + tid] += base;
        }
        __syncthreads();
        for (int i0 = first; i0 < last; i0 += 32) {
            const int i = i0 + lane;
            const unsigned here = __ballot_sync(0xffffffffu, i < last);
            if (i < last) {
                const uint2 e = element(i);
                const int digit = (e.x >> shift) & (bins - 1);
                const unsigned peers = __match_any_sync(here, digit);
                const int at = mine[digit] + __popc(peers & ((1u << lane) - 1));
                __syncwarp(here);
                if (lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
                __stcg(&dst[at], e);
            }
            __syncwarp();
        }
        cluster_sync_all();
    }
    // records: a warp takes 32 places at a time and looks for the ends of the two runs that may reach beyond them
    const uint2* keys = p.keys[(passes - 1) & 1];
    const uint32_t bad = p.V;
    for (int i0 = first; i0 < last; i0 += 32) {
        const int i = i0 + lane;
        const uint2 e = i < T ? __ldcg(&keys[i]) : make_uint2(0xffffffffu, 0);
        const uint32_t left = __shfl_up_sync(0xffffffffu, e.x, 1), edge_l = i0 > 0 ? __ldcg(&keys[i0 - 1]).x : 0xfffffffeu;
        const unsigned heads = __ballot_sync(0xffffffffu, e.x != (lane == 0 ? edge_l : left));
        const uint32_t k0 = __shfl_sync(0xffffffffu, e.x, 0), k31 = __shfl_sync(0xffffffffu, e.x, 31);
        const uint32_t edge_r = i0 + 32 < T ? __ldcg(&keys[i0 + 32]).x : 0xfffffffeu;
        const int begin = heads & 1 ? i0 : emb_lower_bound(keys, T, k0, lane);
        const int end = k31 == edge_r ? emb_lower_bound(keys, T, k31 + 1, lane) : i0 + 32;
        if (i < last) {
            const unsigned upto = heads & (0xffffffffu >> (31 - lane)), after = heads & ~(0xffffffffu >> (31 - lane));
            const int head = upto ? i0 + 31 - __clz(upto) : begin;
            const int tail = after ? i0 + __ffs(after) - 1 : min(end, T);
            uint4 rec = emb_record(e.x, i - head, tail - head, e.y);
            if (e.x == bad) {
                rec.y = 0;
                if (i == head) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
            }
            p.order[i] = e.y;
            p.place[i] = rec;
        }
    }
}

// 16 bytes of bf16 or 32 of fp32 of a table row
template <bool FP32, bool ACC>
__device__ __forceinline__ void emb_store(const EmbedParams& p, long long at, float (&sum)[8]) {
    float old[8] = {};
    if (FP32) {
        float4* d = reinterpret_cast<float4*>(p.d_table) + 2 * at;
        if (ACC) {
            const float4 a = __ldcg(d), b = __ldcg(d + 1);
            old[0] = a.x, old[1] = a.y, old[2] = a.z, old[3] = a.w, old[4] = b.x, old[5] = b.y, old[6] = b.z, old[7] = b.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __fmaf_rn(p.scale, sum[e], old[e]);
        d[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        d[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    } else {
        uint4* d = reinterpret_cast<uint4*>(p.d_table) + at;
        if (ACC) unpack8(__ldcg(d), old);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __fmaf_rn(p.scale, sum[e], old[e]);
        *d = pack8(sum);
    }
}
__device__ __forceinline__ void emb_add(float (&sum)[8], const uint4& v) {
    float f[8];
    unpack8(v, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = __fadd_rn(sum[e], f[e]);
}

// Zeros for the rows without a token, and the pieces' sums.  The zeros need the ids alone, so they start while the sort runs:
// every CTA marks which of its share of the rows occur, and one warp copies zeros over the others by bulk stores,
// which take no other warp's issue slots.  The sort releases its dependents behind its own wait, so whatever came
// before it has completed when this grid starts, and it writes neither ids nor table.
constexpr int EMB_SUM_THREADS = 1024, EMB_SUM_WARPS = EMB_SUM_THREADS / 32;
constexpr int EMB_MARK_ROWS = 32768;                         // rows marked at a time
constexpr int EMB_ZEROS = 8192;                              // bytes of a bulk store
template <bool FP32, bool ACC>
__global__ void __launch_bounds__(EMB_SUM_THREADS) embed_sum_kernel(const EmbedParams p) {
    __shared__ uint32_t present[ACC ? 1 : EMB_MARK_ROWS / 32];
    __shared__ alignas(16) uint4 zeros[ACC ? 1 : EMB_ZEROS / 16];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = static_cast<int>(p.T);
    const int vpr = p.H / 8;
    if (p.T == 0) pdl_wait();                                // no sort came before
    if (!ACC) {
        for (int i = tid; i < EMB_ZEROS / 16; i += EMB_SUM_THREADS) zeros[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        const long long row_bytes = static_cast<long long>(p.H) * (FP32 ? 4 : 2);
        const long long share = (p.V + gridDim.x - 1ll) / gridDim.x, begin = share * blockIdx.x;
        const long long end = begin + share < p.V ? begin + share : p.V;
        for (long long row0 = begin; row0 < end; row0 += EMB_MARK_ROWS) {
            const int rows = static_cast<int>(end - row0 < EMB_MARK_ROWS ? end - row0 : EMB_MARK_ROWS);
            for (int i = tid; i < (rows + 31) / 32; i += EMB_SUM_THREADS) present[i] = 0;
            __syncthreads();
#pragma unroll 8
            for (int i = tid; i < T; i += EMB_SUM_THREADS) {
                const unsigned r = static_cast<unsigned>(__ldcg(&p.ids[i])) - static_cast<unsigned>(row0);
                if (r < static_cast<unsigned>(rows)) atomicOr(&present[r >> 5], 1u << (r & 31));
            }
            __syncthreads();
            if (warp == 0) {
                auto fill = [&](int r, int n) {
                    char* to = static_cast<char*>(p.d_table) + (row0 + r) * row_bytes;
                    for (long long left = n * row_bytes; left > 0;) {
                        const int bytes = left < EMB_ZEROS ? static_cast<int>(left) : EMB_ZEROS;
                        bulk_store(to, smem_u32(zeros), bytes);
                        to += bytes;
                        left -= bytes;
                    }
                };
                for (int w = lane; w < (rows + 31) / 32; w += 32) {
                    const int n = rows - 32 * w < 32 ? rows - 32 * w : 32;
                    uint32_t absent = ~present[w] & (0xffffffffu >> (32 - n));
                    while (absent) {                         // stretches of rows without a token
                        const int r = __ffs(absent) - 1, len = __ffs(~(absent >> r)) - 1;
                        const int rows_here = len < 0 ? 32 - r : len;
                        fill(32 * w + r, rows_here);
                        absent &= rows_here == 32 ? 0u : ~(((1u << rows_here) - 1) << r);
                    }
                }
                tma_store_commit();
            }
            if (row0 + EMB_MARK_ROWS < end) __syncthreads();
        }
    }
    pdl_wait();
    // An item is a piece's 512 columns.  A warp looks up 32 of its items at a time and sums four of them side by side.
    const int slices = (vpr + 63) / 64;
    const long long items = p.T * slices, stride = static_cast<long long>(gridDim.x) * EMB_SUM_WARPS;
    for (long long base = blockIdx.x * EMB_SUM_WARPS + warp; base < items; base += 32 * stride) {
        const long long item = base + lane * stride;
        const int at_place = static_cast<int>(item / slices), at_slice = static_cast<int>(item - static_cast<long long>(at_place) * slices);
        uint4 rec = make_uint4(0, 0, 0, 0);
        if (item < items) rec = __ldcg(&p.place[at_place]);
        unsigned todo = __ballot_sync(0xffffffffu, rec.y != 0);
        while (todo) {
            const int l = __ffs(todo) - 1;
            todo &= todo - 1;
            const int place = __shfl_sync(0xffffffffu, at_place, l), key = __shfl_sync(0xffffffffu, rec.x, l);
            const int c0 = __shfl_sync(0xffffffffu, at_slice, l) * 64 + lane;
            const uint32_t info = __shfl_sync(0xffffffffu, rec.y, l);
            const int len = info & EMB_LEN;
            const int token = lane < len ? __ldcg(&p.order[place + lane]) : 0;
            const uint4* dy = reinterpret_cast<const uint4*>(p.d_y) + c0;
            const bool in0 = c0 < vpr, in1 = c0 + 32 < vpr;
            float s0[8] = {}, s1[8] = {};
#pragma unroll 4
            for (int r = 0; r < len; ++r) {
                const uint4* row = dy + static_cast<long long>(__shfl_sync(0xffffffffu, token, r)) * vpr;
                uint4 a = make_uint4(0, 0, 0, 0), b = a;
                if (in0) a = __ldcg(row);
                if (in1) b = __ldcg(row + 32);
                emb_add(s0, a);
                emb_add(s1, b);
            }
            if (info & EMB_MANY) {
                float4* to = reinterpret_cast<float4*>(p.part + emb_slot(place, len) * p.H) + 2 * c0;
                if (in0) {
                    to[0] = make_float4(s0[0], s0[1], s0[2], s0[3]);
                    to[1] = make_float4(s0[4], s0[5], s0[6], s0[7]);
                }
                if (in1) {
                    to[64] = make_float4(s1[0], s1[1], s1[2], s1[3]);
                    to[65] = make_float4(s1[4], s1[5], s1[6], s1[7]);
                }
            } else {
                const long long at = static_cast<long long>(key) * vpr + c0;
                if (in0) emb_store<FP32, ACC>(p, at, s0);
                if (in1) emb_store<FP32, ACC>(p, at + 32, s1);
            }
        }
    }
    if (!ACC && warp == 0) tma_store_wait_all();
    pdl_launch_dependents();
}

// Runs of several pieces: warp w of a CTA adds up pieces w, w + 8, ... of 256 columns, then the eight sums are added up.
constexpr int EMB_FOLD_WARPS = 8;
template <bool FP32, bool ACC>
__global__ void __launch_bounds__(EMB_FOLD_WARPS * 32) embed_fold_kernel(const EmbedParams p) {
    __shared__ int heads[EMB_FOLD_WARPS * 32], found;
    __shared__ float sums[EMB_FOLD_WARPS][8][32];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) found = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const long long mine = static_cast<long long>(blockIdx.x) * EMB_FOLD_WARPS * 32 + tid;
    if (mine < p.T) {
        const uint32_t info = __ldcg(&p.place[mine]).y;
        if ((info & (EMB_MANY | EMB_HEAD)) == (EMB_MANY | EMB_HEAD)) heads[atomicAdd(&found, 1)] = static_cast<int>(mine);
    }
    __syncthreads();
    const int vpr = p.H / 8, c = blockIdx.y * 32 + lane, n = found;
    for (int h = 0; h < n; ++h) {
        const int place = heads[h];
        const uint4 rec = __ldcg(&p.place[place]);
        const int run = static_cast<int>(rec.z), pieces = (run + EMB_PIECE - 1) / EMB_PIECE;
        float s[8] = {};
        if (c < vpr) {
#pragma unroll 4
            for (int i = warp; i < pieces; i += EMB_FOLD_WARPS) {
                const int at = place + i * EMB_PIECE, len = min(EMB_PIECE, run - i * EMB_PIECE);
                const float4* from = reinterpret_cast<const float4*>(p.part + emb_slot(at, len) * p.H) + 2 * c;
                const float4 a = __ldcg(from), b = __ldcg(from + 1);
                s[0] += a.x, s[1] += a.y, s[2] += a.z, s[3] += a.w, s[4] += b.x, s[5] += b.y, s[6] += b.z, s[7] += b.w;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[warp][e][lane] = s[e];
        __syncthreads();
        if (warp == 0 && c < vpr) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int w = 1; w < EMB_FOLD_WARPS; ++w) s[e] = __fadd_rn(s[e], sums[w][e][lane]);
            }
            emb_store<FP32, ACC>(p, static_cast<long long>(static_cast<int>(rec.x)) * vpr + c, s);
        }
        __syncthreads();
    }
}

static size_t align16(size_t n) { return (n + 15) / 16 * 16; }
size_t embed_bwd_bytes(int64_t T, int, int H) {
    const size_t n = static_cast<size_t>(T);
    return align16(4 * n) + 16 * n + (T > EMB_RANK_TOKENS ? 2 * 8 * n : 0) + (T > EMB_PIECE ? 2 * (n / EMB_PIECE + 1) * 4 * H : 0) + 16;
}

cudaError_t launch_embed(const EmbedParams& p, cudaStream_t stream) {
    const long long n = p.T * (p.H / 8);
    return launch_pdl(embed_kernel, dim3(static_cast<unsigned>((n + EMB_THREADS - 1) / EMB_THREADS)), EMB_THREADS, 0, stream, 1, p);
}

template <bool FP32, bool ACC>
static cudaError_t launch_embed_sums(const EmbedParams& p, cudaStream_t stream) {
    cudaError_t e = launch_pdl(embed_sum_kernel<FP32, ACC>, dim3(static_cast<unsigned>(p.sm_count)), EMB_SUM_THREADS, 0, stream, 1, p);
    if (e != cudaSuccess || p.T <= EMB_PIECE) return e;
    const unsigned blocks = static_cast<unsigned>((p.T + EMB_FOLD_WARPS * 32 - 1) / (EMB_FOLD_WARPS * 32));
    return launch_pdl(embed_fold_kernel<FP32, ACC>, dim3(blocks, (p.H / 8 + 31) / 32), EMB_FOLD_WARPS * 32, 0, stream, 1, p);
}

cudaError_t launch_embed_bwd(EmbedParams& p, void* ws, cudaStream_t stream) {
    char* at = static_cast<char*>(ws);
    p.place = reinterpret_cast<uint4*>(at);
    at += 16 * p.T;
    if (p.T > EMB_RANK_TOKENS)
        for (int i = 0; i < 2; ++i, at += 8 * p.T) p.keys[i] = reinterpret_cast<uint2*>(at);
    p.order = reinterpret_cast<int32_t*>(at);
    p.part = reinterpret_cast<float*>(at + align16(4 * p.T));
    cudaError_t e = cudaSuccess;
    if (p.T > EMB_RANK_TOKENS) {
        static DeviceOnce configured;
        e = configured.run([&]() {
            return cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(EMB_SORT_SMEM));
        });
        if (e != cudaSuccess) return e;
        int bits = 1;
        while (p.V >> bits) ++bits;                          // keys are 0 .. V
        const int passes = (bits + 8) / 9, digit_bits = (bits + passes - 1) / passes;
        e = launch_pdl(embed_sort_kernel, dim3(EMB_CLUSTER), EMB_SORT_THREADS, EMB_SORT_SMEM, stream, EMB_CLUSTER, p, passes, digit_bits);
    } else if (p.T > 0) {
        e = launch_pdl(embed_rank_kernel, dim3(static_cast<unsigned>((p.T + 31) / 32)), EMB_RANK_WARPS * 32, 0, stream, 1, p);
    }
    if (e != cudaSuccess) return e;
    return p.fp32 ? (p.accumulate ? launch_embed_sums<true, true>(p, stream) : launch_embed_sums<true, false>(p, stream))
                  : (p.accumulate ? launch_embed_sums<false, true>(p, stream) : launch_embed_sums<false, false>(p, stream));
}

}  // namespace tik
