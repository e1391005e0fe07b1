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
// Lanes are tokens; the warps of a CTA share the tokens that they are compared with, from shared memory (out of L2 every
// load of the chain waits behind the zeros that are being written meanwhile).
constexpr int EMB_RANK_TOKENS = 4096;
constexpr int EMB_RANK_WARPS = 8;
__global__ void __launch_bounds__(EMB_RANK_WARPS * 32) embed_rank_kernel(const EmbedParams p) {
    __shared__ alignas(16) int keys[EMB_RANK_TOKENS];
    __shared__ int count[EMB_RANK_WARPS][3][32];
    pdl_wait();
    pdl_launch_dependents();
    const int T = static_cast<int>(p.T), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int padded = (T + 4 * EMB_RANK_WARPS - 1) / (4 * EMB_RANK_WARPS) * (4 * EMB_RANK_WARPS);
#pragma unroll 4
    for (int i = threadIdx.x; i < padded; i += EMB_RANK_WARPS * 32) keys[i] = i < T ? emb_key(p, p.ids[i]) : 0x7fffffff;
    __syncthreads();
    const int t = blockIdx.x * 32 + lane, mine = t < T ? keys[t] : -1;
    int less = 0, same = 0, same_before = 0;
    const int per = padded / EMB_RANK_WARPS;
#pragma unroll 4
    for (int i = per * warp; i < per * (warp + 1); i += 4) {
        const int4 k4 = *reinterpret_cast<const int4*>(keys + i);
        const int k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            less += k[j] < mine;
            same += k[j] == mine;
            same_before += k[j] == mine && i + j < t;
        }
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
// warp moves its elements, in order, to where the elements before them end.  ON_CHIP: the list stays in the CTAs' shared
// memory between the passes (up to EMB_CHIP_TOKENS), which the zeros written meanwhile do not slow down; else in global memory.
constexpr int EMB_CLUSTER = 8, EMB_SORT_THREADS = 1024, EMB_SORT_WARPS = EMB_SORT_THREADS / 32;
constexpr int EMB_BINS = 512, EMB_CHIP_TOKENS = 65536;
struct EmbedSortSmem {
    int hist[EMB_SORT_WARPS][EMB_BINS];
    int total[EMB_BINS], base[EMB_BINS];
    int warp_sum[EMB_SORT_WARPS];
    int first_head[EMB_SORT_WARPS], last_head[EMB_SORT_WARPS];
    int cta_first_head, cta_last_head;
    uint2 edge;                                              // the CTA's last element
};
// elements of a warp's stretch: whole windows of 32
inline __host__ __device__ int emb_stretch(int T) {
    return ((T + EMB_CLUSTER * EMB_SORT_WARPS - 1) / (EMB_CLUSTER * EMB_SORT_WARPS) + 31) / 32 * 32;
}

__device__ __forceinline__ int ld_cluster_int(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_uint2(uint32_t addr, uint2 v) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}

template <bool ON_CHIP>
__global__ void __launch_bounds__(EMB_SORT_THREADS) embed_sort_kernel(const EmbedParams p, int passes, int digit_bits) {
    extern __shared__ __align__(16) unsigned char emb_smem[];
    EmbedSortSmem& sm = *reinterpret_cast<EmbedSortSmem*>(emb_smem);
    uint2* list = reinterpret_cast<uint2*>(emb_smem + sizeof(EmbedSortSmem));        // ON_CHIP: two buffers of a CTA's stretch
    const int T = static_cast<int>(p.T), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    pdl_wait();
    pdl_launch_dependents();
    const int bins = 1 << digit_bits;
    const int per = emb_stretch(T), chunk = per * EMB_SORT_WARPS;
    const long long cta_from = static_cast<long long>(chunk) * rank, from = cta_from + per * warp;
    const int first = static_cast<int>(from < T ? from : T), last = static_cast<int>(from + per < T ? from + per : T);
    int* mine = sm.hist[warp];
    // elements of this CTA's stretch before pass `pass` (pass == passes: sorted)
    auto element = [&](int pass, int i) {
        if (pass == 0) return make_uint2(emb_key(p, p.ids[i]), i);
        if (ON_CHIP) return list[(pass & 1) * chunk + static_cast<int>(i - cta_from)];
        return __ldcg(&p.keys[pass & 1][i]);
    };
    cluster_sync_all();                                      // every CTA runs before any writes to another's shared memory
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * digit_bits;
        for (int i = lane; i < bins; i += 32) mine[i] = 0;
        __syncwarp();
        for (int i0 = first; i0 < last; i0 += 32) {
            const int i = i0 + lane;
            const unsigned here = __ballot_sync(0xffffffffu, i < last);
            if (i < last) {
                const int digit = (element(pass, i).x >> shift) & (bins - 1);
                const unsigned peers = __match_any_sync(here, digit);
                if (lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
            }
            __syncwarp();
        }
        __syncthreads();
        int sum = 0;
        if (tid < bins) {                                    // a bin's counts -> counts of the warps before
#pragma unroll
            for (int w = 0; w < EMB_SORT_WARPS; ++w) {
                const int n = sm.hist[w][tid];
                sm.hist[w][tid] = sum;
                sum += n;
            }
            sm.total[tid] = sum;
        }
        __syncwarp();
        cluster_sync_all();
        int before = 0, all = 0;                             // of the CTAs before, of the cluster
        if (tid < bins) {
#pragma unroll
            for (uint32_t r = 0; r < EMB_CLUSTER; ++r) {
                const int n = ld_cluster_int(mapa_cluster(smem_u32(sm.total + tid), r));
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
        if (lane == 31) sm.warp_sum[warp] = scan;
        __syncthreads();
        int below = lane < warp ? sm.warp_sum[lane] : 0;
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) below += __shfl_xor_sync(0xffffffffu, below, off);
        if (tid < bins) sm.base[tid] = scan - all + before + below;
        __syncthreads();
        for (int i0 = first; i0 < last; i0 += 32) {
            const int i = i0 + lane;
            const unsigned here = __ballot_sync(0xffffffffu, i < last);
            if (i < last) {
                const uint2 e = element(pass, i);
                const int digit = (e.x >> shift) & (bins - 1);
                const unsigned peers = __match_any_sync(here, digit);
                const int at = sm.base[digit] + mine[digit] + __popc(peers & ((1u << lane) - 1));
                __syncwarp(here);
                if (lane == __ffs(peers) - 1) mine[digit] += __popc(peers);
                if (ON_CHIP) {
                    const uint32_t to = static_cast<uint32_t>(at) / static_cast<uint32_t>(chunk);
                    st_cluster_uint2(mapa_cluster(smem_u32(list + ((pass + 1) & 1) * chunk + (at - static_cast<int>(to) * chunk)), to), e);
                } else {
                    __stcg(&p.keys[(pass + 1) & 1][at], e);
                }
            }
            __syncwarp();
        }
        cluster_sync_all();
    }
    // Records need the ends of each run.  Heads (first places of runs) of a warp's windows, the first and the last of its stretch,
    // then of its CTA; what a stretch does not hold, the closest stretch before or after it does.
    if (tid == 0 && cta_from < T) sm.edge = element(passes, static_cast<int>(cta_from + chunk < T ? cta_from + chunk : T) - 1);
    cluster_sync_all();
    constexpr int NONE_BEFORE = -1, NONE_AFTER = 0x7fffffff;
    auto heads_of = [&](int i0) {
        const int i = i0 + lane;
        const uint32_t key = i < T ? element(passes, i).x : 0xffffffffu;
        uint32_t left = __shfl_up_sync(0xffffffffu, key, 1);
        if (lane == 0) {
            left = 0xfffffffeu;
            if (i0 > cta_from) left = element(passes, i0 - 1).x;
            else if (rank > 0) left = ld_cluster_int(mapa_cluster(smem_u32(&sm.edge), rank - 1));
        }
        return __ballot_sync(0xffffffffu, key != left);      // (places from T on: the first of them is a head)
    };
    int first_head = NONE_AFTER, last_head = NONE_BEFORE;
    for (int i0 = first; i0 < last; i0 += 32) {
        const unsigned heads = heads_of(i0);
        if (heads == 0) continue;
        if (first_head == NONE_AFTER) first_head = i0 + __ffs(heads) - 1;
        last_head = i0 + 31 - __clz(heads);
    }
    if (lane == 0) {
        sm.first_head[warp] = first_head;
        sm.last_head[warp] = last_head;
    }
    __syncthreads();
    int before = NONE_BEFORE, after = NONE_AFTER;            // closest heads outside the stretch
    {
        int cta_first = sm.first_head[lane], cta_last = sm.last_head[lane];
        before = lane < warp ? cta_last : NONE_BEFORE;
        after = lane > warp ? cta_first : NONE_AFTER;
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) {
            before = max(before, __shfl_xor_sync(0xffffffffu, before, off));
            after = min(after, __shfl_xor_sync(0xffffffffu, after, off));
            cta_first = min(cta_first, __shfl_xor_sync(0xffffffffu, cta_first, off));
            cta_last = max(cta_last, __shfl_xor_sync(0xffffffffu, cta_last, off));
        }
        if (tid == 0) {
            sm.cta_first_head = cta_first;
            sm.cta_last_head = cta_last;
        }
    }
    __syncwarp();
    cluster_sync_all();
    {
        int cta_first = NONE_AFTER, cta_last = NONE_BEFORE;
        if (lane < EMB_CLUSTER) {
            if (lane > static_cast<int>(rank)) cta_first = ld_cluster_int(mapa_cluster(smem_u32(&sm.cta_first_head), lane));
            if (lane < static_cast<int>(rank)) cta_last = ld_cluster_int(mapa_cluster(smem_u32(&sm.cta_last_head), lane));
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) {
            cta_first = min(cta_first, __shfl_xor_sync(0xffffffffu, cta_first, off));
            cta_last = max(cta_last, __shfl_xor_sync(0xffffffffu, cta_last, off));
        }
        before = max(before, cta_last);
        after = min(min(after, cta_first), T);
    }
    const uint32_t bad = p.V;
    int next = -1;                                           // the first head behind the window
    for (int i0 = first; i0 < last; i0 += 32) {
        const int i = i0 + lane;
        const unsigned heads = heads_of(i0);
        const unsigned to_lane = 0xffffffffu >> (31 - lane);
        if (next < i0 + 32) {
            next = after;
            for (int j0 = i0 + 32; j0 < last; j0 += 32) {
                const unsigned more = heads_of(j0);
                if (more) {
                    next = j0 + __ffs(more) - 1;
                    break;
                }
            }
        }
        if (i < last) {
            const uint2 e = element(passes, i);
            const unsigned upto = heads & to_lane, behind = heads & ~to_lane;
            const int head = upto ? i0 + 31 - __clz(upto) : before;
            const int tail = behind ? i0 + __ffs(behind) - 1 : next;
            uint4 rec = emb_record(e.x, i - head, tail - head, e.y);
            if (e.x == bad) {
                rec.y = 0;
                if (i == head) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
            }
            p.order[i] = e.y;
            p.place[i] = rec;
        }
        if (heads) before = i0 + 31 - __clz(heads);
    }
    cluster_sync_all();                                      // no CTA leaves while another may read its shared memory
}

// eight columns of a table row: what is there, and the new value
template <bool FP32>
struct EmbedOld {
    uint4 v[FP32 ? 2 : 1];
};
template <bool FP32>
__device__ __forceinline__ void emb_old(const EmbedParams& p, long long at, EmbedOld<FP32>& old) {
    const uint4* d = reinterpret_cast<const uint4*>(p.d_table) + (FP32 ? 2 : 1) * at;
#pragma unroll
    for (int i = 0; i < (FP32 ? 2 : 1); ++i) old.v[i] = __ldcg(d + i);
}
template <bool FP32, bool ACC>
__device__ __forceinline__ void emb_store(const EmbedParams& p, long long at, const float (&sum)[8], const EmbedOld<FP32>& old) {
    float f[8] = {};
    if (ACC && FP32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4 v = old.v[FP32 ? i : 0];
            f[4 * i] = __uint_as_float(v.x), f[4 * i + 1] = __uint_as_float(v.y);
            f[4 * i + 2] = __uint_as_float(v.z), f[4 * i + 3] = __uint_as_float(v.w);
        }
    } else if (ACC) {
        unpack8(old.v[0], f);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __fmaf_rn(p.scale, sum[e], f[e]);
    if (FP32) {
        float4* d = reinterpret_cast<float4*>(p.d_table) + 2 * at;
        d[0] = make_float4(f[0], f[1], f[2], f[3]);
        d[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
        reinterpret_cast<uint4*>(p.d_table)[at] = pack8(f);
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
constexpr int EMB_SUM_THREADS = 512, EMB_SUM_WARPS = EMB_SUM_THREADS / 32;
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
    // A warp has the same NV * 256 columns of consecutive places.  It looks up 32 places at a time and goes through the rows of
    // the pieces that begin there, whichever piece they belong to, U at a time: most pieces are one row, and one
    // after the other they would leave a few hundred bytes per warp in flight.
    constexpr int NV = ACC ? 1 : 2, U = ACC && FP32 ? 6 : 8; // (16-byte vectors per lane: the old values need registers too)
    struct Item {
        int place, key, len, start;
    };
    __shared__ Item list[EMB_SUM_WARPS][32];
    const int slices = (vpr + 32 * NV - 1) / (32 * NV), warps = gridDim.x * EMB_SUM_WARPS, me = blockIdx.x * EMB_SUM_WARPS + warp;
    const int groups = warps >= slices ? warps / slices : 1, group = warps >= slices ? me / slices : 0;
    const int per = static_cast<int>((p.T + groups - 1) / groups);
    const long long places_from = static_cast<long long>(per) * group;
    const int places_to = static_cast<int>(group >= groups ? 0 : places_from + per < T ? places_from + per : T);
    for (int slice = me % slices; slice < slices; slice += warps) {
        const int c0 = slice * 32 * NV + lane;
        bool in[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) in[v] = c0 + 32 * v < vpr;
        const uint4* dy = reinterpret_cast<const uint4*>(p.d_y) + c0;
        float sum[NV][8] = {};
        for (long long p0 = places_from; p0 < places_to; p0 += 32) {
            uint4 rec = make_uint4(0, 0, 0, 0);
            if (p0 + lane < places_to) rec = __ldcg(&p.place[p0 + lane]);
            const int len = rec.y & EMB_LEN;
            int end = len;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int n = __shfl_up_sync(0xffffffffu, end, off);
                if (lane >= off) end += n;
            }
            const int rows = __shfl_sync(0xffffffffu, end, 31), start = end - len;
            const unsigned pieces = __ballot_sync(0xffffffffu, len > 0), before_lane = (1u << lane) - 1;
            if (len > 0)
                list[warp][__popc(pieces & before_lane)] = {static_cast<int>(p0) + lane, static_cast<int>(rec.x),
                                                            static_cast<int>(rec.y & (EMB_LEN | EMB_MANY)), start};
            __syncwarp();
            for (int r0 = 0; r0 < rows; r0 += 32) {
                // lane l: row r0 + l, its piece (the o-th) and its token
                const unsigned starts = __reduce_or_sync(0xffffffffu, len > 0 && start >= r0 && start < r0 + 32 ? 1u << (start - r0) : 0u);
                const int o = __popc(__ballot_sync(0xffffffffu, len > 0 && start < r0)) + __popc(starts & (before_lane * 2 + 1)) - 1;
                int token = 0;
                bool at_end = false;
                if (r0 + lane < rows) {
                    const Item& it = list[warp][o];
                    const int r = r0 + lane - it.start;
                    token = __ldcg(&p.order[it.place + r]);
                    at_end = r + 1 == static_cast<int>(it.len & EMB_LEN);
                }
                const unsigned ends = __ballot_sync(0xffffffffu, at_end);
                const int n = rows - r0 < 32 ? rows - r0 : 32;
                for (int j = 0; j < n; j += U) {
                    uint4 row[U][NV];
                    EmbedOld<FP32> old[ACC ? U : 1][NV];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const uint4* from = dy + static_cast<long long>(__shfl_sync(0xffffffffu, token, (j + u) & 31)) * vpr;
                        const int ou = __shfl_sync(0xffffffffu, o, (j + u) & 31);
#pragma unroll
                        for (int v = 0; v < NV; ++v)
                            if (j + u < n && in[v]) {
                                row[u][v] = __ldcg(from + 32 * v);
                                if (ACC && (ends >> (j + u) & 1)) emb_old(p, static_cast<long long>(list[warp][ou].key) * vpr + c0 + 32 * v, old[ACC ? u : 0][v]);
                            }
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (j + u >= n) break;
#pragma unroll
                        for (int v = 0; v < NV; ++v) emb_add(sum[v], row[u][v]);
                        const int ou = __shfl_sync(0xffffffffu, o, j + u);
                        if (!(ends >> (j + u) & 1)) continue;
                        const Item it = list[warp][ou];
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            if (in[v] && (it.len & EMB_MANY)) {
                                float4* to = reinterpret_cast<float4*>(p.part + emb_slot(it.place, it.len & EMB_LEN) * p.H) + 2 * (c0 + 32 * v);
                                to[0] = make_float4(sum[v][0], sum[v][1], sum[v][2], sum[v][3]);
                                to[1] = make_float4(sum[v][4], sum[v][5], sum[v][6], sum[v][7]);
                            } else if (in[v]) {
                                emb_store<FP32, ACC>(p, static_cast<long long>(it.key) * vpr + c0 + 32 * v, sum[v], old[ACC ? u : 0][v]);
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) sum[v][e] = 0.0f;
                        }
                    }
                }
            }
            __syncwarp();
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
            const long long at = static_cast<long long>(static_cast<int>(rec.x)) * vpr + c;
            EmbedOld<FP32> old;
            if (ACC) emb_old(p, at, old);
            emb_store<FP32, ACC>(p, at, s, old);
        }
        __syncthreads();
    }
}

static size_t align16(size_t n) { return (n + 15) / 16 * 16; }
size_t embed_bwd_bytes(int64_t T, int, int H) {
    const size_t n = static_cast<size_t>(T);
    return align16(4 * n) + 16 * n + (T > EMB_CHIP_TOKENS ? 2 * 8 * n : 0) + (T > EMB_PIECE ? 2 * (n / EMB_PIECE + 1) * 4 * H : 0) + 16;
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
    const bool on_chip = p.T <= EMB_CHIP_TOKENS;
    if (!on_chip)
        for (int i = 0; i < 2; ++i, at += 8 * p.T) p.keys[i] = reinterpret_cast<uint2*>(at);
    p.order = reinterpret_cast<int32_t*>(at);
    p.part = reinterpret_cast<float*>(at + align16(4 * p.T));
    cudaError_t e = cudaSuccess;
    if (p.T > EMB_RANK_TOKENS) {
        static DeviceOnce configured;
        const size_t base = sizeof(EmbedSortSmem), list = 2ull * sizeof(uint2) * EMB_SORT_WARPS;      // per element of a stretch
        e = configured.run([&]() {
            const cudaError_t e1 = cudaFuncSetAttribute(embed_sort_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                        static_cast<int>(base + list * emb_stretch(EMB_CHIP_TOKENS)));
            return e1 != cudaSuccess ? e1 : cudaFuncSetAttribute(embed_sort_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                                 static_cast<int>(base));
        });
        if (e != cudaSuccess) return e;
        int bits = 1;
        while (p.V >> bits) ++bits;                          // keys are 0 .. V
        const int passes = (bits + 8) / 9, digit_bits = (bits + passes - 1) / passes;
        e = launch_pdl(on_chip ? embed_sort_kernel<true> : embed_sort_kernel<false>, dim3(EMB_CLUSTER), EMB_SORT_THREADS,
                       base + (on_chip ? list * emb_stretch(static_cast<int>(p.T)) : 0), stream, EMB_CLUSTER, p, passes, digit_bits);
    } else if (p.T > 0) {
        e = launch_pdl(embed_rank_kernel, dim3(static_cast<unsigned>((p.T + 31) / 32)), EMB_RANK_WARPS * 32, 0, stream, 1, p);
    }
    if (e != cudaSuccess) return e;
    return p.fp32 ? (p.accumulate ? launch_embed_sums<true, true>(p, stream) : launch_embed_sums<true, false>(p, stream))
                  : (p.accumulate ? launch_embed_sums<false, true>(p, stream) : launch_embed_sums<false, false>(p, stream));
}

}  // namespace tik
