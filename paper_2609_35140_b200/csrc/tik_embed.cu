// Embedding lookup and its gradient by sorted tokens.
#include <cuda_bf16.h>

#include <type_traits>

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

// y[t] = scale * table[ids[t]]; 16-byte vectors, VPT per thread (a block covers 256 * VPT consecutive ones).  A vector is two
// loads one behind the other, id and row, so large calls have four of each in flight per thread (8191 x 4096: 23.6 us with
// one, 17.8 with four); small calls take one, which spreads them over more blocks.
constexpr unsigned EMB_VEC_MAX = 0xfffff000u;                // vectors per launch: 32-bit indices
template <int VPT>
__global__ void __launch_bounds__(EMB_THREADS) embed_kernel(const EmbedParams p, unsigned nvec, unsigned vpr) {
    const unsigned base = blockIdx.x * (EMB_THREADS * VPT) + threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    uint4 v[VPT];
    int id[VPT];
    unsigned c[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const unsigned i = base + EMB_THREADS * j, t = i / vpr;
        c[j] = i - t * vpr;
        id[j] = i < nvec ? p.ids[t] : -1;
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        v[j] = make_uint4(0, 0, 0, 0);
        if (id[j] >= 0 && id[j] < p.V) v[j] = reinterpret_cast<const uint4*>(p.table)[static_cast<size_t>(id[j]) * vpr + c[j]];
    }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
        const unsigned i = base + EMB_THREADS * j;
        if (i >= nvec) break;
        if (c[j] == 0 && (id[j] < 0 || id[j] >= p.V)) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
        reinterpret_cast<uint4*>(p.y)[i] = scaled8(v[j], p.scale);
    }
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
constexpr int EMB_RANK_TOKENS = 4608;                        // (one wave of CTAs; 4097 tokens x 256, added, us: 13.4 so, 18.4 by sorting)
constexpr int EMB_RANK_WARPS = 32;                           // (4000 tokens: 14 us with eight, 9 with 32)
__global__ void __launch_bounds__(EMB_RANK_WARPS * 32) embed_rank_kernel(const EmbedParams p) {
    __shared__ alignas(16) int keys[EMB_RANK_TOKENS];
    __shared__ int count[3][32];
    if (threadIdx.x < 96) (&count[0][0])[threadIdx.x] = 0;
    pdl_wait();
    pdl_launch_dependents();
    const int T = static_cast<int>(p.T), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (blockIdx.x == 0 && threadIdx.x < 2) p.tickets[threadIdx.x] = 0;
    const int padded = (T + 4 * EMB_RANK_WARPS - 1) / (4 * EMB_RANK_WARPS) * (4 * EMB_RANK_WARPS);
#pragma unroll                                               // (all in flight at once)
    for (int j = 0; j < (EMB_RANK_TOKENS + EMB_RANK_WARPS * 32 - 1) / (EMB_RANK_WARPS * 32); ++j) {
        const int i = threadIdx.x + j * EMB_RANK_WARPS * 32;
        if (i < padded) keys[i] = i < T ? emb_key(p, p.ids[i]) : 0x7fffffff;
    }
    __syncthreads();
    const int t0 = blockIdx.x * 32, t = t0 + lane, mine = t < T ? keys[t] : -1;
    // In front of the CTA's tokens an equal id comes earlier in the order, behind them it does not.
    int place = 0, same = 0, same_before = 0;
    const int per = padded / EMB_RANK_WARPS, begin = per * warp, end = begin + per;
    auto four = [&](int i, auto before) {
        const int4 k4 = *reinterpret_cast<const int4*>(keys + i);
        const int k[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            place += decltype(before)::value ? k[j] <= mine : k[j] < mine;
            (decltype(before)::value ? same_before : same) += k[j] == mine;
        }
    };
    int i = begin;
#pragma unroll 4
    for (; i < min(end, t0); i += 4) four(i, std::true_type());
    for (; i < min(end, t0 + 32); ++i) {
        const bool equal = keys[i] == mine;
        place += keys[i] < mine || (equal && i < t);
        (i < t ? same_before : same) += equal;
    }
#pragma unroll 4
    for (; i < end; i += 4) four(i, std::false_type());
    atomicAdd(&count[0][lane], place);
    atomicAdd(&count[1][lane], same);
    atomicAdd(&count[2][lane], same_before);
    __syncthreads();
    if (warp != 0 || t >= T) return;
    place = count[0][lane];
    same = count[1][lane];
    same_before = count[2][lane];
    p.order[place] = t;
    uint4 rec = emb_record(mine, same_before, same_before + same, t);
    if (mine == p.V) {
        atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
        rec.y = 0;
    }
    p.place[place] = rec;
}

// Other calls: a stable radix sort by one cluster of eight CTAs, whose 256 warps own consecutive stretches of the list.  Per
// digit: each warp counts its digits, the CTAs exchange their counts through distributed shared memory, and each
// warp moves its elements, in order, to where the elements before them end.  A stretch is NW windows of 32 elements, held in
// registers, and the list stays in the CTAs' shared memory between the passes, which the zeros that are written meanwhile
// do not slow down.  What a call costs are its few barriers across the cluster (~0.7 us each) and the chains between them.
constexpr int EMB_CLUSTER = 8, EMB_SORT_THREADS = 1024, EMB_SORT_WARPS = EMB_SORT_THREADS / 32;
constexpr int EMB_BINS = 512, EMB_CHIP_TOKENS = 8 * 32 * EMB_SORT_WARPS * EMB_CLUSTER;
struct EmbedSortSmem {
    int hist[EMB_SORT_WARPS][EMB_BINS];
    int total[EMB_BINS], base[EMB_BINS];
    int warp_sum[EMB_SORT_WARPS];
    int first_head[EMB_SORT_WARPS], last_head[EMB_SORT_WARPS];
    int cta_first_head, cta_last_head;
};
constexpr size_t emb_sort_smem(int nw) { return sizeof(EmbedSortSmem) + 2ull * nw * 32 * EMB_SORT_WARPS * sizeof(uint2); }

__device__ __forceinline__ int ld_cluster_int(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_uint2(uint32_t addr, uint2 v) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(v.x), "r"(v.y) : "memory");
}

// A digit's place among those of its kind that this warp has seen; counts it.
__device__ __forceinline__ int emb_count(int* counts, bool valid, int digit, int lane) {
    int at = 0;
    const unsigned here = __ballot_sync(0xffffffffu, valid);
    if (valid) {
        const unsigned peers = __match_any_sync(here, digit);
        at = counts[digit] + __popc(peers & ((1u << lane) - 1));
        __syncwarp(here);
        if (lane == __ffs(peers) - 1) counts[digit] += __popc(peers);
    }
    __syncwarp();
    return at;
}
// The record of place i of 32 that a warp holds, element e; heads: first places of runs among them, before / next: the closest ones
// outside.
__device__ __forceinline__ void emb_write_record(const EmbedParams& p, int i0, uint2 e, unsigned heads, int before, int next, int lane) {
    const unsigned to_lane = 0xffffffffu >> (31 - lane), upto = heads & to_lane, behind = heads & ~to_lane;
    const int i = i0 + lane, head = upto ? i0 + 31 - __clz(upto) : before, tail = behind ? i0 + __ffs(behind) - 1 : next;
    uint4 rec = emb_record(e.x, i - head, tail - head, e.y);
    if (e.x == static_cast<uint32_t>(p.V)) {
        rec.y = 0;
        if (i == head) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
    }
    p.order[i] = e.y;
    p.place[i] = rec;
}

template <int NW>
__global__ void __launch_bounds__(EMB_SORT_THREADS) embed_sort_kernel(const EmbedParams p, int passes, int digit_bits) {
    extern __shared__ __align__(16) unsigned char emb_smem[];
    EmbedSortSmem& sm = *reinterpret_cast<EmbedSortSmem*>(emb_smem);
    uint2* list = reinterpret_cast<uint2*>(emb_smem + sizeof(EmbedSortSmem));        // two buffers of the CTA's elements
    const int T = static_cast<int>(p.T), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_ctarank();
    pdl_wait();
    pdl_launch_dependents();
    if (rank == 0 && tid < 2) p.tickets[tid] = 0;
    const int bins = 1 << digit_bits;
    constexpr int per = 32 * NW, chunk = per * EMB_SORT_WARPS;
    const long long cta_from = static_cast<long long>(chunk) * rank, from = cta_from + per * warp;
    const int first = static_cast<int>(from < T ? from : T), last = static_cast<int>(from + per < T ? from + per : T);
    int* mine = sm.hist[warp];
    // elements of this warp's stretch before pass `pass` (pass == passes: sorted)
    auto element = [&](int pass, int i) {
        if (pass == 0) return make_uint2(emb_key(p, p.ids[i]), i);
        return list[(pass & 1) * chunk + static_cast<int>(i - cta_from)];
    };
    uint2 held[NW];
    int at[NW];
    auto hold = [&](int pass) {
#pragma unroll
        for (int w = 0; w < NW; ++w)
            if (first + 32 * w + lane < last) held[w] = element(pass, first + 32 * w + lane);
    };
    hold(0);
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * digit_bits;
        for (int i = lane; i < bins; i += 32) mine[i] = 0;
        __syncwarp();
#pragma unroll
        for (int w = 0; w < NW; ++w) at[w] = emb_count(mine, first + 32 * w + lane < last, held[w].x >> shift & (bins - 1), lane);
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
        const int below = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[lane] : 0);
        if (tid < bins) sm.base[tid] = scan - all + before + below;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (first + 32 * w + lane >= last) continue;
            const int digit = held[w].x >> shift & (bins - 1), to = sm.base[digit] + mine[digit] + at[w], cta = to / chunk;
            st_cluster_uint2(mapa_cluster(smem_u32(list + ((pass + 1) & 1) * chunk + (to - cta * chunk)), cta), held[w]);
        }
        __syncwarp();
        cluster_sync_all();
        hold(pass + 1);
    }
    // Records need the ends of each run.  Heads (first places of runs) of a warp's windows, the first and the last of its stretch,
    // then of its CTA; what a stretch does not hold, the closest stretch before or after it does.
    constexpr int NONE_BEFORE = -1, NONE_AFTER = 0x7fffffff;
    auto window = [&](int i0) {                              // i0 + lane's element; past the end a key that no token has
        const int i = i0 + lane;
        return i < T ? list[(passes & 1) * chunk + static_cast<int>(i - cta_from)] : make_uint2(0xffffffffu, 0);
    };
    auto heads_of = [&](int i0, uint32_t key) {
        uint32_t left = __shfl_up_sync(0xffffffffu, key, 1);
        if (lane == 0) {
            left = 0xfffffffeu;
            if (i0 > cta_from) left = element(passes, i0 - 1).x;
            else if (rank > 0) left = ld_cluster_int(mapa_cluster(smem_u32(list + (passes & 1) * chunk + chunk - 1), rank - 1));
        }
        return __ballot_sync(0xffffffffu, key != left);      // (places from T on: the first of them is a head)
    };
    int first_head = NONE_AFTER, last_head = NONE_BEFORE;
    for (int i0 = first; i0 < last; i0 += 32) {
        const unsigned heads = heads_of(i0, window(i0).x);
        if (heads == 0) continue;
        if (first_head == NONE_AFTER) first_head = i0 + __ffs(heads) - 1;
        last_head = i0 + 31 - __clz(heads);
    }
    if (lane == 0) {
        sm.first_head[warp] = first_head;
        sm.last_head[warp] = last_head;
    }
    __syncthreads();
    const int first_w = sm.first_head[lane], last_w = sm.last_head[lane];
    int before = __reduce_max_sync(0xffffffffu, lane < warp ? last_w : NONE_BEFORE);         // closest heads outside the stretch
    int after = __reduce_min_sync(0xffffffffu, lane > warp ? first_w : NONE_AFTER);
    if (warp == 0) {
        const int cta_first = __reduce_min_sync(0xffffffffu, first_w), cta_last = __reduce_max_sync(0xffffffffu, last_w);
        if (lane == 0) {
            sm.cta_first_head = cta_first;
            sm.cta_last_head = cta_last;
        }
        __syncwarp();
    }
    cluster_sync_all();
    {
        int cta_first = NONE_AFTER, cta_last = NONE_BEFORE;
        if (lane < EMB_CLUSTER) {
            if (lane > static_cast<int>(rank)) cta_first = ld_cluster_int(mapa_cluster(smem_u32(&sm.cta_first_head), lane));
            if (lane < static_cast<int>(rank)) cta_last = ld_cluster_int(mapa_cluster(smem_u32(&sm.cta_last_head), lane));
        }
        before = max(before, __reduce_max_sync(0xffffffffu, cta_last));
        after = min(min(after, __reduce_min_sync(0xffffffffu, cta_first)), T);
    }
    int next = -1;                                           // the first head behind the window
    for (int i0 = first; i0 < last; i0 += 32) {
        const uint2 e = window(i0);
        const unsigned heads = heads_of(i0, e.x);
        if (next < i0 + 32) {
            next = after;
            for (int j0 = i0 + 32; j0 < last; j0 += 32) {
                const unsigned more = heads_of(j0, window(j0).x);
                if (more) {
                    next = j0 + __ffs(more) - 1;
                    break;
                }
            }
        }
        if (i0 + lane < last) emb_write_record(p, i0, e, heads, before, next, lane);
        if (heads) before = i0 + 31 - __clz(heads);
    }
    __syncwarp();
    cluster_sync_all();                                      // no CTA leaves while another may read its shared memory
}

// More than EMB_CHIP_TOKENS: the list in global memory, EMB_WIDE_CTAS CTAs, two launches a digit -- counts of every CTA, then each
// CTA adds up the counts before it, counts once more and moves its elements -- and one for the records.  (By the cluster above
// out of global memory, for which eight SMs have too few loads in flight, 65 537 tokens took 94 us with the sums of 256 columns and
// 262 144 299; so 54 and 105.  65 536 by the cluster on chip: 60, under the zeros where those are written.)
constexpr int EMB_WIDE_CTAS = 128, EMB_WIDE_AHEAD = 4;       // windows of a warp in flight
struct EmbedWideSmem {
    int hist[EMB_SORT_WARPS][EMB_BINS];
    int base[EMB_BINS], half[2][EMB_BINS], all[2][EMB_BINS], warp_sum[EMB_SORT_WARPS];
};
// f(index, element) for the warp's stretch in order, every lane taking part; index >= last: there is none
template <class F>
__device__ __forceinline__ void emb_wide_elements(const EmbedParams& p, int pass, int lane, F&& f) {
    const int T = static_cast<int>(p.T), warp = blockIdx.x * EMB_SORT_WARPS + (threadIdx.x >> 5);
    const int per = ((T + EMB_WIDE_CTAS * EMB_SORT_WARPS - 1) / (EMB_WIDE_CTAS * EMB_SORT_WARPS) + 31) / 32 * 32;
    const long long from = static_cast<long long>(per) * warp;
    const int first = static_cast<int>(from < T ? from : T), last = static_cast<int>(from + per < T ? from + per : T);
    for (int i0 = first; i0 < last; i0 += 32 * EMB_WIDE_AHEAD) {
        uint2 e[EMB_WIDE_AHEAD];
#pragma unroll
        for (int u = 0; u < EMB_WIDE_AHEAD; ++u) {
            const int i = i0 + 32 * u + lane;
            if (i < last) e[u] = pass == 0 ? make_uint2(emb_key(p, p.ids[i]), i) : __ldcg(&p.keys[pass & 1][i]);
        }
#pragma unroll
        for (int u = 0; u < EMB_WIDE_AHEAD; ++u) f(i0 + 32 * u + lane < last, e[u]);
    }
}
__global__ void __launch_bounds__(EMB_SORT_THREADS) embed_wide_count_kernel(const EmbedParams p, int pass, int digit_bits) {
    extern __shared__ __align__(16) unsigned char emb_smem[];
    EmbedWideSmem& sm = *reinterpret_cast<EmbedWideSmem*>(emb_smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bins = 1 << digit_bits, shift = pass * digit_bits;
    for (int i = lane; i < bins; i += 32) sm.hist[warp][i] = 0;
    __syncwarp();
    pdl_wait();
    pdl_launch_dependents();
    emb_wide_elements(p, pass, lane, [&](bool there, uint2 e) { emb_count(sm.hist[warp], there, e.x >> shift & (bins - 1), lane); });
    __syncthreads();
    if (tid >= bins) return;
    int sum = 0;
#pragma unroll
    for (int w = 0; w < EMB_SORT_WARPS; ++w) sum += sm.hist[w][tid];
    p.counts[blockIdx.x * EMB_BINS + tid] = sum;
}
__global__ void __launch_bounds__(EMB_SORT_THREADS) embed_wide_move_kernel(const EmbedParams p, int pass, int digit_bits) {
    extern __shared__ __align__(16) unsigned char emb_smem[];
    EmbedWideSmem& sm = *reinterpret_cast<EmbedWideSmem*>(emb_smem);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bins = 1 << digit_bits, shift = pass * digit_bits;
    for (int i = lane; i < bins; i += 32) sm.hist[warp][i] = 0;
    __syncwarp();
    pdl_wait();
    pdl_launch_dependents();
    emb_wide_elements(p, pass, lane, [&](bool there, uint2 e) { emb_count(sm.hist[warp], there, e.x >> shift & (bins - 1), lane); });
    {
        const int bin = tid % EMB_BINS, part = tid / EMB_BINS;           // two threads a bin, half of the CTAs each
        int before = 0, all = 0;
        if (bin < bins) {
#pragma unroll 16
            for (int c = part * (EMB_WIDE_CTAS / 2); c < (part + 1) * (EMB_WIDE_CTAS / 2); ++c) {
                const int n = __ldcg(&p.counts[c * EMB_BINS + bin]);
                before += c < static_cast<int>(blockIdx.x) ? n : 0;
                all += n;
            }
        }
        sm.half[part][bin] = before;
        sm.all[part][bin] = all;
    }
    __syncthreads();
    int all = 0, scan = 0;
    if (tid < bins) {
        int sum = sm.half[0][tid] + sm.half[1][tid];                     // of the CTAs before, then of the warps before
#pragma unroll
        for (int w = 0; w < EMB_SORT_WARPS; ++w) {
            const int n = sm.hist[w][tid];
            sm.hist[w][tid] = sum;
            sum += n;
        }
        scan = all = sm.all[0][tid] + sm.all[1][tid];
    }
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int n = __shfl_up_sync(0xffffffffu, scan, off);
        if (lane >= off) scan += n;
    }
    if (lane == 31) sm.warp_sum[warp] = scan;
    __syncthreads();
    const int below = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_sum[lane] : 0);
    if (tid < bins) sm.base[tid] = scan - all + below;
    __syncthreads();
    emb_wide_elements(p, pass, lane, [&](bool there, uint2 e) {
        const int digit = e.x >> shift & (bins - 1), at = emb_count(sm.hist[warp], there, digit, lane);
        if (there) __stcg(&p.keys[(pass + 1) & 1][sm.base[digit] + at], e);
    });
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
// a window of 32 places per warp
constexpr int EMB_RECORD_WARPS = 8;
__global__ void __launch_bounds__(EMB_RECORD_WARPS * 32) embed_wide_record_kernel(const EmbedParams p, int passes) {
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x == 0 && threadIdx.x < 2) p.tickets[threadIdx.x] = 0;
    const int T = static_cast<int>(p.T), lane = threadIdx.x & 31, i0 = (blockIdx.x * EMB_RECORD_WARPS + (threadIdx.x >> 5)) * 32, i = i0 + lane;
    if (i0 >= T) return;
    const uint2* keys = p.keys[passes & 1];
    const uint2 e = i < T ? __ldcg(&keys[i]) : make_uint2(0xffffffffu, 0);
    uint32_t left = __shfl_up_sync(0xffffffffu, e.x, 1);
    if (lane == 0) left = i0 > 0 ? __ldcg(&keys[i0 - 1]).x : 0xfffffffeu;
    const uint32_t right = i0 + 32 < T ? __ldcg(&keys[i0 + 32]).x : 0xfffffffeu;
    const unsigned heads = __ballot_sync(0xffffffffu, e.x != left);
    const uint32_t k0 = __shfl_sync(0xffffffffu, e.x, 0), k31 = __shfl_sync(0xffffffffu, e.x, 31);
    const int before = heads & 1 ? i0 : emb_lower_bound(keys, T, k0, lane);
    const int next = k31 == right ? emb_lower_bound(keys, T, k31 + 1, lane) : min(i0 + 32, T);
    if (i < T) emb_write_record(p, i0, e, heads, before, next, lane);
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
// every CTA marks which rows occur, and its first warp copies zeros over the others by bulk stores, which take no other
// warp's issue slots.  The sort releases its dependents behind its own wait, so whatever came before it has completed when
// this grid starts, and it writes neither ids nor table.  A first part of the rows is shared out evenly; the rest, and the
// sums, are taken in small shares by whoever is free, from counters that the sort has cleared: SMs write at rates that differ by
// a fifth, pieces differ in rows, and a CTA takes a whole SM, so that those on the sort's eight begin when it ends.
constexpr int EMB_SUM_THREADS = 512, EMB_SUM_WARPS = EMB_SUM_THREADS / 32;
constexpr int EMB_MARK_ROWS = 1 << 18;                       // rows marked at a time
constexpr int EMB_ZEROS = 8192;                              // bytes of a bulk store
constexpr int EMB_SHARE = 1 << 18;                           // bytes of a share of the zeros, about
constexpr int EMB_PREFETCH = 64 << 20;                       // bytes of gradients brought to L2 ahead: half of it

// zeros over rows [r, r + n)
__device__ __forceinline__ void emb_fill(char* table, long long row_bytes, uint32_t zeros, long long r, int n) {
    char* to = table + r * row_bytes;
    for (long long left = n * row_bytes; left > 0;) {
        const int bytes = left < EMB_ZEROS ? static_cast<int>(left) : EMB_ZEROS;
        bulk_store(to, zeros, bytes);
        to += bytes;
        left -= bytes;
    }
}
// ... over the absent ones of 32-row words [w0, w1) of the marks, by a whole warp
__device__ __forceinline__ void emb_fill_words(char* table, long long row_bytes, uint32_t zeros, const uint32_t* present, long long row0,
                                               int rows, int w0, int w1, int lane) {
    if (w1 - w0 == 1) {                                      // long rows: one per lane
        const int r = 32 * w0 + lane;
        if (r < rows && !(present[w0] >> lane & 1)) emb_fill(table, row_bytes, zeros, row0 + r, 1);
        return;
    }
    for (int w = w0 + lane; w < w1; w += 32) {
        const int n = rows - 32 * w < 32 ? rows - 32 * w : 32;
        uint32_t absent = ~present[w] & (0xffffffffu >> (32 - n));
        while (absent) {                                     // stretches of rows without a token
            const int r = __ffs(absent) - 1, end = __ffs(~(absent >> r)) - 1, len = end < 0 ? 32 - r : end;
            emb_fill(table, row_bytes, zeros, row0 + 32 * w + r, len);
            absent &= len == 32 ? 0u : ~(((1u << len) - 1) << r);
        }
    }
}

template <bool FP32, bool ACC>
__global__ void __launch_bounds__(EMB_SUM_THREADS) embed_sum_kernel(const EmbedParams p, int late) {
    extern __shared__ uint32_t present[];                    // !ACC: a bit per row, at most EMB_MARK_ROWS
    __shared__ alignas(16) uint4 zeros[ACC ? 1 : EMB_ZEROS / 16];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = static_cast<int>(p.T);
    const int vpr = p.H / 8;
    if (p.T == 0) pdl_wait();                                // no sort came before
    if (!ACC) {
        for (int i = tid; i < EMB_ZEROS / 16; i += EMB_SUM_THREADS) zeros[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        const long long row_bytes = static_cast<long long>(p.H) * (FP32 ? 4 : 2);
        char* table = static_cast<char*>(p.d_table);
        const int fillers = gridDim.x - late, me = blockIdx.x;           // (the last `late` CTAs begin late)
        for (long long row0 = 0; row0 < p.V; row0 += EMB_MARK_ROWS) {
            const int rows = static_cast<int>(p.V - row0 < EMB_MARK_ROWS ? p.V - row0 : EMB_MARK_ROWS), words = (rows + 31) / 32;
            for (int i = tid; i < words; i += EMB_SUM_THREADS) present[i] = 0;
            __syncthreads();
#pragma unroll 8
            for (int i = tid; i < T; i += EMB_SUM_THREADS) {
                const unsigned r = static_cast<unsigned>(__ldcg(&p.ids[i])) - static_cast<unsigned>(row0);
                if (r < static_cast<unsigned>(rows)) atomicOr(&present[r >> 5], 1u << (r & 31));
            }
            __syncthreads();
            if (warp == 0) {
                // a third in even shares, or all of it where nothing has cleared the counters or they are taken
                const bool last = row0 + EMB_MARK_ROWS >= p.V && p.T > 0;
                const int even = last ? words / 3 : words;
                const int w0 = me < fillers ? static_cast<int>(static_cast<long long>(even) * me / fillers) : 0;
                const int w1 = me < fillers ? static_cast<int>(static_cast<long long>(even) * (me + 1) / fillers) : 0;
                for (int w = w0; w < w1; ++w) emb_fill_words(table, row_bytes, smem_u32(zeros), present, row0, rows, w, w + 1, lane);
                if (last) {
                    pdl_wait();
                    const int step = static_cast<int>(EMB_SHARE / (32 * row_bytes) > 1 ? EMB_SHARE / (32 * row_bytes) : 1);
                    int ticket = 0;
                    if (lane == 0) ticket = atomicAdd(&p.tickets[0], 1);
                    for (;;) {
                        const long long w = even + static_cast<long long>(step) * __shfl_sync(0xffffffffu, ticket, 0);
                        if (w >= words) break;
                        if (lane == 0) ticket = atomicAdd(&p.tickets[0], 1);         // (the next one, under this one's stores)
                        const int to = w + step < words ? static_cast<int>(w) + step : words;
                        emb_fill_words(table, row_bytes, smem_u32(zeros), present, row0, rows, static_cast<int>(w), to, lane);
                    }
                }
                tma_store_commit();
            }
            if (row0 + EMB_MARK_ROWS < p.V) __syncthreads();
        }
    }
    if (ACC) {
        // Nothing may be added before the sort is through, but the gradients can be brought to L2 meanwhile (two micro-batches of
        // 6007 x 1536 in fp32, the second one accumulated: 180.2 us without, 174.3 with; the table's rows as well: 176.9).
        const int row = p.H * 2;
        const long long most = EMB_PREFETCH / row, n = p.T < most ? p.T : most;
        for (long long t = blockIdx.x * EMB_SUM_THREADS + tid; t < n; t += gridDim.x * EMB_SUM_THREADS) bulk_prefetch_l2(p.d_y + t * p.H, row);
    }
    pdl_wait();
    // A warp takes `places` consecutive places and NV * 256 columns.  It looks the places up and goes through the rows of
    // the pieces that begin there, whichever piece they belong to, U at a time: most pieces are one row, and one
    // after the other they would leave a few hundred bytes per warp in flight.
    constexpr int NV = ACC ? 1 : 2, U = ACC && FP32 ? 6 : 8; // (16-byte vectors per lane: the old values need registers too)
    constexpr int IDLE = ACC ? 0 : 1;                        // the first warp has the zeros
    struct Item {
        int place, key, len, start;
    };
    __shared__ Item list[EMB_SUM_WARPS][32];
    const int slices = (vpr + 32 * NV - 1) / (32 * NV), warps = gridDim.x * (EMB_SUM_WARPS - IDLE);
    // Two shares a warp of one place at least (a share costs three trips to L2 before its first row; six a warp: 203 us instead of 180 for
    // two micro-batches of 6007 x 1536, fp32) and 16 places at most (32: 97 us instead of 86 for 16 001 x 3584, fp32, added).
    const long long each = p.T * slices / (2ll * warps);
    const int places = each < 1 ? 1 : each > 16 ? 16 : static_cast<int>(each);
    const long long shares = (p.T + places - 1) / places * slices;
    auto look_up = [&](long long share) {
        const long long at = share / slices * places + lane;
        return share < shares && lane < places && at < T ? __ldcg(&p.place[at]) : make_uint4(0, 0, 0, 0);
    };
    // the first two shares are even; the one after the next is asked for, and the next one looked up, under this one's rows
    long long share = warp < IDLE ? shares : static_cast<long long>(warp - IDLE) * gridDim.x + blockIdx.x, next = share + warps;
    uint4 rec = look_up(share), next_rec;
    int ticket = 0;
    for (; share < shares; share = next, next = 2ll * warps + __shfl_sync(0xffffffffu, ticket, 0), rec = next_rec) {
        next_rec = look_up(next);
        if (lane == 0 && next < shares) ticket = atomicAdd(&p.tickets[1], 1);
        const long long p0 = share / slices * places;
        const int c0 = static_cast<int>(share % slices) * 32 * NV + lane;
        bool in[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) in[v] = c0 + 32 * v < vpr;
        const uint4* dy = reinterpret_cast<const uint4*>(p.d_y) + c0;
        float sum[NV][8] = {};
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

// Calls of at most EMB_SMALL_TOKENS tokens whose zeros are little work: one launch and no sort.  A warp takes a token and 256
// columns, finds the tokens of the same id by comparing, and, if its own is the first of them, adds up their rows.  A run of
// several pieces waits until the CTA is through with the others and then gets a warp per piece; eight pieces at most are added
// up in the order of embed_fold_kernel.  256 tokens x 256, vocabulary 2048: 8.9 us by the three kernels, 3.0 by this one.
constexpr int EMB_SMALL_TOKENS = EMB_FOLD_WARPS * EMB_PIECE, EMB_SMALL_WORDS = EMB_SMALL_TOKENS / 32;
constexpr long long EMB_SMALL_BYTES = 128 << 20;             // of the table, where it is written whole: beyond, even shares of the zeros cost more
                                                             // (256 tokens, us: 134 MB 23.1 so and 24.6 by the three kernels, 268 MB 45.7 and 42.5)
constexpr int EMB_SMALL_ROWS = 1 << 16;                      // rows of a CTA's share of the zeros
constexpr int EMB_QUEUE = 32;
template <bool FP32, bool ACC>
__global__ void __launch_bounds__(EMB_SUM_THREADS) embed_small_kernel(const EmbedParams p) {
    __shared__ int keys[EMB_SMALL_TOKENS];
    __shared__ short runs[EMB_SUM_WARPS][EMB_SMALL_TOKENS];  // a warp's run: its tokens
    __shared__ int queue[EMB_QUEUE], queued;                 // items with a long run
    __shared__ float sums[EMB_FOLD_WARPS][8][32];
    __shared__ uint32_t present[ACC ? 1 : EMB_SMALL_ROWS / 32];
    __shared__ alignas(16) uint4 zeros[ACC ? 1 : EMB_ZEROS / 16];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, T = static_cast<int>(p.T), vpr = p.H / 8;
    const long long row_bytes = static_cast<long long>(p.H) * (FP32 ? 4 : 2);
    const int share = (p.V + static_cast<int>(gridDim.x) - 1) / static_cast<int>(gridDim.x), row0 = share * blockIdx.x;
    const int rows = ACC ? 0 : min(share, p.V - row0);
    if (!ACC) {
        for (int i = tid; i < (rows + 31) / 32; i += EMB_SUM_THREADS) present[i] = 0;
        for (int i = tid; i < EMB_ZEROS / 16; i += EMB_SUM_THREADS) zeros[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    if (tid == 0) queued = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    if (tid < EMB_SMALL_TOKENS) {
        const int key = tid < T ? emb_key(p, p.ids[tid]) : -1;
        keys[tid] = key;
        if (!ACC && key >= row0 && key - row0 < rows) atomicOr(&present[(key - row0) >> 5], 1u << ((key - row0) & 31));
        if (key == p.V && blockIdx.x == 0) atomicOr(p.dev_status, TIK_DEV_BAD_TOKEN);
    }
    __syncthreads();
    if (!ACC && warp == EMB_SUM_WARPS - 1) {
        emb_fill_words(static_cast<char*>(p.d_table), row_bytes, smem_u32(zeros), present, row0, rows, 0, (rows + 31) / 32, lane);
        tma_store_commit();
    }
    constexpr int U = 16;                                    // rows in flight
    const int slices = (vpr + 31) / 32;
    // the tokens of `token`'s run into runs[warp]; their number, 0 unless it is the first of them
    auto find = [&](int token) {
        const int mine = keys[token];
        int n = 0;
        bool first = mine != p.V;
#pragma unroll
        for (int w = 0; w < EMB_SMALL_WORDS; ++w) {
            const int i = 32 * w + lane;
            const unsigned same = __ballot_sync(0xffffffffu, keys[i] == mine);
            if (i < token && (same >> lane & 1)) first = false;
            if (same >> lane & 1) runs[warp][n + __popc(same & ((1u << lane) - 1))] = static_cast<short>(i);
            n += __popc(same);
        }
        first = __all_sync(0xffffffffu, first);
        __syncwarp();
        return first ? n : 0;
    };
    // rows [from, to), 32 at most, of the run
    auto add_rows = [&](int from, int to, const uint4* column, float (&sum)[8]) {
        const int token = from + lane < to ? runs[warp][from + lane] : 0;
        for (int r0 = 0; r0 < to - from; r0 += U) {
            uint4 row[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned t = __shfl_sync(0xffffffffu, token, r0 + u);
                if (column && r0 + u < to - from) row[u] = __ldcg(column + static_cast<size_t>(t) * vpr);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (r0 + u < to - from) emb_add(sum, row[u]);
        }
    };
    auto column_of = [&](int c) { return c < vpr ? reinterpret_cast<const uint4*>(p.d_y) + c : nullptr; };
    for (int item = warp * gridDim.x + blockIdx.x; item < T * slices; item += EMB_SUM_WARPS * gridDim.x) {
        const int token = item / slices, c = (item - token * slices) * 32 + lane, n = find(token);
        if (n > EMB_PIECE) {
            int at = 0;
            if (lane == 0) at = atomicAdd(&queued, 1);
            at = __shfl_sync(0xffffffffu, at, 0);
            if (at < EMB_QUEUE) {
                if (lane == 0) queue[at] = item;
                continue;
            }
        }
        const long long at = static_cast<long long>(keys[token]) * vpr + c;
        EmbedOld<FP32> old;
        if (ACC && n > 0 && c < vpr) emb_old(p, at, old);
        float sum[8];
        for (int r = 0; r < n; r += EMB_PIECE) {             // (more than one piece: the queue was full)
            float piece[8] = {};
            add_rows(r, min(n, r + EMB_PIECE), column_of(c), piece);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = r == 0 ? piece[e] : __fadd_rn(sum[e], piece[e]);
        }
        if (n > 0 && c < vpr) emb_store<FP32, ACC>(p, at, sum, old);
        __syncwarp();
    }
    __syncthreads();
    for (int q = 0; q < min(queued, EMB_QUEUE); ++q) {
        const int item = queue[q], token = item / slices, c = (item - token * slices) * 32 + lane, n = find(token);
        const int pieces = (n + EMB_PIECE - 1) / EMB_PIECE;
        float sum[8] = {};
        if (warp < pieces) add_rows(warp * EMB_PIECE, min(n, (warp + 1) * EMB_PIECE), column_of(c), sum);
        if (warp < EMB_FOLD_WARPS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[warp][e][lane] = sum[e];
        }
        __syncthreads();
        if (warp == 0 && c < vpr) {
            const long long at = static_cast<long long>(keys[token]) * vpr + c;
            EmbedOld<FP32> old;
            if (ACC) emb_old(p, at, old);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
                for (int w = 1; w < EMB_FOLD_WARPS; ++w) sum[e] = __fadd_rn(sum[e], sums[w][e][lane]);
            }
            emb_store<FP32, ACC>(p, at, sum, old);
        }
        __syncthreads();
    }
    if (!ACC && warp == EMB_SUM_WARPS - 1) tma_store_wait_all();
}

static size_t align16(size_t n) { return (n + 15) / 16 * 16; }
size_t embed_bwd_bytes(int64_t T, int, int H) {
    const size_t n = static_cast<size_t>(T);
    return align16(4 * n) + 16 * n + (T > EMB_CHIP_TOKENS ? 2 * 8 * n + 4 * EMB_WIDE_CTAS * EMB_BINS : 0) + (T > EMB_PIECE ? 2 * (n / EMB_PIECE + 1) * 4 * H : 0) + 16;      // (16: the counters)
}

cudaError_t launch_embed(const EmbedParams& p0, cudaStream_t stream) {
    EmbedParams p = p0;
    const unsigned vpr = p.H / 8;
    // a launch takes as many rows as 32-bit vector indices count
    for (long long rows, left = p.T; left > 0; left -= rows, p.ids += rows, p.y += rows * p.H) {
        rows = std::min<long long>(left, EMB_VEC_MAX / vpr);
        const unsigned n = static_cast<unsigned>(rows * vpr);
        const bool large = n >= (1u << 20);
        const unsigned per = EMB_THREADS * (large ? 4 : 1);
        const cudaError_t e = launch_pdl(large ? embed_kernel<4> : embed_kernel<1>, dim3((n - 1) / per + 1), EMB_THREADS, 0, stream, 1, p, n, vpr);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <bool FP32, bool ACC>
static cudaError_t launch_embed_small(const EmbedParams& p, cudaStream_t stream) {
    return launch_pdl(embed_small_kernel<FP32, ACC>, dim3(static_cast<unsigned>(p.sm_count)), EMB_SUM_THREADS, 0, stream, 1, p);
}
template <bool FP32, bool ACC>
static cudaError_t launch_embed_sums(const EmbedParams& p, cudaStream_t stream) {
    const int late = p.T > EMB_RANK_TOKENS && p.T <= EMB_CHIP_TOKENS && p.sm_count > 2 * EMB_CLUSTER ? EMB_CLUSTER : 0;
    const size_t marks = ACC ? 0 : (std::min(p.V, EMB_MARK_ROWS) + 31) / 32 * sizeof(uint32_t);
    cudaError_t e = launch_pdl(embed_sum_kernel<FP32, ACC>, dim3(static_cast<unsigned>(p.sm_count)), EMB_SUM_THREADS, marks, stream, 1, p, late);
    if (e != cudaSuccess || p.T <= EMB_PIECE) return e;
    const unsigned blocks = static_cast<unsigned>((p.T + EMB_FOLD_WARPS * 32 - 1) / (EMB_FOLD_WARPS * 32));
    return launch_pdl(embed_fold_kernel<FP32, ACC>, dim3(blocks, (p.H / 8 + 31) / 32), EMB_FOLD_WARPS * 32, 0, stream, 1, p);
}

cudaError_t launch_embed_bwd(EmbedParams& p, void* ws, cudaStream_t stream) {
    char* at = static_cast<char*>(ws);
    p.tickets = reinterpret_cast<int*>(at);
    at += 16;
    p.place = reinterpret_cast<uint4*>(at);
    at += 16 * p.T;
    const bool wide = p.T > EMB_CHIP_TOKENS;
    if (wide) {
        p.counts = reinterpret_cast<int*>(at);
        at += 4 * EMB_WIDE_CTAS * EMB_BINS;
        for (int i = 0; i < 2; ++i, at += 8 * p.T) p.keys[i] = reinterpret_cast<uint2*>(at);
    }
    p.order = reinterpret_cast<int32_t*>(at);
    p.part = reinterpret_cast<float*>(at + align16(4 * p.T));
    cudaError_t e = cudaSuccess;
    const long long table_bytes = static_cast<long long>(p.V) * p.H * (p.fp32 ? 4 : 2);
    if (p.T > 0 && p.T <= EMB_SMALL_TOKENS && (p.accumulate || (table_bytes <= EMB_SMALL_BYTES && p.V / p.sm_count < EMB_SMALL_ROWS)))
        return p.fp32 ? (p.accumulate ? launch_embed_small<true, true>(p, stream) : launch_embed_small<true, false>(p, stream))
                      : (p.accumulate ? launch_embed_small<false, true>(p, stream) : launch_embed_small<false, false>(p, stream));
    if (p.T > EMB_RANK_TOKENS) {
        static DeviceOnce configured;
        e = configured.run([&]() {
            cudaError_t r = cudaSuccess;
            auto allow = [&](auto kern, int nw) {
                if (r == cudaSuccess)
                    r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(emb_sort_smem(nw)));
            };
            if (r == cudaSuccess) r = cudaFuncSetAttribute(embed_wide_count_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(EmbedWideSmem));
            if (r == cudaSuccess) r = cudaFuncSetAttribute(embed_wide_move_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(EmbedWideSmem));
            allow(embed_sort_kernel<1>, 1);
            allow(embed_sort_kernel<2>, 2);
            allow(embed_sort_kernel<4>, 4);
            allow(embed_sort_kernel<8>, 8);
            return r;
        });
        if (e != cudaSuccess) return e;
        int bits = 1;
        while (p.V >> bits) ++bits;                          // keys are 0 .. V
        const int passes = (bits + 8) / 9, digit_bits = (bits + passes - 1) / passes;
        if (wide) {
            for (int pass = 0; pass < passes && e == cudaSuccess; ++pass) {
                e = launch_pdl(embed_wide_count_kernel, dim3(EMB_WIDE_CTAS), EMB_SORT_THREADS, sizeof(EmbedWideSmem), stream, 1, p, pass, digit_bits);
                if (e == cudaSuccess)
                    e = launch_pdl(embed_wide_move_kernel, dim3(EMB_WIDE_CTAS), EMB_SORT_THREADS, sizeof(EmbedWideSmem), stream, 1, p, pass, digit_bits);
            }
            if (e != cudaSuccess) return e;
            const unsigned grid = static_cast<unsigned>((p.T + 32 * EMB_RECORD_WARPS - 1) / (32 * EMB_RECORD_WARPS));
            e = launch_pdl(embed_wide_record_kernel, dim3(grid), EMB_RECORD_WARPS * 32, 0, stream, 1, p, passes);
        } else {
            const long long windows = (p.T + EMB_CHIP_TOKENS / 8 - 1) / (EMB_CHIP_TOKENS / 8);       // per warp
            const int nw = windows <= 1 ? 1 : windows <= 2 ? 2 : windows <= 4 ? 4 : 8;
            auto kern = nw == 1 ? embed_sort_kernel<1> : nw == 2 ? embed_sort_kernel<2> : nw == 4 ? embed_sort_kernel<4> : embed_sort_kernel<8>;
            e = launch_pdl(kern, dim3(EMB_CLUSTER), EMB_SORT_THREADS, emb_sort_smem(nw), stream, EMB_CLUSTER, p, passes, digit_bits);
        }
    } else if (p.T > 0) {
        e = launch_pdl(embed_rank_kernel, dim3(static_cast<unsigned>((p.T + 31) / 32)), EMB_RANK_WARPS * 32, 0, stream, 1, p);
    }
    if (e != cudaSuccess) return e;
    return p.fp32 ? (p.accumulate ? launch_embed_sums<true, true>(p, stream) : launch_embed_sums<true, false>(p, stream))
                  : (p.accumulate ? launch_embed_sums<false, true>(p, stream) : launch_embed_sums<false, false>(p, stream));
}

}  // namespace tik
