// Clipped policy loss with a KL term over packed tokens, and its gradient with respect to the log-probabilities.
//
// Per token, with x = logprob - old_logprob, r = exp(x), advantage A and y = ref_logprob - logprob:
//   policy = max(-A r, -A clamp(r, 1 - clip_low, 1 + clip_high)),  for A < 0 and clip_dual: at most -A clip_dual
//   kl     = exp(y) - y - 1
//   l      = policy + kl_coef kl,      dl/dlogprob = (cut ? 0 : -A r) - kl_coef (exp(y) - 1)
// and over the tokens whose weight w is not 0:  loss = sum_t f_t l_t,  d_logprob = f_t dl_t, with f_t = scale w_t, divided by the
// number of such tokens (of the whole call, or of the token's sequence).
//
// Per token fp32, but where digits would be lost that matter: whether a token is cut is decided on x in 64 bits against the
// logarithms of the thresholds (r in 32 bits would put tokens on the wrong side of a border where the gradient jumps); exp(y) - y - 1 comes
// from its series, not from a difference; -A r goes into the sum as -A and -A (r - 1), the first exact and the second small, and from x = -1 down,
// where r - 1 has lost digits of r (half of them at x = -8, all at -18), as it is, in the gradient too.  Sums over tokens,
// which are of both signs and mostly cancel, are fp64 in one fixed order, counts are integers.  (All of it in fp64 took 275 instructions a token.)
// 20 bytes in and 4 out per token, so a call is all latency: up to 4096 tokens one cluster of up to eight CTAs takes
// it in one launch, a token a thread, counts and sums through distributed shared memory.  Longer calls, whose arithmetic needs all
// SMs, take two: one counts, the other computes, and its last CTA folds the sums.
#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

namespace loss {
constexpr int MAX_CLUSTER = 8;
constexpr int SEQ_CAP = 8192;                // sequences' counts that a CTA of a cluster holds
constexpr int STEPS = 4;                     // tokens of a thread at most, one per 32 tokens of its warp's stretch
constexpr int CLUSTER_THREADS = 512;
constexpr int GRID_THREADS = 256;
constexpr int MAX_CTAS = 592;                // of the two-launch form
constexpr int SUMS = 5;                      // policy, KL, tokens cut, r - 1 - x, tokens that count
}  // namespace loss

// tokens that a sequence may hold
__device__ __forceinline__ void loss_range(const PolicyLossParams& p, int& from, int& to) {
    from = 0;
    to = p.T;
    if (p.cu) {
        from = max(p.cu[0], 0);
        to = min(p.cu[p.S], to);
    }
}

// exp(x) - 1 and exp(x) - 1 - x.  Up to |x| = 1, where nearly all tokens are, from x^2 q(x) with q = sum x^n / (n + 2)! to n = 10 (the next
// term is 4e-9 of q): nothing cancels.  Beyond, where little does, through expf.
struct Exp {
    float less_one, remainder, whole;                      // whole: exp(x), from x = -1 down, where exp(x) - 1 has lost digits of it
};
__device__ __forceinline__ Exp loss_exp(float x) {
    Exp e;
    if (fabsf(x) < 1.0f) {
        float q = 1.0f / 479001600.0f;
        q = fmaf(q, x, 1.0f / 39916800.0f);
        q = fmaf(q, x, 1.0f / 3628800.0f);
        q = fmaf(q, x, 1.0f / 362880.0f);
        q = fmaf(q, x, 1.0f / 40320.0f);
        q = fmaf(q, x, 1.0f / 5040.0f);
        q = fmaf(q, x, 1.0f / 720.0f);
        q = fmaf(q, x, 1.0f / 120.0f);
        q = fmaf(q, x, 1.0f / 24.0f);
        q = fmaf(q, x, 1.0f / 6.0f);
        q = fmaf(q, x, 0.5f);
        e.remainder = x * x * q;
        e.less_one = x + e.remainder;
        e.whole = 0.0f;
    } else {
        e.whole = expf(x);
        e.less_one = e.whole - 1.0f;
        e.remainder = e.less_one - x;
    }
    return e;
}

// A thread's share of the sums
struct LossSums {
    double policy = 0.0, kl = 0.0, remainder = 0.0;
    int cut = 0, tokens = 0;
};
// tokens of a sequence, those of the call (without weights: all count)
__device__ __forceinline__ int loss_length(const PolicyLossParams& p, int s) { return min(p.cu[s + 1], p.T) - max(p.cu[s], 0); }

// Adds a token that counts to the sums and returns its gradient; f: its factor.
__device__ __forceinline__ float loss_token(const PolicyLossParams& p, double f, float lp, float old, float adv, float ref, LossSums& sum) {
    const float x = lp - old;
    const Exp r = loss_exp(x);
    // x against a threshold, in 64 bits where 32 do not settle it
    auto beyond = [&](double mark, float sign) {
        const float d = sign * (x - static_cast<float>(mark));
        if (fabsf(d) > 1e-6f * (fabsf(x) + 1.0f)) return d > 0.0f;
        return sign * ((static_cast<double>(lp) - static_cast<double>(old)) - mark) > 0.0;
    };
    const bool up = adv > 0.0f, down = adv < 0.0f;
    bool cut = (up || down) && beyond(up ? p.log_high : p.log_low, up ? 1.0f : -1.0f);
    float less_one = cut ? (up ? p.high : -p.low) : r.less_one;            // of what the advantage is multiplied with
    if (p.dual && down && !cut && beyond(p.log_dual, 1.0f)) {
        cut = true;
        less_one = p.dual_less_one;
    }
    if (adv == 0.0f && fabsf(x) <= 3.402823466e38f) less_one = 0.0f;       // nothing times a ratio beyond fp32 (x beyond it goes on)
    // -A r from r itself where r is small
    const bool small = !cut && x <= -1.0f;
    const float base = small ? 0.0f : -adv, part = -adv * (small ? r.whole : less_one);
    float grad = cut ? 0.0f : small ? part : fmaf(-adv, less_one, -adv);
    sum.policy = fma(f, static_cast<double>(base), sum.policy);
    sum.policy = fma(f, static_cast<double>(part), sum.policy);
    if (p.ref) {
        const Exp e = loss_exp(ref - lp);
        sum.kl = fma(f, static_cast<double>(e.remainder), sum.kl);
        if (p.kl_coef != 0.0f) grad -= p.kl_coef * e.less_one;             // (0 times what may be beyond fp32)
    }
    sum.cut += cut;
    sum.remainder += r.remainder;
    ++sum.tokens;
    return static_cast<float>(f) * grad;
}

// The sequences of a warp's ascending tokens.  `near`: cu[s0 + 1 + lane], the ends of the sequences from s0 on.
struct LossSeq {
    int s0, near;
    __device__ __forceinline__ void load(const PolicyLossParams& p, int lane) { near = p.cu[min(s0 + 1 + lane, p.S)]; }
    __device__ __forceinline__ void begin(const PolicyLossParams& p, int token, int lane) {
        s0 = warp_find_sequence(p.cu, p.S, token, lane);
        load(p, lane);
    }
    // The sequence of each lane's token (whole warp, tokens ascending over the lanes and from call to call); some
    // sequence for a token that none holds.
    __device__ __forceinline__ int of(const PolicyLossParams& p, int token, int lane) {
        int n = 0;                                         // ends that the token has reached: a prefix of the 32
#pragma unroll
        for (int w = 16; w >= 1; w >>= 1)
            if (__shfl_sync(0xffffffffu, near, n + w - 1) <= token) n += w;
        if (__shfl_sync(0xffffffffu, near, 31) <= token) n = 32;
        int s = s0 + n;
        if (n == 32) {
            int hi = p.S;                                  // cu[s] <= token; the last such s
            while (hi - s > 1) {
                const int mid = s + (hi - s) / 2;
                if (p.cu[mid] <= token) s = mid;
                else hi = mid;
            }
        }
        s = min(s, p.S - 1);
        const int last = __shfl_sync(0xffffffffu, s, 31);
        if (last > s0) {
            s0 = last;
            load(p, lane);
        }
        return s;
    }
};

template <class V>
__device__ __forceinline__ V warp_total(V v) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

__device__ __forceinline__ double dsmem_read(uint32_t addr) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ int dsmem_read_int(uint32_t addr) {
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void dsmem_add(uint32_t addr, int v) {
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

__device__ __forceinline__ void loss_results(const PolicyLossParams& p, const double (&sum)[loss::SUMS]) {
    const double n = sum[4] > 1.0 ? sum[4] : 1.0;
    *p.loss = static_cast<float>(p.kl_coef != 0.0f ? sum[0] + static_cast<double>(p.kl_coef) * sum[1] : sum[0]);
    if (p.stats) {
        p.stats[0] = static_cast<float>(sum[0]);
        p.stats[1] = static_cast<float>(sum[1]);
        p.stats[2] = static_cast<float>(sum[2] / n);
        p.stats[3] = static_cast<float>(sum[3] / n);
        p.stats[4] = static_cast<float>(sum[4]);
    }
}
// Sums of a block's threads: thread 0 gets the totals, warps in ascending order.
__device__ __forceinline__ void loss_block_fold(double (&v)[loss::SUMS], const double (*buf)[loss::SUMS], int warps) {
    __syncthreads();
    if (threadIdx.x == 0)
#pragma unroll
        for (int i = 0; i < loss::SUMS; ++i) {
            v[i] = 0.0;
            for (int w = 0; w < warps; ++w) v[i] += buf[w][i];
        }
}
__device__ __forceinline__ void loss_block_sums(const LossSums& s, double (&v)[loss::SUMS], double (*buf)[loss::SUMS], int warps) {
    const double policy = warp_total(s.policy), kl = warp_total(s.kl), remainder = warp_total(s.remainder);
    const int cut = __reduce_add_sync(0xffffffffu, s.cut), tokens = __reduce_add_sync(0xffffffffu, s.tokens);
    if ((threadIdx.x & 31) == 0) {
        double* const to = buf[threadIdx.x >> 5];
        to[0] = policy, to[1] = kl, to[2] = cut, to[3] = remainder, to[4] = tokens;
    }
    loss_block_fold(v, buf, warps);
}

// One cluster, a token a thread.
__global__ void __launch_bounds__(loss::CLUSTER_THREADS) loss_cluster_kernel(const PolicyLossParams p) {
    using namespace loss;
    extern __shared__ int seq_count[];                     // [per]: tokens of the sequences rank * per ...
    __shared__ double sums[CLUSTER_THREADS / 32][SUMS];
    __shared__ double cta_sums[SUMS];
    __shared__ int cta_count;
    const int tid = threadIdx.x, lane = tid & 31, warps = blockDim.x >> 5;
    const int ctas = static_cast<int>(gridDim.x), rank = static_cast<int>(blockIdx.x);
    const bool per_sequence = p.reduction == LOSS_SEQUENCE_MEAN, count_seq = per_sequence && p.weight;
    const int per = (p.S + ctas - 1) / ctas;
    if (count_seq)
        for (int i = tid; i < per; i += blockDim.x) seq_count[i] = 0;
    if (tid == 0) cta_count = 0;
    pdl_wait();
    pdl_launch_dependents();
    const int t = rank * static_cast<int>(blockDim.x) + tid;
    const bool in = t < p.T;
    float w = in ? (p.weight ? p.weight[t] : 1.0f) : 0.0f, adv = in && !p.adv_per_seq ? p.advantage[t] : 0.0f;
    const float lp = in ? p.logprob[t] : 0.0f, old = in ? p.old_logprob[t] : 0.0f, ref = in && p.ref ? p.ref[t] : 0.0f;
    int from, to, seq = 0;
    loss_range(p, from, to);
    if (t < from || t >= to) w = 0.0f;
    if (p.adv_per_seq || per_sequence) {
        LossSeq q;
        q.begin(p, t - lane, lane);
        seq = q.of(p, t, lane);
        if (p.adv_per_seq && w != 0.0f) adv = p.advantage[seq];
    }
    if (ctas > 1) cluster_sync_all();                      // zeroed counts, and every CTA of the cluster has begun
    else __syncthreads();
    const unsigned on = __ballot_sync(0xffffffffu, w != 0.0f);
    if (lane == 0 && on) atomicAdd(&cta_count, __popc(on));
    if (count_seq) {
        // a warp's tokens are mostly of one sequence: one addition for each run of equal ones
        const int before = __shfl_up_sync(0xffffffffu, seq, 1);
        const unsigned heads = __ballot_sync(0xffffffffu, lane == 0 || before != seq);
        if (heads >> lane & 1u) {
            const unsigned later = lane == 31 ? 0u : heads & (0xffffffffu << (lane + 1));
            const unsigned run = (later ? (1u << (__ffs(later) - 1)) - 1u : 0xffffffffu) & (0xffffffffu << lane);
            const int n = __popc(on & run), owner = seq / per;
            if (n > 0) dsmem_add(mapa_cluster(smem_u32(&seq_count[seq - owner * per]), owner), n);
        }
    }
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
    double f = p.scale;
    if (p.reduction == LOSS_TOKEN_MEAN) {
        int all = 0;
        for (int c = 0; c < ctas; ++c) all += dsmem_read_int(mapa_cluster(smem_u32(&cta_count), c));
        f /= all > 1 ? all : 1;
    }
    LossSums mine;
    float d = 0.0f;
    if (w != 0.0f) {
        f *= w;
        if (per_sequence) {
            const int owner = seq / per;
            const int n = count_seq ? dsmem_read_int(mapa_cluster(smem_u32(&seq_count[seq - owner * per]), owner)) : loss_length(p, seq);
            f /= n > 1 ? n : 1;
        }
        d = loss_token(p, f, lp, old, adv, ref, mine);
    }
    if (p.d_logprob && in) p.d_logprob[t] = d;
    double sum[SUMS];
    loss_block_sums(mine, sum, sums, warps);
    if (ctas == 1) {
        if (tid == 0) loss_results(p, sum);
        return;
    }
    if (tid == 0)
#pragma unroll
        for (int i = 0; i < SUMS; ++i) cta_sums[i] = sum[i];
    cluster_sync_all();
    if (rank == 0 && tid == 0) {
        for (int c = 1; c < ctas; ++c)
#pragma unroll
            for (int i = 0; i < SUMS; ++i) sum[i] += dsmem_read(mapa_cluster(smem_u32(&cta_sums[i]), c));
        loss_results(p, sum);
    }
    cluster_sync_all();                                    // nobody leaves while its sums may still be read
}

// Tokens per sequence (a CTA each, `count` has S entries), or of the CTAs' shares of the call; the ticket of the next kernel.  A CTA counts a million
// tokens in 600 us: calls of a few long sequences wait for the longest (a million tokens in one sequence 636 us, in 8 101, in 1024 21).
__global__ void __launch_bounds__(loss::GRID_THREADS) loss_count_kernel(const PolicyLossParams p) {
    using namespace loss;
    __shared__ int buf[GRID_THREADS / 32];
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x == 0 && tid == 0) *p.ticket = 0;
    if (!p.weight) return;
    int lo, hi;
    loss_range(p, lo, hi);
    unsigned from = lo + blockIdx.x * GRID_THREADS, to = hi, step = gridDim.x * GRID_THREADS;
    if (p.reduction == LOSS_SEQUENCE_MEAN) {
        from = max(lo, p.cu[blockIdx.x]);
        to = max(min(hi, p.cu[blockIdx.x + 1]), 0);
        step = GRID_THREADS;
    } else if (hi < 0) {
        to = 0;
    }
    int n = 0;
#pragma unroll 8
    for (unsigned t = from + tid; t < to; t += step) n += p.weight[t] != 0.0f;
    n = warp_total(n);
    if ((tid & 31) == 0) buf[tid >> 5] = n;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < GRID_THREADS / 32; ++w) n += buf[w];
        p.count[blockIdx.x] = n;
    }
}

__global__ void __launch_bounds__(loss::GRID_THREADS, 4) loss_grid_kernel(const PolicyLossParams p, int counts, int steps) {
    using namespace loss;
    constexpr int WARPS = GRID_THREADS / 32;
    __shared__ double sums[WARPS][SUMS];
    __shared__ int buf[WARPS];
    __shared__ bool last;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool per_sequence = p.reduction == LOSS_SEQUENCE_MEAN, find = p.adv_per_seq || per_sequence;
    pdl_wait();
    pdl_launch_dependents();
    // (unsigned: the last step of a call of nearly 2^31 tokens passes them)
    const unsigned stretch = 32u * steps, step = gridDim.x * WARPS * stretch, T = static_cast<unsigned>(p.T);
    unsigned base = (blockIdx.x * WARPS + warp) * stretch;
    float lp[STEPS], old[STEPS], adv[STEPS], w[STEPS], ref[STEPS];
    auto load = [&]() {
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            const unsigned t = base + 32 * j + lane;
            const bool in = j < steps && t < T;
            w[j] = in ? (p.weight ? p.weight[t] : 1.0f) : 0.0f;
            lp[j] = in ? p.logprob[t] : 0.0f;
            old[j] = in ? p.old_logprob[t] : 0.0f;
            adv[j] = in && !p.adv_per_seq ? p.advantage[t] : 0.0f;
            ref[j] = in && p.ref ? p.ref[t] : 0.0f;
        }
    };
    load();                                                // on its way while the counts are folded
    int lo, hi;
    loss_range(p, lo, hi);
    double f = p.scale;
    if (p.reduction == LOSS_TOKEN_MEAN) {
        int all = hi - lo;
        if (p.weight) {
            int n = 0;
            for (int i = tid; i < counts; i += GRID_THREADS) n += p.count[i];
            n = warp_total(n);
            if (lane == 0) buf[warp] = n;
            __syncthreads();
            all = 0;
            for (int w = 0; w < WARPS; ++w) all += buf[w];
        }
        f /= static_cast<double>(all > 1 ? all : 1);
    }
    LossSums mine;
    while (base < T) {
        LossSeq q;
        if (find) q.begin(p, static_cast<int>(base), lane);
#pragma unroll
        for (int j = 0; j < STEPS; ++j) {
            if (j >= steps) break;
            const unsigned at = base + 32 * j + lane;
            const int t = at < T ? static_cast<int>(at) : p.T - 1;
            const int s = find ? q.of(p, t, lane) : 0;
            float d = 0.0f;
            if (w[j] != 0.0f && t >= lo && t < hi) {
                double fj = f * w[j];
                if (per_sequence) {
                    const int n = p.weight ? p.count[s] : loss_length(p, s);
                    fj /= n > 1 ? n : 1;
                }
                d = loss_token(p, fj, lp[j], old[j], p.adv_per_seq ? p.advantage[s] : adv[j], ref[j], mine);
            }
            if (p.d_logprob && at < T) p.d_logprob[at] = d;
        }
        base += step;
        if (base < T) load();
    }
    double sum[SUMS];
    loss_block_sums(mine, sum, sums, WARPS);
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < SUMS; ++i) p.part[blockIdx.x * SUMS + i] = sum[i];
        __threadfence();
        last = atomicAdd(p.ticket, 1) == static_cast<int>(gridDim.x) - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    // the CTAs' sums in one order, whichever CTA is the last
    double part[(MAX_CTAS + GRID_THREADS - 1) / GRID_THREADS][SUMS];
#pragma unroll
    for (int k = 0; k < (MAX_CTAS + GRID_THREADS - 1) / GRID_THREADS; ++k)
#pragma unroll
        for (int i = 0; i < SUMS; ++i) {
            const int c = tid + k * GRID_THREADS;
            part[k][i] = c < static_cast<int>(gridDim.x) ? __ldcg(&p.part[c * SUMS + i]) : 0.0;
        }
#pragma unroll
    for (int i = 0; i < SUMS; ++i) {
        double v = part[0][i];
#pragma unroll
        for (int k = 1; k < (MAX_CTAS + GRID_THREADS - 1) / GRID_THREADS; ++k) v += part[k][i];
        v = warp_total(v);
        if (lane == 0) sums[warp][i] = v;
    }
    loss_block_fold(sum, sums, WARPS);
    if (tid == 0) loss_results(p, sum);
}

// Scratch: the ticket (16 bytes), the CTAs' sums, and counts of sequences or CTAs.
size_t policy_loss_bytes(int64_t S) {
    const size_t counts = static_cast<size_t>(S > loss::MAX_CTAS ? S : loss::MAX_CTAS);
    return 16 + sizeof(double) * loss::SUMS * loss::MAX_CTAS + (counts * sizeof(int) + 15) / 16 * 16;
}

cudaError_t launch_policy_loss(PolicyLossParams& p, void* ws, cudaStream_t stream) {
    using namespace loss;
    const bool counts_seq = p.reduction == LOSS_SEQUENCE_MEAN && p.weight;
    // (Two tokens a thread of the cluster: 8000 tokens 8.5 us, 7.0 by two launches; 4000 tokens 6.3 either way, and a launch less of the host.)
    if (p.T <= MAX_CLUSTER * CLUSTER_THREADS && (!counts_seq || p.S <= SEQ_CAP)) {
        int ctas = 1;
        while (p.T > ctas * CLUSTER_THREADS) ctas *= 2;
        const int threads = p.T > CLUSTER_THREADS ? CLUSTER_THREADS : p.T > 32 ? (p.T + 31) / 32 * 32 : 32;
        const size_t smem = counts_seq ? static_cast<size_t>((p.S + ctas - 1) / ctas) * sizeof(int) : 0;
        return launch_pdl(loss_cluster_kernel, dim3(ctas), static_cast<unsigned>(threads), smem, stream, static_cast<unsigned>(ctas), p);
    }
    p.ticket = static_cast<int*>(ws);
    p.part = reinterpret_cast<double*>(static_cast<char*>(ws) + 16);
    p.count = reinterpret_cast<int*>(p.part + SUMS * MAX_CTAS);
    // as few tokens a thread as MAX_CTAS allow: what a thread does one after the other is what a call waits for
    const int64_t waves = (p.T + static_cast<int64_t>(MAX_CTAS) * GRID_THREADS - 1) / (static_cast<int64_t>(MAX_CTAS) * GRID_THREADS);
    const int steps = static_cast<int>(waves < STEPS ? waves : STEPS);
    const int64_t stretches = (p.T + static_cast<int64_t>(GRID_THREADS) * steps - 1) / (static_cast<int64_t>(GRID_THREADS) * steps);
    const int ctas = static_cast<int>(stretches < MAX_CTAS ? stretches : MAX_CTAS);
    const int counts = !p.weight ? 1 : p.reduction == LOSS_SEQUENCE_MEAN ? p.S : ctas;
    cudaError_t e = launch_pdl(loss_count_kernel, dim3(static_cast<unsigned>(counts)), GRID_THREADS, 0, stream, 1, p);
    if (e != cudaSuccess) return e;
    return launch_pdl(loss_grid_kernel, dim3(static_cast<unsigned>(ctas)), GRID_THREADS, 0, stream, 1, p, counts, steps);
}

}  // namespace tik
