// The step between two blocks of a layer -- norm after the block, gate, scaled residual sum, norm before the next block --
// and its gradient.
#include <cuda_bf16.h>

#include <type_traits>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int BN_THREADS = 128;

// a row's sum from its warps' totals
template <int ROWS>
__device__ __forceinline__ float bn_row_total(const float* w4, int mine) {
    return ROWS == 4 ? w4[mine] : ROWS == 2 ? __fadd_rn(w4[2 * mine], w4[2 * mine + 1]) : hn_block_total(w4);
}

// One CTA per row with the reduction shape of rmsnorm_kernel (NV 16-byte vectors per thread): without post norm and gate
// and with a scale of 1 the results are those of its residual form, bit for bit.
// FEW (calls of up to BN_FEW_ROWS rows): weights and gate are requested with the row, not when they are needed -- a chain of
// trips to L2 that many resident rows hide, and that a decode step waits for (call after call on the device, us: 64 x 3584 4.2 without
// and 2.4 with FEW; 1024 x 3584 5.4 and 5.8; 9001 x 5120 58 and 92: its registers halve the rows on an SM).
// ROWS: rows of a CTA.  Of up to 256 (512) channels a row's data sit in one (two) of the four warps of that shape, whose totals are then
// the whole sum, so four (two) rows take a CTA and a CTA per row does not wait for its turn to start (60 000 x 256: 50.4 us
// with one row, 24.6 with four).
constexpr long long BN_FEW_ROWS = 512;
template <int NV, bool FEW, int ROWS>
__global__ void __launch_bounds__(BN_THREADS) block_norm_kernel(const BlockNormParams p) {
    constexpr int WIDTH = BN_THREADS / ROWS;
    const int mine = threadIdx.x / WIDTH, tid = threadIdx.x % WIDTH, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = blockIdx.x * static_cast<long long>(ROWS) + mine;
    const bool there = ROWS == 1 || row < p.T;
    const int nvec = there ? p.H / 8 : 0;
    const uint4* x = reinterpret_cast<const uint4*>(p.x) + row * nvec;
    const uint4* res = reinterpret_cast<const uint4*>(p.residual) + row * nvec;
    const uint4* wp = reinterpret_cast<const uint4*>(p.post_weight);
    const uint4* wn = reinterpret_cast<const uint4*>(p.weight);
    __shared__ float tot_x[4], tot_s[4];
    pdl_wait();
    if (gridDim.x <= 2048 || p.H >= 1536) pdl_launch_dependents();       // (many short rows go without: the rule in tik_ffn.cu)
    uint4 xv[NV], rv[NV], wpv[FEW ? NV : 1], gv[FEW ? NV : 1], wnv[FEW ? NV : 1];
    const uint4* gc = p.gate_kind == GATE_CHANNEL ? reinterpret_cast<const uint4*>(p.gate) : nullptr;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + WIDTH * j;
        if (v < nvec) {
            xv[j] = x[v];
            rv[j] = res[v];
            if (FEW) {
                if (wp) wpv[j] = wp[v];
                if (gc) gv[j] = gc[v];
                if (wn) wnv[j] = wn[v];
            }
        }
    }
    const float inv_h = 1.0f / static_cast<float>(p.H);
    float c = p.branch_scale;                                // what all channels have in common
    if (p.gate_kind == GATE_TOKEN) c = __fmul_rn(c, there ? __bfloat162float(p.gate[row]) : 0.0f);
    if (wp) {
        F2 part = f2(0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (tid + WIDTH * j < nvec) {
                const uint32_t xw[4] = {xv[j].x, xv[j].y, xv[j].z, xv[j].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const F2 f = f2_bf16(xw[e]);
                    part = f2_fma(f, f, part);
                }
            }
        const float sum = hn_warp_total(f2_sum(part));
        if (lane == 0) tot_x[warp] = sum;
        __syncthreads();
        c = __fmul_rn(c, prep_inv_rms(bn_row_total<ROWS>(tot_x, mine), inv_h, p.eps));
    }
    const F2 c2 = f2(c);
    uint32_t s[NV][4];
    float part = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + WIDTH * j;
        if (v >= nvec) continue;
        const uint32_t xw[4] = {xv[j].x, xv[j].y, xv[j].z, xv[j].w}, rw[4] = {rv[j].x, rv[j].y, rv[j].z, rv[j].w};
        F2 f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = f2_mul(f2_bf16(xw[e]), c2);
        if (wp) {
            const uint4 w4 = FEW ? wpv[FEW ? j : 0] : wp[v];
            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = f2_mul(f[e], f2_bf16(w[e]));
        }
        if (gc) {
            const uint4 g4 = FEW ? gv[FEW ? j : 0] : gc[v];
            const uint32_t g[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = f2_mul(f[e], f2_bf16(g[e]));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float lo, hi;
            f2_get(f2_add(f2_bf16(rw[e]), f[e]), lo, hi);
            s[j][e] = pack_bf16x2(lo, hi);
            // (one chain in the order of the elements, as rmsnorm_kernel's)
            f2_get(f2_bf16(s[j][e]), lo, hi);
            part = __fmaf_rn(hi, hi, __fmaf_rn(lo, lo, part));
        }
        reinterpret_cast<uint4*>(p.s)[row * nvec + v] = make_uint4(s[j][0], s[j][1], s[j][2], s[j][3]);
    }
    if (!wn) return;
    part = hn_warp_total(part);
    if (lane == 0) tot_s[warp] = part;
    __syncthreads();
    const F2 inv = f2(prep_inv_rms(bn_row_total<ROWS>(tot_s, mine), inv_h, p.eps));
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + WIDTH * j;
        if (v >= nvec) continue;
        const uint4 w4 = FEW ? wnv[FEW ? j : 0] : wn[v];
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float lo, hi;
            f2_get(f2_mul(f2_mul(f2_bf16(s[j][e]), inv), f2_bf16(w[e])), lo, hi);
            o[e] = pack_bf16x2(lo, hi);
        }
        reinterpret_cast<uint4*>(p.y)[row * nvec + v] = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// ---- gradient --------------------------------------------------------------------------------
// Per row of x, s, d_y and d_s two sums over the row have to be known before the next step: (x^2, s^2, d_y w s), which give G, and
// G x (post weight, gate), which gives d_x.  Six planes of T x H cross HBM once, which bounds the kernel, if the instructions
// (four hundred a row and thread) and the waits between them leave room: the first sums of a row are taken beside the second
// of the row before it, so that a row costs one barrier and one reduction of four values.  One persistent CTA per SM,
// made of groups that each take a row at a time; rows arrive by bulk copies into a ring that the groups share.  A thread has the
// same NV x 8 columns of every row, so that the sums over tokens stay in its registers until the end;
// block_norm_fold_kernel adds up the CTAs'.
// Two fp32 values.  (The two-wide instructions of block_norm_kernel make this kernel slower: 12 % fewer instructions, but warps wait
// for them longer than fourteen warps on an SM hide; 16001 x 3584 121.9 us with them, 119.3 without.)
struct S2 {
    float lo, hi;
};
__device__ __forceinline__ S2 s2(float both) { return {both, both}; }
__device__ __forceinline__ S2 s2(float lo, float hi) { return {lo, hi}; }
__device__ __forceinline__ S2 s2_bf16(uint32_t w) { return {__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)}; }
__device__ __forceinline__ S2 s2_fma(S2 a, S2 b, S2 c) { return {__fmaf_rn(a.lo, b.lo, c.lo), __fmaf_rn(a.hi, b.hi, c.hi)}; }
__device__ __forceinline__ S2 s2_mul(S2 a, S2 b) { return {__fmul_rn(a.lo, b.lo), __fmul_rn(a.hi, b.hi)}; }
// a * b + c of bf16 factors with one rounding, which takes no unpacking (the products with d_y so: 8000 calls of 16001 x 3584 in a row, at
// the power limit and its lower clock, 124 us -> 122, of 32000 x 1536 103 -> 102; 24 calls 112 either way.  The squares too: 8000 calls 122,
// 24 calls 120).
__device__ __forceinline__ S2 s2_fma_bf16(uint32_t a, uint32_t b, S2 c) {
    S2 d;
    asm("{\n\t.reg .b16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %2;\n\tmov.b32 {bl, bh}, %3;\n\t"
        "fma.rn.f32.bf16 %0, al, bl, %4;\n\tfma.rn.f32.bf16 %1, ah, bh, %5;\n\t}"
        : "=f"(d.lo), "=f"(d.hi) : "r"(a), "r"(b), "f"(c.lo), "f"(c.hi));
    return d;
}
__device__ __forceinline__ float s2_sum(S2 a) { return __fadd_rn(a.lo, a.hi); }

constexpr int BN_THREADS_MOST = 512, BN_THREADS_WIDE = 640;  // at 128 and at 96 registers

struct BlockNormBwdShape {
    int nv, most, group, groups, ctas, slots, slot_bytes, factor_bytes;  // 16-byte vectors per thread, threads at most, threads of a group
    size_t smem;
};
constexpr int BN_SLOTS = 64;
struct BlockNormBwdSmem {
    unsigned long long full[BN_SLOTS];
    float4 sums[2][BN_THREADS_WIDE / 32];                    // [turn][warp of the CTA]
    int abort_word;
};
constexpr int BN_RING = (sizeof(BlockNormBwdSmem) + 127) / 128 * 128;

// Sums of four values over the lanes that differ in the bits of FIRST and below: a butterfly whose first two steps fold two values
// into one register, one half of the lanes going on with either.  Lane l ends with value l / (FIRST / 2) % 4.
template <int FIRST>
__device__ __forceinline__ float bn_sums4(float a, float b, float c, float d, int lane) {
    const bool up = lane & FIRST, up2 = lane & (FIRST / 2);
    const float ac = (up ? c : a) + __shfl_xor_sync(0xffffffffu, up ? a : c, FIRST);
    const float bd = (up ? d : b) + __shfl_xor_sync(0xffffffffu, up ? b : d, FIRST);
    float t = (up2 ? bd : ac) + __shfl_xor_sync(0xffffffffu, up2 ? ac : bd, FIRST / 2);
#pragma unroll
    for (int off = FIRST / 4; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    return t;
}

// Root of a mean square: it may be subnormal, when eps is 0 or smaller than that, and the forward's root takes it as it is.  rsqrtf's
// scaling of such arguments costs the rows of one vector a thread more than of two (9001 x 5120 107 us, 60 000 x 256 51.6), so there the
// instruction without it comes first and rsqrtf behind a branch that hardly any row takes (104 and 50.8; with two vectors
// 16 001 x 3584 takes 111 us by rsqrtf and 115 so).
template <int NV>
__device__ __forceinline__ float bn_rsqrt(float x) {
    if (NV > 1) return rsqrtf(x);
    float r;
    asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// X: something of x is needed -- it has a norm or a gate.  Without either d_x is G times a number, and x is not read (gradient of
// the norm before a block alone, 16 001 x 3584: 99 us with x, 82 without).
template <int NV, int THREADS, bool X>
__global__ void __launch_bounds__(THREADS, 1) block_norm_bwd_kernel(const BlockNormParams p, const BlockNormBwdShape shape) {
    constexpr int PLANES = X ? 4 : 3;                        // of a slot: d_s, x, s, d_y
    extern __shared__ __align__(128) unsigned char bn_smem[];
    BlockNormBwdSmem& sm = *reinterpret_cast<BlockNormBwdSmem*>(bn_smem);
    // branch_scale * post_weight * gate (per channel) of the columns in fp32; then the ring
    float4* const factors = reinterpret_cast<float4*>(bn_smem + BN_RING);
    unsigned char* const ring = bn_smem + BN_RING + shape.factor_bytes;
    const int width = shape.group, group = threadIdx.x / width, tid = threadIdx.x - group * width;       // threads of a group
    const int lane = threadIdx.x & 31, warps = width >> 5, warp = tid >> 5;
    const int nvec = p.H / 8, row_vecs = NV * width;      // (a row in the ring is as wide as the threads' vectors)
    const float inv_h = 1.0f / static_cast<float>(p.H);
    const bool norm = p.weight != nullptr, post = X && p.post_weight != nullptr, branch = p.d_x != nullptr;
    // What is absent reads as zeros: planes that are not there, vectors behind the row.
    for (int i = threadIdx.x; i < shape.slots * PLANES * row_vecs; i += blockDim.x) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    if (threadIdx.x == 0) {
        for (int i = 0; i < shape.slots; ++i) mbar_init(smem_u32(&sm.full[i]), 1);
        sm.abort_word = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const int planes = (norm ? 2 : 0) + (X ? 1 : 0) + (p.d_s ? 1 : 0);
    // The CTA's n-th row, which group n % groups takes, is row blockIdx.x + n * gridDim.x.
    const unsigned T = static_cast<unsigned>(p.T);           // (below 2^31: a row behind the last one does not wrap)
    auto request = [&](unsigned row, int slot) {
        if (row >= T) return;
        const uint32_t bar = smem_u32(&sm.full[slot]), to = smem_u32(ring + slot * shape.slot_bytes);
        mbar_expect_tx(bar, planes * p.H * 2);
        const __nv_bfloat16* src[4] = {p.d_s, X ? p.x : nullptr, norm ? p.s : nullptr, norm ? p.d_y : nullptr};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (src[i]) bulk_load(to + (X || i == 0 ? i : i - 1) * 16 * row_vecs, src[i] + static_cast<size_t>(row) * p.H, p.H * 2, bar);
    };
    if (threadIdx.x == 0)
        for (int n = 0; n < shape.slots; ++n) request(blockIdx.x + n * gridDim.x, n);
    // [half vector][thread]: 16 bytes a thread and instruction; every group writes the same values and reads what it wrote itself
    uint32_t w[NV][4];
    S2 sum_w[NV][4], sum_c[NV][4];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int v = tid + width * j;
        auto column = [&](const __nv_bfloat16* base, bool there, float (&to)[8]) {
            unpack8(there && v < nvec ? reinterpret_cast<const uint4*>(base)[v] : make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u), to);
        };
        float f[8], g[8];
        column(p.post_weight, post, f);
        column(p.gate, p.gate_kind == GATE_CHANNEL, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = p.branch_scale * (f[e] * g[e]);
        factors[2 * j * width + tid] = make_float4(f[0], f[1], f[2], f[3]);
        factors[(2 * j + 1) * width + tid] = make_float4(f[4], f[5], f[6], f[7]);
        const uint4 wv = norm && v < nvec ? reinterpret_cast<const uint4*>(p.weight)[v] : make_uint4(0, 0, 0, 0);
        w[j][0] = wv.x, w[j][1] = wv.y, w[j][2] = wv.z, w[j][3] = wv.w;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum_w[j][e] = sum_c[j][e] = s2(0.0f);
    }
    int slot = group, turn = 0;                              // (there are more slots than groups)
    uint32_t parity = 0;
    unsigned row = blockIdx.x + group * gridDim.x;
    const unsigned step = gridDim.x * shape.groups;
    auto take = [&](const uint4* at, int plane, int j, uint32_t (&to)[4]) {
        const uint4 v = at[plane * row_vecs + width * j];
        to[0] = v.x, to[1] = v.y, to[2] = v.z, to[3] = v.w;
    };
    auto row_at = [&](int s) { return reinterpret_cast<const uint4*>(ring + s * shape.slot_bytes) + tid; };
    float tx, ts, tq;                                        // a row's first sums: this thread's part
    auto first_sums = [&](int s, uint32_t par) {
        mbar_wait(smem_u32(&sm.full[s]), par, &sm.abort_word, p.dev_status);
        const uint4* at = row_at(s);
        S2 sx = s2(0.0f), ss = s2(0.0f), sq = s2(0.0f);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            uint32_t x[4], s4[4], dy[4];
            if (X) take(at, 1, j, x);
            take(at, PLANES - 2, j, s4);
            take(at, PLANES - 1, j, dy);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const S2 se = s2_bf16(s4[e]);
                if (X) sx = s2_fma(s2_bf16(x[e]), s2_bf16(x[e]), sx);
                ss = s2_fma(se, se, ss);
                sq = s2_fma(s2_fma_bf16(dy[e], w[j][e], s2(0.0f)), se, sq);
            }
        }
        tx = s2_sum(sx), ts = s2_sum(ss), tq = s2_sum(sq);
    };
    // (tx, ts, tq, td) of the group
    auto total = [&](float td, float (&to)[4]) {
        const float part = bn_sums4<16>(tx, ts, tq, td, lane);
        float* mine = reinterpret_cast<float*>(sm.sums[turn] + group * warps);
        if ((lane & 7) == 0) mine[4 * warp + lane / 8] = part;
        if (warps > 1) named_bar_sync(1 + group, width);
        else __syncwarp();
        constexpr int WARPS = NV == 1 ? 32 : 16;             // of a group, at most
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if ((lane & (WARPS - 1)) < warps) v = sm.sums[turn][group * warps + (lane & (WARPS - 1))];
        const float t = bn_sums4<WARPS / 2>(v.x, v.y, v.z, v.w, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = __shfl_sync(0xffffffffu, t, WARPS / 4 * i);
        turn ^= 1;
    };
    float sums[4];
    if (row < T) first_sums(slot, parity);
    // A barrier's parity tells a phase from the next one only, so whoever waits for a slot's row has to know that the row before it
    // in that slot has arrived.  Of later rows it does: a row is requested by a group that has seen the row that many groups
    // behind the old one of that slot.  For the first rows that replace another, which are waited for beside rows of the first
    // fill, it is the groups' first rows that have to be there.
    __syncthreads();
    if (row < T) total(0.0f, sums);
    for (; row < T; row += step) {
        const float gt = p.gate_kind == GATE_TOKEN ? __bfloat162float(p.gate[row]) : 1.0f;
        const float ms = fmaf(sums[1], inv_h, p.eps), mx = fmaf(sums[0], inv_h, p.eps);
        float rs = norm ? bn_rsqrt<NV>(ms) : 0.0f, rx = post ? bn_rsqrt<NV>(mx) : 1.0f;
        if (NV == 1 && (ms < 0x1p-126f || (X && mx < 0x1p-126f))) {
            if (norm) rs = rsqrtf(ms);
            if (post) rx = rsqrtf(mx);
        }
        // G = d_s + r (q - k s): k = r^2 mean(q s), by products in this order, is no larger than r times the rms of q, which is in
        // range where G is.  r^3 is not for rows below 1e-13, nor r^3 mean(q s) below 1e-19.
        const S2 rs2 = s2(rs), ks2 = s2(-(rs * (rs * (sums[2] * inv_h)))), c2 = s2(gt * rx);
        const size_t out_at = static_cast<size_t>(row) * nvec + tid;
        uint32_t x[NV][4];
        S2 Gf[NV][4], td = s2(0.0f);                      // G times its factor
        const uint4* at = row_at(slot);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const float4 f0 = factors[2 * j * width + tid], f1 = factors[(2 * j + 1) * width + tid];
            const S2 f[4] = {s2(f0.x, f0.y), s2(f0.z, f0.w), s2(f1.x, f1.y), s2(f1.z, f1.w)};
            uint32_t ds[4], s[4], dy[4], out[4];
            take(at, 0, j, ds);
            if (X) take(at, 1, j, x[j]);
            take(at, PLANES - 2, j, s);
            take(at, PLANES - 1, j, dy);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const S2 q = s2_fma_bf16(dy[e], w[j][e], s2(0.0f));
                const S2 G = s2_fma(rs2, s2_fma(ks2, s2_bf16(s[e]), q), s2_bf16(ds[e]));
                sum_w[j][e] = s2_fma(rs2, s2_fma_bf16(dy[e], s[e], s2(0.0f)), sum_w[j][e]);
                Gf[j][e] = s2_mul(G, f[e]);
                if (X) {
                    const S2 xe = s2_bf16(x[j][e]);
                    sum_c[j][e] = s2_fma(s2_mul(G, xe), c2, sum_c[j][e]);
                    td = s2_fma(Gf[j][e], xe, td);
                }
                const S2 v = G;
                out[e] = pack_bf16x2(v.lo, v.hi);
            }
            if (tid + width * j < nvec) reinterpret_cast<uint4*>(p.d_residual)[out_at + width * j] = make_uint4(out[0], out[1], out[2], out[3]);
        }
        int next = slot + shape.groups;
        uint32_t next_parity = parity;
        if (next >= shape.slots) {
            next -= shape.slots;
            next_parity ^= 1;
        }
        tx = ts = tq = 0.0f;
        if (row + step < T) first_sums(next, next_parity);
        total(s2_sum(td), sums);
        // everybody in the group is through with the row: a later one takes its slot
        if (tid == 0) request(row + shape.slots * gridDim.x, slot);
        slot = next;
        parity = next_parity;
        if (!branch) continue;
        if (p.gate_kind == GATE_TOKEN && tid == 0) p.d_gate[row] = rx * sums[3];
        const S2 kx2 = s2(-(rx * (rx * (sums[3] * inv_h))));               // d_x likewise
        auto write_dx = [&](auto norm_of_x) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                uint32_t out[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const S2 v = s2_mul(c2, decltype(norm_of_x)::value ? s2_fma(kx2, s2_bf16(x[j][e]), Gf[j][e]) : Gf[j][e]);
                    out[e] = pack_bf16x2(v.lo, v.hi);
                }
                if (tid + width * j < nvec) reinterpret_cast<uint4*>(p.d_x)[out_at + width * j] = make_uint4(out[0], out[1], out[2], out[3]);
            }
        };
        // (without a norm of x its values are in no term of d_x: zero times an infinity would be one)
        if (post) write_dx(std::bool_constant<X>());
        else write_dx(std::false_type());
    }
    // The groups' sums, in their order, through the ring (nothing is on its way there any more).
    const bool column = post || p.gate_kind == GATE_CHANNEL;
    S2* const all = reinterpret_cast<S2*>(ring);             // [plane][half vector][group][thread] of two S2
    __syncthreads();
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = (2 * j + e / 2) * static_cast<int>(blockDim.x) + static_cast<int>(threadIdx.x);
            all[2 * i + e % 2] = sum_w[j][e];
            all[2 * (2 * NV * static_cast<int>(blockDim.x) + i) + e % 2] = sum_c[j][e];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * NV * width; i += blockDim.x) {
        const int part = i / width, t = i - part * width, plane = part / (2 * NV), half = part % (2 * NV);
        if (plane == 0 ? !norm : !column) continue;
        const int c = 2 * (t + width * (half / 2)) + half % 2;               // 4 columns
        if (4 * c >= p.H) continue;
        const float4* from = reinterpret_cast<const float4*>(all) + part * blockDim.x + t;
        float4 s = from[0];
        for (int g = 1; g < shape.groups; ++g) {
            const float4 v = from[g * width];
            s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
        }
        reinterpret_cast<float4*>(p.part + (static_cast<long long>(plane) * gridDim.x + blockIdx.x) * p.H)[c] = s;
    }
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

// Threads for NV vectors each: two, which halves what a row costs beside its columns (28 warps of one vector at 3584 channels 126 us,
// 14 of two 121), but one where two would leave lanes idle (up to 256 channels) or, with x, too few warps on an SM (above 4096
// channels one group is all that fits at 128 registers; 9001 x 5120: 107 us by 20 warps of one, 112 by 10 of two, 134 by two groups
// of 10 at 96 registers, which spill).  Without x 96 registers are enough for the second group there (9001 x 5120 85 -> 66 us; at
// 3584 and 6144 channels, where they would gain no group, 128 are faster, 88 -> 84 and 86 -> 81).  As many groups as the threads
// hold.  The ring: for one group all of shared memory; for two an odd number of slots, which the groups then take in turns (14 000 x
// 4096: six 119 us, five 113; 16 001 x 3584: seven 113, six 115, five 116); for more 164 KB, since rows that are asked for earlier
// only get in the way of the writes (20 000 x 2048: 87 us with 227 KB, 83 with 164, 86 with 140; 32 000 x 1536 104, 98, 102).
// (148 SMs: the number of CTAs and groups decides the order of the sums over tokens, so it does not follow the device.)
constexpr int BN_RING_MANY = 164 * 1024;
static BlockNormBwdShape bwd_shape(int64_t T, int H, bool x) {
    BlockNormBwdShape s;
    s.nv = H <= 256 || (x && H > 4096 && H <= 8 * BN_THREADS_WIDE) ? 1 : 2;
    s.group = (H / 8 + 32 * s.nv - 1) / (32 * s.nv) * 32;
    const bool two = s.group > BN_THREADS_MOST / 2 && s.group <= BN_THREADS_WIDE / 2;
    s.most = s.nv == 1 || (!x && two) ? BN_THREADS_WIDE : BN_THREADS_MOST;
    s.slot_bytes = (x ? 4 : 3) * 16 * s.nv * s.group;
    s.factor_bytes = 32 * s.nv * s.group;
    s.slots = std::min(BN_SLOTS, (227 * 1024 - BN_RING - s.factor_bytes) / s.slot_bytes);
    s.ctas = static_cast<int>(std::min<int64_t>(T, 148));
    const int64_t rows = (T + 147) / 148;                    // of a CTA
    s.groups = static_cast<int>(std::min<int64_t>(std::max(1, s.most / s.group), rows));
    while (s.groups > 1 && 2 * s.groups >= s.slots) --s.groups;
    if (s.groups > 2) s.slots = std::min(s.slots, BN_RING_MANY / s.slot_bytes);
    if (s.groups == 2) s.slots -= s.slots % 2 == 0;
    // (a short call's ring holds its rows; the groups' sums need 64 bytes a thread and vector of it at the end)
    const int sums = (64 * s.nv * s.groups * s.group + s.slot_bytes - 1) / s.slot_bytes;
    s.slots = static_cast<int>(std::min<int64_t>(s.slots, std::max<int64_t>({rows, sums, s.groups + 1})));
    s.smem = BN_RING + s.factor_bytes + static_cast<size_t>(s.slots) * s.slot_bytes;
    return s;
}
size_t block_norm_bwd_bytes(int64_t T, int H) { return static_cast<size_t>(bwd_shape(T, H, true).ctas) * 2 * H * sizeof(float); }

cudaError_t launch_block_norm(const BlockNormParams& p, cudaStream_t stream) {
    const int nv = (p.H / 8 + BN_THREADS - 1) / BN_THREADS;
    auto pick = [&](auto few) {
        constexpr bool FEW = decltype(few)::value;
        return p.H <= 256 ? block_norm_kernel<1, FEW, 4> : p.H <= 512 ? block_norm_kernel<1, FEW, 2> : nv <= 1 ? block_norm_kernel<1, FEW, 1>
             : nv <= 2 ? block_norm_kernel<2, FEW, 1> : nv <= 4 ? block_norm_kernel<4, FEW, 1> : block_norm_kernel<8, FEW, 1>;
    };
    const long long rows = p.H <= 256 ? 4 : p.H <= 512 ? 2 : 1;
    return launch_pdl(p.T <= BN_FEW_ROWS ? pick(std::true_type()) : pick(std::false_type()), dim3(static_cast<unsigned>((p.T + rows - 1) / rows)),
                      BN_THREADS, 0, stream, 1, p);
}

cudaError_t launch_block_norm_bwd(const BlockNormParams& p, cudaStream_t stream) {
    const bool x = p.post_weight || p.gate;
    const BlockNormBwdShape shape = bwd_shape(p.T, p.H, x);
    if (shape.ctas > 0) {
        static DeviceOnce configured;
        cudaError_t e = configured.run([&]() {
            cudaError_t r = cudaSuccess;
            auto allow = [&](auto kern) {
                if (r == cudaSuccess) r = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
            };
            allow(block_norm_bwd_kernel<2, BN_THREADS_MOST, true>);
            allow(block_norm_bwd_kernel<2, BN_THREADS_MOST, false>);
            allow(block_norm_bwd_kernel<2, BN_THREADS_WIDE, false>);
            allow(block_norm_bwd_kernel<1, BN_THREADS_WIDE, true>);
            allow(block_norm_bwd_kernel<1, BN_THREADS_WIDE, false>);
            return r;
        });
        if (e != cudaSuccess) return e;
        const bool wide = shape.most == BN_THREADS_WIDE;
        auto kern = shape.nv == 1 ? (x ? block_norm_bwd_kernel<1, BN_THREADS_WIDE, true> : block_norm_bwd_kernel<1, BN_THREADS_WIDE, false>)
                    : x           ? block_norm_bwd_kernel<2, BN_THREADS_MOST, true>
                    : wide        ? block_norm_bwd_kernel<2, BN_THREADS_WIDE, false>
                                  : block_norm_bwd_kernel<2, BN_THREADS_MOST, false>;
        e = launch_pdl(kern, dim3(shape.ctas), shape.group * shape.groups, shape.smem, stream, 1, p, shape);
        if (e != cudaSuccess) return e;
    }
    if (!p.d_weight && !p.d_post_weight && p.gate_kind != GATE_CHANNEL) return cudaSuccess;
    return launch_pdl(block_norm_fold_kernel, dim3((p.H + 127) / 128, 2), BN_FOLD_WARPS * 32, 0, stream, 1, p, shape.ctas);
}

}  // namespace tik
