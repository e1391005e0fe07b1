// AdamW over a list of tensors in one launch, moments in fp32 or in 8 bits.
//
//   g = clip * grad;  m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
//   p = (1 - lr weight_decay) p - lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps)
// with clip = max_norm / norm where a norm is given and exceeds max_norm (the factor that a clip of the gradients would write back
// to them), and nothing at all where the norm is not finite.  p is the fp32 master copy if there is one, which the weights are
// rounded from; else the weights.
//
// 8-bit moments: m, and the root of v, as e4m3 values in units of a power of two that 32 elements share: the smallest one with
// which the block's largest fits (448).  The root halves the range that the exponents have to cover, and a root that is not
// zero is never stored as zero: the next step divides by it.  Three bits behind the point are off by 2^-4 at most, which moves the step of
// an element by as much; but beta2 = 0.999 changes a root by 0.05 % a step, which rounding to the nearest would never let through.
// So such states are rounded stochastically where a seed is given (up with a probability that is the distance from the value
// below, from 16 bits of a hash of the element's place, the seed and the step), and so are bf16 weights without a master copy.
//
// HBM-bound: 12 bytes of bf16 weights, gradient and 8-bit moments to 28 with a master copy.  The list travels as a kernel parameter;
// chunks of 8192 elements on as many CTAs as the SMs hold.
#include <cuda_fp8.h>

#include <algorithm>
#include <cstdlib>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int ADAM_THREADS = 256;
constexpr int ADAM_CHUNK = 8192;
constexpr int ADAM_BLOCK = 32;                               // elements that share a scale

struct AdamEntry {
    const void* grad;
    void* param;
    float* master;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    long long n;
    long long place;             // of the first element among all of the call's
    unsigned first;              // chunk of the launch with which the tensor begins
    int flags;
};
constexpr int ADAM_PARAM_FP32 = 1, ADAM_GRAD_FP32 = 2;
template <int CAP>
struct AdamList {
    AdamEntry e[CAP];
    int n;
    unsigned chunks;
};
constexpr int ADAM_CAP_SMALL = 32, ADAM_CAP = 400;           // (parameters may take 32764 bytes)

struct AdamStep {                // what a step's numbers come to
    float decay, size, root;     // 1 - lr weight_decay, lr / (1 - beta1^t), (1 - beta2^t)^(-1/2)
    unsigned key;
};
__host__ __device__ inline uint32_t adam_mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x5BD1F3C5u;
    x ^= x >> 15;
    x *= 0x2F4A6E9Bu;
    return x ^ x >> 16;
}
__host__ __device__ inline AdamStep adam_step(const AdamParams& p, double lr, long long step) {
    const double t = step > 1 ? static_cast<double>(step) : 1.0;
    AdamStep s;
    s.decay = static_cast<float>(1.0 - lr * p.weight_decay);
    s.size = static_cast<float>(lr / -expm1(t * p.log_beta1));
    s.root = static_cast<float>(1.0 / sqrt(-expm1(t * p.log_beta2)));
    s.key = adam_mix(p.seed ^ static_cast<uint32_t>(step) * 0x9E3779B9u);
    return s;
}
__device__ __forceinline__ uint32_t adam_random(long long place, uint32_t key) {
    return adam_mix(static_cast<uint32_t>(place) * 0x632BE5ABu + key + static_cast<uint32_t>(place >> 32) * 0x85157AF5u);
}

// A thread's eight elements, in groups of W neighbours, a group of every thread after the other: W = 4 where a tensor lies at multiples of
// 16 bytes (a warp's access is one run of 128 bytes or more, whole sectors), else W = 1.  A block of 32 is a group of 32 / W lanes.
constexpr int ADAM_N = 8;
template <int W>
__device__ __forceinline__ long long adam_place(long long at, int i) { return at + i % W + (i / W) * (W * ADAM_THREADS); }

// What lies at or past n is 0.
template <int W>
__device__ __forceinline__ void adam_load(float (&x)[ADAM_N], const void* src, bool fp32, long long at, long long n) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W == 4 && e + W <= n) {
            if (fp32) {
                const float4 a = __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(src) + e));
                x[i] = a.x, x[i + 1 % W] = a.y, x[i + 2 % W] = a.z, x[i + 3 % W] = a.w;
            } else {
                const uint2 a = __ldcs(reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(src) + e));
                x[i] = __uint_as_float(a.x << 16), x[i + 1 % W] = __uint_as_float(a.x & 0xffff0000u);
                x[i + 2 % W] = __uint_as_float(a.y << 16), x[i + 3 % W] = __uint_as_float(a.y & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                x[i + j] = 0.0f;
                if (e + j < n) x[i + j] = fp32 ? static_cast<const float*>(src)[e + j] : __bfloat162float(static_cast<const __nv_bfloat16*>(src)[e + j]);
            }
        }
    }
}
template <int W>
__device__ __forceinline__ void adam_store(const float (&x)[ADAM_N], void* dst, bool fp32, long long at, long long n) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W == 4 && e + W <= n) {
            if (fp32)
                __stcs(reinterpret_cast<float4*>(static_cast<float*>(dst) + e), make_float4(x[i], x[i + 1 % W], x[i + 2 % W], x[i + 3 % W]));
            else
                __stcs(reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(dst) + e),
                       make_uint2(pack_bf16x2(x[i], x[i + 1 % W]), pack_bf16x2(x[i + 2 % W], x[i + 3 % W])));
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (e + j < n) {
                    if (fp32) static_cast<float*>(dst)[e + j] = x[i + j];
                    else static_cast<__nv_bfloat16*>(dst)[e + j] = __float2bfloat16_rn(x[i + j]);
                }
        }
    }
}

__device__ __forceinline__ float adam_scale_value(unsigned byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
// Stored 8-bit values times their block's scale
template <int W>
__device__ __forceinline__ void adam_load8(float (&x)[ADAM_N], const void* src, const uint8_t* scale, long long at, long long n) {
    const uint8_t* q = static_cast<const uint8_t*>(src);
    unsigned w[2] = {0u, 0u}, byte[ADAM_N / W];
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        byte[i / W] = e < n ? scale[e / ADAM_BLOCK] : 0u;
        if (W == 4 && e + W <= n) {
            w[i / 4] = __ldcs(reinterpret_cast<const unsigned*>(q + e));
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (e + j < n) w[i / 4] |= static_cast<unsigned>(q[e + j]) << (8 * ((i + j) & 3));
        }
    }
#pragma unroll
    for (int i = 0; i < ADAM_N; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[i / 4] >> (8 * (i & 2))), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        x[i] = f.x * adam_scale_value(byte[i / W]);
        x[i + 1] = f.y * adam_scale_value(byte[(i + 1) / W]);
    }
}
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }
// The power of two, as its biased exponent, with which a block whose largest magnitude is `a` fits 448 = 1.75 * 2^8.
__device__ __forceinline__ unsigned adam_scale_of(float a) {
    const unsigned b = __float_as_uint(a);
    const int e = static_cast<int>(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return static_cast<unsigned>(max(e, 0));
}
// y rounded to a value of e4m3 above or below it: |y| in units of the last place there, plus a number from [0, 1), cut off.
__device__ __forceinline__ float adam_round_e4m3(float y, unsigned random16) {
    const unsigned e = max(__float_as_uint(y) >> 23 & 0xffu, 121u);        // 2^-6: below it the places stay those of 2^-6
    const float per_place = __uint_as_float((257u - e) << 23), place = __uint_as_float((e - 3u) << 23);
    const float t = floorf(__fadd_rn(fabsf(y) * per_place, static_cast<float>(random16) * 0x1p-16f));
    return copysignf(t * place, y);
}
// Stores values and, from each block's first lane, its scale.  POSITIVE: the second moment's roots, of which none above 0 becomes 0.
template <int W, bool STOCHASTIC, bool POSITIVE>
__device__ __forceinline__ void adam_store8(const float (&x)[ADAM_N], const uint32_t (&random)[ADAM_N], void* dst, uint8_t* scale, long long at,
                                            long long n) {
    unsigned byte[ADAM_N / W], w[2] = {0u, 0u};
    float y[ADAM_N];
    bool plain = true;                                       // every value is finite, and 0 or in e4m3's normal range
#pragma unroll
    for (int k = 0; k < ADAM_N / W; ++k) {
        float a = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) a = max_or_nan(a, fabsf(x[W * k + j]));
        if (!finite(a)) {                                    // what is not finite does not count
            plain = false;
            a = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (finite(x[W * k + j])) a = fmaxf(a, fabsf(x[W * k + j]));
        }
#pragma unroll
        for (int off = 1; off < ADAM_BLOCK / W; off <<= 1) a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, off));
        byte[k] = adam_scale_of(a);
    }
#pragma unroll
    for (int i = 0; i < ADAM_N; ++i) {
        y[i] = x[i] * __uint_as_float((254u - byte[i / W]) << 23);
        plain = plain && (__float_as_uint(fabsf(y[i])) - 1u >= 0x3c800000u - 1u);
    }
    if (plain) {
        if (STOCHASTIC)
#pragma unroll
            for (int i = 0; i < ADAM_N; ++i) {
                // 20 of 23 places are cut off: the number is added below them.  (The same as below in the normal range.)
                const unsigned r = POSITIVE ? random[i] >> 12 & 0xffff0u : (random[i] & 0xffffu) << 4;
                y[i] = __uint_as_float((__float_as_uint(y[i]) + r) & 0xfff00000u);
            }
#pragma unroll
        for (int i = 0; i < ADAM_N; i += 2)
            w[i / 4] |= static_cast<unsigned>(__nv_cvt_float2_to_fp8x2(make_float2(y[i], y[i + 1]), __NV_SATFINITE, __NV_E4M3)) << (8 * (i & 2));
    } else {
#pragma unroll
        for (int i = 0; i < ADAM_N; ++i) {
            float f = y[i];
            if (STOCHASTIC) f = adam_round_e4m3(f, POSITIVE ? random[i] >> 16 : random[i] & 0xffffu);
            if (!finite(x[i])) f = CUDART_NAN_F;
            unsigned q = __nv_cvt_float_to_fp8(f, __NV_SATFINITE, __NV_E4M3);
            if (POSITIVE && q == 0u && x[i] > 0.0f) q = 1u;
            w[i / 4] |= q << (8 * (i & 3));
        }
    }
    uint8_t* to = static_cast<uint8_t*>(dst);
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W == 4 && e + W <= n) {
            __stcs(reinterpret_cast<unsigned*>(to + e), w[i / 4]);
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (e + j < n) to[e + j] = static_cast<uint8_t>(w[i / 4] >> (8 * ((i + j) & 3)));
        }
        if (e < n && e % ADAM_BLOCK == 0) scale[e / ADAM_BLOCK] = static_cast<uint8_t>(byte[i / W]);
    }
}

// Eight elements of each of a warp's lanes.
template <int W, bool STATE8, bool STOCHASTIC>
__device__ __forceinline__ void adam_elements(const AdamEntry& e, long long at, const AdamParams& p, const AdamStep& s, float clip) {
    const long long n = e.n;
    float x[ADAM_N], g[ADAM_N], m[ADAM_N], v[ADAM_N];
    const bool p32 = e.flags & ADAM_PARAM_FP32;
    adam_load<W>(g, e.grad, e.flags & ADAM_GRAD_FP32, at, n);
    if (STATE8) {
        adam_load8<W>(m, e.m, e.m_scale, at, n);
        adam_load8<W>(v, e.v, e.v_scale, at, n);
    } else {
        adam_load<W>(m, e.m, true, at, n);
        adam_load<W>(v, e.v, true, at, n);
    }
    adam_load<W>(x, e.master ? static_cast<const void*>(e.master) : e.param, e.master ? true : p32, at, n);
    uint32_t random[ADAM_N];
    const float to_m = p.one_minus_beta1 * clip, to_v = p.one_minus_beta2 * clip * clip;
#pragma unroll
    for (int i = 0; i < ADAM_N; ++i) {
        if (STATE8) v[i] = v[i] * v[i];
        m[i] = fmaf(p.beta1, m[i], to_m * g[i]);
        v[i] = fmaf(p.beta2, v[i], to_v * g[i] * g[i]);
        float root;
        asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v[i]));
        float inverse;                                       // (root <= 2^64 and eps >= 2^-126: far inside the range)
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(fmaf(root, s.root, p.eps)));
        x[i] = fmaf(s.decay, x[i], -s.size * m[i] * inverse);
        if (STATE8) v[i] = root;
        random[i] = STOCHASTIC ? adam_random(e.place + adam_place<W>(at, i), s.key) : 0u;
    }
    if (STATE8) {
        adam_store8<W, STOCHASTIC, false>(m, random, e.m, e.m_scale, at, n);
        adam_store8<W, STOCHASTIC, true>(v, random, e.v, e.v_scale, at, n);
    } else {
        adam_store<W>(m, e.m, true, at, n);
        adam_store<W>(v, e.v, true, at, n);
    }
    if (e.master) adam_store<W>(x, e.master, true, at, n);
    if (STOCHASTIC && !e.master && !p32) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < ADAM_N; ++i) top = max_or_nan(top, fabsf(x[i]));
        const bool all = finite(top);
#pragma unroll
        for (int i = 0; i < ADAM_N; ++i)
            if (all || finite(x[i])) x[i] = __uint_as_float((__float_as_uint(x[i]) + (adam_mix(random[i]) & 0xffffu)) & 0xffff0000u);
    }
    adam_store<W>(x, e.param, p32, at, n);
}

// CTAs that an SM holds, and the grid has for it: with more of them than it holds, a second wave of a few would have the chip to itself.
constexpr int adam_ctas_per_sm(int w, bool state8) { return state8 ? (w == 4 ? 3 : 2) : 4; }
template <int CAP, int W, bool STATE8, bool STOCHASTIC>
__global__ void __launch_bounds__(ADAM_THREADS, adam_ctas_per_sm(W, STATE8)) adam_kernel(const __grid_constant__ AdamList<CAP> l, const __grid_constant__ AdamParams p,
                                                            const AdamStep given) {
    __shared__ AdamStep from_device;
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    float clip = 1.0f;
    if (p.norm) {
        const float norm = *p.norm;
        if (!(norm <= 3.402823466e38f)) return;
        if (norm > p.max_norm) clip = __fdiv_rn(p.max_norm, norm);
    }
    AdamStep s = given;
    if (p.lr_device || p.step_device) {
        if (tid == 0) from_device = adam_step(p, p.lr_device ? static_cast<double>(*p.lr_device) : p.lr, p.step_device ? *p.step_device : p.step);
        __syncthreads();
        s = from_device;
    }
    int at = 0;                                              // tensor of the CTA's last chunk
    for (unsigned c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        int lo = l.e[at].first <= c ? at : 0, hi = l.n;      // the last tensor with first <= c
        if (lo + 1 < hi && l.e[lo + 1].first > c) hi = lo + 1;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (l.e[mid].first <= c) lo = mid;
            else hi = mid;
        }
        at = lo;
        const AdamEntry& e = l.e[lo];
        const long long base = static_cast<long long>(c - e.first) * ADAM_CHUNK;
        // a trip of a CTA is eight elements of every thread
#pragma unroll 1
        for (int i = 0; i < ADAM_CHUNK && base + i < e.n; i += ADAM_N * ADAM_THREADS)
            adam_elements<W, STATE8, STOCHASTIC>(e, base + i + W * tid, p, s, clip);
    }
}

template <int W, bool STATE8, bool STOCHASTIC>
static cudaError_t launch_adam_list(const AdamList<ADAM_CAP>& l, const AdamParams& p, const AdamStep& s, cudaStream_t stream) {
    const dim3 ctas(std::min<unsigned>(l.chunks, static_cast<unsigned>(p.sm_count * adam_ctas_per_sm(W, STATE8))));
    if (l.n > ADAM_CAP_SMALL) return launch_pdl(adam_kernel<ADAM_CAP, W, STATE8, STOCHASTIC>, ctas, ADAM_THREADS, 0, stream, 1, l, p, s);
    AdamList<ADAM_CAP_SMALL> few;
    std::copy(l.e, l.e + l.n, few.e);
    few.n = l.n;
    few.chunks = l.chunks;
    return launch_pdl(adam_kernel<ADAM_CAP_SMALL, W, STATE8, STOCHASTIC>, ctas, ADAM_THREADS, 0, stream, 1, few, p, s);
}
template <int W>
static cudaError_t launch_adam_lists(const AdamTensors& t, const AdamParams& p, bool state8, bool stochastic, const AdamStep& s, cudaStream_t stream) {
    long long place = 0;
    for (int at = 0; at < t.n;) {
        AdamList<ADAM_CAP> l;
        l.n = 0;
        long long chunks = 0;
        for (; at < t.n && l.n < ADAM_CAP; ++at) {
            const long long n = t.numel[at];
            if (n == 0) continue;
            AdamEntry e;
            e.grad = t.grads[at];
            e.param = t.params[at];
            e.master = t.master ? t.master[at] : nullptr;
            e.m = t.m[at];
            e.v = t.v[at];
            e.m_scale = state8 ? t.m_scale[at] : nullptr;
            e.v_scale = state8 ? t.v_scale[at] : nullptr;
            e.n = n;
            e.place = place;
            e.first = static_cast<unsigned>(chunks);
            e.flags = (t.param_dtypes[at] == 1 ? ADAM_PARAM_FP32 : 0) | (t.grad_dtypes[at] == 1 ? ADAM_GRAD_FP32 : 0);
            place += n;
            auto bits = [](const void* q) { return reinterpret_cast<uintptr_t>(q); };
            const uintptr_t state = bits(e.m) | bits(e.v);
            const bool vectors = ((bits(e.grad) | bits(e.param) | bits(e.master)) & 15) == 0 && (state & (state8 ? 3 : 15)) == 0;
            if (vectors != (W == 4)) continue;
            l.e[l.n++] = e;
            chunks += (n + ADAM_CHUNK - 1) / ADAM_CHUNK;
        }
        l.chunks = static_cast<unsigned>(chunks);
        if (l.n == 0) continue;
        const cudaError_t err = state8 ? (stochastic ? launch_adam_list<W, true, true>(l, p, s, stream) : launch_adam_list<W, true, false>(l, p, s, stream))
                                       : (stochastic ? launch_adam_list<W, false, true>(l, p, s, stream) : launch_adam_list<W, false, false>(l, p, s, stream));
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

// Tensors that lie at odd addresses take launches of their own, behind the others'.
cudaError_t launch_adamw(const AdamTensors& t, const AdamParams& p, bool state8, bool stochastic, cudaStream_t stream) {
    const AdamStep s = adam_step(p, p.lr, p.step);
    const cudaError_t e = launch_adam_lists<4>(t, p, state8, stochastic, s, stream);
    return e == cudaSuccess ? launch_adam_lists<1>(t, p, state8, stochastic, s, stream) : e;
}

bool adamw_ranges_overlap(const AdamTensors& t, const AdamParams& p, bool state8, bool* no_memory) {
    struct Range {
        uintptr_t from, to;
        bool written;
    };
    *no_memory = false;
    if (t.n <= 0) return false;
    Range* const r = static_cast<Range*>(malloc((7ull * t.n + 3ull) * sizeof(Range)));
    if (!r) return *no_memory = true;
    int n = 0;
    auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
    // one list after the other: mostly ascending already, as views of a flat buffer
    auto add = [&](auto&& address, auto&& bytes, bool written) {
        const int begin = n;
        for (int i = 0; i < t.n; ++i)
            if (t.numel[i] > 0 && address(i)) {
                const uintptr_t a = reinterpret_cast<uintptr_t>(address(i));
                r[n++] = {a, a + static_cast<uintptr_t>(bytes(i)), written};
            }
        if (!std::is_sorted(r + begin, r + n, before)) std::sort(r + begin, r + n, before);
        if (begin > 0 && n > begin && !before(r[begin - 1], r[begin])) std::inplace_merge(r, r + begin, r + n, before);
    };
    const int state = state8 ? 1 : 4;
    add([&](int i) { return t.params[i]; }, [&](int i) { return t.numel[i] * (t.param_dtypes[i] == 1 ? 4 : 2); }, true);
    if (t.master) add([&](int i) { return t.master[i]; }, [&](int i) { return t.numel[i] * 4; }, true);
    add([&](int i) { return t.m[i]; }, [&](int i) { return t.numel[i] * state; }, true);
    add([&](int i) { return t.v[i]; }, [&](int i) { return t.numel[i] * state; }, true);
    if (state8) {
        add([&](int i) { return t.m_scale[i]; }, [&](int i) { return (t.numel[i] + ADAM_BLOCK - 1) / ADAM_BLOCK; }, true);
        add([&](int i) { return t.v_scale[i]; }, [&](int i) { return (t.numel[i] + ADAM_BLOCK - 1) / ADAM_BLOCK; }, true);
    }
    add([&](int i) { return t.grads[i]; }, [&](int i) { return t.numel[i] * (t.grad_dtypes[i] == 1 ? 4 : 2); }, false);
    for (const void* one : {static_cast<const void*>(p.norm), static_cast<const void*>(p.lr_device), static_cast<const void*>(p.step_device)})
        if (one) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(one);
            const Range x = {a, a + 4, false};
            Range* at = std::upper_bound(r, r + n, x, before);
            std::copy_backward(at, r + n, r + n + 1);
            *at = x;
            ++n;
        }
    // ascending by their beginnings: one meets another if it begins before the furthest end of those ahead of it; two that are read may
    bool overlap = false;
    uintptr_t end_written = 0, end_any = 0;
    for (int i = 0; i < n && !overlap; ++i) {
        overlap = r[i].from < (r[i].written ? end_any : end_written);
        end_any = std::max(end_any, r[i].to);
        if (r[i].written) end_written = std::max(end_written, r[i].to);
    }
    free(r);
    return overlap;
}

}  // namespace tik
