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
// a ring of bulk copies in each of as many CTAs as the SMs hold keeps 150 KB and more an SM on their way.
#include <cuda_fp8.h>

#include <algorithm>
#include <cstdlib>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int ADAM_THREADS = 256;
constexpr int ADAM_BLOCK = 32;                               // elements that share a scale

struct AdamEntry {
    const void* grad;
    void* param;
    float* master;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    long long n;
    long long place;             // of the first element among all of the call's
    unsigned first;              // trip of the launch with which the tensor begins
    int flags;
};
constexpr int ADAM_PARAM_FP32 = 1, ADAM_GRAD_FP32 = 2;
template <int CAP>
struct AdamList {
    AdamEntry e[CAP];
    int n;
    unsigned trips;
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

// A thread's eight elements, in groups of W neighbours, a group of every thread after the other.  Where a tensor lies at multiples of 16
// bytes W is 4, so that a warp's access is one run of whole sectors, and with 8-bit moments 8: a block of 32, held by 32 / W lanes, then takes two
// shuffles for a maximum and one thread's scale goes for all its elements.  Else W is 1.
constexpr int ADAM_N = 8;
template <int W>
__device__ __forceinline__ long long adam_place(long long at, int i) { return at + i % W + (i / W) * (W * ADAM_THREADS); }

// From global memory, where what lies at or past n is 0, or from a stage of the ring, which is whole.
template <int W, bool STAGED>
__device__ __forceinline__ void adam_load(float (&x)[ADAM_N], const void* src, bool fp32, long long at, long long n) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W > 1 && (STAGED || e + W <= n)) {
            if (fp32) {
#pragma unroll
                for (int j = 0; j < W; j += 4) {
                    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(src) + e + j);
                    const float4 a = STAGED ? *p : __ldcs(p);
                    x[i + j] = a.x, x[i + j + 1 % W] = a.y, x[i + j + 2 % W] = a.z, x[i + j + 3 % W] = a.w;
                }
            } else {
                const uint2* p = reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(src) + e);
                uint4 a = make_uint4(0, 0, 0, 0);
                if (W == 8) {
                    a = STAGED ? *reinterpret_cast<const uint4*>(p) : __ldcs(reinterpret_cast<const uint4*>(p));
                } else {
                    const uint2 b = STAGED ? *p : __ldcs(p);
                    a.x = b.x;
                    a.y = b.y;
                }
                const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < W; ++j) x[i + j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                x[i + j] = 0.0f;
                if (STAGED || e + j < n) x[i + j] = fp32 ? static_cast<const float*>(src)[e + j] : __bfloat162float(static_cast<const __nv_bfloat16*>(src)[e + j]);
            }
        }
    }
}
// W bf16 from their words
template <int W>
__device__ __forceinline__ void adam_store_words(__nv_bfloat16* to, const unsigned (&w)[4]) {
    if (W == 8) __stcs(reinterpret_cast<uint4*>(to), make_uint4(w[0], w[1], w[2], w[3]));
    else __stcs(reinterpret_cast<uint2*>(to), make_uint2(w[0], w[1]));
}
template <int W, bool WHOLE>
__device__ __forceinline__ void adam_store(const float (&x)[ADAM_N], void* dst, bool fp32, long long at, long long n) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W > 1 && (WHOLE || e + W <= n)) {
            if (fp32) {
#pragma unroll
                for (int j = 0; j < W; j += 4)
                    __stcs(reinterpret_cast<float4*>(static_cast<float*>(dst) + e + j), make_float4(x[i + j], x[i + j + 1 % W], x[i + j + 2 % W], x[i + j + 3 % W]));
            } else {
                unsigned w[4] = {};
#pragma unroll
                for (int j = 0; j < W; j += 2) w[j / 2] = pack_bf16x2(x[i + j], x[i + j + 1 % W]);
                adam_store_words<W>(static_cast<__nv_bfloat16*>(dst) + e, w);
            }
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (WHOLE || e + j < n) {
                    if (fp32) static_cast<float*>(dst)[e + j] = x[i + j];
                    else static_cast<__nv_bfloat16*>(dst)[e + j] = __float2bfloat16_rn(x[i + j]);
                }
        }
    }
}

// The upper halves of fp32 values as bf16
template <int W, bool WHOLE>
__device__ __forceinline__ void adam_store_upper(const float (&x)[ADAM_N], void* dst, long long at, long long n) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W > 1 && (WHOLE || e + W <= n)) {
            unsigned w[4] = {};
#pragma unroll
            for (int j = 0; j < W; j += 2) w[j / 2] = __byte_perm(__float_as_uint(x[i + j]), __float_as_uint(x[i + j + 1 % W]), 0x7632);
            adam_store_words<W>(static_cast<__nv_bfloat16*>(dst) + e, w);
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (WHOLE || e + j < n) static_cast<unsigned short*>(dst)[e + j] = static_cast<unsigned short>(__float_as_uint(x[i + j]) >> 16);
        }
    }
}

__device__ __forceinline__ float adam_scale_value(unsigned byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
// The scales' bytes of a thread's groups
template <int W, bool WHOLE>
__device__ __forceinline__ void adam_load_scales(unsigned (&byte)[ADAM_N / W], const uint8_t* scale, long long at, long long n) {
    const uint8_t* p = scale + (at >> 5);
#pragma unroll
    for (int k = 0; k < ADAM_N / W; ++k)                     // (a group of every thread is ADAM_THREADS W elements)
        byte[k] = WHOLE || adam_place<W>(at, W * k) < n ? p[k * (ADAM_THREADS * W / ADAM_BLOCK)] : 0u;
}
// Stored 8-bit values times their block's scale
template <int W, bool STAGED>
__device__ __forceinline__ void adam_load8(float (&x)[ADAM_N], const void* src, const unsigned (&byte)[ADAM_N / W], long long at, long long n) {
    const uint8_t* q = static_cast<const uint8_t*>(src);
    unsigned w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long e = adam_place<W>(at, i);
        if (W == 8 && (STAGED || e + W <= n)) {
            const uint2* p = reinterpret_cast<const uint2*>(q + e);
            const uint2 a = STAGED ? *p : __ldcs(p);
            w[0] = a.x;
            w[1] = a.y;
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (STAGED || e + j < n) w[(i + j) / 4] |= static_cast<unsigned>(q[e + j]) << (8 * ((i + j) & 3));
        }
    }
#pragma unroll
    for (int i = 0; i < ADAM_N; i += 2) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[i / 4] >> (8 * (i & 2))), __NV_E4M3);
        const float2 f = __half22float2(__half2(h));
        f2_get(f2_mul(f2(f.x, f.y), f2(adam_scale_value(byte[i / W]), adam_scale_value(byte[(i + 1) / W]))), x[i], x[i + 1]);
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
// Whether one of four e4m3 values is at most the least normal one, unless what they stand for, `x`, is all 0.
__device__ __forceinline__ bool adam_small(unsigned w, const float* x) {
    if (((((w & 0x7f7f7f7fu) | 0x80808080u) - 0x09090909u) & 0x80808080u) == 0x80808080u) return false;
    return w != 0u || x[0] != 0.0f || x[1] != 0.0f || x[2] != 0.0f || x[3] != 0.0f;
}
// Stores values and, from each block's first lane, its scale.  POSITIVE: the second moment's roots, of which none above 0 becomes 0.
template <int W, bool STOCHASTIC, bool POSITIVE, bool WHOLE>
__device__ __forceinline__ void adam_store8(const float (&x)[ADAM_N], const uint32_t (&random)[ADAM_N], void* dst, uint8_t* scale, long long at,
                                            long long n) {
    unsigned byte[ADAM_N / W], w[2] = {0u, 0u};
    float y[ADAM_N];
    bool rare = false;
#pragma unroll
    for (int k = 0; k < ADAM_N / W; ++k) {
        float a = 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) a = max_or_nan(a, fabsf(x[W * k + j]));
        if (!finite(a)) {                                    // what is not finite does not count
            rare = true;
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
    for (int i = 0; i < ADAM_N; i += 2)
        f2_get(f2_mul(f2(x[i], x[i + 1]), f2(__uint_as_float((254u - byte[i / W]) << 23), __uint_as_float((254u - byte[(i + 1) / W]) << 23))), y[i], y[i + 1]);
#pragma unroll
    for (int i = 0; i < ADAM_N; i += 2) {
        float z[2] = {y[i], y[i + 1]};
        if (STOCHASTIC)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // in the normal range 20 of 23 places are cut off, and the number is added below them
                const unsigned r = POSITIVE ? random[i + j] >> 16 : random[i + j] & 0xffffu;
                z[j] = __uint_as_float((__float_as_uint(y[i + j]) + 16u * r) & 0xfff00000u);
            }
        w[i / 4] |= static_cast<unsigned>(__nv_cvt_float2_to_fp8x2(make_float2(z[0], z[1]), __NV_SATFINITE, __NV_E4M3)) << (8 * (i & 2));
    }
    // Subnormal values, whose places do not follow their exponents, and zeros that may not be: once more, one by one.
    if (STOCHASTIC || POSITIVE) rare = rare || adam_small(w[0], x) || adam_small(w[1], x + 4);
    if (rare) {
        w[0] = w[1] = 0u;
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
        if (W == 8 && (WHOLE || e + W <= n)) {
            __stcs(reinterpret_cast<uint2*>(to + e), make_uint2(w[0], w[1]));
        } else {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (WHOLE || e + j < n) to[e + j] = static_cast<uint8_t>(w[(i + j) / 4] >> (8 * ((i + j) & 3)));
        }
    }
    uint8_t* s = scale + (at >> 5);
#pragma unroll
    for (int k = 0; k < ADAM_N / W; ++k)                     // (trips begin at multiples of 32)
        if ((static_cast<unsigned>(at) & (ADAM_BLOCK - 1)) == 0u && (WHOLE || adam_place<W>(at, W * k) < n))
            s[k * (ADAM_THREADS * W / ADAM_BLOCK)] = static_cast<uint8_t>(byte[k]);
}

// Where a trip's inputs are: the tensor's own arrays, or a stage of the ring whose first elements are the trip's.
struct AdamInputs {
    const void *grad, *weight, *m, *v;
};
// Random numbers of W neighbours: the places differ in their low words alone unless those wrap.
template <int W>
__device__ __forceinline__ void adam_randoms(uint32_t (&random)[ADAM_N], long long place, uint32_t key) {
#pragma unroll
    for (int i = 0; i < ADAM_N; i += W) {
        const long long first = adam_place<W>(place, i);
        const uint32_t low = static_cast<uint32_t>(first), x = low * 0x632BE5ABu + key + static_cast<uint32_t>(first >> 32) * 0x85157AF5u;
#pragma unroll
        for (int j = 0; j < W; ++j) random[i + j] = adam_mix(x + static_cast<uint32_t>(j) * 0x632BE5ABu);
        if (W > 1 && low > 0xffffffffu - W)
#pragma unroll
            for (int j = 1; j < W; ++j) random[i + j] = adam_random(first + j, key);
    }
}
// The approximate root and reciprocal are off by 2^-23 at most, twice what the rounded ones are, for an instruction each in place of a dozen; in
// 8 bits a value goes to another neighbour for it once in 2^19.  Subnormal v count as 0 where issue slots are what bounds the kernel.
template <bool STATE8>
__device__ __forceinline__ void adam_root(float& root, float v) {
    if (STATE8) asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v));
    else asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(v));
}
// Eight elements of each of a warp's lanes: at `at` of the tensor, and `in` of the inputs.
template <int W, bool STATE8, bool STOCHASTIC, bool STAGED>
__device__ __forceinline__ void adam_elements(const AdamEntry& e, long long at, const AdamInputs& src, long long in, const unsigned (&m_byte)[ADAM_N / W],
                                              const unsigned (&v_byte)[ADAM_N / W], const AdamParams& p, const AdamStep& s, float clip) {
    const long long n = e.n;
    float x[ADAM_N], g[ADAM_N], m[ADAM_N], v[ADAM_N];
    const bool p32 = e.flags & ADAM_PARAM_FP32;
    adam_load<W, STAGED>(g, src.grad, e.flags & ADAM_GRAD_FP32, in, n);
    if (STATE8) {
        adam_load8<W, STAGED>(m, src.m, m_byte, in, n);
        adam_load8<W, STAGED>(v, src.v, v_byte, in, n);
    } else {
        adam_load<W, STAGED>(m, src.m, true, in, n);
        adam_load<W, STAGED>(v, src.v, true, in, n);
    }
    adam_load<W, STAGED>(x, src.weight, e.master || p32, in, n);
    uint32_t random[ADAM_N] = {};
    if (STOCHASTIC) adam_randoms<W>(random, e.place + at, s.key);
    const F2 clip2 = f2(clip), to_m = f2(p.one_minus_beta1), to_v = f2(p.one_minus_beta2), beta1 = f2(p.beta1), beta2 = f2(p.beta2);
    const F2 decay = f2(s.decay), size = f2(-s.size), root2 = f2(s.root), eps = f2(p.eps);
#pragma unroll
    for (int i = 0; i < ADAM_N; i += 2) {
        // (clipped before it is squared: the square of a small clip has no digits in fp32, that of a clipped gradient has)
        const F2 g2 = f2_mul(clip2, f2(g[i], g[i + 1])), v1 = f2(v[i], v[i + 1]);
        const F2 m2 = f2_fma(beta1, f2(m[i], m[i + 1]), f2_mul(to_m, g2));
        const F2 v2 = f2_fma(beta2, STATE8 ? f2_mul(v1, v1) : v1, f2_mul(f2_mul(to_v, g2), g2));
        f2_get(m2, m[i], m[i + 1]);
        f2_get(v2, v[i], v[i + 1]);
        float root[2], inverse[2];
        adam_root<STATE8>(root[0], v[i]);
        adam_root<STATE8>(root[1], v[i + 1]);
        f2_get(f2_fma(f2(root[0], root[1]), root2, eps), inverse[0], inverse[1]);
        // (root <= 2^64 and eps >= 2^-126: far inside the range)
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(inverse[0]));
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(inverse[1]));
        f2_get(f2_fma(decay, f2(x[i], x[i + 1]), f2_mul(f2_mul(size, m2), f2(inverse[0], inverse[1]))), x[i], x[i + 1]);
        if (STATE8) v[i] = root[0], v[i + 1] = root[1];
    }
    if (STATE8) {
        adam_store8<W, STOCHASTIC, false, STAGED>(m, random, e.m, e.m_scale, at, n);
        adam_store8<W, STOCHASTIC, true, STAGED>(v, random, e.v, e.v_scale, at, n);
    } else {
        adam_store<W, STAGED>(m, e.m, true, at, n);
        adam_store<W, STAGED>(v, e.v, true, at, n);
    }
    if (e.master) adam_store<W, STAGED>(x, e.master, true, at, n);
    if (STOCHASTIC && !e.master && !p32) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < ADAM_N; ++i) top = max_or_nan(top, fabsf(x[i]));
        if (finite(top)) {
#pragma unroll
            for (int i = 0; i < ADAM_N; ++i) x[i] = __uint_as_float(__float_as_uint(x[i]) + (adam_mix(random[i]) & 0xffffu));
            adam_store_upper<W, STAGED>(x, e.param, at, n);
            return;
        }
#pragma unroll
        for (int i = 0; i < ADAM_N; ++i)
            if (finite(x[i])) x[i] = __uint_as_float((__float_as_uint(x[i]) + (adam_mix(random[i]) & 0xffffu)) & 0xffff0000u);
    }
    adam_store<W, STAGED>(x, e.param, p32, at, n);
}

// A trip is eight elements of every thread, of one tensor, sixteen with 8-bit moments (whose stages are small).  A CTA's trips come through a ring of stages that one
// thread fills by bulk copies: loads into registers kept too few bytes in flight (466 M elements with 8-bit moments 2435 us).  Bulk
// copies want multiples of 16 bytes: an array that lies otherwise is copied from the 16 bytes around its ends, which are the
// tensor's own unless the trip is its first or last; those trips, and ones that are not whole, are read without a stage.
__host__ __device__ constexpr int adam_rounds(bool state8) { return state8 ? 2 : 1; }          // of eight elements of every thread
__host__ __device__ constexpr int adam_trip(bool state8) { return ADAM_N * ADAM_THREADS * adam_rounds(state8); }
constexpr int ADAM_STAGES = 8;                               // at most
struct AdamRing {
    int stages, stage_bytes;
    int weight_at, m_at, v_at;                               // of a stage; the gradient is at 0
};
struct AdamTrip {
    long long base;
    int entry;                                               // -1: the CTA's last trip is over
    int staged;
};
__device__ __forceinline__ unsigned adam_skew(const void* array, long long bytes) {
    return static_cast<unsigned>((reinterpret_cast<uintptr_t>(array) + bytes) & 15u);
}
// Copies from byte `from` of an array, less what it lies past a multiple of 16, `all` bytes.
__device__ __forceinline__ void adam_fetch(uint32_t dst, const void* array, long long from, unsigned all, uint32_t bar) {
    bulk_load(dst, static_cast<const char*>(array) + from - adam_skew(array, from), static_cast<int>(all), bar);
}

// CTAs that an SM holds, and the grid has for it: with more of them than it holds, a second wave of a few would have the chip to itself.
constexpr int adam_ctas_per_sm(int w, bool state8) { return state8 ? (w == 1 ? 2 : 4) : 3; }
template <int CAP, int W, bool STATE8, bool STOCHASTIC>
__global__ void __launch_bounds__(ADAM_THREADS, adam_ctas_per_sm(W, STATE8)) adam_kernel(const __grid_constant__ AdamList<CAP> l, const __grid_constant__ AdamParams p,
                                                                                         const AdamStep given, const AdamRing ring) {
    constexpr int ROUNDS = adam_rounds(STATE8), TRIP = adam_trip(STATE8);
    extern __shared__ __align__(128) char adam_smem[];
    __shared__ AdamStep from_device;
    __shared__ AdamTrip trips[ADAM_STAGES];
    __shared__ __align__(8) unsigned long long bars[ADAM_STAGES];
    __shared__ int left[ADAM_STAGES];                        // warps that are done with a stage's trip
    __shared__ int abort_word;
    const int tid = threadIdx.x;
    const uint32_t full = smem_u32(bars), stage0 = smem_u32(adam_smem);
    if (tid == 0) {
        for (int i = 0; i < ring.stages; ++i) {
            mbar_init(full + 8 * i, 1);
            left[i] = 0;
        }
        fence_barrier_init();
        abort_word = 0;
    }
    pdl_wait();
    pdl_launch_dependents();
    float clip = 1.0f;
    if (p.norm) {
        const float norm = *p.norm;
        if (!(norm <= 3.402823466e38f)) return;
        if (norm > p.max_norm) clip = __fdiv_rn(p.max_norm, norm);
    }
    if ((p.lr_device || p.step_device) && tid == 0)
        from_device = adam_step(p, p.lr_device ? static_cast<double>(*p.lr_device) : p.lr, p.step_device ? *p.step_device : p.step);
    __syncthreads();
    const AdamStep s = p.lr_device || p.step_device ? from_device : given;

    auto fill = [&](int i, int entry) {                      // trip i of this CTA; entry: tensor of an earlier one
        const int stage = i % ring.stages;
        const unsigned c = blockIdx.x + static_cast<unsigned>(i) * gridDim.x;
        const uint32_t bar = full + 8 * stage;
        AdamTrip t = {0, -1, 0};
        if (c < l.trips) {
            int lo = entry, hi = l.n;                        // the last tensor with first <= c
            if (lo + 1 < hi && l.e[lo + 1].first > c) hi = lo + 1;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (l.e[mid].first <= c) lo = mid;
                else hi = mid;
            }
            const AdamEntry& e = l.e[lo];
            t.entry = lo;
            t.base = static_cast<long long>(c - e.first) * TRIP;
            t.staged = W > 1 ? t.base + TRIP <= e.n : t.base > 0 && t.base + TRIP + 16 <= e.n;
        }
        trips[stage] = t;
        if (!t.staged) {
            mbar_arrive(bar);
            return;
        }
        const AdamEntry& e = l.e[t.entry];
        const uint32_t dst = stage0 + stage * ring.stage_bytes;
        const int g = e.flags & ADAM_GRAD_FP32 ? 4 : 2, w = e.master || (e.flags & ADAM_PARAM_FP32) ? 4 : 2, st = STATE8 ? 1 : 4;
        const void* weight = e.master ? static_cast<const void*>(e.master) : e.param;
        auto size = [&](const void* a, int k) { return (adam_skew(a, t.base * k) + static_cast<unsigned>(TRIP * k) + 15u) & ~15u; };
        mbar_expect_tx(bar, size(e.grad, g) + size(weight, w) + size(e.m, st) + size(e.v, st));
        adam_fetch(dst, e.grad, t.base * g, size(e.grad, g), bar);
        adam_fetch(dst + ring.weight_at, weight, t.base * w, size(weight, w), bar);
        adam_fetch(dst + ring.m_at, e.m, t.base * st, size(e.m, st), bar);
        adam_fetch(dst + ring.v_at, e.v, t.base * st, size(e.v, st), bar);
    };
    if (tid == 0)
        for (int i = 0; i < ring.stages; ++i) fill(i, 0);

    for (int i = 0;; ++i) {
        const int stage = i % ring.stages, use = i / ring.stages;
        mbar_wait(full + 8 * stage, use & 1, &abort_word, p.dev_status);
        if (*static_cast<volatile int*>(&abort_word)) break;
        const AdamTrip t = trips[stage];
        if (t.entry < 0) break;
        const AdamEntry& e = l.e[t.entry];
        const long long at = t.base + W * tid;
        constexpr int ROUND = ADAM_N * ADAM_THREADS;
        unsigned m_byte[ROUNDS][ADAM_N / W] = {}, v_byte[ROUNDS][ADAM_N / W] = {};
        if (t.staged) {
            if (STATE8)
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r) {
                    adam_load_scales<W, true>(m_byte[r], e.m_scale, at + r * ROUND, e.n);
                    adam_load_scales<W, true>(v_byte[r], e.v_scale, at + r * ROUND, e.n);
                }
            const char* src = adam_smem + stage * ring.stage_bytes;
            const int g = e.flags & ADAM_GRAD_FP32 ? 4 : 2, w = e.master || (e.flags & ADAM_PARAM_FP32) ? 4 : 2, st = STATE8 ? 1 : 4;
            const void* weight = e.master ? static_cast<const void*>(e.master) : e.param;
            const AdamInputs in = W > 1 ? AdamInputs{src, src + ring.weight_at, src + ring.m_at, src + ring.v_at}
                                         : AdamInputs{src + adam_skew(e.grad, t.base * g), src + ring.weight_at + adam_skew(weight, t.base * w),
                                                      src + ring.m_at + adam_skew(e.m, t.base * st), src + ring.v_at + adam_skew(e.v, t.base * st)};
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r)
                adam_elements<W, STATE8, STOCHASTIC, true>(e, at + r * ROUND, in, r * ROUND + W * tid, m_byte[r], v_byte[r], p, s, clip);
        } else {
            const AdamInputs in = {e.grad, e.master ? static_cast<const void*>(e.master) : e.param, e.m, e.v};
#pragma unroll 1
            for (int r = 0; r < ROUNDS; ++r) {
                if (STATE8) {
                    adam_load_scales<W, false>(m_byte[0], e.m_scale, at + r * ROUND, e.n);
                    adam_load_scales<W, false>(v_byte[0], e.v_scale, at + r * ROUND, e.n);
                }
                adam_elements<W, STATE8, STOCHASTIC, false>(e, at + r * ROUND, in, at + r * ROUND, m_byte[0], v_byte[0], p, s, clip);
            }
        }
        // the last warp to leave a stage fills it again
        __syncwarp();
        if ((tid & 31) == 0) {
            __threadfence_block();
            if (atomicAdd(&left[stage], 1) == ADAM_THREADS / 32 - 1) {
                left[stage] = 0;
                __threadfence_block();
                fill(i + ring.stages, t.entry);
            }
        }
        __syncwarp();
    }
    if (*static_cast<volatile int*>(&abort_word)) {          // let copies in flight finish before shared memory is released
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 1000000ull) {
        }
    }
}

template <int W, bool STATE8, bool STOCHASTIC>
static cudaError_t launch_adam_list(const AdamList<ADAM_CAP>& l, const AdamParams& p, const AdamStep& s, cudaStream_t stream) {
    // A stage has room for the list's widest tensors, and a CTA for as many stages as its share of the SM's shared memory takes, two at
    // least: a CTA less an SM where the stages are wide (8-bit moments beside a master copy 1515 -> 1417 us).
    int grad = 2, weight = 2;
    for (int i = 0; i < l.n; ++i) {
        if (l.e[i].flags & ADAM_GRAD_FP32) grad = 4;
        if (l.e[i].master || (l.e[i].flags & ADAM_PARAM_FP32)) weight = 4;
    }
    auto room = [](int size) { return adam_trip(STATE8) * size + (W > 1 ? 0 : 128); };
    AdamRing ring;
    ring.weight_at = room(grad);
    ring.m_at = ring.weight_at + room(weight);
    ring.v_at = ring.m_at + room(STATE8 ? 1 : 4);
    ring.stage_bytes = ring.v_at + room(STATE8 ? 1 : 4);
    constexpr int shared = 216 * 1024;
    int per_sm = adam_ctas_per_sm(W, STATE8);
    while (per_sm > 1 && shared / per_sm < 2 * ring.stage_bytes) --per_sm;
    const int most = shared / per_sm, trips = static_cast<int>(std::min<unsigned>(l.trips, 1u << 20));
    ring.stages = std::min(std::min(ADAM_STAGES, most / ring.stage_bytes), 1 + (trips + p.sm_count * per_sm - 1) / (p.sm_count * per_sm));
    const dim3 ctas(std::min<unsigned>(l.trips, static_cast<unsigned>(p.sm_count * per_sm)));
    const size_t smem = static_cast<size_t>(ring.stages) * ring.stage_bytes;
    auto allow = [&](const void* kern, DeviceOnce& once) {
        return once.run([&]() { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, shared); });
    };
    static DeviceOnce many, some;
    if (l.n > ADAM_CAP_SMALL) {
        auto kern = adam_kernel<ADAM_CAP, W, STATE8, STOCHASTIC>;
        const cudaError_t e = allow(reinterpret_cast<const void*>(kern), many);
        return e == cudaSuccess ? launch_pdl(kern, ctas, ADAM_THREADS, smem, stream, 1, l, p, s, ring) : e;
    }
    AdamList<ADAM_CAP_SMALL> few;
    std::copy(l.e, l.e + l.n, few.e);
    few.n = l.n;
    few.trips = l.trips;
    auto kern = adam_kernel<ADAM_CAP_SMALL, W, STATE8, STOCHASTIC>;
    const cudaError_t e = allow(reinterpret_cast<const void*>(kern), some);
    return e == cudaSuccess ? launch_pdl(kern, ctas, ADAM_THREADS, smem, stream, 1, few, p, s, ring) : e;
}
template <bool VECTORS>
static cudaError_t launch_adam_lists(const AdamTensors& t, const AdamParams& p, bool state8, bool stochastic, const AdamStep& s, cudaStream_t stream) {
    long long place = 0;
    for (int at = 0; at < t.n;) {
        AdamList<ADAM_CAP> l;
        l.n = 0;
        long long trips = 0;
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
            e.first = static_cast<unsigned>(trips);
            e.flags = (t.param_dtypes[at] == 1 ? ADAM_PARAM_FP32 : 0) | (t.grad_dtypes[at] == 1 ? ADAM_GRAD_FP32 : 0);
            place += n;
            auto bits = [](const void* q) { return reinterpret_cast<uintptr_t>(q); };
            const uintptr_t state = bits(e.m) | bits(e.v);
            const bool vectors = ((bits(e.grad) | bits(e.param) | bits(e.master)) & 15) == 0 && (state & 15) == 0;
            if (vectors != VECTORS) continue;
            l.e[l.n++] = e;
            trips += (n + adam_trip(state8) - 1) / adam_trip(state8);
        }
        l.trips = static_cast<unsigned>(trips);
        if (l.n == 0) continue;
        constexpr int W8 = VECTORS ? 8 : 1, W32 = VECTORS ? 4 : 1;
        const cudaError_t err = state8 ? (stochastic ? launch_adam_list<W8, true, true>(l, p, s, stream) : launch_adam_list<W8, true, false>(l, p, s, stream))
                                       : (stochastic ? launch_adam_list<W32, false, true>(l, p, s, stream) : launch_adam_list<W32, false, false>(l, p, s, stream));
        if (err != cudaSuccess) return err;
    }
    return cudaSuccess;
}

// Tensors that lie at odd addresses take launches of their own, behind the others'.
cudaError_t launch_adamw(const AdamTensors& t, const AdamParams& p, bool state8, bool stochastic, cudaStream_t stream) {
    const AdamStep s = adam_step(p, p.lr, p.step);
    const cudaError_t e = launch_adam_lists<true>(t, p, state8, stochastic, s, stream);
    return e == cudaSuccess ? launch_adam_lists<false>(t, p, state8, stochastic, s, stream) : e;
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
