// Global gradient norm over a list of tensors, and clipping by it.
#include <cuda_bf16.h>

#include <algorithm>
#include <cstdlib>

#include "tik_core.cuh"
#include "tik_internal.h"
#include "tik_ptx.cuh"

namespace tik {

constexpr int GRAD_THREADS = 256;
constexpr int GRAD_VEC = 8;                                  // 16-byte vectors per thread and chunk
constexpr int GRAD_CHUNK = GRAD_THREADS * GRAD_VEC;          // vectors of a chunk: 32 KiB
// Four CTAs on an SM, and shared memory that nothing uses to keep it at four: with the slots that registers leave, the CTAs of a call
// that starts as its predecessor drains pile up, five on some SMs and three on others, and each has an even share of the list.
constexpr int GRAD_CTAS = 592;
constexpr size_t GRAD_SMEM = 46 * 1024;

// The list travels as a kernel parameter: nothing to copy, and a captured graph holds it.
struct GradEntry {
    const void* in;
    void* out;
    long long n;
    unsigned first;              // chunk of the launch with which the tensor begins
    int fp32;
};
template <int CAP>
struct GradList {
    GradEntry e[CAP];
    int n;
    unsigned chunks;
};
constexpr int GRAD_CAP_SMALL = 64, GRAD_CAP = 1000;          // (parameters may take 32764 bytes)

// A chunk of a tensor.  Vectors start at the first 16-byte boundary; the elements in front of it and behind the last
// whole vector ("ends", fewer than 16) go with the tensor's first chunk.
struct GradChunk {
    const char* in;              // the tensor's first element
    char* out;
    long long n, head, first_vec, nvec, vecs;                // vecs: of this chunk
    int fp32;
};
template <int CAP>
__device__ __forceinline__ GradChunk grad_chunk(const GradList<CAP>& l, unsigned c, int& at) {
    // the last tensor with first <= c (empty ones take no chunk): mostly the one of the CTA's chunk before, `at`
    int lo = l.e[at].first <= c ? at : 0, hi = l.n;
    if (lo + 1 < hi && l.e[lo + 1].first > c) hi = lo + 1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.e[mid].first <= c) lo = mid;
        else hi = mid;
    }
    at = lo;
    const GradEntry& e = l.e[lo];
    GradChunk g;
    g.in = static_cast<const char*>(e.in);
    g.out = static_cast<char*>(e.out);
    g.n = e.n;
    g.fp32 = e.fp32;
    const int size = e.fp32 ? 4 : 2;
    const long long to_boundary = ((16 - (reinterpret_cast<uintptr_t>(e.in) & 15)) & 15) / size;
    g.head = to_boundary < e.n ? to_boundary : e.n;
    g.nvec = (e.n - g.head) * size / 16;
    g.first_vec = static_cast<long long>(c - e.first) * GRAD_CHUNK;
    g.vecs = g.nvec - g.first_vec < GRAD_CHUNK ? g.nvec - g.first_vec : GRAD_CHUNK;
    return g;
}
__device__ __forceinline__ float grad_element(const GradChunk& g, long long i) {
    return g.fp32 ? reinterpret_cast<const float*>(g.in)[i] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(g.in)[i]);
}
// index of the thread's element among the ends, or -1
__device__ __forceinline__ long long grad_end(const GradChunk& g, int tid) {
    if (g.first_vec != 0) return -1;
    const long long behind = g.head + g.nvec * (g.fp32 ? 4 : 8), i = tid < g.head ? tid : behind + (tid - g.head);
    return i < g.n ? i : -1;
}

// Sums of squares in fp32 over one thread's vectors, in fp64 from there on.  A sum that left the range in which fp32
// squares are exact enough is taken again in fp64, from the registers.
__device__ __forceinline__ double grad_squares(const uint4 (&v)[GRAD_VEC], bool fp32) {
    float s[4] = {};
    unsigned any = 0;
#pragma unroll
    for (int j = 0; j < GRAD_VEC; ++j) {
        const unsigned w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (fp32) {
                const float f = __uint_as_float(w[i]);
                s[i] = __fmaf_rn(f, f, s[i]);
                any |= w[i] & 0x7fffffffu;
            } else {
                const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xffff0000u);
                s[i] = __fmaf_rn(lo, lo, s[i]);
                s[i] = __fmaf_rn(hi, hi, s[i]);
                any |= w[i] & 0x7fff7fffu;
            }
        }
    }
    const float t = (s[0] + s[1]) + (s[2] + s[3]);
    if (any == 0 || (t >= 0x1p-80f && t <= 0x1p120f)) return t;
    double d = 0.0;
#pragma unroll
    for (int j = 0; j < GRAD_VEC; ++j) {
        const unsigned w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double a = __uint_as_float(fp32 ? w[i] : w[i] << 16), b = fp32 ? 0.0 : __uint_as_float(w[i] & 0xffff0000u);
            d += a * a + b * b;
        }
    }
    return d;
}

__device__ __forceinline__ double grad_block_sum(double v, double* buf, int tid) {
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    if ((tid & 31) == 0) buf[tid >> 5] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < GRAD_THREADS / 32; ++w) v += buf[w];
    return v;
}

template <int CAP>
__global__ void __launch_bounds__(GRAD_THREADS) grad_norm_kernel(const __grid_constant__ GradList<CAP> l, double* part) {
    __shared__ double buf[GRAD_THREADS / 32];
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    double sum = 0.0;
    int tensor = 0;
    for (unsigned c = blockIdx.x; c < l.chunks; c += gridDim.x) {
        const GradChunk g = grad_chunk(l, c, tensor);
        const uint4* src = reinterpret_cast<const uint4*>(g.in + g.head * (g.fp32 ? 4 : 2)) + g.first_vec;
        uint4 v[GRAD_VEC];
#pragma unroll
        for (int j = 0; j < GRAD_VEC; ++j) v[j] = tid + GRAD_THREADS * j < g.vecs ? src[tid + GRAD_THREADS * j] : make_uint4(0, 0, 0, 0);
        sum += grad_squares(v, g.fp32);
        const long long i = grad_end(g, tid);
        if (i >= 0) {
            const double f = grad_element(g, i);
            sum += f * f;
        }
    }
    sum = grad_block_sum(sum, buf, tid);
    if (tid == 0) part[blockIdx.x] = sum;
}

// fp32 norm from the CTAs' sums, the same bits wherever it is taken
__device__ __forceinline__ float grad_fold(const double* part, int n, double* buf, int tid) {
    double sum = 0.0;
    for (int i = tid; i < n; i += GRAD_THREADS) sum += part[i];
    return static_cast<float>(sqrt(grad_block_sum(sum, buf, tid)));
}
__global__ void __launch_bounds__(GRAD_THREADS) grad_fold_kernel(const double* part, int n, float* norm) {
    __shared__ double buf[GRAD_THREADS / 32];
    pdl_wait();
    pdl_launch_dependents();
    const float v = grad_fold(part, n, buf, threadIdx.x);
    if (threadIdx.x == 0) *norm = v;
}

template <int CAP>
__global__ void __launch_bounds__(GRAD_THREADS) grad_clip_kernel(const __grid_constant__ GradList<CAP> l, const double* part, int nparts,
                                                                 float* norm, float max_norm, bool in_place) {
    __shared__ double buf[GRAD_THREADS / 32];
    const int tid = threadIdx.x;
    pdl_wait();
    pdl_launch_dependents();
    float v;
    if (part) {
        v = grad_fold(part, nparts, buf, tid);
        if (blockIdx.x == 0 && tid == 0) *norm = v;
    } else {
        v = *norm;
    }
    const bool clip = v > max_norm && v <= 3.402823466e38f;
    const float coef = clip ? __fdiv_rn(max_norm, v) : 1.0f;
    if (!clip && in_place) return;
    // Back to front: what the norm read last may still be in L2.
    int tensor = l.n - 1;
    for (unsigned i = blockIdx.x; i < l.chunks; i += gridDim.x) {
        const GradChunk g = grad_chunk(l, l.chunks - 1 - i, tensor);
        if (!clip && g.out == g.in) continue;
        const int size = g.fp32 ? 4 : 2;
        const uint4* src = reinterpret_cast<const uint4*>(g.in + g.head * size) + g.first_vec;
        char* dst = g.out + g.head * size + g.first_vec * 16;
        const bool whole = (reinterpret_cast<uintptr_t>(dst) & 15) == 0;
        uint4 v[GRAD_VEC];
#pragma unroll
        for (int j = 0; j < GRAD_VEC; ++j) if (tid + GRAD_THREADS * j < g.vecs) v[j] = src[tid + GRAD_THREADS * j];
#pragma unroll
        for (int j = 0; j < GRAD_VEC; ++j) {
            const int at = tid + GRAD_THREADS * j;
            if (at >= g.vecs) break;
            unsigned w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
            if (clip) {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] = g.fp32 ? __float_as_uint(__fmul_rn(__uint_as_float(w[k]), coef))
                                  : pack_bf16x2(__fmul_rn(__uint_as_float(w[k] << 16), coef), __fmul_rn(__uint_as_float(w[k] & 0xffff0000u), coef));
            }
            char* to = dst + 16ll * at;
            if (whole) {
                *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
            } else if (g.fp32) {
#pragma unroll
                for (int k = 0; k < 4; ++k) reinterpret_cast<unsigned*>(to)[k] = w[k];
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) reinterpret_cast<unsigned short*>(to)[k] = static_cast<unsigned short>(w[k / 2] >> (16 * (k & 1)));
            }
        }
        const long long end = grad_end(g, tid);
        if (end >= 0) {
            const float f = grad_element(g, end), r = clip ? __fmul_rn(f, coef) : f;
            if (g.fp32) reinterpret_cast<float*>(g.out)[end] = r;
            else reinterpret_cast<__nv_bfloat16*>(g.out)[end] = __float2bfloat16_rn(r);
        }
    }
}

static int64_t grad_launches(int64_t n) { return (n + GRAD_CAP - 1) / GRAD_CAP; }
size_t grad_norm_bytes(int64_t n) { return static_cast<size_t>(grad_launches(n)) * GRAD_CTAS * sizeof(double); }

// Calls f(list, CTAs) for the lists of at most GRAD_CAP tensors that the call is cut into.
template <class F>
static cudaError_t for_lists(const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes, int n, F&& f) {
    for (int at = 0; at < n;) {
        GradList<GRAD_CAP> l;
        l.n = 0;
        long long chunks = 0;
        for (; at < n && l.n < GRAD_CAP; ++at) {
            if (numel[at] == 0) continue;
            const bool fp32 = dtypes[at] == 1;
            const long long most = (numel[at] * (fp32 ? 4 : 2) + 16ll * GRAD_CHUNK - 1) / (16ll * GRAD_CHUNK);
            l.e[l.n++] = {grads[at], out ? out[at] : const_cast<void*>(grads[at]), numel[at], static_cast<unsigned>(chunks), fp32 ? 1 : 0};
            chunks += most;
        }
        l.chunks = static_cast<unsigned>(chunks);
        if (l.n == 0) continue;
        const cudaError_t e = f(l, static_cast<int>(std::min<long long>(chunks, GRAD_CTAS)));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
static size_t grad_smem(int ctas) { return ctas < GRAD_CTAS ? 0 : GRAD_SMEM; }
static GradList<GRAD_CAP_SMALL> small_list(const GradList<GRAD_CAP>& l) {
    GradList<GRAD_CAP_SMALL> s;
    std::copy(l.e, l.e + l.n, s.e);
    s.n = l.n;
    s.chunks = l.chunks;
    return s;
}

static cudaError_t launch_squares(const void* const* grads, const int64_t* numel, const int* dtypes, int n, double* part, int* parts,
                                  cudaStream_t stream) {
    *parts = 0;
    return for_lists(grads, nullptr, numel, dtypes, n, [&](const GradList<GRAD_CAP>& l, int ctas) {
        double* to = part + *parts;
        *parts += ctas;
        return l.n <= GRAD_CAP_SMALL ? launch_pdl(grad_norm_kernel<GRAD_CAP_SMALL>, dim3(ctas), GRAD_THREADS, grad_smem(ctas), stream, 1, small_list(l), to)
                                     : launch_pdl(grad_norm_kernel<GRAD_CAP>, dim3(ctas), GRAD_THREADS, grad_smem(ctas), stream, 1, l, to);
    });
}

cudaError_t launch_grad_norm(const void* const* grads, const int64_t* numel, const int* dtypes, int n, float* norm, double* part,
                             cudaStream_t stream) {
    int parts;
    const cudaError_t e = launch_squares(grads, numel, dtypes, n, part, &parts, stream);
    if (e != cudaSuccess) return e;
    return launch_pdl(grad_fold_kernel, dim3(1), GRAD_THREADS, 0, stream, 1, part, parts, norm);
}

cudaError_t launch_grad_clip(const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes, int n, float max_norm,
                             float* norm, bool norm_known, double* part, cudaStream_t stream) {
    int parts = 0;
    if (!norm_known) {
        const cudaError_t e = launch_squares(grads, numel, dtypes, n, part, &parts, stream);
        if (e != cudaSuccess) return e;
        if (parts == 0) return launch_pdl(grad_fold_kernel, dim3(1), GRAD_THREADS, 0, stream, 1, part, 0, norm);
    }
    const double* from = norm_known ? nullptr : part;
    return for_lists(grads, out, numel, dtypes, n, [&](const GradList<GRAD_CAP>& l, int ctas) {
        return l.n <= GRAD_CAP_SMALL
                   ? launch_pdl(grad_clip_kernel<GRAD_CAP_SMALL>, dim3(ctas), GRAD_THREADS, grad_smem(ctas), stream, 1, small_list(l), from, parts, norm, max_norm, out == nullptr)
                   : launch_pdl(grad_clip_kernel<GRAD_CAP>, dim3(ctas), GRAD_THREADS, grad_smem(ctas), stream, 1, l, from, parts, norm, max_norm, out == nullptr);
    });
}

bool grad_ranges_overlap(const void* const* grads, void* const* out, const int64_t* numel, const int* dtypes, int n, const float* norm,
                         bool norm_known, bool* no_memory) {
    struct Range {
        uintptr_t from, to;
    };
    *no_memory = false;
    if (n <= 0) return false;
    Range* const written = static_cast<Range*>(malloc(2ull * (n + 1ull) * sizeof(Range)));
    if (!written) return *no_memory = true;
    Range* const read = written + n + 1;                     // inputs that are not written in place
    int nw = 0, nr = 0;
    for (int i = 0; i < n; ++i) {
        if (numel[i] == 0) continue;
        const uintptr_t bytes = static_cast<uintptr_t>(numel[i]) * (dtypes[i] == 1 ? 4 : 2);
        const uintptr_t in = reinterpret_cast<uintptr_t>(grads[i]), to = out ? reinterpret_cast<uintptr_t>(out[i]) : in;
        written[nw++] = {to, to + bytes};
        if (to != in) read[nr++] = {in, in + bytes};
    }
    const Range of_norm = {reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm + 1)};
    if (norm_known) read[nr++] = of_norm;
    else written[nw++] = of_norm;
    auto before = [](const Range& a, const Range& b) { return a.from < b.from; };
    auto ascending = [&](Range* r, int count) {              // (lists of a flat buffer's views are already)
        if (!std::is_sorted(r, r + count, before)) std::sort(r, r + count, before);
    };
    ascending(written, nw);
    ascending(read, nr);
    bool overlap = false;
    for (int i = 1; i < nw && !overlap; ++i) overlap = written[i].from < written[i - 1].to;
    for (int i = 0, j = 0; i < nr && !overlap; ++i) {
        while (j < nw && written[j].to <= read[i].from) ++j;
        overlap = j < nw && written[j].from < read[i].to;
    }
    free(written);
    return overlap;
}

}  // namespace tik
