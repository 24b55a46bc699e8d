// The global norm of a list of gradients, and the list scaled to a largest norm.
//
//   N = sqrt(sum over all tensors and elements of g^2)
//   c = max_norm / max(N, max_norm),   out = c * g
//
// Both passes are bound by memory: the norm reads every gradient once, the
// scaling reads it again and writes it.  The tensors travel as a table in the
// kernel arguments (kTableMax of them a launch), so nothing is copied to the
// device beforehand and a call can be captured; a tensor is cut into chunks of
// kChunkBytes, which the workgroups take in turn.  A workgroup leaves one
// partial sum; whoever needs the norm adds all partial sums in their order, so
// that every workgroup of the scaling gets the same bits without a launch
// between the two.  Squares and sums are 64-bit: a square of fp32 neither
// overflows nor vanishes, and with 2^31 elements none passes more than some 160
// additions (64 of its chunk, as many chunks of its workgroup, the trees and the
// partial sums): N is off by less than 2^-45 of it before it is rounded to fp32.
#include <cmath>

#include "conv_common.h"

namespace onexn {
namespace {

constexpr int kTableMax = 176;        // tensors a launch: 3.9 KB of kernel arguments
constexpr int kMaxPartials = 2048;    // workgroups of the norm over all launches (eight a CU)
constexpr int kChunkBytes = 32768;    // eight 16-byte loads a lane
// Short lists go to one workgroup, kOneParts chunks at a time: one launch in
// place of two, 6.8 against 10.2 us of the host.  On the GPU the norm takes 5.0
// us of 8 chunks and 7.5 of 16, against 4.7 in two launches, the clipping 7.0 of
// 4 chunks and 10.8 of 8, against 7.6.
constexpr int kOneParts = 4, kOneNorm = 8, kOneClip = 4;
constexpr int kLoads = kChunkBytes / (kThreads * 16);

struct GradTable {
    const void* g[kTableMax];
    void* out[kTableMax];
    int32_t first[kTableMax + 1];     // first chunk of each tensor
    uint16_t last[kTableMax];         // elements of its last chunk; kBf16: type
    int32_t count;
};
constexpr uint16_t kBf16 = 0x8000;

// 16 bytes of elements at any element alignment (global loads take any).
template <typename T> struct Vec;
template <> struct Vec<float> { typedef float type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Vec<uint16_t> { typedef uint16_t type __attribute__((ext_vector_type(8), aligned(2))); };

struct Chunk {
    int tensor;
    int32_t index, elements;
    bool bf16;
};

// The tensor that holds chunk c: the last one whose first chunk is at most c
// (tensors without elements share their first chunk with the next).
__device__ __forceinline__ Chunk find_chunk(const GradTable& t, int32_t c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid - 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const bool bf16 = t.last[lo] & kBf16;
    return {lo, c - t.first[lo], c + 1 == t.first[lo + 1] ? t.last[lo] & ~kBf16 : kChunkBytes / (bf16 ? 2 : 4), bf16};
}

// A chunk's elements: 16 bytes a lane and step (zeros behind the last whole 16
// bytes), and what is left over, an element for each of the first lanes.
template <typename T> struct Part {
    static constexpr int V = 16 / sizeof(T), FULL = kChunkBytes / int(sizeof(T));
    typedef typename Vec<T>::type vec;
    vec v[kLoads];
    T rest;
    __device__ static int32_t me() { return threadIdx.x % kThreads; }
    __device__ static int32_t at(int k) { return (k * kThreads + me()) * V; }
    __device__ static int32_t rest_at(int32_t n) {      // -1: not this lane's
        return me() < n % V ? n - n % V + me() : -1;
    }
    __device__ void load(const T* __restrict__ g, int32_t n) {
        rest = T(0);
        if (n == FULL) {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) v[k] = *reinterpret_cast<const vec*>(g + at(k));
            return;
        }
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            v[k] = vec{};
            if (at(k) + V <= n) v[k] = *reinterpret_cast<const vec*>(g + at(k));
        }
        if (rest_at(n) >= 0) rest = g[rest_at(n)];
    }
};

// Sum over the workgroup, in lane and wave order; every thread gets it.
template <int THREADS = kThreads>
__device__ __forceinline__ double block_sum(double v, double* lds) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    const int wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) lds[wave] = v;
    __syncthreads();
    double s = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) s += lds[w];
    return s;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const void* g, const Chunk& c) {
    constexpr int V = 16 / sizeof(T);
    Part<T> p;
    p.load(static_cast<const T*>(g) + int64_t(c.index) * Part<T>::FULL, c.elements);
    const double d = to_f32(p.rest);
    double s = d * d;
#pragma unroll
    for (int k = 0; k < kLoads; ++k)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const double d = to_f32(p.v[k][e]);
            s = fma(d, d, s);
        }
    return s;
}

__global__ void __launch_bounds__(kThreads) grad_squares(const GradTable t, double* __restrict__ partial) {
    __shared__ double lds[kThreads / 64];
    const int32_t chunks = t.first[t.count];
    double s = 0;
    for (int32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        const Chunk k = find_chunk(t, c);
        s += k.bf16 ? chunk_squares<uint16_t>(t.g[k.tensor], k) : chunk_squares<float>(t.g[k.tensor], k);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The norm, from all partial sums in their order.
__device__ __forceinline__ double total_norm(const double* __restrict__ partial, int32_t partials, double* lds) {
    double s = 0;
    for (int32_t i = threadIdx.x; i < partials; i += kThreads) s += partial[i];
    return sqrt(block_sum(s, lds));
}

__global__ void __launch_bounds__(kThreads) grad_norm_join(const double* __restrict__ partial, int32_t partials,
                                                           float* __restrict__ norm) {
    __shared__ double lds[kThreads / 64];
    const double N = total_norm(partial, partials, lds);
    if (threadIdx.x == 0) *norm = float(N);
}

// 64 bits, as the norm: finite gradients may have norms of 1e43, and their factor
// is no fp32 number then (0.27 G elements of fp32: 610 us, 600 with a factor in
// fp32; 0.4 G of bf16: 463 and 462).  (A norm that is NaN gives a factor that is
// NaN.)
__device__ __forceinline__ double factor(double N, double max_norm) { return N <= max_norm ? 1. : max_norm / N; }

// c * g, rounded to fp32 and from there to the gradient's type.
template <typename T>
__device__ __forceinline__ T scaled(T g, double c) { return from_f32<T>(float(c * to_f32(g))); }

template <typename T>
__device__ __forceinline__ void chunk_scale(const void* g, void* out, const Chunk& k, double c) {
    typedef typename Part<T>::vec vec;
    const int64_t at = int64_t(k.index) * Part<T>::FULL;
    T* const o = static_cast<T*>(out) + at;
    Part<T> p;
    p.load(static_cast<const T*>(g) + at, k.elements);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
#pragma unroll
        for (int e = 0; e < p.V; ++e) p.v[j][e] = scaled<T>(p.v[j][e], c);
        if (p.at(j) + p.V <= k.elements) __builtin_nontemporal_store(p.v[j], reinterpret_cast<vec*>(o + p.at(j)));
    }
    if (p.rest_at(k.elements) >= 0) o[p.rest_at(k.elements)] = scaled<T>(p.rest, c);
}

__global__ void __launch_bounds__(kThreads) grad_scale(const GradTable t, const double* __restrict__ partial,
                                                       int32_t partials, double max_norm, float* __restrict__ norm) {
    __shared__ double lds[kThreads / 64];
    const double N = total_norm(partial, partials, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = float(N);
    const double c = factor(N, max_norm);
    // Last chunks first: what the norm has read last may still be in the caches.
    for (int32_t i = t.first[t.count] - 1 - int32_t(blockIdx.x); i >= 0; i -= gridDim.x) {
        const Chunk k = find_chunk(t, i);
        const void* const g = t.g[k.tensor];
        void* const out = t.out[k.tensor];
        if (c == 1. && out == g) continue;
        if (k.bf16) chunk_scale<uint16_t>(g, out, k, c);
        else chunk_scale<float>(g, out, k, c);
    }
}

// The norm, and the scaling where max_norm is positive, of a short list: one
// workgroup, kOneParts chunks at a time.
__global__ void __launch_bounds__(kThreads * kOneParts) grad_one(const GradTable t, double max_norm,
                                                                 float* __restrict__ norm) {
    __shared__ double lds[kThreads * kOneParts / 64];
    const int32_t chunks = t.first[t.count], first = __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    double s = 0;
    for (int32_t c = first; c < chunks; c += kOneParts) {
        const Chunk k = find_chunk(t, c);
        s += k.bf16 ? chunk_squares<uint16_t>(t.g[k.tensor], k) : chunk_squares<float>(t.g[k.tensor], k);
    }
    const double N = sqrt(block_sum<kThreads * kOneParts>(s, lds));
    if (norm && threadIdx.x == 0) *norm = float(N);
    if (max_norm <= 0) return;
    const double c = factor(N, max_norm);
    for (int32_t i = first; i < chunks; i += kOneParts) {
        const Chunk k = find_chunk(t, i);
        if (c == 1. && t.out[k.tensor] == t.g[k.tensor]) continue;
        if (k.bf16) chunk_scale<uint16_t>(t.g[k.tensor], t.out[k.tensor], k, c);
        else chunk_scale<float>(t.g[k.tensor], t.out[k.tensor], k, c);
    }
}

int32_t chunk_elements(int32_t dt) { return kChunkBytes / (dt == ONEXN_BF16 ? 2 : 4); }
int64_t chunks_of(int64_t size, int32_t dt) { return (size + chunk_elements(dt) - 1) / chunk_elements(dt); }

onexn_status check_grads(const char* fn, const void* const* g, void* const* out, const int32_t* dt,
                         const int64_t* size, int32_t count, int64_t* total) {
    if (count < 0) return fail(ONEXN_ERR_ARG, "%s: count must be >= 0", fn);
    if (count > 0 && (!g || !dt || !size)) return fail(ONEXN_ERR_NULL, "%s: NULL pointer argument", fn);
    *total = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (dt[i] != ONEXN_F32 && dt[i] != ONEXN_BF16)
            return fail(ONEXN_ERR_DTYPE, "%s: unknown dtype %d of tensor %d", fn, dt[i], i);
        if (size[i] < 0) return fail(ONEXN_ERR_ARG, "%s: tensor %d has a negative size", fn, i);
        if (size[i] > 0 && (!g[i] || (out && !out[i])))
            return fail(ONEXN_ERR_NULL, "%s: tensor %d is NULL", fn, i);
        const uintptr_t align = dt[i] == ONEXN_BF16 ? 1 : 3;
        if ((reinterpret_cast<uintptr_t>(g[i]) & align) || (out && (reinterpret_cast<uintptr_t>(out[i]) & align)))
            return fail(ONEXN_ERR_ARG, "%s: tensor %d is not aligned to its elements", fn, i);
        if (size[i] > INT64_MAX / 4) return fail(ONEXN_ERR_BUFSIZE, "%s: tensor %d is too large", fn, i);
        *total += chunks_of(size[i], dt[i]);
        if (*total > INT32_MAX / 2) return fail(ONEXN_ERR_BUFSIZE, "%s: more than 2^30 chunks of 32 KB", fn);
    }
    return ONEXN_OK;
}

// Table of tensors [at, at + kTableMax), and its chunks.
int32_t fill_table(GradTable& t, const void* const* g, void* const* out, const int32_t* dt, const int64_t* size,
                   int32_t count, int32_t at) {
    t.count = count - at < kTableMax ? count - at : kTableMax;
    int32_t chunks = 0;
    for (int32_t i = 0; i < t.count; ++i) {
        t.g[i] = g[at + i];
        t.out[i] = out ? out[at + i] : const_cast<void*>(g[at + i]);
        const int32_t own = int32_t(chunks_of(size[at + i], dt[at + i])), full = chunk_elements(dt[at + i]);
        t.last[i] = uint16_t((own ? size[at + i] - int64_t(own - 1) * full : 0) | (dt[at + i] == ONEXN_BF16 ? kBf16 : 0));
        t.first[i] = chunks;
        chunks += own;
    }
    t.first[t.count] = chunks;
    return chunks;
}

size_t grad_workspace(int32_t count) { return size_t(kMaxPartials + (count + kTableMax - 1) / kTableMax) * 8; }

onexn_status check_workspace(const char* fn, void* ws, size_t bytes, int32_t count) {
    if (!ws) return fail(ONEXN_ERR_NULL, "%s: NULL workspace", fn);
    if (bytes < grad_workspace(count))
        return fail(ONEXN_ERR_BUFSIZE, "%s: workspace of %zu bytes, %zu needed", fn, bytes, grad_workspace(count));
    if (reinterpret_cast<uintptr_t>(ws) % 8 != 0) return fail(ONEXN_ERR_ARG, "%s: workspace must be 8-byte aligned", fn);
    return ONEXN_OK;
}

onexn_status launched(const char* fn) {
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return fail(ONEXN_ERR_HIP, "%s: launch failed: %s", fn, hipGetErrorString(err));
    return ONEXN_OK;
}

void launch_one(const void* const* g, void* const* out, const int32_t* dt, const int64_t* size, int32_t count,
                double max_norm, float* norm, hipStream_t s) {
    GradTable t;
    fill_table(t, g, out, dt, size, count, 0);
    hipLaunchKernelGGL(grad_one, dim3(1), dim3(kThreads * kOneParts), 0, s, t, max_norm, norm);
}

// The partial sums of all tensors; returns how many there are.
int32_t launch_squares(const void* const* g, const int32_t* dt, const int64_t* size, int32_t count, int64_t total,
                       double* partial, hipStream_t s) {
    int32_t partials = 0;
    for (int32_t at = 0; at < count; at += kTableMax) {
        GradTable t;
        const int32_t chunks = fill_table(t, g, nullptr, dt, size, count, at);
        if (chunks == 0) continue;
        // A launch's share of the partial sums, one at least.
        int64_t grid = total <= kMaxPartials ? chunks : int64_t(chunks) * kMaxPartials / total;
        if (grid < 1) grid = 1;
        hipLaunchKernelGGL(grad_squares, dim3(uint32_t(grid)), dim3(kThreads), 0, s, t, partial + partials);
        partials += int32_t(grid);
    }
    return partials;
}

}  // namespace
}  // namespace onexn

using namespace onexn;

extern "C" size_t onexn_grad_workspace_bytes(int32_t count) { return count < 0 ? 0 : grad_workspace(count); }

extern "C" onexn_status onexn_grad_norm(const void* const* grads, const int32_t* dtypes, const int64_t* sizes,
                                        int32_t count, float* norm_dev, void* workspace_dev,
                                        size_t workspace_bytes, void* stream) {
    clear_error();
    int64_t total = 0;
    if (onexn_status st = check_grads("grad_norm", grads, nullptr, dtypes, sizes, count, &total)) return st;
    if (!norm_dev) return fail(ONEXN_ERR_NULL, "grad_norm: NULL norm");
    if (onexn_status st = check_workspace("grad_norm", workspace_dev, workspace_bytes, count)) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (total <= kOneNorm && count <= kTableMax) {
        launch_one(grads, nullptr, dtypes, sizes, count, 0., norm_dev, s);
        return launched("grad_norm");
    }
    double* partial = static_cast<double*>(workspace_dev);
    const int32_t partials = launch_squares(grads, dtypes, sizes, count, total, partial, s);
    hipLaunchKernelGGL(grad_norm_join, dim3(1), dim3(kThreads), 0, s, partial, partials, norm_dev);
    return launched("grad_norm");
}

extern "C" onexn_status onexn_clip_grads(const void* const* grads, void* const* out, const int32_t* dtypes,
                                         const int64_t* sizes, int32_t count, double max_norm, float* norm_dev,
                                         void* workspace_dev, size_t workspace_bytes, void* stream) {
    clear_error();
    int64_t total = 0;
    if (onexn_status st = check_grads("clip_grads", grads, out, dtypes, sizes, count, &total)) return st;
    if (!(max_norm > 0) || !std::isfinite(max_norm))
        return fail(ONEXN_ERR_ARG, "clip_grads: max_norm must be positive and finite");
    if (onexn_status st = check_workspace("clip_grads", workspace_dev, workspace_bytes, count)) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (total <= kOneClip && count <= kTableMax) {
        launch_one(grads, out, dtypes, sizes, count, max_norm, norm_dev, s);
        return launched("clip_grads");
    }
    double* partial = static_cast<double*>(workspace_dev);
    const int32_t partials = launch_squares(grads, dtypes, sizes, count, total, partial, s);
    bool written = false;
    for (int32_t at = 0; at < count; at += kTableMax) {
        GradTable t;
        const int32_t chunks = fill_table(t, grads, out, dtypes, sizes, count, at);
        if (chunks == 0) continue;
        const int32_t grid = chunks < kMaxPartials ? chunks : kMaxPartials;
        hipLaunchKernelGGL(grad_scale, dim3(uint32_t(grid)), dim3(kThreads), 0, s, t, partial, partials, max_norm,
                           written ? nullptr : norm_dev);
        written = true;
    }
    if (!written && norm_dev)
        hipLaunchKernelGGL(grad_norm_join, dim3(1), dim3(kThreads), 0, s, partial, partials, norm_dev);
    return launched("clip_grads");
}
