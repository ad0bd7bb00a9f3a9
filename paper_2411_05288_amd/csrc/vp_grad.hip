// The norm of all gradients of a step together, and clipping by it.
//
// Bound by HBM: the norm reads every gradient once, clipping reads it again and writes it.  A call has n tensors of any size
// and either type; they are cut into chunks of 32 KB, the chunks are numbered through over all tensors, and the workgroups of
// one launch share them, so a thousand small tensors and eight large ones fill the chip alike.  The tensors travel in the
// kernel arguments, or, where there are more than fit, in a table in the workspace that a small kernel writes from its
// arguments (no copy from host memory, which a captured graph would read again at every replay).
//
// Squares are formed and summed in fp64: an fp32 value's square is exact there and neither over- nor underflows, and the sum
// of 10^9 of them keeps all digits that the fp32 result has.  Order of the sum: every thread its elements in ascending order,
// then fixed trees over the workgroup and over the workgroups' partial sums; no atomics.
#include "vp_internal.h"

namespace vp {

namespace {

constexpr int GRAD_LIST = 120;              // tensors in the kernel arguments
constexpr int GRAD_CHUNK_BYTES = 32768;
constexpr int GRAD_BLOCKS = 1024;           // partial sums at most

struct GradTensor {
    const void* g;
    void* o;
    int64_t count;
    int first;          // number of its first chunk
    int bf16;
};
struct GradList {
    int n;              // tensors here
    int at;             // table: number of the first of them
    GradTensor t[GRAD_LIST];
};

// Element-aligned vectors of 16 bytes: gradients may be views that start anywhere.
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ double block_sum64(double v, double* sh) {      // 256 threads, a fixed tree
    v = wave_sum64(v);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sh[0] + sh[1]) + (sh[2] + sh[3]);
}

// The tensor of chunk c: the last one whose first chunk is not behind it (tensors without elements have no chunks).
__device__ __forceinline__ int tensor_of(const GradTensor* t, int n, int c) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t[mid].first <= c) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ float bf16_to_f32(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ __forceinline__ unsigned short f32_to_bf16(float v) {
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(unsigned short, b);
}

__device__ __forceinline__ void add_squares(double* s, f32x4u v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e & 1] = fma((double)v[e], (double)v[e], s[e & 1]);
}
__device__ __forceinline__ void add_squares(double* s, u16x8u v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double d = bf16_to_f32(v[e]);
        s[e & 1] = fma(d, d, s[e & 1]);
    }
}

// Squares of one chunk: elements [e0, e1) of a tensor.
template <typename V, typename T>
__device__ __forceinline__ void chunk_squares(const T* g, int64_t e0, int64_t e1, double* s) {
    constexpr int E = 16 / sizeof(T), STEPS = GRAD_CHUNK_BYTES / 16 / 256;
    const T* p = g + e0 + threadIdx.x * E;
    if (e1 - e0 == GRAD_CHUNK_BYTES / (int)sizeof(T)) {
        V v[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) v[i] = *reinterpret_cast<const V*>(p + i * 256 * E);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) add_squares(s, v[i]);
        return;
    }
    const int n = (int)(e1 - e0);
    for (int j = threadIdx.x * E; j < n; j += 256 * E, p += 256 * E) {
        if (j + E <= n) {
            add_squares(s, *reinterpret_cast<const V*>(p));
        } else {
            V v = {};
            for (int e = 0; j + e < n; ++e) v[e] = p[e];
            add_squares(s, v);
        }
    }
}

__device__ __forceinline__ f32x4u times(f32x4u v, float f) { return v * f; }
__device__ __forceinline__ u16x8u times(u16x8u v, float f) {
    u16x8u o;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = f32_to_bf16(bf16_to_f32(v[e]) * f);
    return o;
}
__device__ __forceinline__ float times1(float v, float f) { return v * f; }
__device__ __forceinline__ unsigned short times1(unsigned short v, float f) { return f32_to_bf16(bf16_to_f32(v) * f); }

template <typename V, typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* o, int64_t e0, int64_t e1, float f) {
    constexpr int E = 16 / sizeof(T), STEPS = GRAD_CHUNK_BYTES / 16 / 256;
    const T* p = g + e0 + threadIdx.x * E;
    T* q = o + e0 + threadIdx.x * E;
    if (e1 - e0 == GRAD_CHUNK_BYTES / (int)sizeof(T)) {
        V v[STEPS];
#pragma unroll
        for (int i = 0; i < STEPS; ++i) v[i] = *reinterpret_cast<const V*>(p + i * 256 * E);
#pragma unroll
        for (int i = 0; i < STEPS; ++i) *reinterpret_cast<V*>(q + i * 256 * E) = times(v[i], f);
        return;
    }
    const int n = (int)(e1 - e0);
    for (int j = threadIdx.x * E; j < n; j += 256 * E, p += 256 * E, q += 256 * E) {
        if (j + E <= n) {
            *reinterpret_cast<V*>(q) = times(*reinterpret_cast<const V*>(p), f);
        } else {
            for (int e = 0; j + e < n; ++e) q[e] = times1(p[e], f);
        }
    }
}

__global__ __launch_bounds__(128) void grad_table_kernel(GradList l, GradTensor* table) {
    for (int i = threadIdx.x; i < l.n; i += 128) table[l.at + i] = l.t[i];
}

// Sum of the partial sums in a fixed order (all 256 threads get it).
__device__ __forceinline__ float norm_of(const double* part, int parts, double* sh) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    return (float)sqrt(block_sum64(s, sh));
}

// part[b]: workgroup b's sum of squares.  A single workgroup writes the norm itself.
template <bool TABLE>
__global__ __launch_bounds__(256) void grad_squares_kernel(GradList l, const GradTensor* table, int n, int chunks, double* part,
                                                           float* norm) {
    __shared__ double sh[4];
    const GradTensor* ts = TABLE ? table : l.t;
    double s[2] = {0.0, 0.0};
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        const GradTensor t = ts[tensor_of(ts, n, c)];
        if (t.bf16) {
            const int64_t e0 = (int64_t)(c - t.first) * (GRAD_CHUNK_BYTES / 2), e1 = e0 + GRAD_CHUNK_BYTES / 2;
            chunk_squares<u16x8u>((const u16*)t.g, e0, e1 < t.count ? e1 : t.count, s);
        } else {
            const int64_t e0 = (int64_t)(c - t.first) * (GRAD_CHUNK_BYTES / 4), e1 = e0 + GRAD_CHUNK_BYTES / 4;
            chunk_squares<f32x4u>((const float*)t.g, e0, e1 < t.count ? e1 : t.count, s);
        }
    }
    const double sum = block_sum64(s[0] + s[1], sh);
    if (threadIdx.x == 0) {
        part[blockIdx.x] = sum;
        if (gridDim.x == 1 && norm) norm[0] = (float)sqrt(sum);
    }
}

__global__ __launch_bounds__(256) void grad_norm_kernel(const double* part, int parts, float* norm) {
    __shared__ double sh[4];
    const float v = norm_of(part, parts, sh);
    if (threadIdx.x == 0) norm[0] = v;
}

// parts > 0: the norm comes from the partial sums (every workgroup folds them, which spares a launch) and is written by
// workgroup 0; else it is read.  The chunks are taken from the last to the first: what the norm's launch read last is still in
// the 256 MB infinity cache.
template <bool TABLE>
__global__ __launch_bounds__(256) void grad_scale_kernel(GradList l, const GradTensor* table, int n, int chunks, int in_place,
                                                         const double* part, int parts, float max_norm, float* norm) {
    __shared__ double sh[4];
    const GradTensor* ts = TABLE ? table : l.t;
    float v;
    if (parts) {
        v = norm_of(part, parts, sh);
        if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = v;
    } else {
        v = norm[0];
    }
    const float f = v > max_norm && v < INFINITY ? max_norm / v : 1.f;
    if (f == 1.f && in_place) return;
    for (int c = chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) {
        const GradTensor t = ts[tensor_of(ts, n, c)];
        if (t.bf16) {
            const int64_t e0 = (int64_t)(c - t.first) * (GRAD_CHUNK_BYTES / 2), e1 = e0 + GRAD_CHUNK_BYTES / 2;
            chunk_scale<u16x8u>((const u16*)t.g, (u16*)t.o, e0, e1 < t.count ? e1 : t.count, f);
        } else {
            const int64_t e0 = (int64_t)(c - t.first) * (GRAD_CHUNK_BYTES / 4), e1 = e0 + GRAD_CHUNK_BYTES / 4;
            chunk_scale<f32x4u>((const float*)t.g, (float*)t.o, e0, e1 < t.count ? e1 : t.count, f);
        }
    }
}

}  // namespace

size_t grad_workspace(int32_t n) {
    return GRAD_BLOCKS * sizeof(double) + (n > GRAD_LIST ? align_up((size_t)n * sizeof(GradTensor), 256) : 0);
}

hipError_t launch_grad(const void* const* grads, const int64_t* counts, const int32_t* dts, int32_t n, void* const* outs,
                       float max_norm, bool known, float* norm, void* workspace, hipStream_t st) {
    double* part = (double*)workspace;
    GradTensor* table = (GradTensor*)(part + GRAD_BLOCKS);
    const bool in_table = n > GRAD_LIST;
    GradList l;
    l.n = l.at = 0;
    int64_t chunks = 0;
    {
        ProfScope prof(known ? K_GRAD_SCALE : K_GRAD_NORM, st);
        for (int32_t k = 0; k < n; ++k) {
            const int bf16 = dts[k] == VP_BF16;
            l.t[l.n++] = GradTensor{grads[k], outs ? outs[k] : const_cast<void*>(grads[k]), counts[k], (int)chunks, bf16};
            chunks += ceil_div(counts[k] * (bf16 ? 2 : 4), GRAD_CHUNK_BYTES);
            if (in_table && (l.n == GRAD_LIST || k == n - 1)) {
                hipLaunchKernelGGL(grad_table_kernel, dim3(1), dim3(128), 0, st, l, table);
                l.at = k + 1;
                l.n = 0;
            }
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int blocks = chunks < 1 ? 1 : chunks < GRAD_BLOCKS ? (int)chunks : GRAD_BLOCKS;
    if (!known) {
        ProfScope prof(K_GRAD_NORM, st);
        const bool alone = max_norm < 0.f;
        if (in_table)
            hipLaunchKernelGGL(grad_squares_kernel<true>, dim3(blocks), dim3(256), 0, st, l, table, n, (int)chunks, part, alone ? norm : nullptr);
        else
            hipLaunchKernelGGL(grad_squares_kernel<false>, dim3(blocks), dim3(256), 0, st, l, table, n, (int)chunks, part, alone ? norm : nullptr);
        if (alone && blocks > 1) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, st, part, blocks, norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || alone) return e;
    }
    ProfScope prof(K_GRAD_SCALE, st);
    const int parts = known ? 0 : blocks, in_place = outs == nullptr;
    if (in_table)
        hipLaunchKernelGGL(grad_scale_kernel<true>, dim3(blocks), dim3(256), 0, st, l, table, n, (int)chunks, in_place, part, parts, max_norm, norm);
    else
        hipLaunchKernelGGL(grad_scale_kernel<false>, dim3(blocks), dim3(256), 0, st, l, table, n, (int)chunks, in_place, part, parts, max_norm, norm);
    return hipGetLastError();
}

}  // namespace vp
