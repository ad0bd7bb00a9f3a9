// The norm of all gradients of a step together, and clipping by it.
//
// Bound by HBM: the norm reads every gradient once (8 x 4000 x 4096 fp32: 77 us, 6.8 TB/s), clipping reads it again and writes it
// (8 x 16032 x 4096: 301 us, then 765 us, 5.5 TB/s); short lists by the two launches.  A call has n tensors of any size
// and either type; they are cut into chunks of 32 KB, the chunks are numbered through over all tensors, and the workgroups of
// one launch share them, so a thousand small tensors and eight large ones fill the chip alike.  The tensors travel in the
// kernel arguments, or, where there are more than fit, in a table in the workspace that a small kernel writes from its
// arguments (no copy from host memory, which a captured graph would read again at every replay).
//
// Squares are formed and summed in fp64: an fp32 value's square is exact there and neither over- nor underflows, and the sum
// of 10^9 of them keeps all digits that the fp32 result has.  Order of the sum: every thread its elements in ascending order,
// then fixed trees over the workgroup and over the workgroups' partial sums; no atomics.
#include <limits.h>

#include "vp_internal.h"

namespace vp {

namespace {

constexpr int GRAD_LIST = 160;              // tensors in the kernel arguments
constexpr int GRAD_CHUNK_BYTES = 32768;     // 256 threads, eight loads of 16 bytes each
constexpr int GRAD_BLOCKS = 1024;           // workgroups, and partial sums, at most
constexpr int GRAD_KEEP = (192 << 20) / GRAD_CHUNK_BYTES;      // chunks that the infinity cache holds from one launch to the next
constexpr int GRAD_FIRSTS = 2048;           // numbers of first chunks that a workgroup holds in LDS

struct GradTensor {
    const void* g;
    void* o;
    uint64_t size;      // elements * 2, + 1 with bf16
    __host__ __device__ bool bf16() const { return size & 1; }
    __host__ __device__ int64_t count() const { return (int64_t)(size >> 1); }
    __host__ __device__ int64_t bytes() const { return count() * (bf16() ? 2 : 4); }
    __host__ __device__ int chunks() const { return (int)((bytes() + GRAD_CHUNK_BYTES - 1) / GRAD_CHUNK_BYTES); }
};
// (150 tensors of 37 MB, clipped: 31 us through a table, 27 with all of them in the arguments)
struct GradList {
    int n;              // tensors here
    int at, first;      // table: number of the first of them, and of its first chunk
    GradTensor t[GRAD_LIST];
};
struct GradTable {      // more tensors than the arguments hold: entries and the number of the first chunk of each
    GradTensor* t;
    int* first;
};

// Vectors of 16 bytes at the alignment of an element: gradients may be views that start anywhere.  In registers they are words
// (vectors of 16-bit elements that are loaded under a condition take a register per element, words at odd addresses a load per
// element).
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T>
struct Vec;
template <>
struct Vec<float> {
    typedef float type __attribute__((ext_vector_type(4), aligned(4)));
    typedef float loaded __attribute__((ext_vector_type(4)));
};
template <>
struct Vec<u16> {
    typedef unsigned short type __attribute__((ext_vector_type(8), aligned(2)));
    typedef unsigned short loaded __attribute__((ext_vector_type(8)));
};

// (an address from the table is one of global memory)
template <typename T>
__device__ __forceinline__ T* global(T* p) {
    return (T*)(__attribute__((address_space(1))) T*)p;
}

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

// Sum over the lanes up to this one.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false); }
__device__ __forceinline__ int scan64(int v) {
    v = add_moved<0x111, 0xf>(v);      // from 1, 2, 4, 8 lanes before, within 16
    v = add_moved<0x112, 0xf>(v);
    v = add_moved<0x114, 0xf>(v);
    v = add_moved<0x118, 0xf>(v);
    v = add_moved<0x142, 0xa>(v);      // the last lane of 16 into the next 16, of 32 into the next 32
    return add_moved<0x143, 0xc>(v);
}

// The tensors of a launch.  A chunk's tensor is the last one whose first chunk is not behind it (tensors without elements have no
// chunks).  Steps of a search through memory took longer than the chunk itself (150 tensors of 37 MB together: 11.6 us for their
// squares), so every wavefront holds the list's first chunks in registers, and every workgroup the table's in LDS.
template <bool TABLE>
struct Tensors {
    static constexpr int PER_LANE = (GRAD_LIST + 63) / 64;
    const GradList& l;
    const GradTable& table;
    int n;
    int own[PER_LANE];      // list: lane i has the first chunks of tensors i, i + 64, ... (behind the last tensor: never reached)
    int stride;             // table: every stride-th tensor's in LDS
    const int* lds;
    __device__ Tensors(const GradList& l, const GradTable& table, int n, int* lds) : l(l), table(table), n(n), stride(1), lds(lds) {
        if constexpr (TABLE) {
            stride = (n + GRAD_FIRSTS - 1) / GRAD_FIRSTS;
            for (int k = threadIdx.x; k * stride < n; k += 256) lds[k] = table.first[k * stride];
            __syncthreads();
        } else {
            int before = 0;
#pragma unroll
            for (int b = 0; b < PER_LANE; ++b) {
                own[b] = INT_MAX;
                if (b * 64 < n) {
                    const int k = b * 64 + (threadIdx.x & 63), chunks = k < n ? l.t[k].chunks() : 0, v = before + scan64(chunks);
                    if (k < n) own[b] = v - chunks;
                    before = __builtin_amdgcn_readlane(v, 63);
                }
            }
        }
    }
    // also the number of the chunk within its tensor
    __device__ GradTensor of(int c, int& within) const {
        int k, f = 0;
        if constexpr (TABLE) {
            k = search(lds, 0, (n - 1) / stride, c);
            f = lds[k];
            if (stride > 1) {
                const int end = (k + 1) * stride < n ? (k + 1) * stride : n;
                k = search(table.first, k * stride, end - 1, c);
                f = table.first[k];
            }
            k = __builtin_amdgcn_readfirstlane(k);
            within = __builtin_amdgcn_readfirstlane(c - f);
            return table.t[k];
        } else {
            k = -1;
#pragma unroll
            for (int b = 0; b < PER_LANE; ++b)
                if (b * 64 < n) {
                    const int m = __popcll(__ballot(own[b] <= c));
                    if (m) f = __builtin_amdgcn_readlane(own[b], m - 1);
                    k += m;
                }
            within = c - f;
            return l.t[k];
        }
    }
    __device__ static int search(const int* first, int lo, int hi, int c) {
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first[mid] <= c) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
};

__device__ __forceinline__ float bits(uint32_t b) { return __uint_as_float(b); }
__device__ __forceinline__ uint32_t bf16_bits(float v) {
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(unsigned short, b);
}

// s += squares of the elements of a vector, in fp64
template <typename T>
__device__ __forceinline__ void add_squares(double* s, u32x4 v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) {
            const double d = bits(v[e]);
            s[e & 1] = fma(d, d, s[e & 1]);
        } else {
            const double low = bits(v[e] << 16), high = bits(v[e] & 0xffff0000u);
            s[0] = fma(low, low, s[0]);
            s[1] = fma(high, high, s[1]);
        }
    }
}
// the elements times f, rounded to the type
template <typename T>
__device__ __forceinline__ u32x4 times(u32x4 v, float f) {
    u32x4 o;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) o[e] = __float_as_uint(bits(v[e]) * f);
        else o[e] = bf16_bits(bits(v[e] << 16) * f) | bf16_bits(bits(v[e] & 0xffff0000u) * f) << 16;
    }
    return o;
}
__device__ __forceinline__ uint32_t word_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t word_of(u16 v) { return v; }

// A tensor's chunk.  At the end of a tensor the vectors that are whole are asked for four at a time (one after the other, the
// norm of 60 tensors of 17 MB together took 9.6 us in place of 8.2), and the elements behind them go to a thread each.
template <typename T>
struct Chunk {
    static constexpr int E = 16 / sizeof(T), SIZE = GRAD_CHUNK_BYTES / sizeof(T), STEPS = SIZE / (256 * E);
    int64_t first;      // element
    int n;              // elements
    __device__ Chunk(int64_t count, int within) {
        first = (int64_t)within * SIZE;
        n = count - first < SIZE ? (int)(count - first) : SIZE;
    }
    __device__ bool whole() const { return n == SIZE; }
    __device__ static int at(int step) { return (step * 256 + threadIdx.x) * E; }
    __device__ bool has(int step) const { return at(step) + E <= n; }
    // the element behind the whole vectors that is this thread's, or -1
    __device__ int rest() const { return (int)threadIdx.x < n % E ? n / E * E + threadIdx.x : -1; }
};

template <bool KEEP, typename T>
__device__ __forceinline__ void chunk_squares(const T* g, int64_t count, int within, double* s) {
    using C = Chunk<T>;
    using V = typename Vec<T>::type;
    const C c(count, within);
    const T* p = global(g) + c.first;
    auto load = [&](int i) -> u32x4 {
        const V* at = reinterpret_cast<const V*>(p + C::at(i));
        const typename Vec<T>::loaded v = KEEP ? *at : __builtin_nontemporal_load(at);
        return __builtin_bit_cast(u32x4, v);
    };
    if (c.whole()) {
        u32x4 v[C::STEPS];
#pragma unroll
        for (int i = 0; i < C::STEPS; ++i) v[i] = load(i);
#pragma unroll
        for (int i = 0; i < C::STEPS; ++i) add_squares<T>(s, v[i]);
        return;
    }
    u32x4 rest = {};
    if (c.rest() >= 0) rest[0] = word_of(p[c.rest()]);
    for (int k = 0; k < C::STEPS && C::at(k) - C::at(0) < c.n; k += 4) {
        u32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = u32x4{};
            if (c.has(k + i)) v[i] = load(k + i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) add_squares<T>(s, v[i]);
    }
    add_squares<T>(s, rest);
}

template <bool STREAM, typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* o, int64_t count, int within, float f) {
    using C = Chunk<T>;
    using V = typename Vec<T>::type;
    const C c(count, within);
    const T* p = global(g) + c.first;
    T* q = global(o) + c.first;
    auto load = [&](int i) {
        const typename Vec<T>::loaded v = __builtin_nontemporal_load(reinterpret_cast<const V*>(p + C::at(i)));
        return __builtin_bit_cast(u32x4, v);
    };
    auto store = [&](int i, u32x4 v) {
        V* at = reinterpret_cast<V*>(q + C::at(i));
        const auto w = __builtin_bit_cast(typename Vec<T>::loaded, v);
        if constexpr (STREAM) __builtin_nontemporal_store((V)w, at);
        else *at = w;
    };
    if (c.whole()) {
        u32x4 v[C::STEPS];
#pragma unroll
        for (int i = 0; i < C::STEPS; ++i) v[i] = load(i);
#pragma unroll
        for (int i = 0; i < C::STEPS; ++i) store(i, times<T>(v[i], f));
        return;
    }
    const int rest = c.rest();
    u32x4 last = {};
    if (rest >= 0) last[0] = word_of(p[rest]);
    for (int k = 0; k < C::STEPS && C::at(k) - C::at(0) < c.n; k += 4) {
        u32x4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = u32x4{};
            if (c.has(k + i)) v[i] = load(k + i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c.has(k + i)) store(k + i, times<T>(v[i], f));
    }
    if (rest >= 0) {
        const uint32_t w = times<T>(last, f)[0];
        if constexpr (sizeof(T) == 4) q[rest] = bits(w);
        else q[rest] = (u16)w;
    }
}

__global__ __launch_bounds__(64) void grad_table_kernel(GradList l, GradTable table) {
    int before = l.first;
    for (int k0 = 0; k0 < l.n; k0 += 64) {
        const int k = k0 + threadIdx.x, chunks = k < l.n ? l.t[k].chunks() : 0, v = before + scan64(chunks);
        if (k < l.n) {
            table.t[l.at + k] = l.t[k];
            table.first[l.at + k] = v - chunks;
        }
        before = __builtin_amdgcn_readlane(v, 63);
    }
}

// Sum of the partial sums in a fixed order (all 256 threads get it).
__device__ __forceinline__ float norm_of(const double* part, int parts, double* sh) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    return (float)sqrt(block_sum64(s, sh));
}

// part[b]: workgroup b's sum of squares.  A single workgroup writes the norm itself, where that is what is asked for.
template <bool TABLE>
__global__ __launch_bounds__(256) void grad_squares_kernel(GradList l, GradTable table, int n, int chunks, int keep, double* part,
                                                           float* norm) {
    __shared__ double sh[4];
    __shared__ int firsts[TABLE ? GRAD_FIRSTS : 1];
    const Tensors<TABLE> ts(l, table, n, firsts);
    double s[2] = {0.0, 0.0};
    for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
        int within;
        const GradTensor t = ts.of(c, within);
        if (c >= keep) {
            if (t.bf16()) chunk_squares<true>((const u16*)t.g, t.count(), within, s);
            else chunk_squares<true>((const float*)t.g, t.count(), within, s);
        } else {
            if (t.bf16()) chunk_squares<false>((const u16*)t.g, t.count(), within, s);
            else chunk_squares<false>((const float*)t.g, t.count(), within, s);
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
// the 256 MB infinity cache.  STREAM: what is written does not go there (it would only push out what is still to be read; eight
// shards of 4000 x 4096 into other tensors: 300 -> 273 us).
template <bool TABLE, bool STREAM>
__global__ __launch_bounds__(256) void grad_scale_kernel(GradList l, GradTable table, int n, int chunks, int in_place,
                                                         const double* part, int parts, float max_norm, float* norm) {
    __shared__ double sh[4];
    __shared__ int firsts[TABLE ? GRAD_FIRSTS : 1];
    const Tensors<TABLE> ts(l, table, n, firsts);      // (their first chunks arrive while the norm does)
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
        int within;
        const GradTensor t = ts.of(c, within);
        if (t.bf16()) chunk_scale<STREAM>((const u16*)t.g, (u16*)t.o, t.count(), within, f);
        else chunk_scale<STREAM>((const float*)t.g, (float*)t.o, t.count(), within, f);
    }
}

struct GradCall {
    const void* const* grads;
    const int64_t* counts;
    const int32_t* dts;
    int32_t n;
    void* const* outs;
    float max_norm;
    bool known;
    float* norm;
    double* part;
    GradTable table;
    hipStream_t st;
};

template <bool TABLE, bool STREAM>
hipError_t launch_grad_call(const GradCall& a) {
    GradList l;
    l.n = l.at = l.first = 0;
    int64_t chunks = 0;
    for (int32_t k = 0; k < a.n; ++k) {
        const GradTensor t{a.grads[k], a.outs ? a.outs[k] : const_cast<void*>(a.grads[k]),
                           (uint64_t)a.counts[k] * 2 + (a.dts[k] == VP_BF16 ? 1 : 0)};
        l.t[l.n++] = t;
        chunks += t.chunks();
        if (TABLE && (l.n == GRAD_LIST || k == a.n - 1)) {
            ProfScope prof(a.known ? K_GRAD_SCALE : K_GRAD_NORM, a.st);
            hipLaunchKernelGGL(grad_table_kernel, dim3(1), dim3(64), 0, a.st, l, a.table);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            l.at = k + 1;
            l.first = (int)chunks;
            l.n = 0;
        }
    }
    const int blocks = chunks < 1 ? 1 : chunks < GRAD_BLOCKS ? (int)chunks : GRAD_BLOCKS;
    if (!a.known) {
        ProfScope prof(K_GRAD_NORM, a.st);
        const bool alone = a.max_norm < 0.f;
        hipLaunchKernelGGL((grad_squares_kernel<TABLE>), dim3(blocks), dim3(256), 0, a.st, l, a.table, a.n, (int)chunks,
                           (int)(alone ? chunks : chunks - GRAD_KEEP), a.part, alone ? a.norm : nullptr);
        if (alone && blocks > 1) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, a.st, a.part, blocks, a.norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || alone) return e;
    }
    ProfScope prof(K_GRAD_SCALE, a.st);
    hipLaunchKernelGGL((grad_scale_kernel<TABLE, STREAM>), dim3(blocks), dim3(256), 0, a.st, l, a.table, a.n, (int)chunks,
                       a.outs == nullptr, a.part, a.known ? 0 : blocks, a.max_norm, a.norm);
    return hipGetLastError();
}

}  // namespace

size_t grad_workspace(int32_t n) {
    return GRAD_BLOCKS * sizeof(double) + (n > GRAD_LIST ? align_up((size_t)n * (sizeof(GradTensor) + sizeof(int)), 256) : 0);
}

hipError_t launch_grad(const void* const* grads, const int64_t* counts, const int32_t* dts, int32_t n, void* const* outs,
                       float max_norm, bool known, float* norm, void* workspace, hipStream_t st) {
    int64_t bytes = 0;
    for (int32_t k = 0; k < n; ++k) bytes += counts[k] * (dts[k] == VP_BF16 ? 2 : 4);
    double* part = (double*)workspace;
    GradTensor* table = (GradTensor*)(part + GRAD_BLOCKS);
    const GradCall a{grads, counts, dts, n, outs, max_norm, known, norm, part, GradTable{table, (int*)(table + n)}, st};
    const bool stream = bytes > (int64_t)128 << 20;
    if (n > GRAD_LIST) return stream ? launch_grad_call<true, true>(a) : launch_grad_call<true, false>(a);
    return stream ? launch_grad_call<false, true>(a) : launch_grad_call<false, false>(a);
}

}  // namespace vp
