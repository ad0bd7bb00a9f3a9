// Rows of a matrix in 8-bit integers: scale max |x| / 127 of each row, elements 127 x / max |x| to the nearest integer.
//
// Bound by HBM: every element is read once and its integer written once if a row stays in registers between the search for its
// maximum and the division (16000 x 8192 bf16: 98 us, 4.0 TB/s; 16032 x 4096 fp32: 69 us, 4.8 TB/s); a token's by the launch (3.8 us).
//
// The integer is that of the exact quotient (ties to even).  In fp64 it is: 127 x has at most 24 + 7 bits, so it is exact, and a
// quotient of it by a number of 24 bits that is no half integer is further from one than fp64 rounds.  Almost all elements need no
// fp64 (with a division in fp64 for each, 256 x 8192 bf16 took 23 us in place of 6.3): with r = fl(127 / max) the product t = fl(x r) is off by less than 127 (2^-24 + 2^-24) < 2^-16, so its nearest integer is
// the quotient's unless t is within 2^-15 of a half integer.
#include "vp_internal.h"

namespace vp {

namespace {

constexpr int E = 16;      // columns of a vector: 16 bytes of integers
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef unsigned u32x4u __attribute__((ext_vector_type(4), aligned(1)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }

// Sixteen columns as they are stored.  Rows start at any element, and so do vectors.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
    f32x4u v[4];
    __device__ __forceinline__ void load(const float* p) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = reinterpret_cast<const f32x4u*>(p)[k];
    }
    __device__ __forceinline__ void set(int e, float f) { v[e >> 2][e & 3] = f; }
    __device__ __forceinline__ float operator[](int e) const { return v[e >> 2][e & 3]; }
    // largest |x| in bits: they are ordered like the numbers, infinities and NaN above all others
    __device__ __forceinline__ unsigned largest() const {
        unsigned a = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) a = max(a, __float_as_uint((*this)[e]) & 0x7fffffffu);
        return a;
    }
};
template <>
struct Raw<u16> {
    u16x8u v[2];
    __device__ __forceinline__ void load(const u16* p) {
        v[0] = reinterpret_cast<const u16x8u*>(p)[0];
        v[1] = reinterpret_cast<const u16x8u*>(p)[1];
    }
    __device__ __forceinline__ void set(int e, float f) { v[e >> 3][e & 7] = (u16)(__float_as_uint(f) >> 16); }
    __device__ __forceinline__ float operator[](int e) const { return __uint_as_float((unsigned)v[e >> 3][e & 7] << 16); }
    __device__ __forceinline__ unsigned largest() const {
        const u16x8u a = __builtin_elementwise_max(v[0] & (u16)0x7fff, v[1] & (u16)0x7fff);
        unsigned m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, (unsigned)a[e]);
        return m << 16;
    }
};

// Vector k of a row of h columns: one that the row's end cuts is moved back to end there (it then holds columns of the one before,
// which changes neither the maximum nor their integers); in a row shorter than a vector the columns behind are zero.
template <typename T>
__device__ __forceinline__ void load_vector(Raw<T>& x, const T* row, int k, int h) {
    if (h >= E) {
        x.load(row + min(k * E, h - E));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) x.set(e, e < h ? ld(row + e) : 0.f);
    }
}

// What the row's largest |x| makes of its elements.
struct Scale {
    unsigned bits;
    float r, scale;
    bool small, none;      // 127 / max |x| is no fp32 number; all integers are 0
    __device__ explicit Scale(unsigned bits) : bits(bits) {
        const float a = __uint_as_float(bits);
        none = bits == 0 || bits >= 0x7f800000u;
        small = a < 0x1p-118f;
        r = small ? 0.f : 127.f / a;
        scale = bits < 0x7f800000u ? a / 127.f : __uint_as_float(0x7fc00000u);
    }
    template <typename T>
    __device__ __forceinline__ u32x4 integers(const Raw<T>& x) const {
        int q[E];
        bool near = small;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float t = x[e] * r, n = __builtin_rintf(t);
            near |= fabsf(t - n) > 0.5f - 0x1p-15f;
            q[e] = (int)n;
        }
        if (near && !none) {
            const double a = __uint_as_float(bits);
#pragma unroll
            for (int e = 0; e < E; ++e) q[e] = (int)rint((double)x[e] * 127.0 / a);
        }
        u32x4 o;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            o[k] = none ? 0u : (q[4 * k] & 0xff) | (q[4 * k + 1] & 0xff) << 8 | (q[4 * k + 2] & 0xff) << 16 | q[4 * k + 3] << 24;
        return o;
    }
};

// Integers of vector k: all of its 16 columns of a row of integers, zero from column h on.
__device__ __forceinline__ void store_vector(int8_t* row, int k, int h, const u32x4& q) {
    if (k * E + E <= h || h < E) {
        *reinterpret_cast<u32x4*>(row + k * E) = k * E < h ? q : u32x4{};
        return;
    }
    // behind the last column zeros; then, by the same thread, the columns that a vector moved back ends with
    *reinterpret_cast<u32x4*>(row + k * E) = u32x4{};
    if (k * E < h) {
        asm volatile("" ::: "memory");
        *reinterpret_cast<u32x4u*>(row + h - E) = q;
    }
}

template <int LANES>
__device__ __forceinline__ unsigned max_over(unsigned a) {
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) a = max(a, (unsigned)__shfl_xor((int)a, o, 64));
    return a;
}
__device__ __forceinline__ unsigned max_over_group(unsigned a, unsigned* sh) {      // 256 threads
    a = max_over<64>(a);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = a;
    __syncthreads();
    return max(max(sh[0], sh[1]), max(sh[2], sh[3]));
}

// Rows of at most 16 TR C columns: TR threads hold a row in registers, C vectors each.
template <typename T, int TR, int C>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t N, int h, int stride, int8_t* __restrict__ q,
                                                            float* __restrict__ scales) {
    __shared__ unsigned sh[4];
    const int t = threadIdx.x % TR;
    const int64_t row = (int64_t)blockIdx.x * (256 / TR) + threadIdx.x / TR, i = row < N ? row : N - 1;
    Raw<T> v[C];
#pragma unroll
    for (int c = 0; c < C; ++c) load_vector(v[c], x + i * h, c * TR + t, h);
    unsigned a = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) a = max(a, v[c].largest());
    if constexpr (TR < 256) a = max_over<TR>(a);
    else a = max_over_group(a, sh);
    const Scale s(a);
    if (row >= N) return;
#pragma unroll
    for (int c = 0; c < C; ++c)
        if ((c * TR + t) * E < stride) store_vector(q + i * stride, c * TR + t, h, s.integers(v[c]));
    if (t == 0) scales[i] = s.scale;
}

// Longer rows: read twice.
template <typename T>
__global__ __launch_bounds__(256) void quantize_long_rows_kernel(const T* __restrict__ x, int h, int stride, int8_t* __restrict__ q,
                                                                 float* __restrict__ scales) {
    __shared__ unsigned sh[4];
    const int64_t i = blockIdx.x;
    unsigned a = 0;
    Raw<T> v;
    for (int k = threadIdx.x; k * E < h; k += 256) {
        load_vector(v, x + i * h, k, h);
        a = max(a, v.largest());
    }
    const Scale s(max_over_group(a, sh));
    for (int k = threadIdx.x; k * E < stride; k += 256) {
        load_vector(v, x + i * h, k, h);
        store_vector(q + i * stride, k, h, s.integers(v));
    }
    if (threadIdx.x == 0) scales[i] = s.scale;
}

template <typename T>
hipError_t launch(const T* x, int64_t N, int h, int8_t* q, float* scales, hipStream_t st) {
    const int stride = (int)i8_row_stride(h);
    auto rows = [&](auto kernel, int per_group) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(N, per_group)), dim3(256), 0, st, x, N, h, stride, q, scales);
    };
    if (stride <= 256) rows(quantize_rows_kernel<T, 16, 1>, 16);
    else if (stride <= 1024) rows(quantize_rows_kernel<T, 64, 1>, 4);
    else if (stride <= 4096) rows(quantize_rows_kernel<T, 256, 1>, 1);
    else if (stride <= 8192) rows(quantize_rows_kernel<T, 256, 2>, 1);
    else if (stride <= 16384) rows(quantize_rows_kernel<T, 256, 4>, 1);
    else hipLaunchKernelGGL(quantize_long_rows_kernel<T>, dim3((unsigned)N), dim3(256), 0, st, x, h, stride, q, scales);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int64_t N, int64_t h, vp_dtype dt, int8_t* q, float* scales, hipStream_t st) {
    ProfScope prof(K_QUANTIZE, st);
    return dt == VP_F32 ? launch((const float*)x, N, (int)h, q, scales, st) : launch((const u16*)x, N, (int)h, q, scales, st);
}

}  // namespace vp
