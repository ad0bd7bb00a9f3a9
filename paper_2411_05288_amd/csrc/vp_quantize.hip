// Rows of a matrix in 8-bit integers: scale max |x| / 127 of each row, elements 127 x / max |x| to the nearest integer.
//
// The integer is that of the exact quotient (ties to even): 127 x has at most 24 + 7 bits, so it is exact in fp64, and a quotient
// of it by a number of 24 bits that is no half integer is further from one than fp64 rounds.
#include "vp_internal.h"

namespace vp {

namespace {

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const T* __restrict__ x, int64_t N, int h, int stride, int8_t* q, float* scales) {
    __shared__ float sh[4];
    for (int64_t i = blockIdx.x; i < N; i += gridDim.x) {
        const T* row = x + i * h;
        unsigned a = 0;      // |x| in bits: ordered like the numbers, infinities and NaN above all others
        for (int j = threadIdx.x; j < h; j += 256) a = max(a, __float_as_uint(ld(row + j)) & 0x7fffffffu);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) a = max(a, (unsigned)__shfl_xor((int)a, o, 64));
        if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = __uint_as_float(a);
        __syncthreads();
        a = max(max(__float_as_uint(sh[0]), __float_as_uint(sh[1])), max(__float_as_uint(sh[2]), __float_as_uint(sh[3])));
        __syncthreads();
        const bool finite = a < 0x7f800000u;
        const float largest = __uint_as_float(a);
        if (threadIdx.x == 0) scales[i] = finite ? largest / 127.f : __uint_as_float(0x7fc00000u);
        for (int j = threadIdx.x; j < stride; j += 256) {
            double v = 0.0;
            if (j < h && finite && a != 0) v = rint((double)ld(row + j) * 127.0 / (double)largest);
            q[i * stride + j] = (int8_t)v;
        }
    }
}

}  // namespace

hipError_t launch_quantize_rows(const void* x, int64_t N, int64_t h, vp_dtype dt, int8_t* q, float* scales, hipStream_t st) {
    ProfScope prof(K_QUANTIZE, st);
    const int stride = (int)i8_row_stride(h);
    const dim3 grid((unsigned)(N < 65536 ? N : 65536));
    if (dt == VP_F32) hipLaunchKernelGGL(quantize_rows_kernel<float>, grid, dim3(256), 0, st, (const float*)x, N, (int)h, stride, q, scales);
    else hipLaunchKernelGGL(quantize_rows_kernel<u16>, grid, dim3(256), 0, st, (const u16*)x, N, (int)h, stride, q, scales);
    return hipGetLastError();
}

}  // namespace vp
