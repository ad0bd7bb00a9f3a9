// The output layer's logits from 8-bit integers, Y_ij = s_i t_j sum_k H_ik W_jk, with the shard-local softmax statistics.
#include "vp_internal.h"

namespace vp {

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));
typedef int intx16 __attribute__((ext_vector_type(16)));
constexpr float LOG2E = 1.44269504088896340736f;

// 32 tokens and a tile column (256 vocabulary rows) per workgroup, 64 of them per wavefront, operands from global memory.
// With W first, register r of lane l holds token l % 32 and column 8 (r / 4) + 4 (l / 32) + r % 4 of a 32 x 32 product.
__global__ __launch_bounds__(256) void gemm_i8_kernel(GemmI8Group g) {
    __shared__ float xm[4][32], xs[4][32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, hf = lane >> 5;
    int sh = 0;
    for (int i = 1; i < g.n; ++i) sh += (int)blockIdx.x >= g.first[i];
    const GemmI8Shard& s = g.sh[sh];
    const int n0 = ((int)blockIdx.x - g.first[sh]) * GEMM_BN + wave * 64;
    const int m = blockIdx.y * 32 + l32, mc = m < g.N ? m : g.N - 1;
    const int8_t* a = g.H + (size_t)mc * g.k + hf * 16;
    const int8_t* b[2];
    for (int j = 0; j < 2; ++j) {
        const int n = n0 + j * 32 + l32;
        b[j] = s.W + (size_t)(n < s.rows ? n : s.rows - 1) * g.k + hf * 16;
    }
    intx16 acc[2] = {};
    for (int k = 0; k < g.k; k += 32) {
        const intx4 av = *reinterpret_cast<const intx4*>(a + k);
        for (int j = 0; j < 2; ++j)
            acc[j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(*reinterpret_cast<const intx4*>(b[j] + k), av, acc[j], 0, 0, 0);
    }
    const float rs = g.scales[mc];
    const int64_t label = g.labels[mc] - s.offset;
    float y[32], mx = -INFINITY;
    for (int e = 0; e < 32; ++e) {
        const int col = n0 + (e >> 4) * 32 + 8 * ((e & 15) >> 2) + 4 * hf + (e & 3);
        y[e] = -INFINITY;
        if (col >= s.rows) continue;
        y[e] = (float)acc[e >> 4][e & 15] * s.scales[col] * rs;
        mx = fmaxf(mx, y[e]);
        if (m >= g.N) continue;
        if (col == label) g.part_tgt[(size_t)sh * g.N + m] = y[e];
        if (s.out) {
            const size_t at = (size_t)m * s.rows + col;
            if (g.out_f32) ((float*)s.out)[at] = y[e];
            else ((u16*)s.out)[at] = __builtin_bit_cast(u16, (__bf16)y[e]);
        }
    }
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    float sum = 0.f;
    for (int e = 0; e < 32; ++e) sum += __builtin_amdgcn_exp2f((y[e] - mx) * LOG2E);
    sum += __shfl_xor(sum, 32, 64);
    if (hf == 0) {
        xm[wave][l32] = mx;
        xs[wave][l32] = sum;
    }
    __syncthreads();
    if (threadIdx.x >= 32 || m >= g.N) return;
    mx = fmaxf(fmaxf(xm[0][l32], xm[1][l32]), fmaxf(xm[2][l32], xm[3][l32]));
    sum = 0.f;
    for (int w = 0; w < 4; ++w)
        if (xm[w][l32] > -INFINITY) sum += xs[w][l32] * __expf(xm[w][l32] - mx);
    g.part_max[(size_t)blockIdx.x * g.N + m] = mx;
    g.part_sum[(size_t)blockIdx.x * g.N + m] = sum;
}

}  // namespace

hipError_t launch_gemm_i8(const GemmI8Group& g, hipStream_t st) {
    ProfScope prof(K_GEMM_I8, st);
    // (a launch has at most 65535 blocks along its second dimension)
    constexpr int64_t MOST = 65535 * 32;
    for (int64_t m0 = 0; m0 < g.N; m0 += MOST) {
        if (m0) return hipErrorInvalidValue;
        hipLaunchKernelGGL(gemm_i8_kernel, dim3(g.total, (unsigned)ceil_div(g.N, 32)), dim3(256), 0, st, g);
    }
    return hipGetLastError();
}

}  // namespace vp
