// The norms before and after a block of the model with its gate and residual scale, forward and backward (vp.h has the
// formulas).  Bound by HBM: the forward call reads x and y and writes r and H, the backward call reads dH, dr, r and y and
// writes dx and dy, each once if a row stays on the chip between the sums over it and their use.
#include "vp_internal.h"

namespace vp {

namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(u16* p, float v) {
    const __bf16 b = (__bf16)v;
    *p = __builtin_bit_cast(u16, b);
}
// A vector's element, or what an absent one stands for.
template <typename T>
__device__ __forceinline__ float ld_or(const T* p, int j, float absent) { return p ? ld(p + j) : absent; }

// Sums of K values over the workgroup (1024 threads), a fixed tree; sh: K * 16 floats.
template <int K>
__device__ __forceinline__ void block_sums(float* v, float* sh) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < K; ++k) sh[k * 16 + (threadIdx.x >> 6)] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += sh[k * 16 + i];
        v[k] = s;
    }
}

struct Normed {
    float m, rho;
};
// Mean and 1 / deviation of a row whose elements f(j) gives: squares of differences to the mean, which has been summed first.
template <typename F>
__device__ __forceinline__ Normed statistics(F f, int h, int center, float eps, float* sh) {
    Normed n{0.f, 0.f};
    float s;
    if (center) {
        s = 0.f;
        for (int j = threadIdx.x; j < h; j += 1024) s += f(j);
        block_sums<1>(&s, sh);
        n.m = s / h;
    }
    s = 0.f;
    for (int j = threadIdx.x; j < h; j += 1024) {
        const float d = f(j) - n.m;
        s += d * d;
    }
    block_sums<1>(&s, sh);
    n.rho = 1.f / sqrtf(s / h + eps);
    return n;
}

// Rows of any length: a workgroup per row, which is read again for every sum over it.
template <typename T>
__global__ __launch_bounds__(1024) void block_norm_fwd_long_kernel(BlockNorm p) {
    __shared__ float sh[16];
    for (int i = blockIdx.x; i < p.N; i += gridDim.x) {
        const size_t row = (size_t)i * p.h;
        const T *x = (const T*)p.x + row, *y = p.y ? (const T*)p.y + row : nullptr;
        const T* gate = p.gate ? (const T*)p.gate + (size_t)((int64_t)i * p.gate_rows / p.N) * p.h : nullptr;
        Normed a{0.f, 1.f};
        if (p.post) a = statistics([&](int j) { return ld(y + j); }, p.h, p.center, p.eps, sh);
        auto sum = [&](int j) {
            float v = ld(x + j);
            if (!y) return v;
            float u = ld(y + j);
            if (p.post) u = (u - a.m) * a.rho * ld_or((const T*)p.w_post, j, 1.f) + ld_or((const T*)p.b_post, j, 0.f);
            return v + p.scale * ld_or(gate, j, 1.f) * u;
        };
        const Normed n = statistics(sum, p.h, p.center, p.eps, sh);
        for (int j = threadIdx.x; j < p.h; j += 1024) {
            const float v = sum(j);
            if (p.r) put((T*)p.r + row + j, v);
            put((T*)p.H + row + j, (v - n.m) * n.rho * ld_or((const T*)p.w, j, 1.f) + ld_or((const T*)p.b, j, 0.f));
        }
        if (p.stats && threadIdx.x == 0) {
            p.stats[i] = a.m;
            p.stats[(size_t)p.N + i] = a.rho;
            p.stats[2 * (size_t)p.N + i] = n.m;
            p.stats[3 * (size_t)p.N + i] = n.rho;
        }
    }
}

// ---- backward

// The sums over tokens: rows are cut into `chunks` ranges of `each` rows.  A range's sums go to row c of the partial matrices,
// which a last launch adds up in order; with a single range they go to the results themselves.
// dgate: a row of the gate whose tokens lie in one range is written where it ends; one that continues in the next range goes to
// row c of `tail`, one that began before (and ends or continues) to row c of `head`.
struct ColumnSums {
    float *dw, *db, *dw_post, *db_post, *head, *tail;
    int chunks, each;
};

// What the formulas need of a row.
template <typename T, typename TD, typename TG>
struct Row {
    const T *r, *y, *gate;
    const TD* dH;
    const TG* dr;
    float m1, rho1, m2, rho2;
    __device__ Row(const BlockNormGrad& p, int i) {
        const size_t row = (size_t)i * p.h;
        r = (const T*)p.r + row;
        y = p.y ? (const T*)p.y + row : nullptr;
        gate = p.gate ? (const T*)p.gate + (size_t)((int64_t)i * p.gate_rows / p.N) * p.h : nullptr;
        dH = (const TD*)p.dH + row;
        dr = p.dr ? (const TG*)p.dr + row : nullptr;
        m1 = p.stats[i];
        rho1 = p.stats[(size_t)p.N + i];
        m2 = p.stats[2 * (size_t)p.N + i];
        rho2 = p.stats[3 * (size_t)p.N + i];
    }
    __device__ float rh(int j) const { return (ld(r + j) - m2) * rho2; }
    __device__ float yh(int j) const { return (ld(y + j) - m1) * rho1; }
    __device__ float a(const BlockNormGrad& p, int j) const { return ld(dH + j) * ld_or((const T*)p.w, j, 1.f); }
    // dx, from the means of a and a rh
    __device__ float g(const BlockNormGrad& p, int j, float ma, float mar) const {
        return ld_or(dr, j, 0.f) + rho2 * (a(p, j) - ma - rh(j) * mar);
    }
    __device__ float d(const BlockNormGrad& p, int j, float g) const { return p.scale * ld_or(gate, j, 1.f) * g; }
};

// Rows of any length, first step: the means of a, a rh, c and c yh of every row.
template <typename T, typename TD, typename TG>
__global__ __launch_bounds__(1024) void block_norm_bwd_means_kernel(BlockNormGrad p, float4* means) {
    __shared__ float sh[32];
    for (int i = blockIdx.x; i < p.N; i += gridDim.x) {
        const Row<T, TD, TG> q(p, i);
        float s[2] = {0.f, 0.f}, c[2] = {0.f, 0.f};
        for (int j = threadIdx.x; j < p.h; j += 1024) {
            const float a = q.a(p, j);
            s[0] += a;
            s[1] += a * q.rh(j);
        }
        block_sums<2>(s, sh);
        const float ma = p.center ? s[0] / p.h : 0.f, mar = s[1] / p.h;
        if (p.post) {
            for (int j = threadIdx.x; j < p.h; j += 1024) {
                const float v = q.d(p, j, q.g(p, j, ma, mar)) * ld_or((const T*)p.w_post, j, 1.f);
                c[0] += v;
                c[1] += v * q.yh(j);
            }
            block_sums<2>(c, sh);
        }
        if (threadIdx.x == 0) means[i] = make_float4(ma, mar, p.center ? c[0] / p.h : 0.f, c[1] / p.h);
    }
}

// Second step: the sums over tokens, a thread per column and range of rows.
template <typename T, typename TD, typename TG>
__global__ __launch_bounds__(256) void block_norm_bwd_columns_kernel(BlockNormGrad p, const float4* means, ColumnSums s) {
    const int j = blockIdx.x * 256 + threadIdx.x, c = blockIdx.y;
    if (j >= p.h) return;
    const int i0 = c * s.each, i1 = i0 + s.each < p.N ? i0 + s.each : p.N;
    const int L = p.gate_rows ? (int)(p.N / p.gate_rows) : 0;
    const float wp = ld_or((const T*)p.w_post, j, 1.f), bp = ld_or((const T*)p.b_post, j, 0.f);
    float dw = 0.f, db = 0.f, dwp = 0.f, dbp = 0.f, dg = 0.f;
    for (int i = i0; i < i1; ++i) {
        const Row<T, TD, TG> q(p, i);
        const float4 m = means[i];
        const float dH = ld(q.dH + j), g = q.g(p, j, m.x, m.y);
        dw += dH * q.rh(j);
        db += dH;
        if (p.post) {
            const float d = q.d(p, j, g);
            dwp += d * q.yh(j);
            dbp += d;
        }
        if (p.dgate) {
            dg += p.scale * (p.post ? q.yh(j) * wp + bp : ld(q.y + j)) * g;
            const int k = i / L;
            if ((i + 1) % L == 0 || i + 1 == i1) {
                if (k * L < i0) s.head[(size_t)c * p.h + j] = dg;
                else if ((i + 1) % L == 0) p.dgate[(size_t)k * p.h + j] = dg;
                else s.tail[(size_t)c * p.h + j] = dg;
                dg = 0.f;
            }
        }
    }
    const size_t o = (size_t)c * p.h + j;
    if (p.dw) s.dw[o] = dw;
    if (p.db) s.db[o] = db;
    if (p.dw_post) s.dw_post[o] = dwp;
    if (p.db_post) s.db_post[o] = dbp;
}

// Third step: dx and dy.
template <typename T, typename TD, typename TG>
__global__ __launch_bounds__(1024) void block_norm_bwd_rows_kernel(BlockNormGrad p, const float4* means) {
    for (int i = blockIdx.x; i < p.N; i += gridDim.x) {
        const Row<T, TD, TG> q(p, i);
        const float4 m = means[i];
        TG *dx = (TG*)p.dx + (size_t)i * p.h, *dy = p.dy ? (TG*)p.dy + (size_t)i * p.h : nullptr;
        for (int j = threadIdx.x; j < p.h; j += 1024) {
            const float g = q.g(p, j, m.x, m.y);
            if (dy) {
                float d = q.d(p, j, g);
                if (p.post) d = q.rho1 * (d * ld_or((const T*)p.w_post, j, 1.f) - m.z - q.yh(j) * m.w);
                put(dy + j, d);
            }
            put(dx + j, g);
        }
    }
}

// Last step: the ranges' partial sums of dw, db, dw_post and db_post (blockIdx.y 0 .. 3), and of the rows of the gate whose
// tokens lie in several ranges (blockIdx.y - 4).
__global__ __launch_bounds__(256) void block_norm_bwd_sum_kernel(BlockNormGrad p, ColumnSums s) {
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= p.h) return;
    for (int64_t what = blockIdx.y; what < 4 + p.gate_rows; what += gridDim.y) {
        if (what < 4) {
            const float* part = what == 0 ? s.dw : what == 1 ? s.db : what == 2 ? s.dw_post : s.db_post;
            float* out = what == 0 ? p.dw : what == 1 ? p.db : what == 2 ? p.dw_post : p.db_post;
            if (!out) continue;
            float v = 0.f;
            for (int c = 0; c < s.chunks; ++c) v += part[(size_t)c * p.h + j];
            out[j] = v;
        } else if (p.dgate) {
            const int64_t k = what - 4, L = p.N / p.gate_rows;
            const int c0 = (int)(k * L / s.each), c1 = (int)(((k + 1) * L - 1) / s.each);
            if (c0 == c1) continue;      // written already
            // (one that begins with its first range and fills it has not begun before that range)
            float v = s.tail[(size_t)c0 * p.h + j];
            for (int c = c0 + 1; c <= c1; ++c) v += s.head[(size_t)c * p.h + j];
            p.dgate[(size_t)k * p.h + j] = v;
        }
    }
}

// Ranges of rows whose sums are kept apart: enough to fill the chip with a column per thread, and partial matrices of 16 MB at most.
int long_chunks(int64_t N, int64_t h) {
    int64_t c = ((int64_t)1 << 22) / h;
    c = c < 1 ? 1 : c > 512 ? 512 : c;
    return (int)(c < N ? c : N);
}

constexpr int MAX_ROW_BLOCKS = 1 << 16;

}  // namespace

hipError_t launch_block_norm_fwd(const BlockNorm& p, vp_dtype dt, hipStream_t st) {
    ProfScope prof(K_BLOCK_NORM_FWD, st);
    const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
    if (dt == VP_BF16) hipLaunchKernelGGL(block_norm_fwd_long_kernel<u16>, dim3(blocks), dim3(1024), 0, st, p);
    else hipLaunchKernelGGL(block_norm_fwd_long_kernel<float>, dim3(blocks), dim3(1024), 0, st, p);
    return hipGetLastError();
}

size_t block_norm_bwd_workspace(int64_t N, int64_t h, int64_t gate_rows, bool post) {
    const int kinds = 2 + (post ? 2 : 0) + (gate_rows ? 2 : 0);
    return align_up((size_t)N * sizeof(float4), 256) + align_up((size_t)kinds * long_chunks(N, h) * h * sizeof(float), 256);
}

template <typename T, typename TD, typename TG>
static hipError_t launch_bwd(const BlockNormGrad& p, void* workspace, hipStream_t st) {
    float4* means = (float4*)workspace;
    float* part = (float*)((char*)workspace + align_up((size_t)p.N * sizeof(float4), 256));
    ColumnSums s{};
    s.chunks = long_chunks(p.N, p.h);
    s.each = (int)ceil_div(p.N, s.chunks);
    s.chunks = (int)ceil_div(p.N, s.each);
    const size_t m = (size_t)s.chunks * p.h;
    s.dw = s.chunks > 1 ? part : p.dw;
    s.db = s.chunks > 1 ? part + m : p.db;
    part += 2 * m;
    s.dw_post = s.chunks > 1 ? part : p.dw_post;
    s.db_post = s.chunks > 1 ? part + m : p.db_post;
    if (p.post) part += 2 * m;
    s.head = part;
    s.tail = part + m;
    const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
    const unsigned cols = (unsigned)ceil_div(p.h, 256);
    const bool sums = p.dw || p.db || p.dw_post || p.db_post || p.dgate;
    hipLaunchKernelGGL((block_norm_bwd_means_kernel<T, TD, TG>), dim3(blocks), dim3(1024), 0, st, p, means);
    // (before dx is written: it may be dr)
    if (sums) hipLaunchKernelGGL((block_norm_bwd_columns_kernel<T, TD, TG>), dim3(cols, s.chunks), dim3(256), 0, st, p, means, s);
    hipLaunchKernelGGL((block_norm_bwd_rows_kernel<T, TD, TG>), dim3(blocks), dim3(1024), 0, st, p, means);
    if (sums && s.chunks > 1) {
        const int64_t what = 4 + (p.dgate ? p.gate_rows : 0);
        hipLaunchKernelGGL(block_norm_bwd_sum_kernel, dim3(cols, (unsigned)(what < 65535 ? what : 65535)), dim3(256), 0, st, p, s);
    }
    return hipGetLastError();
}

hipError_t launch_block_norm_bwd(const BlockNormGrad& p, vp_dtype dt, vp_dtype dH_dt, vp_dtype grad_dt, void* workspace,
                                 hipStream_t st) {
    ProfScope prof(K_BLOCK_NORM_BWD, st);
    if (dt == VP_F32) return launch_bwd<float, float, float>(p, workspace, st);
    if (dH_dt == VP_F32)
        return grad_dt == VP_F32 ? launch_bwd<u16, float, float>(p, workspace, st) : launch_bwd<u16, float, u16>(p, workspace, st);
    return grad_dt == VP_F32 ? launch_bwd<u16, u16, float>(p, workspace, st) : launch_bwd<u16, u16, u16>(p, workspace, st);
}

}  // namespace vp
