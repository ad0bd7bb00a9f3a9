// The norms before and after a block of the model with its gate and residual scale, forward and backward (vp.h has the
// formulas).  Bound by HBM: the forward call reads x and y and writes r and H, the backward call reads dH, dr, r and y and
// writes dx and dy, each once if a row stays on the chip between the sums over it and their use.
#include "vp_internal.h"

namespace vp {

namespace {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));
constexpr int K_ROW_SUMS = 32;      // two sums of 16 wavefronts

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

// Eight columns of a row as they are stored.  Rows of lengths that are no multiple of eight start at any element, so vectors are
// element-aligned (the hardware takes 16-byte accesses at any address); only the `n` < 8 columns that a row has left at its end
// go one by one.
template <typename T>
struct Raw8;
template <>
struct Raw8<u16> {
    u16x8u v;
    __device__ float operator[](int e) const { return __uint_as_float((unsigned)v[e] << 16); }
};
template <>
struct Raw8<float> {
    f32x4u a, b;
    __device__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
};
__device__ __forceinline__ void whole(Raw8<u16>& o, const u16* p) { o.v = *reinterpret_cast<const u16x8u*>(p); }
__device__ __forceinline__ void whole(Raw8<float>& o, const float* p) {
    o.a = *reinterpret_cast<const f32x4u*>(p);
    o.b = *reinterpret_cast<const f32x4u*>(p + 4);
}
__device__ __forceinline__ void set(Raw8<u16>& o, int e, u16 v) { o.v[e] = v; }
__device__ __forceinline__ void set(Raw8<float>& o, int e, float v) { if (e < 4) o.a[e] = v; else o.b[e - 4] = v; }
template <typename T>
__device__ __forceinline__ T bits_of(float v);
template <>
__device__ __forceinline__ float bits_of<float>(float v) { return v; }
template <>
__device__ __forceinline__ u16 bits_of<u16>(float v) {
    const __bf16 b = (__bf16)v;
    return __builtin_bit_cast(u16, b);
}
// `absent` where p is NULL; columns that the row does not have are 0.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int j, int n, float absent = 0.f) {
    Raw8<T> o;
    if (p && n >= 8) {
        whole(o, p + j);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) set(o, e, e < n ? (p ? p[j + e] : bits_of<T>(absent)) : bits_of<T>(0.f));
    }
    return o;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int j, int n, const float* v) {
    Raw8<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) set(o, e, bits_of<T>(v[e]));
    if (n >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u16x8u*>(p + j) = o.v;
        } else {
            *reinterpret_cast<f32x4u*>(p + j) = o.a;
            *reinterpret_cast<f32x4u*>(p + j + 4) = o.b;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n) put(p + j + e, v[e]);
    }
}

// Sums of K values over the TR threads of a row, a fixed tree.  Up to a wavefront: shuffles; more: a workgroup is one row, and
// the wavefronts meet in LDS, in the half of `sh` that `turn` names (so that one barrier per sum is enough).
template <int K, int TR>
__device__ __forceinline__ void row_sums(float* v, float (*sh)[K_ROW_SUMS], int& turn) {
    constexpr int W = TR < 64 ? TR : 64;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int o = W / 2; o > 0; o >>= 1) v[k] += __shfl_xor(v[k], o, 64);
    if constexpr (TR > 64) {
        constexpr int N = TR / 64;
        float* at = sh[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) at[k * N + (threadIdx.x >> 6)] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) s += at[k * N + i];
            v[k] = s;
        }
    }
}

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

// Rows of at most 8 C TR columns: TR threads hold a row in registers, C vectors of eight columns each, from the only read of x
// and y to the only write of r and H.
template <typename T, int TR, int C>
__global__ __launch_bounds__(TR < 128 ? 256 : TR) void block_norm_fwd_kernel(BlockNorm p) {
    __shared__ float sh[2][K_ROW_SUMS];
    int turn = 0;
    constexpr int ROWS = TR < 128 ? 256 / TR : 1;
    const int t = threadIdx.x % TR, row = blockIdx.x * ROWS + threadIdx.x / TR;
    const bool live = row < p.N;
    const int i = live ? row : p.N - 1;      // (a workgroup's rows past the last one take part in nothing but the sums)
    const size_t at = (size_t)i * p.h;
    const T *x = (const T*)p.x + at, *y = (const T*)p.y;
    const T* gate = p.gate ? (const T*)p.gate + (size_t)((int64_t)i * p.gate_rows / p.N) * p.h : nullptr;
    int n[C];
    Raw8<T> rx[C], ry[C], rg[C];
    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = (c * TR + t) * 8;
        n[c] = p.h - j < 0 ? 0 : p.h - j;
        rx[c] = load8(x, j, n[c]);
        if (y) ry[c] = load8(y + at, j, n[c]);
        if (gate) rg[c] = load8(gate, j, n[c]);
    }
    // the mean and the deviation of what v holds: squares of differences to the mean, which has been summed first
    auto statistics = [&]() {
        Normed m{0.f, 0.f};
        float s;
        if (p.center) {
            s = 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += v[c][e];      // (columns that do not exist hold 0)
            row_sums<1, TR>(&s, sh, turn);
            m.m = s / p.h;
        }
        s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = e < n[c] ? v[c][e] - m.m : 0.f;
                s += d * d;
            }
        row_sums<1, TR>(&s, sh, turn);
        m.rho = 1.f / sqrtf(s / p.h + p.eps);
        return m;
    };
    Normed a{0.f, 1.f};
    if (y) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = ry[c][e];
        if (p.post) a = statistics();
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = (c * TR + t) * 8;
        if (y && p.post) {
            const Raw8<T> w = load8((const T*)p.w_post, j, n[c], 1.f), b = load8((const T*)p.b_post, j, n[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = (v[c][e] - a.m) * a.rho * w[e] + b[e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = y ? rx[c][e] + (gate ? p.scale * rg[c][e] : p.scale) * v[c][e] : rx[c][e];
        if (p.r && live) store8((T*)p.r + at, j, n[c], v[c]);
    }
    const Normed m = statistics();
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = (c * TR + t) * 8;
        const Raw8<T> w = load8((const T*)p.w, j, n[c], 1.f), b = load8((const T*)p.b, j, n[c]);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (v[c][e] - m.m) * m.rho * w[e] + b[e];
        if (live) store8((T*)p.H + at, j, n[c], o);
    }
    if (p.stats && t == 0 && live) {
        p.stats[i] = a.m;
        p.stats[(size_t)p.N + i] = a.rho;
        p.stats[2 * (size_t)p.N + i] = m.m;
        p.stats[3 * (size_t)p.N + i] = m.rho;
    }
}

// ---- backward

// The sums over tokens: rows are cut into `chunks` ranges of `each` rows.  A range's sums go to row c of the partial matrices,
// which a last launch adds up in order; with a single range they go to the results themselves.
// dgate: a row of the gate whose tokens lie in one range is written where it ends; one that continues in the next range goes to
// row c of `tail`, one that began before (and ends or continues) to row c of `head`.
struct ColumnSums {
    float *dw, *db, *dw_post, *db_post, *head, *tail;
    int chunks, each, pitch;      // (rows of the partial matrices are `pitch` floats apart)
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
                if (k * L < i0) s.head[(size_t)c * s.pitch + j] = dg;
                else if ((i + 1) % L == 0) p.dgate[(size_t)k * p.h + j] = dg;
                else s.tail[(size_t)c * s.pitch + j] = dg;
                dg = 0.f;
            }
        }
    }
    const size_t o = (size_t)c * s.pitch + j;
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

// Rows of at most 8 C TR columns in one pass: a row's values stay in registers between the sums over it and dx and dy, and a
// thread's columns are the same in every row of its range, so the sums over tokens stay in registers too.
template <typename T, typename TD, typename TG, int TR, int C>
__global__ __launch_bounds__(TR < 128 ? 256 : TR) void block_norm_bwd_kernel(BlockNormGrad p, ColumnSums s) {
    __shared__ float sh[2][K_ROW_SUMS];
    int turn = 0;
    constexpr int ROWS = TR < 128 ? 256 / TR : 1;
    const int t = threadIdx.x % TR, c0 = blockIdx.x * ROWS + threadIdx.x / TR;
    const int i0 = c0 * s.each, i1 = i0 + s.each < p.N ? i0 + s.each : p.N;
    if (c0 >= s.chunks) return;      // (a workgroup of several rows has no barriers)
    const int L = p.gate_rows ? (int)(p.N / p.gate_rows) : 0;
    const float inv_h = 1.f / p.h;
    int n[C];
    Raw8<T> w[C], wp[C], bp[C];
    float dw[C][8], db[C][8], dwp[C][8], dbp[C][8], dg[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = (c * TR + t) * 8;
        n[c] = p.h - j < 0 ? 0 : p.h - j;
        w[c] = load8((const T*)p.w, j, n[c], 1.f);
        wp[c] = load8((const T*)p.w_post, j, n[c], 1.f);
        bp[c] = load8((const T*)p.b_post, j, n[c]);
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = db[c][e] = dwp[c][e] = dbp[c][e] = dg[c][e] = 0.f;
    }
    for (int i = i0; i < i1; ++i) {
        const size_t at = (size_t)i * p.h;
        const float m1 = p.stats[i], rho1 = p.stats[(size_t)p.N + i], m2 = p.stats[2 * (size_t)p.N + i], rho2 = p.stats[3 * (size_t)p.N + i];
        Raw8<TD> qd[C];
        Raw8<TG> qr[C];
        Raw8<T> rr[C], ry[C], rg[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * TR + t) * 8;
            qd[c] = load8((const TD*)p.dH + at, j, n[c]);
            rr[c] = load8((const T*)p.r + at, j, n[c]);
            qr[c] = load8(p.dr ? (const TG*)p.dr + at : nullptr, j, n[c]);
            ry[c] = load8(p.y ? (const T*)p.y + at : nullptr, j, n[c]);
            rg[c] = load8(p.gate ? (const T*)p.gate + (size_t)(i / L) * p.h : nullptr, j, n[c], 1.f);
        }
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float dH = qd[c][e], rh = (rr[c][e] - m2) * rho2, a = dH * w[c][e];
                dw[c][e] += dH * rh;
                db[c][e] += dH;
                sums[0] += a;
                sums[1] += a * rh;
            }
        row_sums<2, TR>(sums, sh, turn);
        const float ma = p.center ? sums[0] * inv_h : 0.f, mar = sums[1] * inv_h;
        float g[C][8];
        float more[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int j = (c * TR + t) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                g[c][e] = qr[c][e] + rho2 * (qd[c][e] * w[c][e] - ma - (rr[c][e] - m2) * rho2 * mar);
            store8((TG*)p.dx + at, j, n[c], g[c]);
            if (p.y) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float yh = (ry[c][e] - m1) * rho1;
                    dg[c][e] += p.scale * (yh * wp[c][e] + bp[c][e]) * g[c][e];
                    const float d = p.scale * rg[c][e] * g[c][e];
                    dwp[c][e] += d * yh;
                    dbp[c][e] += d;
                    // (0 in columns that do not exist, whose weight is 0)
                    g[c][e] = d * wp[c][e];
                    more[0] += g[c][e];
                    more[1] += g[c][e] * yh;
                }
            }
        }
        if (p.y) {
            if (p.post) row_sums<2, TR>(more, sh, turn);
            const float mk = p.center ? more[0] * inv_h : 0.f, mky = more[1] * inv_h;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int j = (c * TR + t) * 8;
                if (p.post)
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[c][e] = rho1 * (g[c][e] - mk - (ry[c][e] - m1) * rho1 * mky);
                store8((TG*)p.dy + at, j, n[c], g[c]);
            }
        }
        if (p.dgate && ((i + 1) % L == 0 || i + 1 == i1)) {
            const int k = i / L;
            float* o = k * L < i0 ? s.head + (size_t)c0 * s.pitch
                                  : (i + 1) % L == 0 ? p.dgate + (size_t)k * p.h : s.tail + (size_t)c0 * s.pitch;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                store8(o, (c * TR + t) * 8, n[c], dg[c]);
#pragma unroll
                for (int e = 0; e < 8; ++e) dg[c][e] = 0.f;
            }
        }
    }
    const size_t o = (size_t)c0 * s.pitch;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = (c * TR + t) * 8;
        if (p.dw) store8(s.dw + o, j, n[c], dw[c]);
        if (p.db) store8(s.db + o, j, n[c], db[c]);
        if (p.dw_post) store8(s.dw_post + o, j, n[c], dwp[c]);
        if (p.db_post) store8(s.db_post + o, j, n[c], dbp[c]);
    }
}

// Last step: the ranges' partial sums of dw, db, dw_post and db_post (blockIdx.y 0 .. 3), and of the rows of the gate whose
// tokens lie in several ranges (blockIdx.y - 4: the row, or, where the gate has more rows than there are ranges, the range in
// which it begins).  A workgroup takes 32 columns: eight threads of four columns side by side, 32 slices of the ranges.
__global__ __launch_bounds__(256) void block_norm_bwd_sum_kernel(BlockNormGrad p, ColumnSums s) {
    __shared__ float4 sh[32][8];
    const int slice = threadIdx.x >> 3, j = blockIdx.x * 32 + (threadIdx.x & 7) * 4, what = blockIdx.y;
    const float *first, *rest;      // the first range's row, and where the others lie
    float* out;
    int c0 = 0, c1 = s.chunks - 1;
    if (what < 4) {
        first = rest = what == 0 ? s.dw : what == 1 ? s.db : what == 2 ? s.dw_post : s.db_post;
        out = what == 0 ? p.dw : what == 1 ? p.db : what == 2 ? p.dw_post : p.db_post;
        if (!out) return;
    } else {
        const int64_t L = p.N / p.gate_rows;
        int64_t k = what - 4;
        if (p.gate_rows > s.chunks) {
            const int64_t end = k + 1 < s.chunks ? (k + 1) * s.each : p.N;
            if ((end - 1) / L * L < k * s.each) return;      // the row at the end of this range began before it
            k = (end - 1) / L;
        }
        c0 = (int)(k * L / s.each);
        c1 = (int)(((k + 1) * L - 1) / s.each);
        if (c0 == c1) return;      // written already
        first = s.tail;
        rest = s.head;
        out = p.dgate + k * p.h;
    }
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j < p.h)
        for (int c = c0 + slice; c <= c1; c += 32) {
            const float4 q = *reinterpret_cast<const float4*>((c == c0 ? first : rest) + (size_t)c * s.pitch + j);
            v.x += q.x;
            v.y += q.y;
            v.z += q.z;
            v.w += q.w;
        }
    sh[slice][threadIdx.x & 7] = v;
    __syncthreads();
    if (threadIdx.x < 32 && blockIdx.x * 32 + threadIdx.x < p.h) {
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < 32; ++q) sum += reinterpret_cast<const float*>(sh[q])[threadIdx.x];
        out[blockIdx.x * 32 + threadIdx.x] = sum;
    }
}

// Threads of a row that one pass holds in registers (0: rows that are too long for that).
int row_threads(int64_t h, int most) {
    int t = 16;
    while (t < most && t * 8 < h) t *= t < 64 ? 4 : 2;
    return t;
}

// Ranges of rows whose sums over tokens are kept apart.
// One pass: as many as fill the chip with TR threads each (partial matrices of 8 MB at most).
// Long rows: enough to fill it with a thread per column, and partial matrices of 16 MB at most.
constexpr int BWD_MAX_COLUMNS = 8192;
int ranges(int64_t N, int64_t h) {
    int64_t c = h <= BWD_MAX_COLUMNS ? (1 << 18) / row_threads(h, 1024) : ((int64_t)1 << 22) / h;
    if (h > BWD_MAX_COLUMNS) c = c < 1 ? 1 : c > 512 ? 512 : c;
    return (int)(c < N ? c : N);
}
int pitch_of(int64_t h) { return (int)((h + 3) / 4 * 4); }

constexpr int MAX_ROW_BLOCKS = 1 << 16;

}  // namespace

hipError_t launch_block_norm_fwd(const BlockNorm& p, vp_dtype dt, hipStream_t st) {
    ProfScope prof(K_BLOCK_NORM_FWD, st);
    const bool bf16 = dt == VP_BF16;
#define VP_FWD(TR, C)                                                                                                          \
    do {                                                                                                                       \
        const dim3 grid((unsigned)ceil_div(p.N, TR < 128 ? 256 / TR : 1)), block(TR < 128 ? 256 : TR);                         \
        if (bf16) hipLaunchKernelGGL((block_norm_fwd_kernel<u16, TR, C>), grid, block, 0, st, p);                              \
        else hipLaunchKernelGGL((block_norm_fwd_kernel<float, TR, C>), grid, block, 0, st, p);                                 \
        return hipGetLastError();                                                                                              \
    } while (0)
    switch (row_threads(p.h, 1024)) {
        case 16: VP_FWD(16, 1);
        case 64: VP_FWD(64, 1);
        case 128: VP_FWD(128, 1);
        case 256: VP_FWD(256, 1);
        case 512: VP_FWD(512, 1);
    }
    if (p.h <= 8192) VP_FWD(1024, 1);
    if (p.h <= 16384) VP_FWD(1024, 2);
#undef VP_FWD
    const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
    if (bf16) hipLaunchKernelGGL(block_norm_fwd_long_kernel<u16>, dim3(blocks), dim3(1024), 0, st, p);
    else hipLaunchKernelGGL(block_norm_fwd_long_kernel<float>, dim3(blocks), dim3(1024), 0, st, p);
    return hipGetLastError();
}

size_t block_norm_bwd_workspace(int64_t N, int64_t h, int64_t gate_rows, bool post) {
    const int kinds = 2 + (post ? 2 : 0) + (gate_rows ? 2 : 0);
    return (h > BWD_MAX_COLUMNS ? align_up((size_t)N * sizeof(float4), 256) : 0) +
           align_up((size_t)kinds * ranges(N, h) * pitch_of(h) * sizeof(float), 256);
}

template <typename T, typename TD, typename TG>
static hipError_t launch_bwd(const BlockNormGrad& p, void* workspace, hipStream_t st) {
    const bool one_pass = p.h <= BWD_MAX_COLUMNS;
    float4* means = (float4*)workspace;
    float* part = (float*)((char*)workspace + (one_pass ? 0 : align_up((size_t)p.N * sizeof(float4), 256)));
    ColumnSums s{};
    s.chunks = ranges(p.N, p.h);
    s.each = (int)ceil_div(p.N, s.chunks);
    s.chunks = (int)ceil_div(p.N, s.each);
    s.pitch = pitch_of(p.h);
    const size_t m = (size_t)s.chunks * s.pitch;
    s.dw = s.chunks > 1 ? part : p.dw;
    s.db = s.chunks > 1 ? part + m : p.db;
    part += 2 * m;
    s.dw_post = s.chunks > 1 ? part : p.dw_post;
    s.db_post = s.chunks > 1 ? part + m : p.db_post;
    if (p.post) part += 2 * m;
    s.head = part;
    s.tail = part + m;
    const bool sums = p.dw || p.db || p.dw_post || p.db_post || p.dgate;
#define VP_BWD(TR)                                                                                                             \
    case TR:                                                                                                                   \
        hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, TR, 1>), dim3((unsigned)ceil_div(s.chunks, TR < 128 ? 256 / TR : 1)), \
                           dim3(TR < 128 ? 256 : TR), 0, st, p, s);                                                            \
        break
    if (one_pass) {
        switch (row_threads(p.h, 1024)) {
            VP_BWD(16);
            VP_BWD(64);
            VP_BWD(128);
            VP_BWD(256);
            VP_BWD(512);
            VP_BWD(1024);
        }
    } else {
        const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
        hipLaunchKernelGGL((block_norm_bwd_means_kernel<T, TD, TG>), dim3(blocks), dim3(1024), 0, st, p, means);
        // (before dx is written: it may be dr)
        if (sums)
            hipLaunchKernelGGL((block_norm_bwd_columns_kernel<T, TD, TG>), dim3((unsigned)ceil_div(p.h, 256), s.chunks), dim3(256),
                               0, st, p, means, s);
        hipLaunchKernelGGL((block_norm_bwd_rows_kernel<T, TD, TG>), dim3(blocks), dim3(1024), 0, st, p, means);
    }
#undef VP_BWD
    if (sums && s.chunks > 1) {
        const int64_t rows = p.dgate ? (p.gate_rows < s.chunks ? p.gate_rows : p.gate_rows < p.N ? s.chunks : 0) : 0;
        hipLaunchKernelGGL(block_norm_bwd_sum_kernel, dim3((unsigned)ceil_div(p.h, 32), (unsigned)(4 + rows)), dim3(256), 0, st, p, s);
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
