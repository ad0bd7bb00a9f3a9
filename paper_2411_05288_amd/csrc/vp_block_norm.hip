// The norms before and after a block of the model with its gate and residual scale, forward and backward (vp.h has the
// formulas).  Bound by HBM: the forward call reads x and y and writes r and H, the backward call reads dH, dr, r and y and
// writes dx and dy, each once if a row stays on the chip between the sums over it and their use.  N=4096 h=4096 bf16, RMS norms
// on both sides: forward 26.5 us (5.1 TB/s), backward with fp32 dH 47.5 us (5.1 TB/s) and 4.8 us for the last sums over tokens; a
// single token 3.4 us.
#include "vp_block_norm.h"

namespace vp {

namespace {

// Sums of K values over the workgroup (up to 16 wavefronts), a fixed tree; sh: K * 16 floats.
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
        for (int i = 0; i < (int)(blockDim.x >> 6); ++i) s += sh[k * 16 + i];
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
        for (int j = threadIdx.x; j < h; j += blockDim.x) s += f(j);
        block_sums<1>(&s, sh);
        n.m = s / h;
    }
    s = 0.f;
    for (int j = threadIdx.x; j < h; j += blockDim.x) {
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
    for (int64_t i = blockIdx.x; i < p.N; i += gridDim.x) {
        const size_t row = (size_t)i * p.h;
        const T *x = (const T*)p.x + row, *y = p.y ? (const T*)p.y + row : nullptr;
        const T* gate = p.gate ? (const T*)p.gate + (size_t)(i * p.gate_rows / p.N) * p.h : nullptr;
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
        for (int j = threadIdx.x; j < p.h; j += blockDim.x) {
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

// Rows of at most 8 C TR columns: TR lanes (TR <= 64) or the workgroup's up to TR threads hold a row in registers, C vectors of
// eight columns each, from the only read of x and y to the only write of r and H.
template <typename T, int TR, int C, bool STREAM>
__global__ __launch_bounds__(TR <= 64 ? 256 : TR) void block_norm_fwd_kernel(BlockNorm p) {
    __shared__ float sh[2][K_ROW_SUMS];
    int turn = 0;
    constexpr int ROWS = TR <= 64 ? 256 / TR : 1;
    constexpr bool EARLY = TR < 1024;      // (of the longest rows two workgroups fit a CU without)
    const int t = threadIdx.x % TR, threads = TR <= 64 ? TR : blockDim.x, row = blockIdx.x * ROWS + threadIdx.x / TR;
    const bool live = row < p.N;
    const int i = live ? row : p.N - 1;      // (a workgroup's rows past the last one take part in nothing but the sums)
    const size_t at = (size_t)i * p.h;
    const T *x = (const T*)p.x + at, *y = (const T*)p.y;
    const T* gate = p.gate ? (const T*)p.gate + (size_t)((int64_t)i * p.gate_rows / p.N) * p.h : nullptr;
    int j[C], skip[C];
    Raw8<T> rx[C], ry[C], rg[C], w[C], wp[C], bp[C];
    float v[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const Columns cols(c * threads + t, p.h);
        j[c] = cols.j;
        skip[c] = cols.skip;
        rx[c] = load8<STREAM>(x, j[c]);
        if (y) ry[c] = load8<STREAM>(y + at, j[c]);
        if (gate) rg[c] = load8(gate, j[c]);
    }
    auto load_post = [&](int c) {
        wp[c] = load8((const T*)p.w_post, j[c], 1.f);
        bp[c] = load8((const T*)p.b_post, j[c]);
    };
    // asked for before the first sum, as after it they would be waited for
    if constexpr (EARLY)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (p.post) load_post(c);
            w[c] = load8((const T*)p.w, j[c], 1.f);
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
                for (int e = 0; e < 8; ++e) s += e >= skip[c] ? v[c][e] : 0.f;
            row_sums<1, TR == 16 ? 16 : 64>(&s, sh, turn, 0, threads >> 6);
            m.m = s / p.h;
        }
        s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v[c][e] - m.m;
                s += e >= skip[c] ? d * d : 0.f;
            }
        row_sums<1, TR == 16 ? 16 : 64>(&s, sh, turn, 0, threads >> 6);
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
        if (p.post) {
            if constexpr (!EARLY) load_post(c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[c][e] = (v[c][e] - a.m) * a.rho * wp[c][e] + bp[c][e];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = y ? rx[c][e] + (gate ? p.scale * rg[c][e] : p.scale) * v[c][e] : rx[c][e];
        if (p.r && live) store8((T*)p.r + at, j[c], skip[c], v[c]);
    }
    const Normed m = statistics();
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if constexpr (!EARLY) w[c] = load8((const T*)p.w, j[c], 1.f);
        const Raw8<T> b = load8((const T*)p.b, j[c]);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (v[c][e] - m.m) * m.rho * w[c][e] + b[e];
        if (live) store8((T*)p.H + at, j[c], skip[c], o);
    }
    if (p.stats && t == 0 && live) {
        p.stats[i] = a.m;
        p.stats[(size_t)p.N + i] = a.rho;
        p.stats[2 * (size_t)p.N + i] = m.m;
        p.stats[3 * (size_t)p.N + i] = m.rho;
    }
}

// ---- backward

// What the formulas need of a row.
template <typename T, typename TD, typename TG>
struct Row {
    const T *r, *y, *gate;
    const TD* dH;
    const TG* dr;
    float m1, rho1, m2, rho2;
    __device__ Row(const BlockNormGrad& p, int64_t i) {
        const size_t row = (size_t)i * p.h;
        r = (const T*)p.r + row;
        y = p.y ? (const T*)p.y + row : nullptr;
        gate = p.gate ? (const T*)p.gate + (size_t)(i * p.gate_rows / p.N) * p.h : nullptr;
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
    for (int64_t i = blockIdx.x; i < p.N; i += gridDim.x) {
        const Row<T, TD, TG> q(p, i);
        float s[2] = {0.f, 0.f}, c[2] = {0.f, 0.f};
        for (int j = threadIdx.x; j < p.h; j += blockDim.x) {
            const float a = q.a(p, j);
            s[0] += a;
            s[1] += a * q.rh(j);
        }
        block_sums<2>(s, sh);
        const float ma = p.center ? s[0] / p.h : 0.f, mar = s[1] / p.h;
        if (p.post) {
            for (int j = threadIdx.x; j < p.h; j += blockDim.x) {
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
    const int64_t i0 = (int64_t)c * s.each, i1 = i0 + s.each < p.N ? i0 + s.each : p.N;
    const int L = p.gate_rows ? (int)(p.N / p.gate_rows) : 0;
    const float wp = ld_or((const T*)p.w_post, j, 1.f), bp = ld_or((const T*)p.b_post, j, 0.f);
    float dw = 0.f, db = 0.f, dwp = 0.f, dbp = 0.f, dg = 0.f;
    for (int64_t i = i0; i < i1; ++i) {
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
            const int64_t k = i / L;
            if (L == p.N) continue;
            if ((i + 1) % L == 0 || i + 1 == i1) {
                if (k * L < i0) s.head[(size_t)c * s.pitch + j] = dg;
                else if ((i + 1) % L == 0) p.dgate[(size_t)k * p.h + j] = dg;
                else s.tail[(size_t)c * s.pitch + j] = dg;
                dg = 0.f;
            }
        }
    }
    const size_t o = (size_t)c * s.pitch + j;
    if (s.dw) s.dw[o] = dw;
    if (s.db) s.db[o] = db;
    if (s.dw_post) s.dw_post[o] = dwp;
    if (s.db_post) s.db_post[o] = dbp;
    if (s.dgate) s.dgate[o] = dg;
}

// Third step: dx and dy.
template <typename T, typename TD, typename TG>
__global__ __launch_bounds__(1024) void block_norm_bwd_rows_kernel(BlockNormGrad p, const float4* means) {
    for (int64_t i = blockIdx.x; i < p.N; i += gridDim.x) {
        const Row<T, TD, TG> q(p, i);
        const float4 m = means[i];
        TG *dx = (TG*)p.dx + (size_t)i * p.h, *dy = p.dy ? (TG*)p.dy + (size_t)i * p.h : nullptr;
        for (int j = threadIdx.x; j < p.h; j += blockDim.x) {
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

// Last step: the workgroups' partial sums of dw, db, dw_post, db_post and the single row of a gate (blockIdx.y 0 .. 4), and of
// the rows of a larger gate whose tokens lie in several ranges (blockIdx.y - 5: the row, or, where the gate has more rows than
// there are ranges, the range in which it begins).  A workgroup takes 32 columns: eight threads of four columns side by side, 32
// slices of the partial sums.
__global__ __launch_bounds__(256) void block_norm_bwd_sum_kernel(BlockNormGrad p, ColumnSums s) {
    __shared__ float4 sh[32][8];
    const int slice = threadIdx.x >> 3, j = blockIdx.x * 32 + (threadIdx.x & 7) * 4, what = blockIdx.y;
    const float *first, *rest;      // where the first range's row and the others lie
    float* out;
    int c0 = 0, c1 = s.parts - 1;
    if (what < 5) {
        first = rest = what == 0 ? s.dw : what == 1 ? s.db : what == 2 ? s.dw_post : what == 3 ? s.db_post : s.dgate;
        out = what == 0 ? p.dw : what == 1 ? p.db : what == 2 ? p.dw_post : what == 3 ? p.db_post : p.dgate;
        if (!first || !out || (what == 4 && p.gate_rows > 1)) return;
    } else {
        const int64_t L = p.N / p.gate_rows;
        int64_t k = what - 5;
        if (p.gate_rows > s.ranges) {
            const int64_t begin = k * s.each, end = begin + s.each < p.N ? begin + s.each : p.N;
            k = (end - 1) / L;
            if (k * L < begin) return;      // the row at the end of this range began before it
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
#pragma unroll 4
        for (int c = c0 + slice; c <= c1; c += 32) {
            const float4 q = *reinterpret_cast<const float4*>((c == c0 ? first : rest) + (size_t)c * s.pitch + j);
            v.x += q.x;
            v.y += q.y;
            v.z += q.z;
            v.w += q.w;
        }
    sh[slice][threadIdx.x & 7] = v;
    __syncthreads();
    if (threadIdx.x < 32 && (int)(blockIdx.x * 32 + threadIdx.x) < p.h) {
        // a tree: added up in a row, the slices cost 31 roundings (N=128 h=256 fp32, error against 64 bits: in a row 1.4e-7, so 0.9e-7)
        float sum[32];
#pragma unroll
        for (int q = 0; q < 32; ++q) sum[q] = reinterpret_cast<const float*>(sh[q])[threadIdx.x];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int q = 0; q < o; ++q) sum[q] += sum[q + o];
        out[blockIdx.x * 32 + threadIdx.x] = sum[0];
    }
}

// How rows are cut for the sums over tokens.
// One pass: a workgroup per CU, and at least a row at a time for each of its groups of threads.
// Other rows: enough ranges to fill the chip with a thread per column, and partial matrices of 16 MB at most.
constexpr int CUS = 256;
ColumnSums cut(int64_t N, int64_t h, int64_t gate_rows) {
    ColumnSums s{};
    int64_t parts;
    s.rows = 1;
    if (bwd_in_one_pass(h)) {
        // (us, N=100000 bf16: h=100, 16 lanes 35.9, a wavefront 53.3; h=136 with everything, 32 lanes 55.3, a wavefront 69.7)
        const int64_t vectors = ceil_div(h, 8);
        s.threads = h <= 128 ? 16 : h <= 256 ? 32 : (int)(ceil_div(ceil_div(vectors, bwd_vectors(h)), 64) * 64);
        s.rows = 1024 / s.threads;
        parts = CUS;
    } else {
        parts = ((int64_t)1 << 22) / h;
        parts = parts < 1 ? 1 : parts > 512 ? 512 : parts;
    }
    s.step = 1;
    s.each = (int)ceil_div(N, parts * s.rows);
    s.ranges = (int)ceil_div(N, s.each);
    s.parts = (int)ceil_div(s.ranges, s.rows);
    if (bwd_in_one_pass(h)) {
        // few rows: on one CU, if it holds all of them at once (nothing is left to add up then: N=16 h=256 7.1 -> 5.2 us), else on as
        // many CUs as there are
        s.rows = s.ranges <= s.rows ? s.ranges : (int)ceil_div(s.ranges, CUS);
        s.parts = (int)ceil_div(s.ranges, s.rows);
    }
    if (bwd_in_one_pass(h) && (gate_rows <= 1 || gate_rows == N)) s.step = s.ranges = s.parts * s.rows;
    s.pitch = (int)((h + 3) / 4 * 4);
    return s;
}

constexpr int MAX_ROW_BLOCKS = 1 << 16;
// Threads of a row of any length: a wavefront where it is shorter than a vector (N=100000 h=4: 50 us, with 1024 threads 895).
int long_threads(int64_t h) { return h < MIN_COLUMNS ? 64 : 1024; }

}  // namespace

hipError_t launch_block_norm_fwd(const BlockNorm& p, vp_dtype dt, hipStream_t st) {
    ProfScope prof(K_BLOCK_NORM_FWD, st);
    // bf16 inputs that the infinity cache cannot have held since they were written are read past the caches: N=4096 h=4096 28.0 ->
    // 26.3 us, h=8192 with an element-wise gate 62.4 -> 59.8; smaller ones may still be there (N=2048 h=4096: 13.5 -> 16.1)
    const bool bf16 = dt == VP_BF16, stream = bf16 && (int64_t)p.N * p.h * 8 > (int64_t)96 << 20;
#define VP_FWD(TR, C, THREADS)                                                                                                 \
    do {                                                                                                                       \
        const dim3 grid((unsigned)ceil_div(p.N, TR <= 64 ? 256 / TR : 1)), block(TR <= 64 ? 256 : (THREADS));                   \
        if (stream) hipLaunchKernelGGL((block_norm_fwd_kernel<u16, TR, C, true>), grid, block, 0, st, p);                      \
        else if (bf16) hipLaunchKernelGGL((block_norm_fwd_kernel<u16, TR, C, false>), grid, block, 0, st, p);                  \
        else hipLaunchKernelGGL((block_norm_fwd_kernel<float, TR, C, false>), grid, block, 0, st, p);                          \
        return hipGetLastError();                                                                                              \
    } while (0)
    // As few threads per row as hold it with one or two vectors each: fewer steps in its sums, and no lane without columns (us,
    // the choice against the next one: N=100000 h=100 bf16, 16 lanes 17.6, a wavefront 47.9; h=256, 16 lanes with two vectors
    // 38.6, a wavefront 53.7; N=16384 h=600 layer norms, a wavefront 21.3, a workgroup 25.9; N=8192 h=2048, four wavefronts
    // 27.5, one with four vectors 30.3; N=4096 h=4096, two vectors 26.3, one 26.8; N=2048 h=16384, 1024 threads with two 56, 512
    // with four 69; N=512 h=32768, 1024 with four 31, a row that is read again for every sum 126).
    if (p.h >= MIN_COLUMNS && p.N <= 1 << 27) {      // (a launch has less than 2^32 threads)
        if (p.h <= 128) VP_FWD(16, 1, 256);
        if (p.h <= 256) VP_FWD(16, 2, 256);
        if (p.h <= 512) VP_FWD(64, 1, 256);
        if (p.h <= 1024) VP_FWD(64, 2, 256);
        if (p.h <= 2048) VP_FWD(256, 1, (int)ceil_div(p.h, 512) * 64);
        if (p.h <= 8192) VP_FWD(512, 2, (int)ceil_div(p.h, 1024) * 64);
        if (p.h <= 16384) VP_FWD(1024, 2, (int)ceil_div(p.h, 1024) * 64);
        if (p.h <= 32768) VP_FWD(1024, 4, (int)ceil_div(p.h, 2048) * 64);
    }
#undef VP_FWD
    const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
    if (bf16) hipLaunchKernelGGL(block_norm_fwd_long_kernel<u16>, dim3(blocks), dim3(long_threads(p.h)), 0, st, p);
    else hipLaunchKernelGGL(block_norm_fwd_long_kernel<float>, dim3(blocks), dim3(long_threads(p.h)), 0, st, p);
    return hipGetLastError();
}

// Bytes of the row means (long rows), then of the partial matrices: dw, db, the post norm's, dgate or head and tail.
static size_t means_bytes(int64_t N, int64_t h) { return bwd_in_one_pass(h) ? 0 : align_up((size_t)N * sizeof(float4), 256); }
size_t block_norm_bwd_workspace(int64_t N, int64_t h, int64_t gate_rows, bool post) {
    const ColumnSums s = cut(N, h, gate_rows);
    size_t rows = (size_t)s.parts * (2 + (post ? 2 : 0) + (gate_rows ? 1 : 0));
    if (gate_rows > 1 && gate_rows < N) rows += 2 * (size_t)s.ranges;
    return means_bytes(N, h) + align_up(rows * s.pitch * sizeof(float), 256);
}

template <typename T, typename TD, typename TG>
static hipError_t launch_bwd_long(const BlockNormGrad& p, const ColumnSums& s, float4* means, hipStream_t st) {
    const int blocks = p.N < MAX_ROW_BLOCKS ? p.N : MAX_ROW_BLOCKS;
    hipLaunchKernelGGL((block_norm_bwd_means_kernel<T, TD, TG>), dim3(blocks), dim3(long_threads(p.h)), 0, st, p, means);
    // (before dx is written: it may be dr)
    if (p.dw || p.db || p.dw_post || p.db_post || p.dgate)
        hipLaunchKernelGGL((block_norm_bwd_columns_kernel<T, TD, TG>), dim3((unsigned)ceil_div(p.h, 256), s.parts), dim3(256), 0, st,
                           p, means, s);
    hipLaunchKernelGGL((block_norm_bwd_rows_kernel<T, TD, TG>), dim3(blocks), dim3(long_threads(p.h)), 0, st, p, means);
    return hipGetLastError();
}

hipError_t launch_block_norm_bwd(const BlockNormGrad& p, vp_dtype dt, vp_dtype dH_dt, vp_dtype grad_dt, void* workspace,
                                 hipStream_t st) {
    ProfScope prof(K_BLOCK_NORM_BWD, st);
    ColumnSums s = cut(p.N, p.h, p.gate_rows);
    float4* means = (float4*)workspace;
    float* part = (float*)((char*)workspace + means_bytes(p.N, p.h));
    const size_t m = (size_t)s.parts * s.pitch;
    const bool single = s.parts == 1, one_gate = p.gate_rows == 1;
    auto next = [&](float* out) {
        float* at = part;
        part += m;
        return !out ? nullptr : single ? out : at;
    };
    s.dw = next(p.dw);
    s.db = next(p.db);
    if (p.post) {
        s.dw_post = next(p.dw_post);
        s.db_post = next(p.db_post);
    }
    if (one_gate) s.dgate = next(p.dgate);
    else if (p.gate) s.dgate = part, part += m;      // (where a gate of several rows may be summed)
    s.head = part;
    s.tail = part + (size_t)s.ranges * s.pitch;
    hipError_t e;
    if (bwd_in_one_pass(p.h)) {
        e = dt == VP_F32 ? launch_bwd_one_pass_f32(p, s, st) : launch_bwd_one_pass_bf16(p, dH_dt, grad_dt, s, st);
    } else if (dt == VP_F32) {
        e = launch_bwd_long<float, float, float>(p, s, means, st);
    } else if (dH_dt == VP_F32) {
        e = grad_dt == VP_F32 ? launch_bwd_long<u16, float, float>(p, s, means, st) : launch_bwd_long<u16, float, u16>(p, s, means, st);
    } else {
        e = grad_dt == VP_F32 ? launch_bwd_long<u16, u16, float>(p, s, means, st) : launch_bwd_long<u16, u16, u16>(p, s, means, st);
    }
    if (e != hipSuccess) return e;
    // the rows of a gate whose tokens lie in several ranges: at most one begins in a range
    int64_t rows = 0;
    if (p.dgate && !one_gate && p.gate_rows < p.N && s.ranges > 1) rows = p.gate_rows < s.ranges ? p.gate_rows : s.ranges;
    const bool vectors = !single && (s.dw || s.db || s.dw_post || s.db_post || (one_gate && s.dgate));
    if (vectors || rows) {
        ColumnSums q = s;
        if (single) q.dw = q.db = q.dw_post = q.db_post = q.dgate = nullptr;      // they are where they belong
        hipLaunchKernelGGL(block_norm_bwd_sum_kernel, dim3((unsigned)ceil_div(p.h, 32), (unsigned)(5 + rows)), dim3(256), 0, st, p, q);
    }
    return hipGetLastError();
}

}  // namespace vp
