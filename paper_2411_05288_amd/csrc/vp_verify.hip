// Verification of drafted tokens over the shards' logits and the draw of the next token, and the statistics of stored logits that
// it takes (vp.h has the formulas).
//
// Two launches: the sums of the weights of every segment of 512 tokens of the row that the next token is drawn from, then the
// search for the segment and the token in it.  Which row that is, every wavefront of the first launch finds out by itself: a draft
// takes one logit of each model.
// Probabilities and sums are in fp64: with 256000 tokens of like probability, an error of 1e-7 of the running sum would change
// one draw in 40.
//
// Small calls are bound by the chain of loads that leads to the row (one sequence of 4 drafts, V=32000: 6.3 us for the sums, 3.9 for
// the search), large ones by vector instructions, most of them fp64 and 40 for a token's two weights as the exponential is computed
// here (256 sequences of up to 8 drafts, V=256000 bf16: 93 us for the sums, 2.2 TB/s; the vector units are busy for 0.68 of the
// launch, and for 0.93 of the time that their compute unit has work).  Loops one segment ahead, workgroups that are not all resident
// at once, a launch of its own for the rows and exponentials of bf16 numbers from two tables in LDS (30 % fewer instructions) made no
// difference of more than 8 % there and cost the smaller calls as much.
#include <climits>

#include "vp_internal.h"

namespace vp {

namespace {

constexpr int E = 8, SEGMENT = 64 * E, THREADS = 256, WAVES = THREADS / 64;
constexpr int FILL = 8192;      // wavefronts that the chip holds at a time

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }
// Eight logits as they are stored (vectors start at any element).
template <typename T>
struct Raw;
template <>
struct Raw<float> {
    f32x4u a, b;
    __device__ __forceinline__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4u*>(p);
        b = *reinterpret_cast<const f32x4u*>(p + 4);
    }
    __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
    __device__ __forceinline__ void set(int e, float f) { if (e < 4) a[e] = f; else b[e - 4] = f; }
};
template <>
struct Raw<u16> {
    u16x8u a;
    __device__ __forceinline__ void load(const u16* p) { a = *reinterpret_cast<const u16x8u*>(p); }
    __device__ __forceinline__ float operator[](int e) const { return __uint_as_float((unsigned)a[e] << 16); }
    __device__ __forceinline__ void set(int e, float f) { a[e] = (u16)(__float_as_uint(f) >> 16); }
};
// Columns j .. j + 7 of a row of n, -inf past its end.
template <typename T>
__device__ __forceinline__ void load8(Raw<T>& y, const T* row, int j, int n) {
    if (j + E <= n) {
        y.load(row + j);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) y.set(e, j + e < n ? ld(row + j + e) : -INFINITY);
    }
}

// exp(x) = 2^(n / 128) exp(r), n the integer nearest to 128 x / ln 2: a table of 2^(i / 128), i = 0 .. 127, and four terms of
// the series of exp(r) - 1, |r| <= ln 2 / 256 (the fifth is below 2e-15).  The library's function takes twice the instructions.
constexpr int TABLE = 128;
__device__ __forceinline__ void fill_table(double* table) {
    if (threadIdx.x < TABLE) table[threadIdx.x] = exp2((double)threadIdx.x / TABLE);
    __syncthreads();
}
// `low` keeps the integer in its range (exp(-800) is 0; y = -inf would leave none).  From 2^28 on, fp32 numbers are 32 and more
// apart, later thousands, and m - 800 would become m itself: the logits of such a row are shifted by m first (`close`), which is
// exact where the difference counts.
struct Exp {
    float shift, low;
    double m, f;      // f exp(y - m)
    __device__ Exp(float top, double f) : shift(fabsf(top) >= 0x1p28f ? top : 0.f), low(top - shift - 800.f), m(top - shift), f(f) {}
    template <typename T>
    __device__ __forceinline__ void close(Raw<T>& y) const {
        if (shift == 0.f) return;
#pragma unroll
        for (int e = 0; e < E; ++e) y.set(e, y[e] - shift);
    }
    __device__ __forceinline__ double operator()(float y, const double* table) const {
        const double x = (double)__builtin_elementwise_maximum(y, low) - m;      // (a NaN stays one)
        constexpr double MAGIC = 6755399441055744.0;      // 1.5 2^52: a sum with it ends in the nearest integer
        const double t = fma(x, TABLE / 0.693147180559945309417, MAGIC), n = t - MAGIC;
        const double r = fma(n, -0.693147180559945309417 / TABLE, x);
        double p = fma(r, 1.0 / 24, 1.0 / 6);
        p = fma(p, r, 0.5);
        p = fma(p, r, 1.0);
        p *= r;
        const int k = __double2loint(t);
        const double a = table[k & (TABLE - 1)];
        return ldexp(fma(a, p, a), k >> 7) * f;
    }
};

// What a lane holds of the shard of its number: reading the arguments one shard after the other takes a memory latency each.
struct Lanes {
    int64_t offset;
    int first, rows;
    __device__ explicit Lanes(const Verify& v) {
        const int l = threadIdx.x & 63;
        offset = 0;
        first = INT_MAX;
        rows = 0;
        if (l < v.p) {
            offset = v.sh[l].offset;
            first = v.sh[l].first;
            rows = v.sh[l].rows;
        }
    }
    __device__ __forceinline__ int shard_of(int segment) const { return __popcll(__ballot(segment >= first)) - 1; }
};

// A sequence's rows, and the row of the next token.
struct Rows {
    int64_t first, last;
    __device__ Rows(const Verify& v, int b) {
        first = bounded(v.starts[b], v.N);
        last = bounded(v.starts[b + 1], v.N) - 1;
    }
    __device__ static int64_t bounded(int64_t s, int64_t N) { return s < 0 ? 0 : s > N ? N : s; }
    __device__ bool any() const { return last >= first; }
};
// What the first launch leaves for the second.
struct Found {
    int64_t at;
    float m, s, mz, sz;
};

// Where a token's logit of row i lies: the shard and the element, or shard -1.
struct Place {
    int shard;
    size_t at;
};
__device__ __forceinline__ Place place_of(const Lanes& shards, int p, int64_t i, int64_t token) {
    Place at{-1, 0};
    for (int r = 0; r < p; ++r) {
        const int64_t first = (int64_t)(unsigned)__builtin_amdgcn_readlane((int)shards.offset, r) |
                              (int64_t)__builtin_amdgcn_readlane((int)(shards.offset >> 32), r) << 32;
        const int rows = __builtin_amdgcn_readlane(shards.rows, r);
        const int64_t j = token - first;
        if (token >= first && j < rows) at = {r, (size_t)i * rows + (size_t)j};
    }
    return at;
}

// Row of the first draft that is rejected, or the last row.
template <typename T>
__device__ __forceinline__ int64_t first_rejected(const Verify& v, const Lanes& shards, const Rows& rows) {
    for (int64_t i0 = rows.first; i0 < rows.last; i0 += 64) {
        const int64_t i = i0 + (threadIdx.x & 63);
        bool ok = true;
        if (i < rows.last) {
            const double m = v.gmax[i], s = v.gsum[i], u = v.uniforms[i];
            const double mz = v.zmax ? v.zmax[i] : 0.f, sz = v.zmax ? v.zsum[i] : 0.f;
            const Place at = place_of(shards, v.p, i, v.drafts[i]);
            double p = 0.0, q = 1.0;
            if (at.shard >= 0) {
                p = exp((double)ld((const T*)v.sh[at.shard].Y + at.at) - m) / s;
                if (v.zmax) q = exp((double)ld((const T*)v.sh[at.shard].Z + at.at) - mz) / sz;
            }
            ok = u * q < p;
        }
        const unsigned long long no = __ballot(!ok);
        if (no) return i0 + __builtin_ctzll(no);
    }
    return rows.last;
}

// Weights of the row of the next token.
template <typename T>
struct Weights {
    const Verify& v;
    const double* table;
    int64_t at, skip;      // skip: a token of weight 0
    bool model;
    Exp p, q;
    Raw<T> y, z;           // eight logits of each model, of shard `shard` from column j on
    int shard, j;
    __device__ Weights(const Verify& v, const Found& f, bool rejected, const double* table)
        : v(v), table(table), at(f.at), skip(rejected && !v.zmax ? v.drafts[f.at] : -1), model(rejected && v.zmax), p(f.m, 1.0 / f.s),
          q(f.mz, 1.0 / f.sz) {}
    // This lane's eight of a segment.
    __device__ __forceinline__ void load(const Lanes& shards, int segment) {
        shard = shards.shard_of(segment);
        const VerifyShard& s = v.sh[shard];
        j = (segment - s.first) * SEGMENT + (threadIdx.x & 63) * E;
        const size_t row = (size_t)at * s.rows;
        load8(y, (const T*)s.Y + row, j, s.rows);
        if (model) load8(z, (const T*)s.Z + row, j, s.rows);
        p.close(y);
        if (model) q.close(z);
    }
    __device__ __forceinline__ void get(double (&w)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = p(y[e], table);
        if (model) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] -= q(z[e], table);
                w[e] = fmax(w[e], 0.0) + w[e] * 0.0;      // (the second term is NaN where the first would hide one)
            }
        }
        const int64_t k = skip - v.sh[shard].offset - j;
        if (skip >= 0 && k >= 0 && k < E) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k == e) w[e] = 0.0;
        }
    }
    __device__ __forceinline__ static double sum(const double (&w)[E]) {
        return ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    }
    __device__ __forceinline__ double sum() const {
        double w[E];
        get(w);
        return sum(w);
    }
};

// Sum over the lanes up to this one (the last lane's: over all).
template <int CTRL, int ROWS>
__device__ __forceinline__ double add_moved(double x) {      // + 0 where no lane moves in
    const int low = __builtin_amdgcn_update_dpp(0, __double2loint(x), CTRL, ROWS, 0xf, false);
    const int high = __builtin_amdgcn_update_dpp(0, __double2hiint(x), CTRL, ROWS, 0xf, false);
    return x + __hiloint2double(high, low);
}
__device__ __forceinline__ double wave_scan(double x) {
    x = add_moved<0x111, 0xf>(x);      // from 1, 2, 4, 8 lanes before, within 16
    x = add_moved<0x112, 0xf>(x);
    x = add_moved<0x114, 0xf>(x);
    x = add_moved<0x118, 0xf>(x);
    x = add_moved<0x142, 0xa>(x);      // the last lane of 16 into the next 16, of 32 into the next 32
    return add_moved<0x143, 0xc>(x);
}
__device__ __forceinline__ double last_lane(double x) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(x), 63), __builtin_amdgcn_readlane(__double2loint(x), 63));
}

// Sequence b has the workgroups b * groups .. + groups - 1, whose wavefronts take its segments in turn.
template <typename T>
__global__ __launch_bounds__(THREADS, 8) void verify_sums_kernel(Verify v, int segments, int groups, double* part, Found* found) {
    __shared__ double table[TABLE];
    const int b = blockIdx.x / groups, wave = (blockIdx.x % groups) * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Rows rows(v, b);
    const Lanes shards(v);
    fill_table(table);
    if (!rows.any()) return;
    Found f{first_rejected<T>(v, shards, rows), 0.f, 1.f, 0.f, 1.f};
    const bool rejected = f.at < rows.last;
    f.m = v.gmax[f.at];
    f.s = v.gsum[f.at];
    if (rejected && v.zmax) {
        f.mz = v.zmax[f.at];
        f.sz = v.zsum[f.at];
    }
    if (wave == 0 && (threadIdx.x & 63) == 0) found[b] = f;
    Weights<T> w(v, f, rejected, table);
    for (int g = wave; g < segments; g += groups * WAVES) {
        w.load(shards, g);
        const double sum = wave_scan(w.sum());
        if ((threadIdx.x & 63) == 63) part[(size_t)b * segments + g] = sum;
    }
}

// Of places in order, one to a lane (x its weight, upto the sum of them up to it): the first at which `upto` exceeds the target, or
// where rounding leaves none the last one that has a weight; -1 if none has.
__device__ __forceinline__ int choose(double x, double upto, double target) {
    const unsigned long long some = __ballot(x > 0.0), hit = __ballot(x > 0.0 && upto > target);
    return hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : -1;
}

// The token of a segment (for a whole wavefront): target is the share of its sum, not yet the sums before.
template <typename T>
__device__ __forceinline__ int64_t token_of(Weights<T>& weights, const Lanes& shards, int segment, double target) {
    weights.load(shards, segment);
    double w[E];
    weights.get(w);
    const double mine = weights.sum(w), upto = wave_scan(mine);
    const int l = choose(mine, upto, target);
    int token = -1;
    double run = upto - mine;
    bool done = false;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        run += w[e];
        if (w[e] > 0.0 && !done) {
            token = weights.j + e;
            done = run > target;
        }
    }
    return weights.v.sh[weights.shard].offset + __shfl(token, l, 64);
}

// The draw from p itself, where nothing is left of the difference: every wavefront walks a quarter of the row, then all of them the
// quarter in which the target is reached.
template <typename T>
__device__ int64_t plain_token(const Verify& v, const Found& f, const Lanes& shards, double u, int segments, const double* table,
                               double* sh) {
    Weights<T> weights(v, f, false, table);
    const int wave = threadIdx.x >> 6;
    auto from = [&](int w) { return (int)((int64_t)segments * w / WAVES); };
    auto sum_of = [&](int g) {
        weights.load(shards, g);
        return last_lane(wave_scan(weights.sum()));
    };
    double mine = 0.0;
    for (int g = from(wave); g < from(wave + 1); ++g) mine += sum_of(g);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[wave] = mine;
    __syncthreads();
    double total = 0.0, base = 0.0;
    for (int w = 0; w < WAVES; ++w) total += sh[w];
    if (!(total > 0.0) || !(total < INFINITY)) return -1;
    const double target = u * total;
    int chosen = -1;
    double run = 0.0;
    for (int w = 0; w < WAVES; ++w) {
        if (sh[w] > 0.0) {
            chosen = w;
            base = run;
            if (run + sh[w] > target) break;
        }
        run += sh[w];
    }
    int segment = -1;
    double before = 0.0;
    for (int g = from(chosen); g < from(chosen + 1); ++g) {
        const double s = sum_of(g);
        if (s > 0.0) {
            segment = g;
            before = base;
            if (base + s > target) break;
        }
        base += s;
    }
    return token_of(weights, shards, segment, target - before);
}

template <typename T>
__global__ __launch_bounds__(THREADS) void verify_pick_kernel(Verify v, int segments, const double* part, const Found* found) {
    __shared__ double table[TABLE], sums[WAVES], chosen_base;
    __shared__ int chosen_segment;
    const int b = blockIdx.x, wave = threadIdx.x >> 6;
    const Rows rows(v, b);
    const Found f = found[b];      // (a sequence without rows has none, nor sums: what is read is not used)
    const Lanes shards(v);
    // the segments, an equal number of neighbours to every thread
    part += (size_t)b * segments;
    const int each = (segments + THREADS - 1) / THREADS, g0 = threadIdx.x * each, g1 = min(segments, g0 + each);
    double mine = 0.0;
    for (int g = g0; g < g1; ++g) mine += part[g];
    const double in_wave = wave_scan(mine);
    if ((threadIdx.x & 63) == 63) sums[wave] = in_wave;
    fill_table(table);
    if (!rows.any()) {
        if (threadIdx.x == 0) v.accepted[b] = 0;
        return;
    }
    const double u = v.uniforms[rows.last];
    const double total = ((sums[0] + sums[1]) + sums[2]) + sums[3], target = u * total;
    int64_t token = -1;
    const bool rejected = f.at < rows.last;
    if (total > 0.0 && total < INFINITY) {
        // every wavefront knows all sums: the first one in which the target is reached, or the last one with a weight
        double base = 0.0, run = 0.0;
        int w = -1;
        for (int k = 0; k < WAVES; ++k) {
            if (sums[k] > 0.0 && !(w >= 0 && run > target)) {
                w = k;
                base = run;
            }
            run += sums[k];
        }
        if (wave == w) {
            const int l = choose(mine, base + in_wave, target);
            if ((int)(threadIdx.x & 63) == l) {
                int segment = -1;
                double before = 0.0, at = base + in_wave - mine;
                for (int g = g0; g < g1; ++g) {
                    const double s = part[g];
                    if (s > 0.0) {
                        segment = g;
                        before = at;
                        if (at + s > target) break;
                    }
                    at += s;
                }
                chosen_segment = segment;
                chosen_base = before;
            }
        }
        __syncthreads();
        Weights<T> weights(v, f, rejected, table);
        token = token_of(weights, shards, __builtin_amdgcn_readfirstlane(chosen_segment), target - chosen_base);
    } else if (total == 0.0 && rejected) {
        token = plain_token<T>(v, f, shards, u, segments, table, sums);
    }
    if (threadIdx.x == 0) v.accepted[b] = (int32_t)(f.at - rows.first);
    for (int64_t i = rows.first + threadIdx.x; i <= rows.last; i += THREADS)
        v.tokens[i] = i < f.at ? v.drafts[i] : i == f.at ? token : -1;
}

// ---- statistics of stored logits: a wavefront for every CHUNK columns of a row, then one for every row, which joins them.
//
// Bound by reading the logits: 1276 rows of V=256000 bf16 128 us (5.1 TB/s), 226 of V=128256 14.8, 64 of V=128256 fp32 11.2; a few
// rows by the two launches (5 of V=32000: 9.0).
constexpr int SETS = 4, CHUNK = SETS * SEGMENT;

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o, 64));
    return x;
}
template <typename X>
__device__ __forceinline__ X wave_sum(X x) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    return x;
}
// What exponents are taken around: 0 where there is no number, so that -inf adds nothing and a NaN stays one.
__device__ __forceinline__ float around(float m) { return m == -INFINITY ? 0.f : m; }

// The columns stay in registers between the maximum and the sum, so they are read once.  Exponentials are of 32 bits: a term is off
// by its distance from the maximum times 2^-23, which its size outweighs.
template <typename T>
__global__ __launch_bounds__(THREADS) void logits_stats_kernel(Verify v, int chunks, float2* __restrict__ part) {
    const Lanes shards(v);
    const int c = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (c >= chunks) return;
    const VerifyShard& s = v.sh[shards.shard_of(c)];
    const int j = (c - s.first) * CHUNK + (threadIdx.x & 63) * E;
    for (int64_t i = blockIdx.x; i < v.N; i += gridDim.x) {
        Raw<T> y[SETS];
#pragma unroll
        for (int k = 0; k < SETS; ++k) load8(y[k], (const T*)s.Y + (size_t)i * s.rows, j + k * SEGMENT, s.rows);
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < SETS; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) m = fmaxf(m, y[k][e]);
        m = wave_max(m);
        const float a = around(m);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < SETS; ++k) {
            float x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = __builtin_amdgcn_exp2f((y[k][e] - a) * 1.44269504088896340736f);
            sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        sum = wave_sum(sum);
        if ((threadIdx.x & 63) == 0) part[(size_t)i * chunks + c] = make_float2(m, sum);
    }
}

__global__ __launch_bounds__(THREADS) void join_stats_kernel(const float2* __restrict__ part, int chunks, int64_t N, float* __restrict__ gmax,
                                                             float* __restrict__ gsum) {
    for (int64_t i = (int64_t)blockIdx.x * WAVES + (threadIdx.x >> 6); i < N; i += (int64_t)gridDim.x * WAVES) {
        float m = -INFINITY;
        double sum = 0.0;
        for (int c = threadIdx.x & 63; c < chunks; c += 64) {
            const float2 q = part[(size_t)i * chunks + c];
            const float top = fmaxf(m, q.x);
            const double a = around(top);
            sum = sum * exp(m - a) + q.y * exp(q.x - a);
            m = top;
        }
        const float top = wave_max(m);
        sum = wave_sum(sum * exp(m - (double)around(top)));
        if ((threadIdx.x & 63) == 0) {
            gmax[i] = top;
            gsum[i] = (float)sum;
        }
    }
}

}  // namespace

static int64_t stats_chunks(int32_t p, const int64_t* rows) {
    int64_t n = 0;
    for (int32_t r = 0; r < p; ++r) n += ceil_div(rows[r], CHUNK);
    return n;
}
size_t logits_stats_workspace(int32_t p, int64_t N, const int64_t* rows) {
    return align_up((size_t)(N * stats_chunks(p, rows)) * sizeof(float2), 256);
}

hipError_t launch_logits_stats(const Verify& v0, vp_dtype dt, float* gmax, float* gsum, void* workspace, hipStream_t st) {
    ProfScope prof(K_LOGITS_STATS, st);
    Verify v = v0;
    int chunks = 0;
    for (int r = 0; r < v.p; ++r) {
        v.sh[r].first = chunks;
        chunks += (int)ceil_div(v.sh[r].rows, CHUNK);
    }
    // a workgroup for every row where a launch has fewer than 2^31 threads then
    const int waves = chunks < WAVES ? chunks : WAVES;
    const int64_t groups = ceil_div(chunks, waves), most = ((int64_t)1 << 23) / groups;
    const dim3 grid((unsigned)(v.N < most ? v.N : most), (unsigned)groups);
    float2* part = (float2*)workspace;
    if (dt == VP_F32) hipLaunchKernelGGL(logits_stats_kernel<float>, grid, dim3(64 * waves), 0, st, v, chunks, part);
    else hipLaunchKernelGGL(logits_stats_kernel<u16>, grid, dim3(64 * waves), 0, st, v, chunks, part);
    const int64_t joins = ceil_div(v.N, WAVES);
    hipLaunchKernelGGL(join_stats_kernel, dim3((unsigned)(joins < 65536 ? joins : 65536)), dim3(THREADS), 0, st, part, chunks, v.N, gmax, gsum);
    return hipGetLastError();
}

// The segments' sums, and the rows found.
size_t verify_workspace(int64_t sequences, int64_t V) {
    return align_up((size_t)sequences * ((V / SEGMENT + VERIFY_MAX_SHARDS) * sizeof(double) + sizeof(Found)), 256);
}

template <typename T>
static void launch_verify_t(const Verify& v, int segments, int groups, double* part, Found* found, hipStream_t st) {
    hipLaunchKernelGGL(verify_sums_kernel<T>, dim3(v.sequences * groups), dim3(THREADS), 0, st, v, segments, groups, part, found);
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(v.sequences), dim3(THREADS), 0, st, v, segments, part, found);
}

hipError_t launch_verify(const Verify& v0, vp_dtype dt, void* workspace, hipStream_t st) {
    ProfScope prof(K_VERIFY, st);
    Verify v = v0;
    int segments = 0;
    for (int r = 0; r < v.p; ++r) {
        v.sh[r].first = segments;
        segments += (int)ceil_div(v.sh[r].rows, SEGMENT);
    }
    Found* found = (Found*)workspace;
    double* part = (double*)(found + v.sequences);
    // a wavefront for every segment where there are few, else as many as fit
    const int most = (int)ceil_div(segments, WAVES), some = (int)ceil_div(FILL / WAVES, v.sequences);
    const int groups = most < some ? most : some;
    if (dt == VP_F32) launch_verify_t<float>(v, segments, groups, part, found, st);
    else launch_verify_t<u16>(v, segments, groups, part, found, st);
    return hipGetLastError();
}

}  // namespace vp
