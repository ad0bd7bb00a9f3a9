// Verification of drafted tokens over the shards' logits and the draw of the next token (vp.h has the formulas).
//
// Two launches: the sums of the weights of every chunk of the row that the next token is drawn from, then the search for the
// chunk and the token in it.  Every workgroup finds out by itself which row that is: a draft takes one logit of each model.
// Probabilities and sums are in fp64: with 256000 tokens of like probability, an error of 1e-7 of the running sum would change
// one draw in 40.
#include "vp_internal.h"

namespace vp {

namespace {

constexpr int CHUNK = 4096, THREADS = 256, EACH = CHUNK / THREADS;

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }

// The row of the next token, of a sequence that has rows.
struct Row {
    int64_t first, last, at;
    double m, f, mz, fz;      // p = exp(Y - m) f, q = exp(Z - mz) fz
    bool rejected;
};

// Where a token's logits of row i lie: the shard and the element, or -1.
struct Place {
    int shard;
    size_t at;
};
__device__ Place place_of(const Verify& v, int64_t i, int64_t token) {
    Place p{-1, 0};
    for (int r = 0; r < v.p; ++r) {
        const int64_t j = token - v.sh[r].offset;
        if (token >= v.sh[r].offset && j < v.sh[r].rows) p = {r, (size_t)i * v.sh[r].rows + (size_t)j};
    }
    return p;
}

// Whether sequence b has rows; its row of the next token.
template <typename T>
__device__ bool find_row(const Verify& v, int b, Row& r) {
    auto bounded = [&](int64_t s) { return s < 0 ? 0 : s > v.N ? v.N : s; };
    r.first = bounded(v.starts[b]);
    r.last = bounded(v.starts[b + 1]) - 1;
    if (r.last < r.first) return false;
    r.at = r.last;
    r.rejected = false;
    for (int64_t i0 = r.first; i0 < r.last; i0 += 64) {
        const int64_t i = i0 + (threadIdx.x & 63);
        bool ok = true;
        if (i < r.last) {
            const Place at = place_of(v, i, v.drafts[i]);
            double p = 0.0, q = 1.0;
            if (at.shard >= 0) {
                p = exp((double)ld((const T*)v.sh[at.shard].Y + at.at) - v.gmax[i]) / v.gsum[i];
                if (v.zmax) q = exp((double)ld((const T*)v.sh[at.shard].Z + at.at) - v.zmax[i]) / v.zsum[i];
            }
            ok = (double)v.uniforms[i] * q < p;
        }
        const unsigned long long no = __ballot(!ok);
        if (no) {
            r.at = i0 + __builtin_ctzll(no);
            r.rejected = true;
            break;
        }
    }
    r.m = v.gmax[r.at];
    r.f = 1.0 / v.gsum[r.at];
    r.mz = r.fz = 0.0;
    if (r.rejected && v.zmax) {
        r.mz = v.zmax[r.at];
        r.fz = 1.0 / v.zsum[r.at];
    }
    return true;
}

// Weight of column j of a shard; PLAIN: p alone.
template <typename T, bool PLAIN>
__device__ double weight(const Verify& v, const Row& r, const VerifyShard& s, int j) {
    const size_t at = (size_t)r.at * s.rows + j;
    double w = exp((double)ld((const T*)s.Y + at) - r.m) * r.f;
    if (PLAIN || !r.rejected) return w;
    if (v.zmax) w -= exp((double)ld((const T*)s.Z + at) - r.mz) * r.fz;
    else if (v.drafts[r.at] == s.offset + j) w = 0.0;
    return w < 0.0 ? 0.0 : w;      // (a NaN stays one)
}

__device__ __forceinline__ int shard_of(const Verify& v, int chunk) {
    int r = 0;
    while (r + 1 < v.p && chunk >= v.sh[r + 1].first) ++r;
    return r;
}

// Sum over the workgroup, in a fixed tree, in all threads; before: the sum over the threads before this one.
__device__ double block_scan(double x, double& before, double* sh) {
    double s = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double t = __shfl_up(s, o, 64);
        if ((int)(threadIdx.x & 63) >= o) s += t;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    double base = 0.0;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) base += sh[w];
    before = base + s - x;
    return ((sh[0] + sh[1]) + sh[2]) + sh[3];
}

// A thread's part of a chunk: EACH consecutive columns.
template <typename T, bool PLAIN>
__device__ double thread_sum(const Verify& v, const Row& r, const VerifyShard& s, int chunk) {
    const int j0 = (chunk - s.first) * CHUNK + threadIdx.x * EACH;
    double sum = 0.0;
    for (int j = j0; j < j0 + EACH && j < s.rows; ++j) sum += weight<T, PLAIN>(v, r, s, j);
    return sum;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void verify_sums_kernel(Verify v, int chunks, double* part) {
    __shared__ double sh[4];
    Row r;
    if (!find_row<T>(v, blockIdx.y, r)) return;
    double before;
    const double sum = block_scan(thread_sum<T, false>(v, r, v.sh[shard_of(v, blockIdx.x)], blockIdx.x), before, sh);
    if (threadIdx.x == 0) part[(size_t)blockIdx.y * chunks + blockIdx.x] = sum;
}

// Smallest value over the workgroup.
__device__ int block_min(int x, int* sh) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x = min(x, __shfl_xor(x, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = x;
    __syncthreads();
    return min(min(sh[0], sh[1]), min(sh[2], sh[3]));
}

// The first of n places, in order, at which the running sum exceeds `share` of the whole; or the last of positive weight, where
// rounding leaves none.  sums(i): weights of the places, the same each time.  -1: no place of positive weight, or a sum that is
// no number.
template <typename F>
__device__ int64_t pick(F sums, int n, double target, double& base, double* sh, int* shi) {
    int last = -1;
    double run = base;
    for (int i0 = 0; i0 < n; i0 += THREADS) {
        const int i = i0 + threadIdx.x;
        const double x = i < n ? sums(i) : 0.0;
        double before;
        const double all = block_scan(x, before, sh);
        const bool hit = x > 0.0 && run + before + x > target;
        const int found = block_min(hit ? (int)threadIdx.x : THREADS, shi);
        const int most = -block_min(x > 0.0 ? -(int)threadIdx.x - 1 : 0, shi) - 1;
        if (found < THREADS) {
            __syncthreads();
            if ((int)threadIdx.x == found) sh[0] = run + before;
            __syncthreads();
            base = sh[0];
            return i0 + found;
        }
        if (most >= 0) {
            last = i0 + most;
            __syncthreads();
            if ((int)threadIdx.x == most) sh[0] = run + before;
            __syncthreads();
            base = sh[0];
            __syncthreads();
        }
        run += all;
    }
    return last;
}

template <typename T, bool PLAIN>
__device__ int64_t draw(const Verify& v, const Row& r, int chunks, double* part, double* sh, int* shi) {
    double total = 0.0, before;
    if (PLAIN) {
        for (int c = 0; c < chunks; ++c) {
            const double s = block_scan(thread_sum<T, true>(v, r, v.sh[shard_of(v, c)], c), before, sh);
            if (threadIdx.x == 0) part[c] = s;
        }
        __syncthreads();
    }
    for (int c0 = 0; c0 < chunks; c0 += THREADS) total += block_scan(c0 + (int)threadIdx.x < chunks ? part[c0 + threadIdx.x] : 0.0, before, sh);
    if (!(total < INFINITY)) return -1;
    if (total == 0.0) return -2;
    const double target = (double)v.uniforms[r.last] * total;
    double base = 0.0;
    const int c = (int)pick([&](int i) { return part[i]; }, chunks, target, base, sh, shi);
    const VerifyShard& s = v.sh[shard_of(v, c)];
    const int j0 = (c - s.first) * CHUNK, n = min(CHUNK, s.rows - j0);
    const int64_t j = pick([&](int i) { return weight<T, PLAIN>(v, r, s, j0 + i); }, n, target, base, sh, shi);
    return s.offset + j0 + j;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void verify_pick_kernel(Verify v, int chunks, double* part) {
    __shared__ double sh[4];
    __shared__ int shi[4];
    const int b = blockIdx.x;
    Row r;
    if (!find_row<T>(v, b, r)) {
        if (threadIdx.x == 0) v.accepted[b] = 0;
        return;
    }
    part += (size_t)b * chunks;
    int64_t token = draw<T, false>(v, r, chunks, part, sh, shi);
    if (token == -2) token = r.rejected ? draw<T, true>(v, r, chunks, part, sh, shi) : -1;
    if (token < 0) token = -1;
    if (threadIdx.x == 0) v.accepted[b] = (int32_t)(r.at - r.first);
    for (int64_t i = r.first + threadIdx.x; i <= r.last; i += THREADS)
        v.tokens[i] = i < r.at ? v.drafts[i] : i == r.at ? token : -1;
}

}  // namespace

size_t verify_workspace(int64_t sequences, int64_t V) {
    return align_up((size_t)sequences * (V / CHUNK + VERIFY_MAX_SHARDS) * sizeof(double), 256);
}

hipError_t launch_verify(const Verify& v0, vp_dtype dt, void* workspace, hipStream_t st) {
    ProfScope prof(K_VERIFY, st);
    Verify v = v0;
    int chunks = 0;
    for (int r = 0; r < v.p; ++r) {
        v.sh[r].first = chunks;
        chunks += (int)ceil_div(v.sh[r].rows, CHUNK);
    }
    double* part = (double*)workspace;
    if (dt == VP_F32) {
        hipLaunchKernelGGL(verify_sums_kernel<float>, dim3(chunks, v.sequences), dim3(THREADS), 0, st, v, chunks, part);
        hipLaunchKernelGGL(verify_pick_kernel<float>, dim3(v.sequences), dim3(THREADS), 0, st, v, chunks, part);
    } else {
        hipLaunchKernelGGL(verify_sums_kernel<u16>, dim3(chunks, v.sequences), dim3(THREADS), 0, st, v, chunks, part);
        hipLaunchKernelGGL(verify_pick_kernel<u16>, dim3(v.sequences), dim3(THREADS), 0, st, v, chunks, part);
    }
    return hipGetLastError();
}

}  // namespace vp
