// What the kernels of the norms around a block share: rows in vectors of eight columns, sums over the threads of a row, and the
// one-pass backward kernel, which is compiled for many types and parts (vp_block_norm_bwd_*.hip).
#pragma once

#include "vp_internal.h"

namespace vp {

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned short u16x8u __attribute__((ext_vector_type(8), aligned(2)));
constexpr int K_ROW_SUMS = 32;      // two sums of 16 wavefronts

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const u16* p) { return __uint_as_float((unsigned)*p << 16); }
// A vector's element, or what an absent one stands for.
template <typename T>
__device__ __forceinline__ float ld_or(const T* p, int j, float absent) { return p ? ld(p + j) : absent; }

// Eight columns of a row as they are stored.  Rows of lengths that are no multiple of eight start at any element, so vectors are
// element-aligned (the hardware takes 16-byte accesses at any address).
template <typename T>
struct Raw8;
template <>
struct Raw8<u16> {
    u16x8u v;
    __device__ float operator[](int e) const { return __uint_as_float((unsigned)v[e] << 16); }
    __device__ void load(const u16* p) { v = *reinterpret_cast<const u16x8u*>(p); }
    // past the caches: for what is not read again
    __device__ void load_last(const u16* p) { v = __builtin_nontemporal_load(reinterpret_cast<const u16x8u*>(p)); }
    __device__ void store(u16* p) const { *reinterpret_cast<u16x8u*>(p) = v; }
    __device__ void set(int e, float f) {
        const __bf16 b = (__bf16)f;
        v[e] = __builtin_bit_cast(u16, b);
    }
    // makes the compiler take the registers for changed
    __device__ void keep() { asm volatile("" : "+v"(v)); }
};
template <>
struct Raw8<float> {
    f32x4u a, b;
    __device__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
    __device__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4u*>(p);
        b = *reinterpret_cast<const f32x4u*>(p + 4);
    }
    __device__ void load_last(const float* p) { load(p); }      // (two vectors share a line)
    __device__ void store(float* p) const {
        *reinterpret_cast<f32x4u*>(p) = a;
        *reinterpret_cast<f32x4u*>(p + 4) = b;
    }
    __device__ void set(int e, float f) { if (e < 4) a[e] = f; else b[e - 4] = f; }
    __device__ void keep() { asm volatile("" : "+v"(a), "+v"(b)); }
};
// Columns j .. j + 7 (`absent` eight times where p is NULL).
template <bool LAST = false, typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p, int j, float absent = 0.f) {
    Raw8<T> o;
    if (p) {
        if constexpr (LAST) o.load_last(p + j);
        else o.load(p + j);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) o.set(e, absent);
    }
    return o;
}
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(u16* p, float v) {
    const __bf16 b = (__bf16)v;
    *p = __builtin_bit_cast(u16, b);
}
// Columns j + skip .. j + 7.
template <typename T>
__device__ __forceinline__ void store8(T* p, int j, int skip, const float* v) {
    if (skip == 0) {
        Raw8<T> o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.set(e, v[e]);
        o.store(p + j);
    } else {
#pragma unroll
        for (int e = 1; e < 8; ++e)
            if (e >= skip) put(p + j + e, v[e]);
    }
}
// The columns of vector k of a row of h >= 8: the last vector of a row of no whole number of vectors is moved back to the row's
// end and has `skip` columns of the one before it, which count for nothing: they are left out of the sums over a row and not
// stored (where a result takes an input's place they may have been read after another thread wrote them).  A vector behind the
// last one (skip = 8) reads as that.  So no load of a row has a branch: with elements one by one at the end of a row, N=1003
// h=2050 took three times as long.
struct Columns {
    int j, skip;
    __device__ Columns(int k, int h) {
        j = k * 8 < h - 8 ? k * 8 : h - 8;
        skip = k * 8 - j < 8 ? k * 8 - j : 8;
    }
};

// Sum over 16 lanes, in all of them: every lane adds the same values in the same tree.
template <int ROT>
__device__ __forceinline__ float add_rotated(float v) {
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + ROT, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum16(float v) {
    return add_rotated<1>(add_rotated<2>(add_rotated<4>(add_rotated<8>(v))));
}
__device__ __forceinline__ float lane(float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); }
__device__ __forceinline__ float sum32(float v) {      // (two halves of a wavefront, each in all of its lanes)
    v = sum16(v);
    return v + __shfl_xor(v, 16, 64);
}
__device__ __forceinline__ float sum64(float v) {
    v = sum16(v);
    return (lane(v, 0) + lane(v, 16)) + (lane(v, 32) + lane(v, 48));
}

// Sums of K values over the threads of a row, a fixed tree: rows are held by 16 or 32 LANES, or (LANES = 64) by `waves` whole
// wavefronts of the workgroup, the first of them `wave0`.  Several meet in LDS, in the half of `sh` that `turn` names (so that one
// barrier per sum is enough: a thread that writes a half has passed the barrier behind which all others have read what it held).
template <int K, int LANES>
__device__ __forceinline__ void row_sums(float* v, float (*sh)[K_ROW_SUMS], int& turn, int wave0, int waves) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = LANES == 16 ? sum16(v[k]) : LANES == 32 ? sum32(v[k]) : sum64(v[k]);
    if (LANES == 64 && waves > 1) {
        float* at = sh[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) at[(threadIdx.x >> 6) * K + k] = v[k];
        __syncthreads();
        const int l = threadIdx.x & 15;      // (at most 16 wavefronts)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum16(l < waves ? at[(wave0 + l) * K + k] : 0.f);
    }
}

// The sums over tokens: `ranges` groups of threads (`rows` groups of `threads` threads in a workgroup) take up to `each` rows, one
// at a time: group c rows c, c + ranges, ... (`step` = ranges: what the chip reads at one time lies together), or, under a gate of
// several rows, `each` rows from c * each on (step = 1), so that a row of the gate has few groups to be summed over.  What
// workgroup b has summed goes to row b of the partial matrices (there are `parts`), which a last launch adds up in order; with a
// single workgroup it goes to the results themselves.
// dgate with several rows: a row of the gate whose tokens lie in one range is written where it ends; one that continues in the
// next range goes to row c of `tail`, one that began before (and ends or continues) to row c of `head`, c the range.
struct ColumnSums {
    float *dw, *db, *dw_post, *db_post, *dgate, *head, *tail;
    int ranges, each, parts, pitch;      // (rows of the partial matrices are `pitch` floats apart)
    int rows, threads, step;
};

// Parts of the formulas that a kernel is compiled for.
enum : int { NORM_POST = 1, NORM_GATE = 2, NORM_FULL = 4 };      // FULL: layer norms, or db or db_post is wanted

// Where the sums over tokens of a thread's columns are kept: kind 0 is dw, the others are numbered as they are there.  C = 1
// (up to 8192 columns): two kinds in registers, the others in LDS.  C = 2 (up to 16384): two in LDS, one in registers, the others
// in the workgroup's row of the partial matrices, which the L2 holds.  C = 4 (up to 32768): one in LDS, the others there.
template <int C, int PARTS>
struct Kinds {
    static constexpr bool POST = PARTS & NORM_POST, GATE = PARTS & NORM_GATE, FULL = PARTS & NORM_FULL;
    static constexpr int DW = 0, DWP = 1, DG = 1 + POST, DB = 1 + POST + GATE, DBP = DB + 1;
    static constexpr int COUNT = 1 + POST + GATE + FULL * (1 + POST);
    static constexpr int LDS0 = C == 1 ? 2 : 0, LDS1 = C == 1 ? COUNT : C == 4 || COUNT < 2 ? 1 : 2;      // kinds in LDS
    static constexpr bool in_registers(int kind) { return C == 1 ? kind < 2 : C == 2 && kind == 2; }
    static constexpr int SLOTS = LDS1 > LDS0 ? LDS1 - LDS0 : (C == 1 ? 1 : 0);
};

// Rows of 8 to 8192 C columns in one pass (N=512 h=32768 bf16: 117 us, with a launch for each step 290).  C = 1: a row's values
// stay in registers between the sums over it and dx and dy, and a thread's columns are the same in every row of its range, so the
// sums over tokens stay on the chip too.  C > 1: the inputs are read again for every step, from the caches (below), and some of the
// sums over tokens go through the L2 (Kinds, above).
//
// Of 128 registers a thread, 68 of the 200 instances spill: with C = 4 all (bf16 2 to 82 registers, fp32 28 to 107), and with a post norm
// and a gate together most others (1 to 26; bf16 with whole wavefronts and C = 1 at most 2).
//
// A workgroup fills a CU (up to 1024 threads of up to 128 registers), with as many rows at a time as it holds: fewer partial sums
// to write and add up than with a workgroup per row (N=4096 h=4096: 256 rows of them in place of 512).
template <typename T, typename TD, typename TG, int C, int LANES, int PARTS>
__global__ __launch_bounds__(1024) void block_norm_bwd_kernel(BlockNormGrad p, ColumnSums s) {
    using K = Kinds<C, PARTS>;
    constexpr bool POST = K::POST, GATE = K::GATE, FULL = K::FULL;
    __shared__ float sh[2][K_ROW_SUMS];
    __shared__ float4 lds[K::SLOTS ? K::SLOTS * 2 * C * 1024 : 1];
    int turn = 0;
    const int threads = LANES < 64 ? LANES : s.threads, waves = threads >> 6;
    const int group = LANES < 64 ? threadIdx.x / LANES : __builtin_amdgcn_readfirstlane(threadIdx.x / threads);
    const int t = threadIdx.x - group * threads, c0 = blockIdx.x * s.rows + group;
    const int64_t first = s.step == 1 ? (int64_t)c0 * s.each : c0;
    const int i0 = first < p.N ? (int)first : p.N, i1 = s.step == 1 && p.N - i0 > s.each ? i0 + s.each : p.N;
    const int L = GATE ? (int)(p.N / p.gate_rows) : 1;
    const float inv_h = 1.f / p.h;
    int j[C], skip[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const Columns cols(c * threads + t, p.h);
        j[c] = cols.j;
        skip[c] = cols.skip;
    }
    float reg[C == 4 ? 4 : 2][8];      // of a kind (C = 1), of a vector (C = 2), nothing (C = 4)
    auto in_reg = [&](int kind, int c) -> float* { return reg[C == 1 ? (kind < 2 ? kind : 0) : c]; };
    auto slot = [&](int kind, int c, int half) -> float4& {
        return lds[(((kind - K::LDS0) * C + c) * 2 + half) * 1024 + threadIdx.x];
    };
    auto matrix = [&](int kind) {
        if (POST && kind == K::DWP) return s.dw_post;
        if (GATE && kind == K::DG) return s.dgate;
        return kind == K::DW ? s.dw : kind == K::DB ? s.db : s.db_post;
    };
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) reg[k][e] = 0.f;
#pragma unroll
    for (int k = K::LDS0; k < K::LDS1; ++k)
#pragma unroll
        for (int c = 0; c < C; ++c) slot(k, c, 0) = slot(k, c, 1) = make_float4(0.f, 0.f, 0.f, 0.f);
    // the values of a kind that is not in registers: v, or what is kept with `add` more
    auto kept = [&](int kind, int c, bool fresh, float* v) {
        if (kind < K::LDS1) {
            const float4 a = slot(kind, c, 0), b = slot(kind, c, 1);
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
            v[4] += b.x; v[5] += b.y; v[6] += b.z; v[7] += b.w;
        } else if (!fresh) {
            const Raw8<float> a = load8(matrix(kind) + (size_t)blockIdx.x * s.pitch, j[c]);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += a[e];
        }
    };
    auto keep = [&](int kind, int c, const float* v) {
        if (kind < K::LDS1) {
            slot(kind, c, 0) = make_float4(v[0], v[1], v[2], v[3]);
            slot(kind, c, 1) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            store8(matrix(kind) + (size_t)blockIdx.x * s.pitch, j[c], skip[c], v);
        }
    };
    auto add = [&](int kind, int c, bool fresh, float* v) {
        if (K::in_registers(kind)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) in_reg(kind, c)[e] += v[e];
        } else if (kind < K::LDS1 || matrix(kind)) {
            kept(kind, c, fresh, v);
            keep(kind, c, v);
        }
    };
    // What is read of a row.  C = 1: once, and kept in registers from the first sums to the last.  C > 1: again in every step, from
    // the caches (two vectors of everything at once do not fit: N=2048 h=16384, kept, 124 us for bf16 RMS norms, 215 for fp32 ones
    // and 270 with everything; read again, 127, 196 and 257, which a third kind of sums in registers made 227).
    struct Values {
        Raw8<TD> dH;
        Raw8<TG> dr;
        Raw8<T> r, y, gate;
    };
    struct Statistics {
        float m1, rho1, m2, rho2;
    };
    auto load_statistics = [&](int i) {
        Statistics q;
        i = i < p.N ? i : p.N - 1;
        if constexpr (POST) {
            q.m1 = p.stats[i];
            q.rho1 = p.stats[(size_t)p.N + i];
        }
        q.m2 = p.stats[2 * (size_t)p.N + i];
        q.rho2 = p.stats[3 * (size_t)p.N + i];
        return q;
    };
    auto load_first = [&](Values& v, int i, int c) {
        const size_t at = (size_t)(i < p.N ? i : p.N - 1) * p.h;
        v.dH = load8((const TD*)p.dH + at, j[c]);
        v.r = load8((const T*)p.r + at, j[c]);
    };
    auto load_second = [&](Values& v, int i, int c) {
        i = i < p.N ? i : p.N - 1;
        const size_t at = (size_t)i * p.h;
        v.dr = load8(p.dr ? (const TG*)p.dr + at : nullptr, j[c]);
        if constexpr (POST || GATE) v.y = load8((const T*)p.y + at, j[c]);
        if constexpr (GATE) v.gate = load8((const T*)p.gate + (size_t)(i / L) * p.h, j[c]);
    };
    struct Vectors {
        Raw8<T> w, wp, bp;
    };
    auto load_vectors = [&](int c) {
        Vectors q;
        q.w = load8((const T*)p.w, j[c], 1.f);
        if constexpr (POST) q.wp = load8((const T*)p.w_post, j[c], 1.f);
        if constexpr (POST && GATE) q.bp = load8((const T*)p.b_post, j[c]);
        // what a skipped column would add to the sums over a row has its weight as a factor
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            q.w.set(e, e < skip[c] ? 0.f : q.w[e]);
            if constexpr (POST) q.wp.set(e, e < skip[c] ? 0.f : q.wp[e]);
        }
        return q;
    };
    Values v;
    Vectors q;
    Statistics u = load_statistics(i0);
    if constexpr (C == 1) {
        load_first(v, i0, 0);
        load_second(v, i0, 0);
        q = load_vectors(0);
    }
    for (int it = 0; it < s.each; ++it) {
        const int i = i0 + it * s.step;
        const bool live = i < i1, fresh = it == 0;      // (a workgroup's groups go through the same barriers)
        // (the vectors stay as they are stored: converted ahead of the loop they take twice the registers)
        if constexpr (C == 1) {
            q.w.keep();
            if constexpr (POST) q.wp.keep();
            if constexpr (POST && GATE) q.bp.keep();
        }
        const size_t at = (size_t)(live ? i : 0) * p.h;
        constexpr int M = FULL ? 2 : 1;      // sums over a row: of a value times rh or yh and, for its mean, of the value
        float rh[8], g[C][8], sums[2] = {0.f, 0.f};
        auto first_step = [&](int c) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                rh[e] = (FULL ? v.r[e] - u.m2 : v.r[e]) * u.rho2;
                g[c][e] = v.dH[e] * q.w[e];
            }
        };
        auto normed_y = [&](const Raw8<T>& y, float m1, float rho1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) rh[e] = (FULL ? y[e] - m1 : y[e]) * rho1;
        };
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (C > 1) {
                load_first(v, i, c);
                q = load_vectors(c);
            }
            first_step(c);
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o[e] = v.dH[e] * rh[e];
                sums[0] += g[c][e] * rh[e];
                if constexpr (FULL) sums[1] += g[c][e];
            }
            if (live) add(K::DW, c, fresh, o);
            if constexpr (FULL) {
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = v.dH[e];
                if (live) add(K::DB, c, fresh, o);
            }
        }
        row_sums<M, LANES>(sums, sh, turn, group * waves, waves);
        const float mar = sums[0] * inv_h, ma = FULL && p.center ? sums[1] * inv_h : 0.f;
        float more[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (C > 1) {
                load_first(v, i, c);
                load_second(v, i, c);
                q = load_vectors(c);
                first_step(c);
            }
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) g[c][e] = v.dr[e] + u.rho2 * ((FULL ? g[c][e] - ma : g[c][e]) - rh[e] * mar);
            if (live) store8((TG*)p.dx + at, j[c], skip[c], g[c]);
            if constexpr (POST) normed_y(v.y, u.m1, u.rho1);      // from here on, rh is yh
            if constexpr (GATE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = p.scale * (POST ? rh[e] * q.wp[e] + q.bp[e] : v.y[e]) * g[c][e];
                // (sums of one row of the gate begin where it does)
                if (live) add(K::DG, c, fresh || (L < p.N && i % L == 0), o);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) g[c][e] *= GATE ? p.scale * v.gate[e] : p.scale;
            if constexpr (POST) {
                if constexpr (FULL) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = g[c][e];
                    if (live) add(K::DBP, c, fresh, o);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = g[c][e] * rh[e];
                    g[c][e] *= q.wp[e];
                    more[0] += g[c][e] * rh[e];
                    if constexpr (FULL) more[1] += g[c][e];
                }
                if (live) add(K::DWP, c, fresh, o);
            }
        }
        // nothing of the row itself is needed from here on: the next row's values come while this one's second sums are formed
        const float m1 = u.m1, rho1 = u.rho1;
        if (it + 1 < s.each) {
            u = load_statistics(i + s.step);
            if constexpr (C == 1) {
                load_first(v, i + s.step, 0);
                load_second(v, i + s.step, 0);
            }
        }
        if constexpr (POST) {
            row_sums<M, LANES>(more, sh, turn, group * waves, waves);
            const float mky = more[0] * inv_h, mk = FULL && p.center ? more[1] * inv_h : 0.f;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if constexpr (C > 1) normed_y(load8((const T*)p.y + at, j[c]), m1, rho1);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[c][e] = rho1 * ((FULL ? g[c][e] - mk : g[c][e]) - rh[e] * mky);
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c)
            if (p.dy && live) store8((TG*)p.dy + at, j[c], skip[c], g[c]);
        if (GATE && L < p.N && p.dgate && live && (L == 1 || (i + 1) % L == 0 || i + 1 == i1)) {
            const int k = i / L;
            float* o = (int64_t)k * L < i0 ? s.head + (size_t)c0 * s.pitch
                                           : (i + 1) % L == 0 ? p.dgate + (size_t)k * p.h : s.tail + (size_t)c0 * s.pitch;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float o8[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (K::in_registers(K::DG)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        o8[e] = in_reg(K::DG, c)[e];
                        in_reg(K::DG, c)[e] = 0.f;
                    }
                } else {
                    kept(K::DG, c, false, o8);
                    if (K::DG < K::LDS1) slot(K::DG, c, 0) = slot(K::DG, c, 1) = make_float4(0.f, 0.f, 0.f, 0.f);
                }
                store8(o, j[c], skip[c], o8);
            }
        }
    }
    // What the groups of the workgroup have summed, added up in order in LDS.  (Kinds in registers come last: they take a slot.)
#pragma unroll
    for (int k = K::COUNT - 1; k >= 0; --k) {
        if (C == 1 && k < 2) {
            __syncthreads();
            lds[threadIdx.x] = make_float4(reg[k][0], reg[k][1], reg[k][2], reg[k][3]);
            lds[1024 + threadIdx.x] = make_float4(reg[k][4], reg[k][5], reg[k][6], reg[k][7]);
        }
        float* out = matrix(k);
        if (!out || (GATE && k == K::DG && L < p.N)) continue;
        if (C > 1 && k >= K::LDS1) {      // (a workgroup is one group)
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (K::in_registers(k)) store8(out + (size_t)blockIdx.x * s.pitch, j[c], skip[c], in_reg(k, c));
            continue;
        }
        __syncthreads();
        const float* from = reinterpret_cast<const float*>(lds + (C == 1 && k < 2 ? 0 : (k - K::LDS0) * C * 2 * 1024));
        for (int col = threadIdx.x; col < p.h; col += blockDim.x) {
            int vec = col >> 3;
            const int e = col - Columns(vec, p.h).j, c = C == 1 ? 0 : vec / threads;
            vec -= c * threads;
            float q = 0.f;
            for (int r = 0; r < s.rows; ++r) q += from[((c * 2 + (e >> 2)) * 1024 + r * threads + vec) * 4 + (e & 3)];
            out[(size_t)blockIdx.x * s.pitch + col] = q;
        }
    }
}

// Whether rows of h columns are held by threads in the backward pass.
constexpr int MIN_COLUMNS = 8, BWD_MAX_COLUMNS = 32768;
static inline int bwd_vectors(int64_t h) { return h <= 8192 ? 1 : h <= 16384 ? 2 : 4; }      // of a thread
static inline bool bwd_in_one_pass(int64_t h) { return h >= MIN_COLUMNS && h <= BWD_MAX_COLUMNS; }

template <typename T, typename TD, typename TG, int PARTS>
static void launch_bwd_parts(const BlockNormGrad& p, const ColumnSums& s, hipStream_t st) {
    const dim3 grid(s.parts), block(s.rows * s.threads);
    if (s.threads == 16) hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, 1, 16, PARTS>), grid, block, 0, st, p, s);
    else if (s.threads == 32) hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, 1, 32, PARTS>), grid, block, 0, st, p, s);
    else if (bwd_vectors(p.h) == 1) hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, 1, 64, PARTS>), grid, block, 0, st, p, s);
    else if (bwd_vectors(p.h) == 2) hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, 2, 64, PARTS>), grid, block, 0, st, p, s);
    else hipLaunchKernelGGL((block_norm_bwd_kernel<T, TD, TG, 4, 64, PARTS>), grid, block, 0, st, p, s);
}
template <typename T, typename TD, typename TG>
static hipError_t launch_bwd_one_pass(const BlockNormGrad& p, const ColumnSums& s, hipStream_t st) {
    switch ((p.post ? NORM_POST : 0) | (p.gate ? NORM_GATE : 0) | (p.center || p.db || p.db_post ? NORM_FULL : 0)) {
        case 0: launch_bwd_parts<T, TD, TG, 0>(p, s, st); break;
        case 1: launch_bwd_parts<T, TD, TG, 1>(p, s, st); break;
        case 2: launch_bwd_parts<T, TD, TG, 2>(p, s, st); break;
        case 3: launch_bwd_parts<T, TD, TG, 3>(p, s, st); break;
        case 4: launch_bwd_parts<T, TD, TG, 4>(p, s, st); break;
        case 5: launch_bwd_parts<T, TD, TG, 5>(p, s, st); break;
        case 6: launch_bwd_parts<T, TD, TG, 6>(p, s, st); break;
        case 7: launch_bwd_parts<T, TD, TG, 7>(p, s, st); break;
    }
    return hipGetLastError();
}
hipError_t launch_bwd_one_pass_f32(const BlockNormGrad& p, const ColumnSums& s, hipStream_t st);
hipError_t launch_bwd_one_pass_bf16(const BlockNormGrad& p, vp_dtype dH_dt, vp_dtype grad_dt, const ColumnSums& s, hipStream_t st);

}  // namespace vp
