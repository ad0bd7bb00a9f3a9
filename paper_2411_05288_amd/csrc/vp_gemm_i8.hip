// The output layer's logits from 8-bit integers.  Many tokens: the fast kernel (vp_gemm_bf16_fast.h) with integer products, whose
// operands of 16 bytes hold 16 integers in place of 8 numbers; data movement, tiles and tile order are the same.  It is bound by the
// power limit, like the bf16 products (main loops at 1.5 to 1.7 GHz of 2.4): N=4096 h=8192 V=256000 2.5 POP/s, h=4096 V=128256
// 2.4.  Short sums: tiles in pairs, bound by their statistics and stores.  Few tokens: a kernel that is bound by reading W.
#include <climits>

#include "vp_gemm_bf16_fast.h"

namespace vp {

namespace {

typedef unsigned uintx4u __attribute__((ext_vector_type(4), aligned(2)));

// Few tokens: 32 TI of them and 32 WAVES vocabulary rows in a workgroup of WAVES wavefronts, which take 32 rows each.  W is read
// once, so what counts is that enough of it is on its way: a ring of SLOTS k tiles of 128 integers, all but one of them in flight.
// Up to 32 tokens two workgroups share a compute unit (80 KB of LDS each), so that one loads while the other is at its ends; beyond
// that one has it to itself (96 KB up to 64 tokens, 144 up to 128).  A load instruction takes 8 whole lines of 128 bytes (past the caches: W is not read again), 16 bytes per lane, straight into LDS.
//
// A slot holds rows of 128 bytes, of W and then of H.  Chunk c of row r (16 bytes) sits at position c ^ (r / 2 % 8): 16
// consecutive rows, which a read of LDS serves at a time, have the same chunk in 16 different groups of banks.
//
// N=1 h=4096 V=128256: 78 us (6.7 TB/s).  With the integers of H and the fold 87 us; 116 in the fast kernel; where all workgroups
// begin at the same k tile, whose lines lie in the same few memory channels, 11 more.
// Up to 64 tokens all sums, up to 128 the long ones: fast kernel -> this one, N=128 h=4096 V=128256 122 -> 110, h=8192 V=256000
// 413 -> 391, N=65 h=4096 V=128256 112 -> 102.
constexpr int FEW_K = 128, FEW_MOST = 128;
template <int TI, int WAVES, int SLOTS>
struct Few {
    static constexpr int COLS = 32 * WAVES, ROWS = 32 * TI, SLOT = (COLS + ROWS) * FEW_K;
    static constexpr int LOADS_W = COLS / 8 / WAVES, LOADS_H = (ROWS / 8 + WAVES - 1) / WAVES;
    // outputs of 32 tokens are staged in a slot; rows padded by 16 bytes
    static constexpr int STAGE_ROW = COLS * 4 + 16;
    static_assert(32 * STAGE_ROW <= SLOT, "staging exceeds a slot");
};

template <int TI, int WAVES, int SLOTS>
__global__ __launch_bounds__(64 * WAVES, 2) void gemm_i8_few_kernel(GemmI8Group gg) {
    using F = Few<TI, WAVES, SLOTS>;
    __shared__ __attribute__((aligned(1024))) char slot0[F::SLOT];
    __shared__ __attribute__((aligned(1024))) char slot1[F::SLOT];
    __shared__ __attribute__((aligned(1024))) char slot2[F::SLOT];
    __shared__ __attribute__((aligned(1024))) char slot3[SLOTS == 4 ? F::SLOT : 16];
    static_assert(SLOTS == 3 || SLOTS == 4, "slots");
    const GemmBf16Params& g = gg.base;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, hf = lane >> 5;
    int tile_m, tile_n;      // (one row of tiles)
    tile_of_block(blockIdx.x, gridDim.x, gridDim.x, 1, gg.total, tile_m, tile_n);
    const int shard = shard_of(gg, tile_n);
    const GemmBf16Shard& s = gg.sh[shard];
    const int n0 = (tile_n - gg.first[shard]) * F::COLS, k = g.K * 2;
    const unsigned w_bytes = (unsigned)s.rows * (unsigned)k, h_bytes = (unsigned)g.M * (unsigned)k;

    // this lane's columns are cbase + 8 (r / 4) + r % 4
    const int cbase = n0 + wave * 32 + 4 * hf;
    const float* col_scales = gg.col_scales[shard];
    float cs[16], rs[TI];
    int64_t label[TI];
#pragma unroll
    for (int r = 0; r < 16; ++r) cs[r] = col_scales[min(cbase + 8 * (r >> 2) + (r & 3), s.rows - 1)];
#pragma unroll
    for (int t = 0; t < TI; ++t) {
        const int m = min(t * 32 + l32, g.M - 1);
        rs[t] = gg.row_scales[m];
        label[t] = g.labels[m];
    }

    unsigned w_off[F::LOADS_W], h_off[F::LOADS_H];
#pragma unroll
    for (int i = 0; i < F::LOADS_W; ++i) {
        const int row = (wave * F::LOADS_W + i) * 8 + (lane >> 3), c = (lane & 7) ^ (row >> 1 & 7);
        w_off[i] = (unsigned)(n0 + row) * (unsigned)k + (unsigned)c * 16u;
    }
#pragma unroll
    for (int i = 0; i < F::LOADS_H; ++i) {
        const int row = (wave * F::LOADS_H + i) * 8 + (lane >> 3), c = (lane & 7) ^ (row >> 1 & 7);
        h_off[i] = (unsigned)row * (unsigned)k + (unsigned)c * 16u;
    }
    auto slot = [&](auto i) -> char* {
        constexpr int S = decltype(i)::value % SLOTS;
        if constexpr (S == 0) return slot0;
        else if constexpr (S == 1) return slot1;
        else if constexpr (S == 2) return slot2;
        else return slot3;
    };
    // The k advance is applied to the descriptors: a k tile past the end has empty ones, no access is made and zeros arrive, as
    // they do for rows past the end of W or H.  Every workgroup begins at another k tile (sums of integers have no order).
    const int nkt = k / FEW_K, turn = tile_n % nkt;
    auto load = [&](auto i, int kt) {
        char* to = slot(i);
        const int at = kt + turn < nkt ? kt + turn : kt + turn - nkt;
        const unsigned adv = (unsigned)(at * FEW_K);
        const unsigned wa = kt < nkt ? adv : w_bytes, ha = kt < nkt ? adv : h_bytes;
        const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)s.B + wa), 0, (int)(w_bytes - wa), 0x00020000);
        const __amdgpu_buffer_rsrc_t rh = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)g.A + ha), 0, (int)(h_bytes - ha), 0x00020000);
#pragma unroll
        for (int j = 0; j < F::LOADS_W; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, (lds_ptr)(to + (wave * F::LOADS_W + j) * 1024), 16, (int)w_off[j], 0, 0, 2);
#pragma unroll
        for (int j = 0; j < F::LOADS_H; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rh, (lds_ptr)(to + F::COLS * FEW_K + (wave * F::LOADS_H + j) * 1024), 16, (int)h_off[j], 0, 0, 0);
    };
    int w_at[4], h_at[4];      // of the four 32-wide steps of a k tile
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
        const int pos = ((2 * kk + hf) ^ (l32 >> 1 & 7)) * 16;
        w_at[kk] = (wave * 32 + l32) * FEW_K + pos;
        h_at[kk] = F::COLS * FEW_K + l32 * FEW_K + pos;
    }
    intx16 acc[TI] = {};
    auto multiply = [&](auto i) {
        const char* from = slot(i);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const intx4 w = *reinterpret_cast<const intx4*>(from + w_at[kk]);
#pragma unroll
            for (int t = 0; t < TI; ++t)
                acc[t] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, *reinterpret_cast<const intx4*>(from + h_at[kk] + t * 32 * FEW_K), acc[t], 0, 0, 0);
        }
    };
    // k tile kt: its loads are the oldest of those on their way; behind the barrier all wavefronts' have landed, and the slot of the
    // tile before is free.
    constexpr int PER = F::LOADS_W + F::LOADS_H, LATER = (SLOTS - 2) * PER;
    static_assert(LATER < 64, "memory counter");
    auto step = [&](auto i, int kt) {
        __builtin_amdgcn_s_waitcnt((LATER & 15) | ((LATER >> 4) << 14) | 0x70);      // vmcnt(LATER), lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load(std::integral_constant<int, decltype(i)::value + SLOTS - 1>{}, kt + SLOTS - 1);
        multiply(i);
    };
    constexpr std::integral_constant<int, 0> I0;
    constexpr std::integral_constant<int, 1> I1;
    constexpr std::integral_constant<int, 2> I2;
    constexpr std::integral_constant<int, 3> I3;
    load(I0, 0);
    load(I1, 1);
    if constexpr (SLOTS == 4) load(I2, 2);
    int kt = 0;
    for (int it = nkt / SLOTS; it > 0; --it, kt += SLOTS) {
        step(I0, kt);
        step(I1, kt + 1);
        step(I2, kt + 2);
        if constexpr (SLOTS == 4) step(I3, kt + 3);
    }
    if (kt < nkt) {
        step(I0, kt);
        if (kt + 1 < nkt) {
            step(I1, kt + 1);
            if (SLOTS == 4 && kt + 2 < nkt) step(I2, kt + 2);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0): nor do zeros past the end arrive in a slot any more
    __syncthreads();      // no wavefront reads a slot
    // the statistics of the wavefronts' columns; outputs are staged in slot 0
    float(*xm)[F::ROWS] = reinterpret_cast<float(*)[F::ROWS]>(slot1), (*xs)[F::ROWS] = xm + WAVES;

#pragma unroll
    for (int t = 0; t < TI; ++t) {
        if (t * 32 >= g.M) break;
        const int m = t * 32 + l32;
        float y[16], v = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            y[r] = cbase + 8 * (r >> 2) + (r & 3) < s.rows ? (float)acc[t][r] * cs[r] * rs[t] : -INFINITY;
            v = fmaxf(v, y[r]);
        }
        v = fmaxf(v, __shfl_xor(v, 32, 64));
        const float around = v == -INFINITY ? NO_MAX : v;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += exp2_fast((y[r] - around) * LOG2E);
        sum += __shfl_xor(sum, 32, 64);
        if (hf == 0) {
            xm[wave][m] = v;
            xs[wave][m] = sum;
        }
        const int64_t at = label[t] - s.offset - cbase;
        if (label[t] >= 0 && at >= 0 && at < 32 && (at & 4) == 0 && at + cbase < s.rows && m < g.M) {
            float target = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (at == 8 * (r >> 2) + (r & 3)) target = y[r];
            g.part_tgt[(size_t)shard * g.M + m] = target;
        }
        if (s.out) {
            if (t) __syncthreads();
            const int cols = min(F::COLS, s.rows - n0), rows = min(32, g.M - t * 32);
            const int elem = gg.out_f32 ? 4 : 2, per_row = F::COLS * elem / 16;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                char* to = slot0 + l32 * F::STAGE_ROW + (wave * 32 + 8 * q + 4 * hf) * elem;
                if (gg.out_f32) *reinterpret_cast<floatx4*>(to) = floatx4{y[4 * q], y[4 * q + 1], y[4 * q + 2], y[4 * q + 3]};
                else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(y[4 * q], y[4 * q + 1]), pack_bf16x2(y[4 * q + 2], y[4 * q + 3]));
            }
            __syncthreads();
            for (int i = threadIdx.x; i < rows * per_row; i += 64 * WAVES) {
                const int row = i / per_row, c = i % per_row * (16 / elem);
                const char* from = slot0 + row * F::STAGE_ROW + c * elem;
                char* to = (char*)s.out + ((size_t)(t * 32 + row) * s.ld + n0 + c) * elem;
                if (c + 16 / elem <= cols) *reinterpret_cast<uintx4u*>(to) = *reinterpret_cast<const uintx4*>(from);
                else
                    for (int e = 0; c + e < cols; ++e) {
                        if (gg.out_f32) ((float*)to)[e] = ((const float*)from)[e];
                        else ((u16*)to)[e] = ((const u16*)from)[e];
                    }
            }
        }
    }
    __syncthreads();
    for (int m = threadIdx.x; m < g.M; m += 64 * WAVES) {
        float v = xm[0][m], sum = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v = fmaxf(v, xm[w][m]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += part_sum_i8(xm[w][m], xs[w][m], v);
        g.part_max[(size_t)tile_n * g.M + m] = part_max_i8(v, sum);
        g.part_sum[(size_t)tile_n * g.M + m] = sum;
    }
}

// Tiles of 128 tokens and 256 vocabulary rows, two workgroups on a compute unit, so that one multiplies while the other is at its
// ends: where the sum is short, the statistics and stores of a tile take as long as its products.  A ring of three slots of 64
// integers (A's 128 rows, then B's 256, 64 bytes each, laid out as in vp_gemm_bf16_fast.h), one multiplied while two are on their
// way, one barrier per slot.  Tiles go in rounds of two for each compute unit, the last of them as long as a full one: N=509 V=50001 in
// 3 shards has 792 tiles for 512 places: 23 % of the places of two rounds stay empty.
// Where it is taken: sums of up to PAIR_MOST_K integers.  The fast kernel -> this one, us: N=509 h=1001 V=50001 fp32 76 -> 57, N=1000
// h=1536 V=50001 bf16 129 -> 111, N=4096 h=1024 V=32000 224 -> 182, h=2048 V=64000 647 -> 638, h=2560 V=64000 746 -> 791.
// STREAM: outputs bypass the caches where there is more than one round of tiles, as in the fast kernel, but not fp32 rows that
// share lines (N=509 h=1001 V=50001 in 3 shards: 78 us with it, 57 without; in whole lines, V=49152, 50 and 51).
constexpr int PAIR_MOST_K = 2048;
constexpr int PAIR_ROWS = 128, PAIR_K = 64, PAIR_SLOT = (PAIR_ROWS + BN) * PAIR_K;
static_assert(2 * StageF32<64>::BYTES <= PAIR_SLOT && StageBf16<128>::BYTES <= StageF32<64>::BYTES, "staging of two wavefronts exceeds a slot");

template <bool STREAM>
__global__ __launch_bounds__(256, 2) void gemm_i8_pair_kernel(GemmI8Group gg) {
    __shared__ __attribute__((aligned(1024))) char slot0[PAIR_SLOT];
    __shared__ __attribute__((aligned(1024))) char slot1[PAIR_SLOT];
    __shared__ __attribute__((aligned(1024))) char slot2[PAIR_SLOT];
    __shared__ __attribute__((aligned(16))) char xchg[EPI_XCHG_BYTES];
    const GemmBf16Params& g = gg.base;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int tiles_m = (g.M + PAIR_ROWS - 1) / PAIR_ROWS;
    int tile_m, tile_n;
    tile_of_block(blockIdx.x, gridDim.x, gridDim.x, tiles_m, gg.total, tile_m, tile_n);
    const int shard = shard_of(gg, tile_n);
    tile_n -= gg.first[shard];
    const GemmBf16Shard& s = gg.sh[shard];
    const int m0 = tile_m * PAIR_ROWS, n0 = tile_n * BN;
    const unsigned a_bytes = (unsigned)g.M * (unsigned)g.lda * 2u, b_bytes = (unsigned)s.rows * (unsigned)g.ldb * 2u;
    I8Inputs in;
    in.load(g, gg.row_scales, gg.col_scales[shard], m0, n0, s.rows);

    unsigned avoff[2], bvoff[4];
    half_voffsets<true, 2>(avoff, m0, g.lda, wave, lane);
    half_voffsets<true, 4>(bvoff, n0, g.ldb, wave, lane);
    int abase[4], bbase[4];
    frag_offsets<true, 2>(abase, wm, lane);
    frag_offsets<true>(bbase, wn, lane);
    auto slot = [&](auto i) -> char* {
        constexpr int S = decltype(i)::value % 3;
        if constexpr (S == 0) return slot0;
        else if constexpr (S == 1) return slot1;
        else return slot2;
    };
    const int steps = g.K * 2 / PAIR_K;
    auto load = [&](auto i, int at) {      // (past the end: empty descriptors, see gemm_i8_few_kernel)
        char* to = slot(i);
        const unsigned adv = at < steps ? (unsigned)(at * PAIR_K) : ~0u, aa = min(adv, a_bytes), ba = min(adv, b_bytes);
        const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)g.A + aa), 0, (int)(a_bytes - aa), 0x00020000);
        const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc((void*)((const char*)s.B + ba), 0, (int)(b_bytes - ba), 0x00020000);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (lds_ptr)(to + (wave * 2 + j) * 1024), 16, (int)avoff[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, (lds_ptr)(to + PAIR_ROWS * PAIR_K + (wave * 4 + j) * 1024), 16, (int)bvoff[j], 0, 0, 0);
    };
    floatx16 acc[2][4] = {};
    auto multiply = [&](auto i) {
        const char* from = slot(i);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            bf16x8 a[2], b[4];
#pragma unroll
            for (int t = 0; t < 2; ++t) a[t] = read_operand<true>(from, abase, t, kk);
#pragma unroll
            for (int t = 0; t < 4; ++t) b[t] = read_operand<true>(from + PAIR_ROWS * PAIR_K, bbase, t, kk);
            mfma_step<Epi::LogitsI8, 2>(acc, a, b);
        }
    };
    auto step = [&](auto i, int at) {
        __builtin_amdgcn_s_waitcnt(6 | 0x70);      // vmcnt(6): all but the last slot's loads; lgkmcnt(0)
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        load(std::integral_constant<int, decltype(i)::value + 2>{}, at + 2);
        multiply(i);
    };
    constexpr std::integral_constant<int, 0> I0;
    constexpr std::integral_constant<int, 1> I1;
    constexpr std::integral_constant<int, 2> I2;
    load(I0, 0);
    load(I1, 1);
    int at = 0;
    for (int it = steps / 3; it > 0; --it, at += 3) {
        step(I0, at);
        step(I1, at + 1);
        step(I2, at + 2);
    }
    if (at < steps) {
        step(I0, at);
        if (at + 1 < steps) step(I1, at + 1);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0)
    __syncthreads();

    GemmBf16Params e = g;
    e.N = s.rows;
    e.Y = (u16*)s.out;
    e.ldy = s.ld;
    e.shard_offset = s.offset;
    e.part_max = g.part_max + (size_t)gg.first[shard] * g.M;
    e.part_sum = g.part_sum + (size_t)gg.first[shard] * g.M;
    e.part_tgt = g.part_tgt + (size_t)shard * g.M;
    char* region = (wave < 2 ? slot0 : slot1) + (wave & 1) * StageF32<64>::BYTES;
    gemm_epilogue_i8<STREAM, 2, false>(acc, e, gg.out_f32, in, tile_m, tile_n, xchg, region);
}

}  // namespace

// Columns of a tile: a row of partial statistics each.
int gemm_i8_columns(int64_t N) { return N <= I8_NARROW_MOST ? 128 : BN; }

hipError_t launch_gemm_i8(const GemmI8Group& g0, hipStream_t st) {
    ProfScope prof(K_GEMM_I8, st);
    GemmI8Group g = g0;
    const int cols = gemm_i8_columns(g.base.M);
    g.total = 0;
    for (int r = 0; r < GEMM_GROUP_MAX; ++r) {
        g.first[r] = r < g.n ? g.total : INT_MAX;
        if (r < g.n) g.total += (int)ceil_div(g.sh[r].rows, cols);
    }
    g.slices = 1;
    auto few = [&](auto kernel, int waves) {
        hipLaunchKernelGGL(kernel, dim3(g.total), dim3(64 * waves), 0, st, g);
        return hipGetLastError();
    };
    if (g.base.M <= 32) return few(gemm_i8_few_kernel<1, 4, 4>, 4);
    if (g.base.M <= I8_NARROW_MOST) return few(gemm_i8_few_kernel<2, 4, 4>, 4);
    if (g.base.M <= FEW_MOST && g.base.K * 2 > PAIR_MOST_K) return few(gemm_i8_few_kernel<4, 8, 3>, 8);
    if (g.base.K * 2 > PAIR_MOST_K) return launch_fast_t<true, true, Epi::LogitsI8>(g, st);
    const int tiles = g.total * (int)ceil_div(g.base.M, PAIR_ROWS);
    bool stream = tiles > 2 * compute_unit_count();
    for (int r = 0; r < g.n; ++r) stream &= !(g.out_f32 && g.sh[r].ld % 16);
    if (stream) hipLaunchKernelGGL(gemm_i8_pair_kernel<true>, dim3(tiles), dim3(256), 0, st, g);
    else hipLaunchKernelGGL(gemm_i8_pair_kernel<false>, dim3(tiles), dim3(256), 0, st, g);
    return hipGetLastError();
}

}  // namespace vp
