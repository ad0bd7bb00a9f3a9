// The epilogue of the logits product of 8-bit integers: Y_ij = s_i t_j (integer sum), the statistics of pass S over Y, and Y in
// bf16 or fp32 where it is kept.  Accumulator layout, staging and stores as in vp_gemm_bf16_common.h.
//
// A lane has one token per row block and 64 columns, so the columns' scales come from LDS (four columns to a read, the same
// address in 32 lanes) and the token's scale is a factor of the exponent: exp(Y - m) = 2^(x c - x_max c) with x = t_j (integer
// sum) and c = s_i log2(e), which takes no more instructions per logit than exp alone.  (s_i is not negative, so x_max is the x of
// the largest Y.)
#pragma once

#include "vp_gemm_bf16_common.h"

namespace vp {

// What a thread brings in before the main loop: row m0 + tid's scale and label, column n0 + tid's scale.
struct I8Inputs {
    float row, col;
    int64_t label;
    __device__ __forceinline__ void load(const GemmBf16Params& g, const float* row_scales, const float* col_scales, int m0, int n0,
                                         int cols) {
        const int m = min(m0 + (int)threadIdx.x, g.M - 1), n = min(n0 + (int)threadIdx.x, cols - 1);
        row = row_scales[m];
        label = g.labels[m];
        col = col_scales[n];
    }
};

// Sums around a maximum: a NaN among the logits makes them NaN, also where a maximum, which leaves NaN out, has nothing else.  The
// exponents are then taken around NO_MAX, so a sum over nothing but columns past the end is 0 and one with a NaN is NaN.
constexpr float NO_MAX = -1e38f;
// What a wavefront's sum adds to the tile's, whose maximum is m.
__device__ __forceinline__ float part_sum_i8(float own, float sum, float m) { return own > -INFINITY ? sum * __expf(own - m) : sum; }
// The tile's maximum as it is stored: the fold leaves out sums around -inf, which those that are NaN must not be.
__device__ __forceinline__ float part_max_i8(float m, float sum) { return sum != sum ? fmaxf(m, -3.402823466e38f) : m; }

// Wavefront-private staging block -> global memory, fp32 (see flush_stage_bf16).
template <typename St, bool STREAM>
__device__ __forceinline__ void flush_stage_f32(const char* region, __amdgpu_buffer_rsrc_t rs, unsigned off, unsigned row_bytes,
                                                int orow, int ochunk, bool tail, unsigned off_tail, int n_tail, int rows_left) {
#pragma unroll
    for (int s0 = 0; s0 < St::STEPS; s0 += 8) {
        uintx4 v[8];
#pragma unroll
        for (int s = 0; s < 8; ++s)
            v[s] = *reinterpret_cast<const uintx4*>(region + ((s0 + s) * St::RPI + orow) * St::RS + ochunk * 16);
#pragma unroll
        for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(v[s]));
#pragma unroll
        for (int s = 0; s < 8; ++s)
            __builtin_amdgcn_raw_buffer_store_b128(v[s], rs, (int)(off + (unsigned)((s0 + s) * St::RPI) * row_bytes), 0, STREAM ? 2 : 0);
        if (tail) {
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                if ((s0 + s) * St::RPI >= rows_left) break;      // (uniform)
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    __builtin_amdgcn_raw_buffer_store_b32(
                        v[s][e], rs, (int)(e < n_tail ? off_tail + (unsigned)((s0 + s) * St::RPI) * row_bytes + 4u * e : OOB_OFFSET), 0, 0);
            }
        }
    }
}

// ALONE: the wavefront has its SIMD to itself.  Then the columns' scales stay in registers for all row blocks (read in every one they
// are waited for each time; N=4096 h=8192 V=256000: 10.4 -> 9.3 us a tile), and fp32 outputs are staged 128 columns at a time, else
// 64 (a region of 16.5 or 8.5 KB).
template <bool STREAM, int MI, bool ALONE = true>
__device__ __forceinline__ void gemm_epilogue_i8(floatx16 (&acc)[MI][4], const GemmBf16Params& g, int out_f32, const I8Inputs& in,
                                                 int tile_m, int tile_n, char* xchg, char* region) {
    constexpr int NJ = 4, WN = 2, WCOLS = 128, TM = 64 * MI;
    int lane = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
    asm volatile("" : "+v"(lane));      // (computed here, per tile: see gemm_epilogue_bf16)
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tid = wave * 64 + lane;
    const int wm = wave / WN, wn = wave % WN;
    const int l32 = lane & 31, hf = lane >> 5;
    const int m0 = tile_m * TM, n0 = tile_n * BN;
    float* xm = reinterpret_cast<float*>(xchg);      // [WN][256]
    float* xs = xm + WN * 256;                         // [WN][256]
    float* rows = xs + WN * 256;                       // [256]: scales of the tile's tokens
    float* cols = rows + 256;                          // [256]: of its columns
    int* labels = reinterpret_cast<int*>(cols + 256);  // [256]: the label's column in the tile, or -1
    static_assert((4 * 256 + 3 * 256) * 4 <= EPI_XCHG_BYTES, "exchange area");
    {
        const int64_t at = in.label - g.shard_offset - n0;
        rows[tid] = in.row;
        cols[tid] = in.col;
        labels[tid] = in.label >= 0 && at >= 0 && at < BN && at + n0 < g.N && m0 + tid < g.M ? (int)at : -1;
    }
    __syncthreads();
    const bool ragged = n0 + BN > g.N;      // (uniform)
    const int nvalid = g.N - (n0 + wn * WCOLS + 4 * hf);

    // OUT: 0 the statistics alone, 1 bf16, 2 fp32
    auto blocks = [&](auto out_c) {
        constexpr int OUT = decltype(out_c)::value;
        constexpr int SCOLS = OUT == 2 && !ALONE ? 64 : WCOLS, PARTS = WCOLS / SCOLS, PJ = NJ / PARTS;
        typedef typename std::conditional<OUT == 2, StageF32<SCOLS>, StageBf16<SCOLS>>::type St;
        constexpr int ELEM = OUT == 2 ? 4 : 2, PER = 16 / ELEM;
        const int orow = lane / St::LPR, ochunk = lane % St::LPR;
        const unsigned row_bytes = (unsigned)g.ldy * (unsigned)ELEM;
        const __amdgpu_buffer_rsrc_t rs =
            tile_rows_rsrc(OUT ? (char*)g.Y + (size_t)m0 * g.ldy * ELEM : nullptr, OUT ? (g.M - m0 < TM ? g.M - m0 : TM) : 0, row_bytes);
        const bool tail = n0 + WN * WCOLS > g.N && g.N % PER != 0;
        auto scales = [&](int j, int q) { return *reinterpret_cast<const floatx4*>(cols + wn * WCOLS + j * 32 + 8 * q + 4 * hf); };
        floatx4 kept[NJ][4];
        if constexpr (ALONE)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) kept[j][q] = scales(j, q);
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            __builtin_amdgcn_sched_barrier(0);      // one row block at a time (see gemm_epilogue_bf16)
            const int lr = wm * (32 * MI) + i * 32 + l32;
            float scale = rows[lr];
            const int at = labels[lr] - wn * WCOLS - 4 * hf;
            const int lab = at >= 0 && at < WCOLS && (at & 4) == 0 ? at : -1;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const floatx4 t = ALONE ? kept[j][q] : scales(j, q);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[i][j][4 * q + e] = (float)__builtin_bit_cast(int, (float)acc[i][j][4 * q + e]) * t[e];
                }
            if (ragged) {      // columns past the end of the shard: -inf, which leaves the maximum alone and adds 0 to the sum
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        acc[i][j][r] = j * 32 + 8 * (r >> 2) + (r & 3) < nvalid ? acc[i][j][r] * scale : -INFINITY;
                scale = 1.f;
            }
            float v = acc[i][0][0];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) v = fmaxf(v, acc[i][j][r]);
            v = fmaxf(v, __shfl_xor(v, 32, 64));
            // (-inf: no column but past the shard's end, which add 0, or NaN)
            const float c = scale * LOG2E, vc = (v == -INFINITY ? NO_MAX : v) * c;
            // (eight exponentials at a time: each has to be waited for)
            float part[8] = {};
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    float x[8];
#pragma unroll
                    for (int r = 0; r < 8; ++r) x[r] = fmaf(acc[i][j][8 * q + r], c, -vc);
#pragma unroll
                    for (int r = 0; r < 8; ++r) x[r] = exp2_fast(x[r]);
#pragma unroll
                    for (int r = 0; r < 8; ++r) part[r] += x[r];
                }
            float s = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
            s += __shfl_xor(s, 32, 64);
            if (hf == 0) {
                xm[wn * 256 + lr] = v * scale;
                xs[wn * 256 + lr] = s;
            }
            if (__builtin_amdgcn_ballot_w64(lab >= 0) != 0) {      // at most one element per row
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (lab == j * 32 + 8 * (r >> 2) + (r & 3)) x = acc[i][j][r];
                if (lab >= 0) g.part_tgt[m0 + lr] = x * scale;
            }
            if constexpr (OUT) {
#pragma unroll
                for (int part = 0; part < PARTS; ++part) {
                    const int ocol = n0 + wn * WCOLS + part * SCOLS + ochunk * PER;
                    const unsigned off_row = (unsigned)(wm * (32 * MI) + i * 32 + orow) * row_bytes + (unsigned)ocol * (unsigned)ELEM;
                    const unsigned off = ocol + PER <= g.N ? off_row : OOB_OFFSET;
                    const int n_tail = ocol + PER > g.N && ocol < g.N ? g.N - ocol : 0;
#pragma unroll
                    for (int j = 0; j < PJ; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            float y[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) y[e] = acc[i][part * PJ + j][4 * q + e] * scale;
                            char* to = region + l32 * St::RS + (j * 32 + 8 * q + 4 * hf) * ELEM;
                            if constexpr (OUT == 2) *reinterpret_cast<floatx4*>(to) = floatx4{y[0], y[1], y[2], y[3]};
                            else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
                        }
                    wave_lds_fence();
                    const int left = g.M - (m0 + wm * (32 * MI) + i * 32);
                    if constexpr (OUT == 2) flush_stage_f32<St, STREAM>(region, rs, off, row_bytes, orow, ochunk, tail, off_row, n_tail, left);
                    else flush_stage_bf16<St, STREAM>(region, rs, off, row_bytes, orow, ochunk, tail, off_row, n_tail, left);
                    wave_lds_fence();
                }
            }
        }
    };
    if (!g.Y) blocks(std::integral_constant<int, 0>{});
    else if (out_f32) blocks(std::integral_constant<int, 2>{});
    else blocks(std::integral_constant<int, 1>{});
    __syncthreads();
    if (tid < TM && m0 + tid < g.M) {
        const float a = xm[tid], b = xm[256 + tid], m = fmaxf(a, b);
        const float s = part_sum_i8(a, xs[tid], m) + part_sum_i8(b, xs[256 + tid], m);
        g.part_max[(size_t)tile_n * g.M + m0 + tid] = part_max_i8(m, s);
        g.part_sum[(size_t)tile_n * g.M + m0 + tid] = s;
    }
}

}  // namespace vp
