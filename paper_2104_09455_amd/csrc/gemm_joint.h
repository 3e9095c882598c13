// Small linear layers of 16-bit activations in one launch (int8 weights in either order at any address, up to 1024 values of k,
// unprotected or thread-level): quantised and multiplied by the same workgroup, all of k at once.
//
// A workgroup of eight wavefronts takes 32 rows and 64 columns.  Each wavefront asks for its k tile of weights (128 values of k of all the
// columns) before anything else, then for its four rows of activations, which it quantises into LDS; the rows of all meet there, each
// wavefront multiplies its k tile, the eight partial tiles meet in LDS, and wavefront (b, r) adds, compares and stores rows 16 b + 4 g + r,
// four adjacent columns to a lane.  So the round trips to memory are two side by side, where the quantisation as a launch of its own and a
// product behind it have two launches and four of them in series.
//   Weights N x K: whole lines through 2 KB of LDS of the wavefront's own into fragments; rows off the dword in whole dwords, shifted.
//   Weights K x N: a lane reads four columns of sixteen k and turns them in registers (16 x 4 bytes), which are the fragments of
//   four MFMAs: fragment j of lane c is column 4 c + j, for the other order too, so that a lane holds four columns of its rows.
// Checked: every MFMA goes out twice, the second into one block for the four fragments of a row block; its elements and the sum of
// the four fragments' agree modulo 2^32 (replication with single accumulation, Sec. 5.1), and a flipped bit never changes a sum by a
// multiple of that.
// Bound: latencies; at 1024 values of k the quantisation (1 us) and the partial tiles' way through LDS beside them.  Measured, bf16, residual,
// thread-level, us in a graph (two launches / so): 16 x 1000 x 1000 5.4 / 6.9, 64 x 512 x 512 5.5 / 5.9, 300 x 1000 x 1000 8.9 / 7.3, K x N
// 64 x 512 x 512 8.4 / 5.8, 300 x 1000 x 1000 10.1 / 7.9 (unprotected 0.3 less); a launch less is 3.3 us less of the host's time, which is what a
// program that does not record a graph waits for (calls in a row: 16 x 1000 x 1000 8.7 / 7.2, 64 x 512 x 512 8.3 / 6.4).
// Beyond a round of workgroups the tilings are level or ahead: 300 x 2048 x 1024 (320 of them) 13.0 / 13.1, K x N 10.9 / 13.9, 1500 x 512 x 512 (376)
// 12.2 / 10.9, K x N 8.7 / 10.9.
#pragma once
#include "quantize.h"

namespace abft {

enum { JOINT_NK = 0, JOINT_NK_BYTES = 1, JOINT_KN = 2 };   // weights N x K in rows at whole dwords, at any address; K x N
constexpr int JOINT_WAVES = 8, JOINT_M = 32, JOINT_N = 64, JOINT_MAX_K = 1024;
constexpr int joint_row(int k) { return (k + 127) / 128 * 128; }   // bytes of a row of A in LDS
constexpr int joint_lds_bytes(int k, int layout, bool checked) {
    const int held = JOINT_M * joint_row(k) + (layout == JOINT_KN ? 0 : JOINT_WAVES * 2048), sums = JOINT_WAVES * 8 * (checked ? 1280 : 1024);
    return held > sums ? held : sums;
}

template <int OUT, int EPI, int LAYOUT, bool CHECKED>
__global__ __launch_bounds__(64 * JOINT_WAVES, 4) void gemm_joint_kernel(const GemmArgs p) {
    typedef Mma<DT_I8, 16> MMA;
    typedef MMA::Acc Acc;
    constexpr int W = JOINT_WAVES;
    constexpr bool KN = LAYOUT == JOINT_KN, BYTES = LAYOUT == JOINT_NK_BYTES;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ float scales[JOINT_M];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lrow = lane & 15, lgrp = lane >> 4, crow = lane >> 3, chunk = (lane & 7) * 16;
    const int M = p.M, N = p.N, K = p.K;
    int tile_m, tile_n;
    tile_of_block((int)blockIdx.x, p.tiles_m, p.tiles_n, tile_m, tile_n);
    const int bm0 = tile_m * JOINT_M, bn0 = tile_n * JOINT_N;
    const int nkt = (K + 127) >> 7, arow = nkt * 128;
    const int kt = wave;         // this wavefront's k tile
    const bool busy = kt < nkt;

    // ---- weights: the k tile of 64 columns in 32 registers (off the dword: 40)
    struct Tile {
        i32x4 v[KN ? 1 : 8];
        int more[BYTES ? 8 : 1];
        int row[KN ? 32 : 1];   // K x N: four columns of k = 64 s + 16 lgrp + e at 16 s + e
    };
    // N x K: load q covers rows 8 (q % 2) + crow of turn q / 2, whose row r is column 4 r + q / 2.  Columns outside take the last one's weights,
    // and their sums are not stored.
    const char* const base = p.B + (KN ? 0 : (long long)bn0 * p.ldb);
    unsigned at_row[KN ? 1 : 8];
    if constexpr (!KN) {
#pragma unroll
        for (int q = 0; q < 8; ++q) at_row[q] = (unsigned)min(4 * ((q & 1) * 8 + crow) + (q >> 1), N - 1 - bn0) * (unsigned)p.ldb;
    }
    // K x N: this lane's four columns, read early by `over` bytes where N ends inside them
    const int col4 = bn0 + 4 * lrow, over = KN ? min(max(col4 + 4 - N, 0), 3) : 0;
    const unsigned at_col = KN ? (unsigned)min(col4, N - 4) : 0u;
    const unsigned chunk_at = (unsigned)min(kt * 128 + chunk, K - 16);
    Tile t;
    if (busy) {
        if constexpr (KN) {
            if ((kt + 1) * 128 <= K) {
                const unsigned mine = (unsigned)(lgrp * 16) * (unsigned)p.ldb + at_col;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 16; ++e) t.row[16 * s + e] = ld4u(base + (long long)(kt * 128 + s * 64 + e) * p.ldb + mine);
            } else {
                // (rows beyond K, multiplied with zeros: the last one again)
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        t.row[16 * s + e] = ld4u(base + (long long)min(kt * 128 + s * 64 + lgrp * 16 + e, K - 1) * p.ldb + at_col);
            }
        } else {
            // (chunks beyond K, multiplied with zeros, and one that K cuts: the last 16 bytes of the row)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const char* const from = base + (at_row[q] + chunk_at);
                if constexpr (BYTES) {
                    const int by = (int)(reinterpret_cast<uintptr_t>(from) & 3u);
                    t.v[q] = ld16u(from - by);
                    t.more[q] = ld4u(from - by + (by ? 16 : 12));
                } else {
                    t.v[q] = ld16u(from);
                }
            }
        }
    }

    // ---- A: row m's 16 bytes c at c ^ (m % 8), zeros behind K.  A wavefront's four rows, up to two chunks of eight values to a lane of each
    char* const as = smem;
    i32x4 x[4][2];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const char* const row = p.A + min(bm0 + wave * 4 + r, M - 1) * p.lda * 2;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int k = (c * 64 + lane) * 8;
            x[r][c] = k < K ? row_chunk16(row, k, K) : i32x4{0, 0, 0, 0};
        }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const unsigned top = (unsigned)chunk_magnitude(x[r][1], chunk_magnitude(x[r][0], 0));
        const GroupScale g = group_scale<OUT>(wave_max(max(top & 0xffffu, top >> 16)));
        const int m = wave * 4 + r;
        if (lane == 0) scales[m] = g.scale;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int k = (c * 64 + lane) * 8;
            if (k < arow) *reinterpret_cast<i32x2*>(as + m * arow + (((k >> 4) ^ (m & 7)) << 4) + (k & 8)) = quantize_chunk<OUT>(x[r][c], g);
        }
    }
    __syncthreads();

    // ---- products: acc[b][j] of row block b and fragment j
    Acc acc[2][4], chk[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][j] = Acc{0, 0, 0, 0};
        int zero = 0;
        if constexpr (CHECKED) asm("" : "+v"(zero));   // (or the block would be the first fragment's as far as the two agree, and be merged with it)
        chk[b] = Acc{zero, 0, 0, 0};
    }
    char* const own = smem + JOINT_M * arow + wave * 2048;   // (N x K)
    int to[2], at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) to[h] = (h * 8 + crow) * 128 + (chunk ^ ((crow >> 1) * 16 + 64 * h));
#pragma unroll
    for (int s = 0; s < 2; ++s) at[s] = lrow * 128 + ((4 * s + lgrp) ^ (lrow >> 1)) * 16;
    if (busy) {
        if constexpr (KN) {
            if (bn0 + JOINT_N > N) {
#pragma unroll
                for (int e = 0; e < 32; ++e) t.row[e] = (int)((unsigned)t.row[e] >> (8 * over));
            }
        }
        i32x4 a[2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int b = 0; b < 2; ++b) a[b][s] = *reinterpret_cast<const i32x4*>(as + (b * 16 + lrow) * arow + (((kt * 8 + 4 * s + lgrp) ^ (lrow & 7)) << 4));
        const bool cut = (kt + 1) * 128 > K;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            i32x4 w[2];
            if constexpr (KN) {
                // column 4 c + j of sixteen k: byte j of sixteen registers
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        const unsigned sel = 0x04000400u + 0x01010101u * (unsigned)j;
                        const unsigned lo = __builtin_amdgcn_perm((unsigned)t.row[16 * s + 4 * d + 1], (unsigned)t.row[16 * s + 4 * d], sel);
                        const unsigned hi = __builtin_amdgcn_perm((unsigned)t.row[16 * s + 4 * d + 3], (unsigned)t.row[16 * s + 4 * d + 2], sel);
                        w[s][d] = (int)__builtin_amdgcn_perm(hi, lo, 0x05040100u);
                    }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    i32x4 x = t.v[2 * j + h];
                    if constexpr (BYTES) {
                        const unsigned by = (unsigned)(reinterpret_cast<uintptr_t>(base + (at_row[2 * j + h] + chunk_at)) & 3u);
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            x[d] = (int)__builtin_amdgcn_alignbyte((unsigned)(d < 3 ? t.v[2 * j + h][d + 1] : t.more[2 * j + h]), (unsigned)t.v[2 * j + h][d], by);
                    }
                    if (cut) x = shift_down(x, min(max(kt * 128 + chunk - (K - 16), 0), 15));
                    *reinterpret_cast<i32x4*>(own + to[h]) = x;
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) w[s] = *reinterpret_cast<const i32x4*>(own + at[s]);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    acc[b][j] = MMA::run(a[b][s], w[s], acc[b][j]);
                    if constexpr (CHECKED) chk[b] = MMA::run(a[b][s], w[s], chk[b]);
                }
        }
    }
    // ---- what this wavefront needs at the end: row 16 b + 4 lgrp + r, columns col4 .. col4 + 3
    const int b_end = wave >> 2, r_end = wave & 3, m_end = bm0 + 16 * b_end + 4 * lgrp + r_end;
    float col_scale[4], col_bias[4], res[EPI == EPI_ADD ? 4 : 1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = min(col4 + j, N - 1);
        col_scale[j] = p.col_scale[n];
        col_bias[j] = p.bias ? p.bias[n] : 0.f;
        if constexpr (EPI == EPI_ADD) res[j] = value16<OUT>(p.res + (min(m_end, M - 1) * p.ldr + n) * 2);
    }

    // test hook: a bit of one element, of the finished partial sum that holds k = K - 1 (-1) or of the finished sum (-2)
    if (p.f_row >= 0 && p.f_kt == -1 && kt == nkt - 1) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (bm0 + 16 * b + 4 * lgrp + r == p.f_row && col4 + j == p.f_col) acc[b][j][r] ^= 1 << p.f_bit;
    }
    __syncthreads();   // (the operands' place is the partial tiles')
    i32x4* const red = reinterpret_cast<i32x4*>(smem);
    int* const red_chk = reinterpret_cast<int*>(smem + W * 8 * 1024);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            red[(wave * 8 + 4 * b + r) * 64 + lane] = i32x4{acc[b][0][r], acc[b][1][r], acc[b][2][r], acc[b][3][r]};
            if constexpr (CHECKED) red_chk[(wave * 8 + 4 * b + r) * 64 + lane] = chk[b][r];
        }
    __syncthreads();
    i32x4 sum = red[wave * 64 + lane];
    unsigned twin = CHECKED ? (unsigned)red_chk[wave * 64 + lane] : 0u;
#pragma unroll
    for (int w = 1; w < W; ++w) {
        sum += red[(w * 8 + wave) * 64 + lane];
        if constexpr (CHECKED) twin += (unsigned)red_chk[(w * 8 + wave) * 64 + lane];
    }
    if (p.f_row >= 0 && p.f_kt == -2 && m_end == p.f_row) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (col4 + j == p.f_col) sum[j] ^= 1 << p.f_bit;
    }
    if constexpr (CHECKED) {
        // comparison (Sec. 5.2.2): four elements with their twin
        const unsigned four = ((unsigned)sum[0] + (unsigned)sum[1]) + ((unsigned)sum[2] + (unsigned)sum[3]);
        if (__any(four != twin) && lane == 0) atomicOr(p.flag, 1u);
    }
    if (m_end >= M) return;
    const float row_scale = scales[16 * b_end + 4 * lgrp + r_end];
    float z[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = scaled_value(sum[j], row_scale, col_scale[j], col_bias[j], 0);
    struct __attribute__((packed, aligned(2))) Any2 { int v; };
    struct __attribute__((packed, aligned(2))) Any4 { i32x2 v; };
    with_activation(p.act, [&](auto act) {
        if constexpr (EPI == EPI_GATED) {
            const int out = pack_out16<OUT>(as_float(act(z[0]) * z[1]), as_float(act(z[2]) * z[3])), left = (N - col4) / 2;
            char* const dst = p.C + (m_end * p.ldc + col4 / 2) * 2;
            if (left >= 2) reinterpret_cast<Any2*>(dst)->v = out;
            else if (left == 1) *reinterpret_cast<short*>(dst) = (short)out;
        } else {
            const int left = N - col4;
            char* const dst = p.C + (m_end * p.ldc + col4) * 2;
            float o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = as_float(act(z[j]) + res[j]);
            if (left >= 4) {
                reinterpret_cast<Any4*>(dst)->v = i32x2{pack_out16<OUT>(o[0], o[1]), pack_out16<OUT>(o[2], o[3])};
            } else {
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (j < left) store16<OUT>(dst + 2 * j, o[j]);
            }
        }
    });
}

}  // namespace abft
