// Products of few rows whose activations stay in registers (int8, weights N x K in 16-byte chunks, unprotected or thread-level): what
// decoding does with large weights, and bound by their bytes.
//
// A workgroup of eight wavefronts takes columns by the sixteen, one run of them after the other, and each wavefront one eighth of k, the
// same for all of them: its fragments of A (16 rows, 2 T of 64 values of k each) are read, or quantised, once and stay.  Weights go through registers, D k tiles of 16 columns x 128 bytes ahead and on into the next sixteen columns, and through
// 2 KB of LDS of the wavefront's own into fragments (loaded by whole lines: with a lane per row, as the fragments want them, an
// instruction of 1 KB takes the vector memory path 64 clocks, so 17).  An eighth of k is one run of a row, so that a workgroup
// reads eight places of each row at a time, spread over it.  The partial tiles of sixteen columns meet in LDS, two of them in turn with one
// barrier each; the wavefronts take turns to add them up, compare and store, while the others go on.
// Every product is issued twice where it is checked, into accumulators of its own (thread-level scheme on a tile of one
// fragment: replication); both sides are equal to the last bit unless something failed.
// Bound: the weights' bytes.  Measured, from memory, us (the tilings' kernels and a quantisation of its own / here): gated 1 x 12288 x 4096,
// 100 MB, 41 / 22 (launch and first latency 4, the rest at 5.6 TB/s), 1 x 8192 x 8192 43 / 28; a residual, 1 x 4096 x 12288 17.8 / 14.0, 1 x 4096 x
// 4096 7.6 / 5.6, 16 rows of it 10.4 / 8.7; pre-quantised gated 16 x 8192 x 4096 19.6 / 18.5, 16 x 8192 x 8192 33.1 / 29.9.  Two blocks of
// sixteen rows, level to 8 % ahead from 4096 values of k on and 10 to 30 % behind below, and four, behind by a fifth, were left to the tilings.
#pragma once
#include "gemm_configs.h"
#include "quantize.h"

namespace abft {

constexpr int RES_WAVES = 8;
// FROM16: chunks of eight values that a lane holds at most; 2^lg wavefronts share a row of up to eight, each takes two of up to sixteen; rows
// that are more are quantised by a launch of their own
constexpr int RES_HELD = 16;
constexpr int resident_parts_lg(int rows) { return rows <= 1 ? 3 : rows <= 2 ? 2 : rows <= 4 ? 1 : 0; }
constexpr bool resident_quantises(int rows, int k) {
    return rows <= 16 && (rows > RES_WAVES ? 2 : 1) * ((k + (512 << resident_parts_lg(rows)) - 1) / (512 << resident_parts_lg(rows))) <= RES_HELD;
}
constexpr int resident_lds_bytes(bool checked) { return RES_WAVES * (2048 + 2 * (checked ? 2 : 1) * 1024); }
constexpr int RES_DEEP = 8;   // k tiles ahead at most

struct ResidentArgs {
    GemmArgs g;      // FROM16: g.A and g.lda are the 16-bit activations'
    int unit, per, more;   // columns of a workgroup come by the unit, `per` of them, and the first `more` have one more
};

// T: k tiles of 128 of a wavefront at most; FROM16: A is not quantised yet (type OUT)
template <int OUT, int EPI, int T, bool CHECKED, bool FROM16>
__global__ __launch_bounds__(64 * RES_WAVES, (T <= 4 ? 4 : 2)) void gemm_resident_kernel(const ResidentArgs args) {
    typedef Mma<DT_I8, 16> MMA;
    typedef MMA::Acc Acc;
    constexpr int W = RES_WAVES, D = T <= RES_DEEP ? T : T / 2, RED = W * (CHECKED ? 2 : 1);
    static_assert(T % D == 0, "a slot's k tiles are known at compile time");
    extern __shared__ __attribute__((aligned(16))) char smem[];   // each wavefront's 2 KB, then the partial tiles
    typedef Acc Partial[RED][64];
    Partial* const red = reinterpret_cast<Partial*>(smem + W * 2048);
    __shared__ unsigned tops[16];
    __shared__ __attribute__((aligned(16))) float scales[16];
    const GemmArgs& p = args.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lrow = lane & 15, lgrp = lane >> 4, crow = lane >> 3, chunk = (lane & 7) * 16;
    const int M = p.M, N = p.N, K = p.K;
    // this wavefront's k tiles: a run of them, of a row's nkt
    const int nkt = (K + 127) >> 7, share = nkt / W, more = nkt % W;
    const int n_own = share + (wave < more ? 1 : 0), k0 = resident_first(nkt, wave) * 128;   // (k0 = nkt * 128 without one)
    // this workgroup's columns, by the sixteen (runs of workgroups of one die are runs of columns)
    const int wgs = (int)gridDim.x;
    int lin = (int)blockIdx.x;
    if ((wgs & 7) == 0) lin = (lin & 7) * (wgs >> 3) + (lin >> 3);
    const int first = (lin * args.per + min(lin, args.more)) * args.unit, last = min(first + (args.per + (lin < args.more ? 1 : 0)) * args.unit, N);

    // (k tiles beyond this wavefront's, and chunks beyond K, are multiplied with zeros of A: any place in the row will do)
    i32x4 v[D][2];
    // (a base for all lanes, a lane's own 32 bits, and a constant where the tile is a whole one)
    const char* base;
    unsigned rows[2];
    auto columns = [&](int col0) {
        base = p.B + (long long)col0 * p.ldb + k0;
#pragma unroll
        for (int q = 0; q < 2; ++q) rows[q] = (unsigned)min(q * 8 + crow, last - 1 - col0) * (unsigned)p.ldb;
    };
    auto fetch = [&](int slot, int t) {
        // (beyond eight k tiles worked out where it is used, since the registers are full: kept / so, us, from memory, 1 x 4096 x 12288 added 14.1 / 13.4,
        // 16 x 4096 x 16384 21.3 / 20.3, from integers 17.3 / 16.1; unprotected level, 4 x 4096 x 16384 18.6 / 18.8)
        int c = chunk;
        if (T > RES_DEEP && !resident_whole(T, t)) asm volatile("" : "+v"(c));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            if (resident_whole(T, t)) v[slot][q] = ld16g(base + (rows[q] + (unsigned)chunk) + t * 128);
            else v[slot][q] = ld16g(base + (int)(rows[q] + (unsigned)resident_at(T, t, c, K - k0)));
        }
    };
    // the turn of sixteen rows of 128 bytes: whole lines in, fragments out (a wavefront's LDS operations execute in order)
    char* const own = smem + wave * 2048;
    int to[2], at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) to[h] = (h * 8 + crow) * 128 + (chunk ^ ((crow >> 1) * 16 + 64 * h));
#pragma unroll
    for (int s = 0; s < 2; ++s) at[s] = lrow * 128 + ((4 * s + lgrp) ^ (lrow >> 1)) * 16;

    // ---- A: fragment f holds values k0 + 64 f + 16 lgrp .. + 15 of row lrow
    i32x4 a[2 * T];
    auto at_k = [&](int f) { return k0 + f * 64 + lgrp * 16; };
    auto there = [&](int f) { return lrow < M && f < 2 * n_own && at_k(f) < K; };
    auto first_columns = [&]() {
        columns(first);
#pragma unroll
        for (int t = 0; t < D; ++t) fetch(t, t);
    };
    if constexpr (FROM16) {
        // A wavefront takes a row, or two of them, or a part of one, chunks of eight values to a lane: asked for ahead of the weights, quantised
        // into LDS while those are on their way, row r's 16 bytes c at c ^ (r % 8).
        const bool two = M > W;
        const int lg = resident_parts_lg(M), part = wave & ((1 << lg) - 1), row0 = wave >> lg;
        i32x4 x[RES_HELD];
        auto row_of = [&](int c) { return two && (c & 1) ? row0 + W : row0; };
        auto chunk_k = [&](int c) { return ((((two ? c >> 1 : c) << lg) + part) * 64 + lane) * 8; };
        auto begins = [&](int c) { return chunk_k(c) - lane * 8 < K; };   // (the same for all lanes)
#pragma unroll
        for (int c = 0; c < RES_HELD; ++c) {
            if (!begins(c)) break;
            x[c] = ld16u(chunk_k(c) < K && row_of(c) < M ? p.A + (row_of(c) * p.lda + chunk_k(c)) * 2 : g_zero_chunk);
        }
        first_columns();
        if (tid < 16) tops[tid] = 0;
        int top[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < RES_HELD; ++c) {
            if (!begins(c)) break;
            top[c & 1] = chunk_magnitude(x[c], top[c & 1]);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned best = wave_max(max((unsigned)top[h] & 0xffffu, (unsigned)top[h] >> 16));
            if (lane == 0 && row_of(h) < M) atomicMax(&tops[row_of(h)], best);
        }
        __syncthreads();
        GroupScale g[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) g[h] = group_scale<OUT>(tops[min(row_of(h), M - 1)]);
#pragma unroll
        for (int c = 0; c < RES_HELD; ++c) {
            const int r = row_of(c), k = chunk_k(c);
            if (!begins(c)) break;
            if (k < K && r < M) *reinterpret_cast<i32x2*>(smem + r * (nkt * 128) + (((k >> 4) ^ (r & 7)) << 4) + (k & 8)) = quantize_chunk<OUT>(x[c], g[c & 1]);
        }
        if (tid < 16) scales[tid] = group_scale<OUT>(tops[tid]).scale;   // (there before the first sums are, which a barrier is ahead of)
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 2 * T; ++f) {
            a[f] = i32x4{0, 0, 0, 0};
            if (there(f)) a[f] = *reinterpret_cast<const i32x4*>(smem + lrow * (nkt * 128) + (((at_k(f) >> 4) ^ (lrow & 7)) << 4));
        }
        __syncthreads();   // (from here on the rows' place is the partial tiles')
    } else {
        // (rows outside: the last one again, whose sums are not stored; k outside: zeros)
        i32x4 x[T][2];
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int q = 0; q < 2; ++q) x[t][q] = ld16u(p.A + min(q * 8 + crow, M - 1) * p.lda + min(k0 + t * 128 + chunk, K - 16));
        first_columns();
#pragma unroll
        for (int t = 0; t < T; ++t) {
#pragma unroll
            for (int q = 0; q < 2; ++q) *reinterpret_cast<i32x4*>(own + to[q]) = x[t][q];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                a[2 * t + s] = *reinterpret_cast<const i32x4*>(own + at[s]);
                if (!there(2 * t + s)) a[2 * t + s] = i32x4{0, 0, 0, 0};
            }
        }
        if (tid < 16) scales[tid] = p.row_scale[min(tid, M - 1)];
    }


    int turn_of = 0, buf = 0;   // whose turn it is to add up
    auto sixteen = [&](int col0, auto more_c) {
        constexpr bool MORE = decltype(more_c)::value;   // (another sixteen columns follow)
        // what the wavefront whose turn it is needs at the end, on its way before the products
        const bool mine = wave == turn_of;
        const int col = col0 + lrow, n = min(col, last - 1);
        float col_scale = 0.f, col_bias = 0.f, res[EPI == EPI_ADD ? 4 : 1];
        if (mine) {
            col_scale = p.col_scale[n];
            if (p.bias) col_bias = p.bias[n];
            if constexpr (EPI == EPI_ADD) {
#pragma unroll
                for (int r = 0; r < 4; ++r) res[r] = value16<OUT>(p.res + (min(4 * lgrp + r, M - 1) * p.ldr + n) * 2);
            }
        }
        Acc acc = {0, 0, 0, 0}, chk = {0, 0, 0, 0};
        if constexpr (CHECKED) {
            int zero = 0;
            asm("" : "+v"(zero));   // (blocks that take the same products stay apart)
            chk[0] = zero;
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
#pragma unroll
            for (int q = 0; q < 2; ++q) *reinterpret_cast<i32x4*>(own + to[q]) = v[t % D][q];
            // (in flight before anything waits for the fragments)
            if (MORE && t + D == T) columns(col0 + 16);
            if (MORE || t + D < T) fetch(t % D, t + D < T ? t + D : t + D - T);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const i32x4 w = *reinterpret_cast<const i32x4*>(own + at[s]);
                acc = MMA::run(a[2 * t + s], w, acc);
                if constexpr (CHECKED) chk = MMA::run(a[2 * t + s], w, chk);
            }
        }
        // test hook: a bit of one element, of the finished partial sum that holds k = K - 1 (-1) or of the finished sum (-2)
        auto flip = [&](Acc& of, int which) {
            if (p.f_row < 0 || p.f_kt != which || col != p.f_col || col >= last) return;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (4 * lgrp + r == p.f_row) of[r] ^= 1 << p.f_bit;
        };
        if (n_own > 0 && k0 + n_own * 128 >= K) flip(acc, -1);
        red[buf][wave][lane] = acc;
        if constexpr (CHECKED) red[buf][W + wave][lane] = chk;
        __syncthreads();
        if (mine) {
            Acc sum = red[buf][0][lane];
#pragma unroll
            for (int w = 1; w < W; ++w) sum += red[buf][w][lane];
            flip(sum, -2);
            if constexpr (CHECKED) {
                Acc twin = red[buf][W][lane];
#pragma unroll
                for (int w = 1; w < W; ++w) twin += red[buf][W + w][lane];
                // comparison (Sec. 5.2.2) of a 16 x 16 block with its checksum block
                int differ = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) differ |= sum[r] ^ twin[r];
                if (__any(differ)) {
                    long long s = 0, c = 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        s += sum[r];
                        c += twin[r];
                    }
                    if (wave_sum(s) != wave_sum(c) && lane == 0) atomicOr(p.flag, 1u);
                }
            }
            const f32x4 row_scale = *reinterpret_cast<const f32x4*>(&scales[4 * lgrp]);
            float z[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) z[r] = scaled_value(sum[r], row_scale[r], col_scale, col_bias, 0);
            with_activation(p.act, [&](auto act) {
                if constexpr (EPI == EPI_GATED) {
                    const bool odd = lane & 1;
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float o = gated_pair(z[r], z[r + 1], odd, act);
                        const int m = 4 * lgrp + r + (odd ? 1 : 0);
                        if (m < M && col < last) store16<OUT>(p.C + (m * p.ldc + (col >> 1)) * 2, o);
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int m = 4 * lgrp + r;
                        if (m < M && col < last) store16<OUT>(p.C + (m * p.ldc + col) * 2, as_float(act(z[r]) + res[r]));
                    }
                }
            });
        }
        turn_of = (turn_of + 1) & (W - 1);
        buf ^= 1;
    };
    int col0 = first;
    for (; col0 + 16 < last; col0 += 16) sixteen(col0, std::true_type());
    sixteen(col0, std::false_type());
}

}  // namespace abft
