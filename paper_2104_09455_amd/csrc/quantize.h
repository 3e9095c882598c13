// Symmetric 8-bit quantisation of a group of 16-bit values (a token's activations, a token's key of one head):
//   a = max |x|,   scale = a / 127,   q = 127 x / a rounded to nearest, halves away from zero
// and a group of zeros has the scale 0.  A group that holds an infinity or a NaN has the scale NaN and integers 0, so that
// everything computed from it is NaN, as it would be from the values themselves.
//
// The rounding is exact without a division per value.  x and a have at most 11 significant bits, so 127 x / a is either a
// half exactly or off every half by 2^-19 of itself; x times fl(127 / a) (1 + 2^-20) is off by less than 2^-22 beside the
// factor, which carries exact halves outwards and nothing else over one.  The magnitudes are compared as integers, two to an
// instruction, where infinities and NaN come out on top.
#pragma once
#include "gemm_common.h"

namespace abft {

typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// the larger magnitude, as a pair of 16-bit patterns, of `top` and of the two values in `packed`
__device__ __forceinline__ int larger_magnitudes(int packed, int top) {
    return bitcast<int>(__builtin_elementwise_max(bitcast<u16x2>(packed & 0x7fff7fff), bitcast<u16x2>(top)));
}
__device__ __forceinline__ int chunk_magnitude(const i32x4& v, int top) {
#pragma unroll
    for (int d = 0; d < 4; ++d) top = larger_magnitudes(v[d], top);
    return top;
}

// A group's scale, and the factor that its values are multiplied with: (lift x) * factor, where lift is not 1 only for
// groups below 2^-100 (bf16), whose factor would overflow.
struct GroupScale {
    float scale, factor, lift;
    bool finite;
};
template <int DT>
__device__ __forceinline__ GroupScale group_scale(unsigned top) {   // the largest magnitude's 16-bit pattern
    GroupScale g;
    float a;
    if constexpr (DT == DT_F16) a = (float)bitcast<_Float16>((unsigned short)top);
    else a = bitcast<float>(top << 16);
    g.finite = top < (DT == DT_F16 ? 0x7c00u : 0x7f80u);
    g.lift = a < 7.8886091e-31f ? 18446744073709551616.f : 1.f;   // 2^-100, 2^64
    g.scale = g.finite ? a / 127.f : __builtin_nanf("");
    g.factor = g.finite && top != 0 ? 127.f / (a * g.lift) * (1.f + 0x1p-20f) : 0.f;
    return g;
}

// Four integers, one to a byte, of the four values in two registers.  The sum with 1.5 * 2^23 has the rounded integer in its
// low byte.
template <int DT, bool LIFT>
__device__ __forceinline__ int quantize4(int p0, int p1, const GroupScale& g) {
    constexpr float MAGIC = 12582912.f;
    unsigned u[4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int p = e ? p1 : p0;
        float lo, hi;
        if constexpr (LIFT) {
            const float x0 = DT == DT_F16 ? mul_add_half<DT, 0>(p, g.lift, 0.f) : bf16_lo(p) * g.lift;
            const float x1 = DT == DT_F16 ? mul_add_half<DT, 1>(p, g.lift, 0.f) : bf16_hi(p) * g.lift;
            lo = __builtin_fmaf(x0, g.factor, MAGIC);
            hi = __builtin_fmaf(x1, g.factor, MAGIC);
        } else {
            lo = mul_add_half<DT, 0>(p, g.factor, MAGIC);
            hi = mul_add_half<DT, 1>(p, g.factor, MAGIC);
        }
        u[2 * e] = bitcast<unsigned>(lo);
        u[2 * e + 1] = bitcast<unsigned>(hi);
    }
    const unsigned a = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), b = __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu);
    return (int)(a | b);
}
// the eight integers of a 16-byte chunk
template <int DT>
__device__ __forceinline__ i32x2 quantize_chunk(const i32x4& v, const GroupScale& g) {
    i32x2 q = {0, 0};
    if (!g.finite) return q;
    if (DT == DT_BF16 && g.lift != 1.f) {
        q[0] = quantize4<DT, true>(v[0], v[1], g);
        q[1] = quantize4<DT, true>(v[2], v[3], g);
    } else {
        q[0] = quantize4<DT, false>(v[0], v[1], g);
        q[1] = quantize4<DT, false>(v[2], v[3], g);
    }
    return q;
}

// up to eight 16-bit values of a row from element k on (k < K), zeros behind its end; at any address
__device__ __forceinline__ i32x4 row_chunk16(const char* row, int k, int K) {
    if (k + 8 <= K) return ld16u(row + 2ll * k);
    if (K >= 8) return shift_down(ld16u(row + 2ll * (K - 8)), 2 * (k + 8 - K));
    return gather16<2>(row + 2ll * k, 2, K - k);
}

struct QuantizeArgs {
    const char* X;
    signed char* Q;
    float* scale;
    int M, K;
    long long ldx, ldq;
};

// Rows of a matrix.  TPR threads share a row and hold it in registers between the two passes (NV chunks of eight values each);
// with NV = 0 they read it twice.
// Bound: the row's bytes once, 2 K in and K out; few rows: one round trip to them.  Measured: 8192 x 8192 29.7 us (6.8 TB/s), 64 x
// 8192 3.0 us.
template <int DT, int TPR, int NV>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantizeArgs p) {
    __shared__ unsigned tops[4];
    const int tid = threadIdx.x, t = tid % TPR;
    const long long m = (long long)blockIdx.x * (256 / TPR) + tid / TPR;
    if (TPR == 64 && m >= p.M) return;   // (a wavefront's row: no barrier in this case)
    const char* const row = p.X + m * p.ldx * 2;
    const int K = p.K;
    i32x4 v[NV ? NV : 1];
    int top = 0;
    if constexpr (NV != 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            v[c] = k < K ? row_chunk16(row, k, K) : i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) top = chunk_magnitude(v[c], top);
    } else {
        for (long long k = t * 8; k < K; k += TPR * 8) top = chunk_magnitude(row_chunk16(row, (int)k, K), top);
    }
    unsigned best = max((unsigned)top & 0xffffu, (unsigned)top >> 16);
    best = wave_max(best);
    if constexpr (TPR == 256) {
        if ((tid & 63) == 0) tops[tid >> 6] = best;
        __syncthreads();
        best = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    const GroupScale g = group_scale<DT>(best);
    if (t == 0) p.scale[m] = g.scale;
    signed char* const out = p.Q + m * p.ldq;
    auto store = [&](long long k, const i32x4& x) {
        const i32x2 q = quantize_chunk<DT>(x, g);
        if (k + 8 <= K) {
            struct __attribute__((packed)) Any { i32x2 v; };
            reinterpret_cast<Any*>(out + k)->v = q;
        } else {
            for (int e = 0; e < K - k; ++e) out[k + e] = (signed char)(q[e >> 2] >> (8 * (e & 3)));
        }
    };
    if constexpr (NV != 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            if (k < K) store(k, v[c]);
        }
    } else {
        for (long long k = t * 8; k < K; k += TPR * 8) store(k, row_chunk16(row, (int)k, K));
    }
}

template <int DT>
inline hipError_t launch_quantize_rows(const QuantizeArgs& a, hipStream_t stream) {
    // (a wavefront per row where four chunks a lane hold it and there are rows enough to fill the chip so; else a workgroup.  us,
    // wavefront / workgroup: 8192 x 512 3.6 / 5.8, 64 x 512 2.35 / 2.42; 8192 x 2048 8.6 / 9.8, 4096 x 1024 3.6 / 4.3, 1024 x 2048 level, 256 x 2048
    // 2.9 / 2.5.  Rows that do not fit the registers are read twice.)
    void (*kern)(const QuantizeArgs);
    int rows = 1;
    if (a.K <= 512) { kern = quantize_rows_kernel<DT, 64, 1>; rows = 4; }
    else if (a.K <= 2048 && a.M >= 1024) { kern = quantize_rows_kernel<DT, 64, 4>; rows = 4; }
    else if (a.K <= 2048) kern = quantize_rows_kernel<DT, 256, 1>;
    else if (a.K <= 8192) kern = quantize_rows_kernel<DT, 256, 4>;
    else kern = quantize_rows_kernel<DT, 256, 0>;
    // (a launch holds fewer than 2^32 threads)
    constexpr long long BLOCKS = 1 << 23;
    for (long long m = 0; m < a.M; m += BLOCKS * rows) {
        QuantizeArgs b = a;
        b.X += m * a.ldx * 2;
        b.Q += m * a.ldq;
        b.scale += m;
        b.M = (int)(a.M - m < BLOCKS * rows ? a.M - m : BLOCKS * rows);
        hipLaunchKernelGGL(kern, dim3((unsigned)((b.M + rows - 1) / rows)), dim3(256), 0, stream, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace abft
