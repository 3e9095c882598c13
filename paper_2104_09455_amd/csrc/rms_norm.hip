// Root-mean-square norm of rows, with the residual's addition before it and, behind it, 16-bit values, int8 with a scale per row, or both:
//   s = round(x + r),   y = round(s / sqrt(mean s^2 + eps) * w),   (q, scale) = y quantised as abft_quantize_rows does
// A row stays in its threads' registers from the sum to the integers, so every value is read and written once.
// Bound: bytes, 2 K each for x, r, s and y; few rows: a chain of two round trips to memory and two sums over the row.  Measured, bf16, with a
// residual, both of s and y: 8192 x 8192 95.8 us (5.6 TB/s), 4096 x 4096 25.3, 600 x 5000 7.5, 1 x 4096 3.7 in a graph.  Rows off the
// dword: 1861 x 3789 16.9, at even pitches 15.0, whole 16-byte chunks (3784, 3792) 13.7.  An odd width: 1001 x 2047 without a residual 4.8, 2048 3.9 (the
// last chunk is stored value by value); every other row off the dword 5.1.
#include <hip/hip_runtime.h>

#include "../../include/abft.h"
#include "quantize.h"

using namespace abft;

namespace {

struct NormArgs {
    const char *X, *R;       // R: null without a residual
    char *S, *Y;             // the sum and the normed rows, or null
    signed char* Q;          // or null
    float* scale;
    const float* weight;     // or null: ones
    int M, K;
    long long ldx, ldr, lds, ldy, ldq;
    float eps;
};

// (results leave past the L2, which the rows on their way in then have for themselves: 8192 x 8192 98.9 -> 95.8 us, 8192 x 5120 63.4 -> 59.7, 600 x 5000
// 9.3 -> 7.5, few rows level)
typedef int AnyChunk __attribute__((ext_vector_type(4), aligned(2)));
typedef int AnyHalf __attribute__((ext_vector_type(2), aligned(1)));

template <int DT>
__device__ __forceinline__ void unpack(const i32x4& v, float (&f)[8]) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        f[2 * d] = mul_add_half<DT, 0>(v[d], 1.f, 0.f);
        f[2 * d + 1] = mul_add_half<DT, 1>(v[d], 1.f, 0.f);
    }
}
// x + r of a chunk, rounded
template <int DT>
__device__ __forceinline__ i32x4 add_chunk(const i32x4& x, const i32x4& r) {
    i32x4 s;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        s[d] = pack_out16<DT>(mul_add_half<DT, 0>(x[d], 1.f, mul_add_half<DT, 0>(r[d], 1.f, 0.f)),
                              mul_add_half<DT, 1>(x[d], 1.f, mul_add_half<DT, 1>(r[d], 1.f, 0.f)));
    return s;
}
template <int DT>
__device__ __forceinline__ float square_chunk(const i32x4& v, float lift, float sum) {
    float f[8];
    unpack<DT>(v, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(f[e] * lift, f[e] * lift, sum);
    return sum;
}
// the first n values of a chunk (8: all)
__device__ __forceinline__ void store_chunk(char* to, const i32x4& v, int n) {
    if (n >= 8) __builtin_nontemporal_store(v, reinterpret_cast<AnyChunk*>(to));
    else
        for (int e = 0; e < n; ++e) reinterpret_cast<short*>(to)[e] = (short)(v[e >> 1] >> (16 * (e & 1)));
}
__device__ __forceinline__ void store_integers(signed char* to, const i32x2& q, int n) {
    if (n >= 8) __builtin_nontemporal_store(q, reinterpret_cast<AnyHalf*>(to));
    else
        for (int e = 0; e < n; ++e) to[e] = (signed char)(q[e >> 2] >> (8 * (e & 3)));
}
// weights of a chunk; behind the row's end whatever
__device__ __forceinline__ void weights(const float* w, int k, int K, float (&f)[8]) {
    if (!w) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = 1.f;
    } else if (k <= K - 8) {
        const f32x4 a = load_global_unaligned<f32x4>(reinterpret_cast<const char*>(w + k));
        const f32x4 b = load_global_unaligned<f32x4>(reinterpret_cast<const char*>(w + k + 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f[e] = a[e];
            f[4 + e] = b[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = w[min(k + e, K - 1)];
    }
}
// s times inv (lift s first where squares would overflow) times w, rounded
template <int DT>
__device__ __forceinline__ i32x4 norm_chunk(const i32x4& s, float lift, float inv, const float (&w)[8]) {
    float f[8];
    unpack<DT>(s, f);
    i32x4 y;
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = pack_out16<DT>(f[2 * d] * lift * inv * w[2 * d], f[2 * d + 1] * lift * inv * w[2 * d + 1]);
    return y;
}

constexpr float LIFT = 0x1p-80f;   // (its square is no float)

// DT: the type of the values; TPR threads share a row and hold it (NV chunks of eight values each); with NV = 0 they go over it again
template <int DT, int TPR, int NV>
__global__ __launch_bounds__(256) void rms_norm_kernel(const NormArgs p) {
    __shared__ float sums[4];
    __shared__ unsigned tops[4];
    const int tid = threadIdx.x, t = tid % TPR, K = p.K;
    const long long m = (long long)blockIdx.x * (256 / TPR) + tid / TPR;
    if (TPR == 64 && m >= p.M) return;   // (a wavefront's row: no barrier in this case)
    const char *const x = p.X + m * p.ldx * 2, *const r = p.R ? p.R + m * p.ldr * 2 : nullptr;
    char *const s = p.S ? p.S + m * p.lds * 2 : nullptr, *const y = p.Y ? p.Y + m * p.ldy * 2 : nullptr;
    signed char* const q = p.Q ? p.Q + m * p.ldq : nullptr;
    // the row's chunk at k, added up
    auto chunk = [&](int k) {
        const i32x4 v = row_chunk16(x, k, K);
        return r ? add_chunk<DT>(v, row_chunk16(r, k, K)) : v;
    };
    // the sum of a value over the row's threads
    auto row_sum = [&](float v) {
        v = wave_sum(v);
        if constexpr (TPR == 256) {
            if ((tid & 63) == 0) sums[tid >> 6] = v;
            __syncthreads();
            v = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        }
        return v;
    };
    i32x4 v[NV ? NV : 1];
    float total = 0.f;
    double many = 0.;   // (a thread's chunks of a row that is not held: up to 2^20 of them)
    if constexpr (NV != 0) {
        i32x4 a[NV], b[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            a[c] = k < K ? row_chunk16(x, k, K) : i32x4{0, 0, 0, 0};
            b[c] = r && k < K ? row_chunk16(r, k, K) : i32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            v[c] = r ? add_chunk<DT>(a[c], b[c]) : a[c];
            if (s && k < K) store_chunk(s + 2ll * k, v[c], K - k);
            total = square_chunk<DT>(v[c], 1.f, total);
        }
    } else {
        for (long long k = t * 8; k < K; k += TPR * 8) {
            const i32x4 c = chunk((int)k);
            if (s) store_chunk(s + 2 * k, c, (int)(K - k));
            many += square_chunk<DT>(c, 1.f, 0.f);
        }
        total = (float)many;
    }
    // (the sum may lie where an operand was: from here on it is read, by the thread that wrote it)
    auto again = [&](int k) { return s ? row_chunk16(s, k, K) : chunk(k); };
    total = row_sum(total);
    float lift = 1.f, mean = total / (float)K + p.eps;
    if (DT == DT_BF16 && !(mean < __builtin_huge_valf())) {
        // squares of bf16 values above 2^64 are no floats: once more, 2^80 smaller (fp16 has none)
        lift = LIFT;
        total = 0.f;
        if constexpr (NV != 0) {
#pragma unroll
            for (int c = 0; c < NV; ++c) total = square_chunk<DT>(v[c], lift, total);
        } else {
            many = 0.;
            for (long long k = t * 8; k < K; k += TPR * 8) many += square_chunk<DT>(again((int)k), lift, 0.f);
            total = (float)many;
        }
        if constexpr (TPR == 256) __syncthreads();   // (everyone has read the first sums)
        mean = row_sum(total) / (float)K + p.eps * LIFT * LIFT;
    }
    const float inv = 1.f / __builtin_sqrtf(mean);
    int top = 0;
    auto normed = [&](int k, const i32x4& c) {
        float w[8];
        weights(p.weight, k, K, w);
        i32x4 o = norm_chunk<DT>(c, lift, inv, w);
        if (K - k < 8) o = shift_down(shift_up(o, 2 * (8 - (K - k))), 2 * (8 - (K - k)));   // (zeros behind the row's end)
        if (y) store_chunk(y + 2ll * k, o, K - k);
        return o;
    };
    if constexpr (NV != 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            if (k < K) v[c] = normed(k, v[c]);
            if (q) top = chunk_magnitude(v[c], top);
        }
    } else {
        for (long long k = t * 8; k < K; k += TPR * 8) top = chunk_magnitude(normed((int)k, again((int)k)), top);
    }
    if (!q) return;
    unsigned best = wave_max(max((unsigned)top & 0xffffu, (unsigned)top >> 16));
    if constexpr (TPR == 256) {
        if ((tid & 63) == 0) tops[tid >> 6] = best;
        __syncthreads();
        best = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
    }
    const GroupScale g = group_scale<DT>(best);
    if (t == 0) p.scale[m] = g.scale;
    if constexpr (NV != 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * TPR + t) * 8;
            if (k < K) store_integers(q + k, quantize_chunk<DT>(v[c], g), K - k);
        }
    } else {
        for (long long k = t * 8; k < K; k += TPR * 8) {
            float w[8];
            weights(p.weight, (int)k, K, w);
            store_integers(q + k, quantize_chunk<DT>(norm_chunk<DT>(again((int)k), lift, inv, w), g), (int)(K - k));
        }
    }
}

// Many rows of up to 2048 NV values: a workgroup goes from row to row, the weights in its registers and the next row on its way
template <int DT, int NV>
__global__ __launch_bounds__(256) void rms_norm_rows_kernel(const NormArgs p) {
    __shared__ float sums[2][4];
    __shared__ unsigned tops[2][4];
    const int tid = threadIdx.x, K = p.K;
    float w[NV][8];
    i32x4 a[NV], b[NV];
    auto load = [&](long long m) {
        const char *const x = p.X + m * p.ldx * 2, *const r = p.R ? p.R + m * p.ldr * 2 : nullptr;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * 256 + tid) * 8;
            a[c] = k < K ? row_chunk16(x, k, K) : i32x4{0, 0, 0, 0};
            if (r) b[c] = k < K ? row_chunk16(r, k, K) : i32x4{0, 0, 0, 0};
        }
    };
    load(blockIdx.x);
#pragma unroll
    for (int c = 0; c < NV; ++c) weights(p.weight, min((c * 256 + tid) * 8, K - 1), K, w[c]);
    int buf = 0;
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x, buf ^= 1) {
        char *const s = p.S ? p.S + m * p.lds * 2 : nullptr, *const y = p.Y ? p.Y + m * p.ldy * 2 : nullptr;
        i32x4 v[NV];
        float total = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * 256 + tid) * 8;
            v[c] = p.R ? add_chunk<DT>(a[c], b[c]) : a[c];
            if (s && k < K) store_chunk(s + 2ll * k, v[c], K - k);
            total = square_chunk<DT>(v[c], 1.f, total);
        }
        if (m + gridDim.x < p.M) load(m + gridDim.x);
        total = wave_sum(total);
        if ((tid & 63) == 0) sums[buf][tid >> 6] = total;
        __syncthreads();
        total = (sums[buf][0] + sums[buf][1]) + (sums[buf][2] + sums[buf][3]);
        float lift = 1.f, mean = total / (float)K + p.eps;
        if (DT == DT_BF16 && !(mean < __builtin_huge_valf())) {
            lift = LIFT;
            total = 0.f;
#pragma unroll
            for (int c = 0; c < NV; ++c) total = square_chunk<DT>(v[c], lift, total);
            total = wave_sum(total);
            __syncthreads();   // (everyone has read the first sums)
            if ((tid & 63) == 0) sums[buf][tid >> 6] = total;
            __syncthreads();
            mean = ((sums[buf][0] + sums[buf][1]) + (sums[buf][2] + sums[buf][3])) / (float)K + p.eps * LIFT * LIFT;
        }
        const float inv = 1.f / __builtin_sqrtf(mean);
        int top = 0;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * 256 + tid) * 8;
            if (k < K) {
                v[c] = norm_chunk<DT>(v[c], lift, inv, w[c]);
                if (K - k < 8) v[c] = shift_down(shift_up(v[c], 2 * (8 - (K - k))), 2 * (8 - (K - k)));
                if (y) store_chunk(y + 2ll * k, v[c], K - k);
            }
            top = chunk_magnitude(v[c], top);
        }
        if (!p.Q) continue;
        unsigned best = wave_max(max((unsigned)top & 0xffffu, (unsigned)top >> 16));
        if ((tid & 63) == 0) tops[buf][tid >> 6] = best;
        __syncthreads();
        best = max(max(tops[buf][0], tops[buf][1]), max(tops[buf][2], tops[buf][3]));
        const GroupScale g = group_scale<DT>(best);
        if (tid == 0) p.scale[m] = g.scale;
        signed char* const q = p.Q + m * p.ldq;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int k = (c * 256 + tid) * 8;
            if (k < K) store_integers(q + k, quantize_chunk<DT>(v[c], g), K - k);
        }
    }
}

// Chunks of eight values that each of 256 threads holds of a row of k
constexpr int held_chunks(int k) { return (k - 1) / 2048 + 1; }

template <int DT>
hipError_t launch(const NormArgs& a, hipStream_t stream) {
    void (*kern)(const NormArgs);
    int rows = 1;
    // (a workgroup for each row / rows in turn, us, bf16 with a residual: 8192 x 8192 105 / 98.7, 8192 x 5120 65 / 63, 4096 x 4096 28.5 / 25.5, 2048 x 4096 15.4 / 15.0,
    // 1024 x 8192 16.1 / 15.2; 8192 x 2048 25.2 / 26.2, 8192 x 1024 15.2 / 17.3)
    const int nv = held_chunks(a.K), wgs = nv == 2 ? 1024 : 512;   // (as many as their registers let the chip hold)
    if (nv >= 2 && nv <= 4 && a.M >= 2 * wgs) {
        kern = nv == 2 ? rms_norm_rows_kernel<DT, 2> : nv == 3 ? rms_norm_rows_kernel<DT, 3> : rms_norm_rows_kernel<DT, 4>;
        hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 0, stream, a);
        return hipGetLastError();
    }
    if (a.K <= 512) { kern = rms_norm_kernel<DT, 64, 1>; rows = 4; }
    else if (a.K <= 2048 && a.M >= 1024) { kern = rms_norm_kernel<DT, 64, 4>; rows = 4; }
    else if (a.K <= 2048) kern = rms_norm_kernel<DT, 256, 1>;
    else if (a.K <= 8192) kern = rms_norm_kernel<DT, 256, 4>;
    else if (a.K <= 16384) kern = rms_norm_kernel<DT, 256, 8>;
    else kern = rms_norm_kernel<DT, 256, 0>;
    // (a launch holds fewer than 2^32 threads)
    constexpr long long BLOCKS = 1 << 23;
    for (long long m = 0; m < a.M; m += BLOCKS * rows) {
        NormArgs b = a;
        b.X += m * a.ldx * 2;
        if (b.R) b.R += m * a.ldr * 2;
        if (b.S) b.S += m * a.lds * 2;
        if (b.Y) b.Y += m * a.ldy * 2;
        if (b.Q) {
            b.Q += m * a.ldq;
            b.scale += m;
        }
        b.M = (int)(a.M - m < BLOCKS * rows ? a.M - m : BLOCKS * rows);
        hipLaunchKernelGGL(kern, dim3((unsigned)((b.M + rows - 1) / rows)), dim3(256), 0, stream, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

extern "C" int abft_rms_norm(int M, int K, const void* X, int64_t ldx, int dtype, const float* weight, float eps, const void* R, int64_t ldr,
                             void* S, int64_t lds, void* Y, int64_t ldy, void* Q, int64_t ldq, float* scale, void* stream) {
    if (dtype != ABFT_F16 && dtype != ABFT_BF16) return ABFT_E_ENUM;
    if (M <= 0 || K <= 0) return ABFT_E_SHAPE;
    if (!X || (!Y && !Q) || (Q && !scale) || (S && !R)) return ABFT_E_NULL;
    if (ldx < K || (R && ldr < K) || (S && lds < K) || (Y && ldy < K) || (Q && ldq < K)) return ABFT_E_LD;
    if (!(eps > 0.f) || !(eps < __builtin_huge_valf())) return ABFT_E_VALUE;
    NormArgs a;
    a.X = reinterpret_cast<const char*>(X);
    a.R = reinterpret_cast<const char*>(R);
    a.S = reinterpret_cast<char*>(S);
    a.Y = reinterpret_cast<char*>(Y);
    a.Q = reinterpret_cast<signed char*>(Q);
    a.scale = scale;
    a.weight = weight;
    a.M = M; a.K = K; a.ldx = ldx; a.ldr = ldr; a.lds = lds; a.ldy = ldy; a.ldq = ldq;
    a.eps = eps;
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    return (dtype == ABFT_F16 ? launch<DT_F16>(a, st) : launch<DT_BF16>(a, st)) == hipSuccess ? ABFT_OK : ABFT_E_HIP;
}
