// Writing keys and values of new tokens to a paged cache, quantised on the way if it is int8, and reading them back.
//
// A group of lanes, eight values to a lane, takes one token's key and value of one head: both are on their
// way at once, the largest magnitude is an exchange inside the group, and each lane stores the eight integers of its eight values.
// Bound: bytes (2 dim in, dim + 4 out for each key and value, the other way round in reading); few tokens: one round trip to
// the slot and one to the values.  Measured, fp16 to int8, 8 heads of 128: 64 tokens 2.9 us written, 2.4 read; 8192 tokens 11.0 and
// 10.5 us (4.6 and 4.9 TB/s), 16384 18.8 and 18.3 (5.4 and 5.6); 8192 in a 16-bit cache 11.5 and 12.2 (5.9 and 5.5).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kv_cache.h"
#include "quantize.h"

using namespace abft;

namespace {

struct KvArgs {
    char *k, *v;             // the cache
    float *k_scale, *v_scale;
    char *K, *V;             // the tokens' values
    const int64_t* slots;
    long long ldk, ldv;      // elements
    unsigned pairs;          // tokens x heads of the launch
    int heads, dim, page_size;
    int slots_in_cache;
};

// where a token's values of one head are in the cache, in tokens of one head (page_size of them per page and head); -1: nowhere
__device__ __forceinline__ long long place(const KvArgs& p, int token, int head) {
    const int64_t slot = p.slots[token];
    if (slot < 0 || slot >= p.slots_in_cache) return -1;
    const unsigned page = (unsigned)slot / (unsigned)p.page_size, off = (unsigned)slot - page * (unsigned)p.page_size;
    return ((long long)page * p.heads + head) * p.page_size + off;
}

// DT: the type of the tokens' values; I8: of the cache, else the same; LANES: lanes of a head, of eight values each
template <int DT, bool I8, int LANES>
__global__ __launch_bounds__(256) void kv_write_kernel(const KvArgs p) {
    const int t = threadIdx.x % LANES;
    // (groups without a pair or a place go along, so that the exchange below has all its lanes; the values are asked for before the
    // slot has come)
    const unsigned pair = min(blockIdx.x * (256u / LANES) + threadIdx.x / LANES, p.pairs - 1), token = pair / (unsigned)p.heads;
    const int head = (int)(pair - token * (unsigned)p.heads);
    const bool in = t * 8 < p.dim;
    const long long e = (long long)head * p.dim + (in ? t * 8 : 0);
    const i32x4 k = ld16u(p.K + (token * p.ldk + e) * 2), v = ld16u(p.V + (token * p.ldv + e) * 2);
    const long long at = place(p, (int)token, head);
    const bool on = at >= 0 && in && blockIdx.x * (256u / LANES) + threadIdx.x / LANES < p.pairs;
    const i32x4 none = {0, 0, 0, 0};
    const i32x4 x[2] = {in ? k : none, in ? v : none};
    if constexpr (!I8) {
        if (on) {
            *reinterpret_cast<i32x4*>(p.k + (at * p.dim + t * 8) * 2) = x[0];
            *reinterpret_cast<i32x4*>(p.v + (at * p.dim + t * 8) * 2) = x[1];
        }
    } else {
        unsigned top[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int m = chunk_magnitude(x[q], 0);
            top[q] = max((unsigned)m & 0xffffu, (unsigned)m >> 16);
#pragma unroll
            for (int s = 1; s < LANES; s <<= 1) top[q] = max(top[q], (unsigned)__shfl_xor((int)top[q], s));
        }
        if (on) {
            const GroupScale gk = group_scale<DT>(top[0]), gv = group_scale<DT>(top[1]);
            *reinterpret_cast<i32x2*>(p.k + at * p.dim + t * 8) = quantize_chunk<DT>(x[0], gk);
            *reinterpret_cast<i32x2*>(p.v + at * p.dim + t * 8) = quantize_chunk<DT>(x[1], gv);
            if (t == 0) {
                p.k_scale[at] = gk.scale;
                p.v_scale[at] = gv.scale;
            }
        }
    }
}

// eight integers times a scale, rounded to 16 bits
template <int DT>
__device__ __forceinline__ i32x4 dequantize_chunk(const i32x2& q, float scale) {
    i32x4 out;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int w = q[d >> 1] >> (16 * (d & 1));
        out[d] = pack_out16<DT>((float)(signed char)w * scale, (float)(signed char)(w >> 8) * scale);
    }
    return out;
}

struct __attribute__((packed)) AnyChunk { i32x4 v; };

template <int DT, bool I8, int LANES>
__global__ __launch_bounds__(256) void kv_read_kernel(const KvArgs p) {
    const int t = threadIdx.x % LANES;
    const unsigned pair = blockIdx.x * (256u / LANES) + threadIdx.x / LANES, token = pair / (unsigned)p.heads;
    const int head = (int)(pair - token * (unsigned)p.heads);
    if (pair >= p.pairs || t * 8 >= p.dim) return;
    const long long at = place(p, (int)token, head);
    i32x4 x[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    if (at >= 0) {
        if constexpr (I8) {
            const i32x2 k = *reinterpret_cast<const i32x2*>(p.k + at * p.dim + t * 8);
            const i32x2 v = *reinterpret_cast<const i32x2*>(p.v + at * p.dim + t * 8);
            x[0] = dequantize_chunk<DT>(k, p.k_scale[at]);
            x[1] = dequantize_chunk<DT>(v, p.v_scale[at]);
        } else {
            x[0] = ld16(p.k + (at * p.dim + t * 8) * 2);
            x[1] = ld16(p.v + (at * p.dim + t * 8) * 2);
        }
    }
    const long long e = (long long)head * p.dim + t * 8;
    reinterpret_cast<AnyChunk*>(p.K + (token * p.ldk + e) * 2)->v = x[0];
    reinterpret_cast<AnyChunk*>(p.V + (token * p.ldv + e) * 2)->v = x[1];
}

template <int DT, bool I8, int LANES>
hipError_t launch(bool write, const KvArgs& all, int tokens, hipStream_t st) {
    constexpr unsigned PER = 256 / LANES;
    // (a launch holds fewer than 2^32 threads)
    const int step = std::max((int)((1ll << 31) / LANES / all.heads), 1);
    for (int t = 0; t < tokens; t += std::min(step, tokens - t)) {
        KvArgs a = all;
        a.K += t * a.ldk * 2;
        a.V += t * a.ldv * 2;
        a.slots += t;
        a.pairs = (unsigned)std::min(step, tokens - t) * (unsigned)a.heads;
        const dim3 grid((a.pairs + PER - 1) / PER);
        if (write) hipLaunchKernelGGL((kv_write_kernel<DT, I8, LANES>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((kv_read_kernel<DT, I8, LANES>), grid, dim3(256), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int kv_move(bool write, const abft_kv_cache_t* c, int tokens, const int64_t* slots, char* K, long long ldk, char* V, long long ldv,
            int dtype, void* stream) {
    const int rc = kv_validate(c, dtype);
    if (rc != ABFT_OK) return rc;
    if (tokens < 0) return ABFT_E_SHAPE;
    if (tokens == 0) return ABFT_OK;
    if (!slots || !K || !V) return ABFT_E_NULL;
    const long long row = (long long)c->heads * c->head_dim;
    if (ldk < row || ldv < row) return ABFT_E_LD;
    if ((long long)tokens * c->heads > 0x7fffffffll) return ABFT_E_SHAPE;
    KvArgs a;
    a.k = reinterpret_cast<char*>(c->k); a.v = reinterpret_cast<char*>(c->v);
    a.k_scale = c->k_scale; a.v_scale = c->v_scale;
    a.K = K; a.V = V; a.slots = slots; a.ldk = ldk; a.ldv = ldv;
    a.pairs = 0; a.heads = c->heads; a.dim = c->head_dim; a.page_size = c->page_size;
    a.slots_in_cache = c->pages * c->page_size;
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const bool i8 = c->dtype == ABFT_I8, f16 = dtype == ABFT_F16;
    auto of_lanes = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        if (f16) return i8 ? launch<DT_F16, true, L>(write, a, tokens, st) : launch<DT_F16, false, L>(write, a, tokens, st);
        return i8 ? launch<DT_BF16, true, L>(write, a, tokens, st) : launch<DT_BF16, false, L>(write, a, tokens, st);
    };
    const hipError_t e = c->head_dim <= 32   ? of_lanes(std::integral_constant<int, 4>())
                         : c->head_dim <= 64 ? of_lanes(std::integral_constant<int, 8>())
                                             : of_lanes(std::integral_constant<int, 16>());
    return e == hipSuccess ? ABFT_OK : ABFT_E_HIP;
}

}  // namespace

extern "C" {

int abft_kv_write(const abft_kv_cache_t* cache, int tokens, const int64_t* slots, const void* K, int64_t ldk, const void* V,
                  int64_t ldv, int dtype, void* stream) {
    return kv_move(true, cache, tokens, slots, reinterpret_cast<char*>(const_cast<void*>(K)), ldk,
                   reinterpret_cast<char*>(const_cast<void*>(V)), ldv, dtype, stream);
}

int abft_kv_read(const abft_kv_cache_t* cache, int tokens, const int64_t* slots, void* K, int64_t ldk, void* V, int64_t ldv,
                 int dtype, void* stream) {
    return kv_move(false, cache, tokens, slots, reinterpret_cast<char*>(K), ldk, reinterpret_cast<char*>(V), ldv, dtype, stream);
}

}  // extern "C"
