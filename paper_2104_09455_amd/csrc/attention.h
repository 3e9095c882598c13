// Attention of new tokens over a paged cache of keys and values, for gfx950 (MI355X).
//
// Row (token, query head) with query q sees some of its sequence's keys and becomes sum_j w_j v_j / sum_j w_j with
// w_j = 2^(c q.k_j - m), c = scale log2(e), in one pass over the keys: m is a running maximum, and sums that were taken under a
// smaller one are scaled down when it moves.  m only has to be near the maximum, so it moves when a value passes it by more than
// 2^8, which after a row's first keys hardly happens.  Weights of fp16 are kept 2^7 larger than that: up to 2^15, so that what
// vanishes below the type's smallest value is less than 2^-32 of the largest (2^-25 of it, for each of a million keys, were 3 %).
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T.  The first leaves in each lane weights of one row (its column)
// and of keys 4 g .. 4 g + 3 of every eight or sixteen, g the lane's group, and that is what the second takes as its operand
// along k once two such runs are put behind one another: the sum over keys does not ask for an order, so V is read in the same
// one.  Weights never leave their lane, and a row's statistics are its lane's.
//
// int8 caches: keys and values are integers, exact in 16 bits; a key's scale goes into c, and a value's into the exponent, w'_j =
// 2^(c s_j q.k_j + log2 t_j - m), so that weights rounded to 16 bits are in range whatever the scales are; the sum of weights takes
// w'_j / t_j.
#pragma once
#include "gemm_common.h"
#include "kv_cache.h"
#include "quantize.h"

namespace abft {

struct AttnArgs {
    // cache: pages x heads x page_size x dim; scales of int8
    const char *K, *V;
    const float *ks, *vs;
    int pages, page_size, heads, dim;
    unsigned page_blocks, page_magic;   // page_size / 16, and 2^31 / that, rounded up (blocks of 16 keys -> pages)
    // sequences
    const int *q_start, *kv_len, *table;
    long long ld_table;
    int n_seqs, total_q, max_q, max_kv;
    // rows
    const char* Q;
    char* O;
    long long ldq, ldo;                 // elements
    int group;                          // query heads for each head of the cache
    float c;                            // scale log2(e)
    int causal, window;
    // Sequences of one new token have a program of their own (single: they are left to it): `single_groups` workgroups, and two
    // places each for sums of keys that are not all of a row's: group rows of dim floats, and of two (m, the sum of weights).
    int single, single_groups;
    unsigned* counters;                 // one for each of them or of the row tiles below, zero before and after a launch
    float *single_o, *single_ml;
    // The others: at most `tiles` row tiles; up to tile_split of them their keys may be divided, and the pieces' sums go here, row tiles of the same.
    int tiles, tile_split, tile_counters;   // tile_counters: how many counters are theirs
    float *tile_o, *tile_ml;
};

constexpr int ATTN_BLOCK_KEYS = 64;     // keys of a tile
constexpr int ATTN_GROUP_MAX = 16;      // query heads a head's single-token block holds

struct SeqInfo {
    int q0, nq, kv;
};
// (cut to what the host was told)
__device__ __forceinline__ SeqInfo seq_info(const AttnArgs& p, int s) {
    SeqInfo i;
    i.q0 = min(max(p.q_start[s], 0), p.total_q);
    i.nq = min(min(max(p.q_start[s + 1], i.q0), p.total_q) - i.q0, p.max_q);
    i.kv = min(max(p.kv_len[s], 0), p.max_kv);
    return i;
}
// a key block's place: its first key's index among a head's tokens (all pages of all heads behind one another)
// (exact: a block is below 2^20 and a page has at most 2^8, and their product stays below 2^31)
__device__ __forceinline__ unsigned page_of(const AttnArgs& p, unsigned block) { return __umulhi(2 * block, p.page_magic); }
__device__ __forceinline__ long long block_place(const AttnArgs& p, unsigned block, unsigned page_index, int entry, int head) {
    const unsigned page = min((unsigned)max(entry, 0), (unsigned)(p.pages - 1));
    return ((long long)page * p.heads + head) * p.page_size + (long long)(block - page_index * p.page_blocks) * 16;
}

// eight int8 values (two registers) as 16-bit floats
template <int DT>
__device__ __forceinline__ i32x4 widen8(int lo, int hi) {
    i32x4 out;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
        const int w = d < 2 ? lo : hi, sh = 16 * (d & 1);
        out[d] = pack_out16<DT>((float)(signed char)(w >> sh), (float)(signed char)(w >> (sh + 8)));
    }
    return out;
}

template <int DT>
__device__ __forceinline__ bool is_finite16(unsigned bits) { return (bits & 0x7fffu) < (DT == DT_F16 ? 0x7c00u : 0x7f80u); }
template <int DT>
__device__ __forceinline__ bool any_not_finite(const i32x4& v) {
    const unsigned top = (unsigned)chunk_magnitude(v, 0);
    return !is_finite16<DT>(top & 0xffffu) || !is_finite16<DT>(top >> 16);
}
// two values, zeros in the place of what is not finite
template <int DT>
__device__ __forceinline__ int only_finite(int v) {
    return (is_finite16<DT>(v & 0xffff) ? v & 0xffff : 0) | (is_finite16<DT>((unsigned)v >> 16) ? v & (int)0xffff0000 : 0);
}
template <int DT>
__device__ __forceinline__ float widen16(unsigned short v) {
    if constexpr (DT == DT_F16) return (float)bitcast<_Float16>(v);
    else return bitcast<float>((unsigned)v << 16);
}
// four keys' values of one column each, out of four rows that the lane's group of sixteen reads 8 bytes of
__device__ __forceinline__ i32x2 read_transposed(const char* p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return bitcast<i32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
}

__device__ __forceinline__ float swap_halves(float v) { return __shfl_xor(v, 32); }

// log2 of a value's scale and its inverse (a group of zeros: any scale does; NaN stays).  Smaller scales are taken for the least one: 2^-64,
// nothing in an output of fp16 (and 2^24 weights of 2^15, each times its inverse, stay inside fp32), or 2^-100 for bf16.
template <int DT>
__device__ __forceinline__ void value_scale(float t, float& log2_t, float& inv_t) {
    constexpr float LEAST = DT == DT_F16 ? 0x1p-64f : 0x1p-100f;
    t = t < LEAST ? LEAST : t;
    log2_t = __builtin_amdgcn_logf(t);
    inv_t = __builtin_amdgcn_rcpf(t);
}

// two floats that workgroups on other dies read in the same launch, and read so
__device__ __forceinline__ void put_shared(float* p, float a, float b) {
    const unsigned long long v = (unsigned long long)bitcast<unsigned>(b) << 32 | bitcast<unsigned>(a);
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_shared(const float* p) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return float2{bitcast<float>((unsigned)v), bitcast<float>((unsigned)(v >> 32))};
}

constexpr float ATTN_NONE = -3.402823466e+38f;   // the running maximum before the first key
constexpr float ATTN_SLACK = 8.f;                // how far (as powers of two) a value may pass it
// how far below the running maximum the exponents' base is (see above; 2^15 (1 + rounding) is below fp16's 65504)
template <int DT>
constexpr float ATTN_LIFT = DT == DT_F16 ? 7.f : 0.f;

}  // namespace abft
