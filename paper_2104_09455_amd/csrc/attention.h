// Attention of new tokens over a paged cache of keys and values, for gfx950 (MI355X).
//
// Row (token, query head) with query q sees some of its sequence's keys and becomes sum_j w_j v_j / sum_j w_j with
// w_j = 2^(c q.k_j - m), c = scale log2(e), in one pass over the keys: m is a running maximum, and sums that were taken under a
// smaller one are scaled down when it moves.  m only has to be near the maximum, so it moves when a value passes it by more than
// 2^8 (the weights stay far inside 16 bits, the sums inside fp32), which after a row's first keys hardly happens.
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
    unsigned page_blocks, page_magic;   // page_size / 16, and 2^32 / that, rounded up (blocks of 16 keys -> pages)
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
    // Splits of a sequence's keys, `chunk` each, and where their sums go: rows x splits of dim floats, and of two (m, the sum of
    // weights).  Sequences of one new token ("single": a kernel of their own) and the others.
    int single;                         // sequences with one new token are left to the kernel for them
    int single_chunk, single_splits, tile_chunk, tile_splits;
    float *single_o, *single_ml, *tile_o, *tile_ml;
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
// (exact: block < 2^20 and a page has at most 2^8 blocks, and 2^20 * 2^8 < 2^32; one block to a page has no magic, 0)
__device__ __forceinline__ unsigned page_of(const AttnArgs& p, unsigned block) { return p.page_magic ? __umulhi(block, p.page_magic) : block; }
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

// log2 of a value's scale and its inverse (a group of zeros: any scale does; NaN stays)
__device__ __forceinline__ void value_scale(float t, float& log2_t, float& inv_t) {
    t = t < 7.8886091e-31f ? 7.8886091e-31f : t;
    log2_t = __builtin_amdgcn_logf(t);
    inv_t = __builtin_amdgcn_rcpf(t);
}

constexpr float ATTN_NONE = -3.402823466e+38f;   // the running maximum before the first key
constexpr float ATTN_SLACK = 8.f;                // how far (as powers of two) a value may pass it

// ------------------------------------------------------------------------------------------------------------------ //
// Many rows: a workgroup of four wavefronts takes 32 rows each of one sequence and head of the cache (rows are the new
// tokens' query heads of that head, token by token), and all keys that these rows see, 64 at a time, in 16 bits in LDS.
// ------------------------------------------------------------------------------------------------------------------ //
template <int DP>
struct AttnTile {
    static constexpr int PITCH = DP <= 64 ? 128 : 256;            // bytes of a key's row in LDS
    static constexpr int ROWS = 128;                              // rows of a workgroup
    static constexpr int KEYS = ATTN_BLOCK_KEYS;
    static constexpr int HALF = KEYS * PITCH;                     // K, or V
    static constexpr int STAGE = 2 * HALF + 3 * KEYS * 4;         // and three floats a key
    static constexpr int LDS_BYTES = 2 * STAGE + 16;
    // 16-byte chunk c of row r lies at chunk c ^ swizzle(r): the 16 rows that a fragment of K is read from at once, and the
    // 4 (x 64 bytes) of V, lie in different banks
    static __device__ __forceinline__ int k_swizzle(int r) { return PITCH == 256 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_swizzle(int r) { return PITCH == 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// which sequence and which of its row tiles the t-th tile of the launch is; false: there is none
__device__ __forceinline__ bool find_tile(const AttnArgs& p, int t, int rows, int& seq, int& tile, int& tiles) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
        const int s = s0 + lane;
        int n = 0;
        if (s < p.n_seqs) {
            const SeqInfo i = seq_info(p, s);
            if (!(p.single && i.nq == 1)) n = (i.nq * p.group + rows - 1) / rows;
        }
        int sum = n;   // of this lane's and all lower ones
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
        const unsigned long long at = __ballot(before + sum > t);
        if (at != 0) {
            const int first = __builtin_ctzll(at);
            seq = s0 + first;
            tiles = __shfl(n, first);
            tile = t - (before + __shfl(sum, first) - tiles);
            return true;
        }
        before += __shfl(sum, 63);
    }
    return false;
}

// What a tile's V held that is not finite, and the product therefore left out: for each such value, the rows that see its key
// take it times their weight.  One key after the other, the weights formed anew; this is for results that end as infinities
// and NaN, not for speed.
template <int DT, int DP>
__device__ __forceinline__ void add_not_finite(const AttnArgs& p, f32x16 (&o)[DP / 32], float m, int k0, const SeqInfo& si, const int* pages,
                                                         int head, int token, int qh, int lo, int hi, int h) {
    const unsigned short* const q = reinterpret_cast<const unsigned short*>(p.Q) + token * p.ldq + (long long)qh * p.dim;
    for (int key = k0; key < min(k0 + ATTN_BLOCK_KEYS, si.kv); ++key) {
        const unsigned block = (unsigned)key >> 4, pi = page_of(p, block);
        const long long at = (block_place(p, block, pi, pages[pi], head) + (key & 15)) * p.dim;
        const unsigned short* const k = reinterpret_cast<const unsigned short*>(p.K) + at;
        const unsigned short* const v = reinterpret_cast<const unsigned short*>(p.V) + at;
        float dot = 0.f;
        for (int d = 0; d < p.dim; ++d) dot = __builtin_fmaf(widen16<DT>(q[d]), widen16<DT>(k[d]), dot);
        const bool seen = key >= lo && key < hi;
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(dot, p.c, -m));
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int d = 32 * b + 8 * (r >> 2) + 4 * h + (r & 3);
                const unsigned short x = d < p.dim ? v[d] : 0;
                if (seen && !is_finite16<DT>(x)) o[b][r] += w * widen16<DT>(x);
            }
    }
}

template <int DT, bool I8, int DP>
__global__ __launch_bounds__(256, 2) void attn_tile_kernel(const AttnArgs p) {
    typedef AttnTile<DP> T;
    typedef Mma<DT, 32> MMA;
    constexpr int STEPS = DP / 16, BLOCKS = DP / 32, KEYS = T::KEYS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;   // this lane's row of the wavefront's 32, its half of the keys

    const int head = (int)blockIdx.x % p.heads;
    int seq, tile, tiles;
    if (!find_tile(p, (int)blockIdx.x / p.heads, T::ROWS, seq, tile, tiles)) return;
    seq = __builtin_amdgcn_readfirstlane(seq);
    tile = tiles - 1 - __builtin_amdgcn_readfirstlane(tile);   // (the rows that see most first)
    const SeqInfo si = seq_info(p, seq);
    const int split = blockIdx.y, rows = si.nq * p.group, before = si.kv - si.nq;
    const int chunks = max(1, (si.kv + p.tile_chunk - 1) / p.tile_chunk);
    if (split >= chunks) return;

    // ---- rows: the workgroup's, the wavefront's, this lane's, and the keys that they see, lo .. hi - 1
    auto lo_of = [&](int r) { return p.window > 0 ? max(before + r / p.group - p.window + 1, 0) : 0; };
    auto hi_of = [&](int r) { return p.causal ? min(before + r / p.group + 1, si.kv) : si.kv; };
    const int row0 = tile * T::ROWS, row_end = min(row0 + T::ROWS, rows) - 1;
    const int wrow0 = min(row0 + wave * 32, rows - 1), wrow_end = min(row0 + wave * 32 + 31, rows - 1);
    const bool wave_on = row0 + wave * 32 < rows;
    const int my_row = min(row0 + wave * 32 + col, rows - 1);
    const bool row_on = row0 + wave * 32 + col < rows;
    const int my_lo = lo_of(my_row), my_hi = hi_of(my_row);
    const int from = max(lo_of(row0), split * p.tile_chunk), to = min(hi_of(row_end), min(si.kv, (split + 1) * p.tile_chunk));
    const int full_from = lo_of(row_end), full_to = hi_of(row0);            // keys that all rows of the workgroup see
    const int w_from = lo_of(wrow0), w_to = hi_of(wrow_end), w_full_from = lo_of(wrow_end), w_full_to = hi_of(wrow0);
    const int t0 = from / KEYS, t1 = to > from ? (to + KEYS - 1) / KEYS : t0;   // tiles of keys

    // ---- this lane's query, as the fragments of the first product want it: values 16 s + 8 h .. + 7 of its row
    const int token = si.q0 + my_row / p.group, qh = head * p.group + my_row % p.group;
    i32x4 q[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = 16 * s + 8 * h;
        q[s] = row_on && d < p.dim ? ld16(p.Q + (token * p.ldq + (long long)qh * p.dim + d) * 2) : i32x4{0, 0, 0, 0};
    }

    // ---- copies: 16 bytes a thread, thread's chunk of rows tid / CPR + PASS i of a tile
    constexpr int CPR = I8 ? T::PITCH / 32 : T::PITCH / 16, PASS = 256 / CPR, NP = KEYS / PASS;
    const int chunk = tid % CPR, crow = tid / CPR;
    const bool chunk_on = chunk * 16 < p.dim * (I8 ? 1 : 2);
    const int* const pages = p.table + seq * p.ld_table;
    const int row_bytes = p.dim * (I8 ? 1 : 2);
    i32x4 kreg[NP], vreg[NP];
    float scale_reg = 0.f;
    auto load_tile = [&](int kt) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int key = kt * KEYS + crow + i * PASS;
            kreg[i] = vreg[i] = i32x4{0, 0, 0, 0};
            if (key < si.kv && chunk_on) {
                const unsigned block = (unsigned)key >> 4, pi = page_of(p, block);
                const long long at = (block_place(p, block, pi, pages[pi], head) + (key & 15)) * row_bytes + chunk * 16;
                kreg[i] = ld16(p.K + at);
                vreg[i] = ld16(p.V + at);
            }
        }
        if constexpr (I8) {
            const int key = kt * KEYS + (tid & 63);
            scale_reg = 0.f;
            if (tid < 128 && key < si.kv) {
                const unsigned block = (unsigned)key >> 4, pi = page_of(p, block);
                const long long at = block_place(p, block, pi, pages[pi], head) + (key & 15);
                scale_reg = (tid < 64 ? p.ks : p.vs)[at];
            }
        }
    };
    int* const special = reinterpret_cast<int*>(smem + 2 * T::STAGE);   // per stage: a tile whose V holds something not finite
    auto write_tile = [&](int kt, int stage) {
        char* const ks = smem + stage * T::STAGE;
        char* const vs = ks + T::HALF;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int r = crow + i * PASS;
            if constexpr (I8) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int c = 2 * chunk + e;
                    *reinterpret_cast<i32x4*>(ks + r * T::PITCH + ((c ^ T::k_swizzle(r)) * 16)) = widen8<DT>(kreg[i][2 * e], kreg[i][2 * e + 1]);
                    *reinterpret_cast<i32x4*>(vs + r * T::PITCH + ((c ^ T::v_swizzle(r)) * 16)) = widen8<DT>(vreg[i][2 * e], vreg[i][2 * e + 1]);
                }
            } else {
                *reinterpret_cast<i32x4*>(ks + r * T::PITCH + ((chunk ^ T::k_swizzle(r)) * 16)) = kreg[i];
                // a key that some rows of the tile do not see must not reach them as 0 times infinity: such values stay out of
                // the product and are added one by one, where they are seen
                if (kt * KEYS < full_from || (kt + 1) * KEYS > full_to) {
                    if (any_not_finite<DT>(vreg[i])) {
                        bad = true;
#pragma unroll
                        for (int d = 0; d < 4; ++d) vreg[i][d] = only_finite<DT>(vreg[i][d]);
                    }
                }
                *reinterpret_cast<i32x4*>(vs + r * T::PITCH + ((chunk ^ T::v_swizzle(r)) * 16)) = vreg[i];
            }
        }
        if (bad) special[stage] = kt;
        if constexpr (I8) {
            float* const f = reinterpret_cast<float*>(vs + T::HALF);
            if (tid < 64) {
                f[tid] = scale_reg * p.c;
            } else if (tid < 128) {
                float l, v;
                value_scale(scale_reg, l, v);
                f[tid] = l;
                f[tid + 64] = v;
            }
        }
    };

    typename MMA::Acc o[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    float m = ATTN_NONE, l = 0.f;   // (m: as a power of two)

    if (tid < 2) special[tid] = -1;
    __syncthreads();
    if (t1 > t0) {
        load_tile(t0);
        write_tile(t0, 0);
    }
    __syncthreads();
    for (int kt = t0; kt < t1; ++kt) {
        const int stage = (kt - t0) & 1;
        if (kt + 1 < t1) load_tile(kt + 1);
        const int k0 = kt * KEYS;
        // (a wavefront whose rows see nothing of the tile leaves it out)
        if (wave_on && k0 < w_to && k0 + KEYS > w_from) {
            const char* const ks = smem + stage * T::STAGE;
            const char* const vs = ks + T::HALF;
            // ---- S^T: two blocks of 32 keys
            typename MMA::Acc s[2];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    const int r = kb * 32 + col;
                    const i32x4 a = *reinterpret_cast<const i32x4*>(ks + r * T::PITCH + (((2 * st + h) ^ T::k_swizzle(r)) * 16));
                    s[kb] = MMA::run(a, q[st], s[kb]);
                }
            }
            // key of register r in block kb: k0 + 32 kb + 8 (r / 4) + 4 h + r % 4
            const float* const fs = reinterpret_cast<const float*>(vs + T::HALF) + 4 * h;
            if constexpr (I8) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r4 = 0; r4 < 4; ++r4) {
                        const f32x4 kc = *reinterpret_cast<const f32x4*>(fs + 32 * kb + 8 * r4);
                        const f32x4 lt = *reinterpret_cast<const f32x4*>(fs + KEYS + 32 * kb + 8 * r4);
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[kb][4 * r4 + r] = __builtin_fmaf(s[kb][4 * r4 + r], kc[r], lt[r]);
                    }
            }
            const bool masked = k0 < w_full_from || k0 + KEYS > w_full_to;
            if (masked) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int key = k0 + 32 * kb + 8 * (r >> 2) + 4 * h + (r & 3);
                        s[kb][r] = key >= my_lo && key < my_hi ? s[kb][r] : -__builtin_huge_valf();
                    }
            }
            // ---- the running maximum
            float top = s[0][0];
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[kb][r]);
            if constexpr (!I8) top *= p.c;
            if (__any(top - m > ATTN_SLACK)) {
                top = __builtin_fmaxf(__builtin_fmaxf(top, swap_halves(top)), m);
                const float f = __builtin_amdgcn_exp2f(m - top);
                m = top;
                l *= f;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[b][r] *= f;
            }
            // ---- weights and their sum
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] = __builtin_amdgcn_exp2f(I8 ? s[kb][r] - m : __builtin_fmaf(s[kb][r], p.c, -m));
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    if constexpr (I8) {
                        f32x4 inv = *reinterpret_cast<const f32x4*>(fs + 2 * KEYS + 32 * kb + 8 * r4);
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            // (a key that is not seen may have any scale)
                            if (masked) inv[r] = s[kb][4 * r4 + r] == 0.f ? 0.f : inv[r];
                            l = __builtin_fmaf(s[kb][4 * r4 + r], inv[r], l);
                        }
                    } else {
                        l += (s[kb][4 * r4] + s[kb][4 * r4 + 1]) + (s[kb][4 * r4 + 2] + s[kb][4 * r4 + 3]);
                    }
                }
            // ---- O^T += V^T P^T: sixteen keys at a time, 32 kb + 16 half + {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    i32x4 w;
#pragma unroll
                    for (int d = 0; d < 4; ++d) w[d] = pack_out16<DT>(s[kb][8 * half + 2 * d], s[kb][8 * half + 2 * d + 1]);
#pragma unroll
                    for (int b = 0; b < BLOCKS; ++b) {
                        // (a transposing read: sixteen lanes bring four keys' rows of sixteen values and get a column each)
                        i32x4 a;
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int r = 32 * kb + 16 * half + 8 * e + 4 * h + ((lane & 15) >> 2);
                            const int byte = 64 * b + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
                            const i32x2 v = read_transposed(vs + r * T::PITCH + (((byte >> 4) ^ T::v_swizzle(r)) * 16) + (byte & 15));
                            a[2 * e] = v[0];
                            a[2 * e + 1] = v[1];
                        }
                        o[b] = MMA::run(a, w, o[b]);
                    }
                }
            if constexpr (!I8) {
                if (__builtin_expect(special[stage] == kt, 0)) add_not_finite<DT, DP>(p, o, m, k0, si, pages, head, token, qh, my_lo, row_on ? my_hi : 0, h);
            }
        }
        if (kt + 1 < t1) write_tile(kt + 1, stage ^ 1);
        __syncthreads();
    }

    // ---- out: this lane's row, values 32 b + 8 (r / 4) + 4 h + r % 4
    l += swap_halves(l);
    if (!row_on) return;
    if (chunks == 1) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        char* const dst = p.O + (token * p.ldo + (long long)qh * p.dim) * 2;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d = 32 * b + 2 * r + 4 * h;
                i32x2 v;
                v[0] = pack_out16<DT>(o[b][r] * inv, o[b][r + 1] * inv);
                v[1] = pack_out16<DT>(o[b][r + 2] * inv, o[b][r + 3] * inv);
                if (d < p.dim) *reinterpret_cast<i32x2*>(dst + 2 * d) = v;
            }
    } else {
        const long long at = ((long long)token * p.heads * p.group + qh) * p.tile_splits + split;
        float* const dst = p.tile_o + at * p.dim;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int d = 32 * b + 2 * r + 4 * h;
                if (d < p.dim) *reinterpret_cast<f32x4*>(dst + d) = f32x4{o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]};
            }
        if (h == 0) {
            p.tile_ml[2 * at] = m;
            p.tile_ml[2 * at + 1] = l;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ //
// One new token: its rows are the up to sixteen query heads of a head of the cache.  A workgroup takes a chunk of the keys, its four
// wavefronts 32 keys each in turn, straight from memory into fragments (nothing is read twice, so nothing goes through LDS);
// at the end their sums meet in LDS.
// ------------------------------------------------------------------------------------------------------------------ //
template <int DT, bool I8, int DP>
struct SingleTile {
    static constexpr int ES = I8 ? 1 : 2;
    static constexpr int KB = DP / 4 * ES / 16;    // 16-byte pieces of a key in a lane: a quarter of its values
    static constexpr int VD = DP / 16;             // values of a V row in a lane
    static constexpr int VW = VD * ES / 4;         // registers of them
    i32x4 k[2][KB];
    int v[8][VW];
    f32x4 ks[2], vs[2];
};

template <int DT, bool I8, int DP>
__global__ __launch_bounds__(256) void attn_single_kernel(const AttnArgs p) {
    typedef SingleTile<DT, I8, DP> ST;
    typedef Mma<DT, 16> MMA;
    constexpr int ES = ST::ES, VD = ST::VD, STEPS = DP / 32;
    __shared__ __attribute__((aligned(16))) float out_o[4][16][DP];
    __shared__ float out_m[4][16], out_l[4][16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int head = (int)blockIdx.x % p.heads, rest = (int)blockIdx.x / p.heads;
    const int split = rest % p.single_splits, seq = rest / p.single_splits;
    const SeqInfo si = seq_info(p, seq);
    if (si.nq != 1) return;
    const int chunks = max(1, (si.kv + p.single_chunk - 1) / p.single_chunk);
    if (split >= chunks) return;
    // keys that the token sees: it is the last one, and sees all but what the window leaves out
    const int lo = p.window > 0 ? max(si.kv - p.window, 0) : 0, hi = si.kv;
    const int c_from = split * p.single_chunk, c_to = min(hi, c_from + p.single_chunk);
    const int from = max(c_from, lo) & ~31;
    const int n_tiles = c_to > from ? (c_to - from + 31) >> 5 : 0;
    const int n_own = n_tiles > wave ? (n_tiles - wave + 3) >> 2 : 0;

    // page numbers of the own tiles' two blocks of sixteen keys: lane 2 i + b holds that of block b of tile i
    int entry = 0;
    {
        const unsigned key = (unsigned)from + 32u * (wave + 4 * (lane >> 1)) + 16u * (lane & 1);
        if ((lane >> 1) < n_own && (int)key < c_to) entry = p.table[seq * p.ld_table + page_of(p, key >> 4)];
    }
    i32x4 q[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = g * (DP / 4) + 8 * s;
        q[s] = col < p.group && d < p.dim ? ld16(p.Q + (si.q0 * p.ldq + (long long)(head * p.group + col) * p.dim + d) * 2) : i32x4{0, 0, 0, 0};
    }

    const int row_bytes = p.dim * ES;
    const bool v_on = col * VD < p.dim;
    auto load = [&](ST& t, int i) {
        const int k0 = from + 32 * (wave + 4 * i);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int kb = k0 + 16 * b;
            const unsigned block = (unsigned)kb >> 4;
            const int e = __builtin_amdgcn_readlane(entry, 2 * i + b);
            const bool in = kb < c_to;    // (a block of keys that there are some of; it lies in one page)
            const long long at = in ? block_place(p, block, page_of(p, block), e, head) : 0;
            const char* const kp = p.K + (at + col) * row_bytes + g * (DP / 4) * ES;
#pragma unroll
            for (int c = 0; c < ST::KB; ++c) t.k[b][c] = in && (g * (DP / 4) * ES + 16 * c) < row_bytes ? ld16(kp + 16 * c) : i32x4{0, 0, 0, 0};
            const char* const vp = p.V + (at + 4 * g) * row_bytes + col * VD * ES;
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                // (keys that are not seen: whatever lies there, zeros here)
                const int key = kb + 4 * g + e4;
                const bool on = v_on && key >= lo && key < c_to;
                const char* const src = vp + e4 * row_bytes;
                int* const dst = t.v[4 * b + e4];
                if constexpr (ST::VW == 4) {
                    const i32x4 x = on ? ld16(src) : i32x4{0, 0, 0, 0};
#pragma unroll
                    for (int d = 0; d < 4; ++d) dst[d] = x[d];
                } else if constexpr (ST::VW == 2) {
                    const i32x2 x = on ? *reinterpret_cast<const i32x2*>(src) : i32x2{0, 0};
                    dst[0] = x[0];
                    dst[1] = x[1];
                } else {
                    dst[0] = on ? *reinterpret_cast<const int*>(src) : 0;
                }
            }
            if constexpr (I8) {
                t.ks[b] = *reinterpret_cast<const f32x4*>(p.ks + at + 4 * g);
                t.vs[b] = *reinterpret_cast<const f32x4*>(p.vs + at + 4 * g);
            }
        }
    };

    typename MMA::Acc o[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) o[j] = typename MMA::Acc{0.f, 0.f, 0.f, 0.f};
    float m = ATTN_NONE, l = 0.f;
    auto take = [&](const ST& t, int i) {
        const int k0 = from + 32 * (wave + 4 * i);
        float s[2][4], inv[2][4];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            typename MMA::Acc acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                i32x4 a;
                if constexpr (I8) a = widen8<DT>(t.k[b][st >> 1][2 * (st & 1)], t.k[b][st >> 1][2 * (st & 1) + 1]);
                else a = t.k[b][st];
                acc = MMA::run(a, q[st], acc);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                inv[b][r] = 1.f;
                if constexpr (I8) {
                    float lt;
                    value_scale(t.vs[b][r], lt, inv[b][r]);
                    s[b][r] = __builtin_fmaf(acc[r], t.ks[b][r] * p.c, lt);
                } else {
                    s[b][r] = acc[r] * p.c;
                }
            }
        }
        if (k0 < lo || k0 + 32 > c_to) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = k0 + 16 * b + 4 * g + r;
                    const bool seen = key >= lo && key < c_to;
                    s[b][r] = seen ? s[b][r] : -__builtin_huge_valf();
                    inv[b][r] = seen ? inv[b][r] : 0.f;
                }
        }
        float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(s[0][0], s[0][1]), __builtin_fmaxf(s[0][2], s[0][3])),
                                    __builtin_fmaxf(__builtin_fmaxf(s[1][0], s[1][1]), __builtin_fmaxf(s[1][2], s[1][3])));
        if (__any(top - m > ATTN_SLACK)) {
            top = __builtin_fmaxf(top, __shfl_xor(top, 16));
            top = __builtin_fmaxf(__builtin_fmaxf(top, __shfl_xor(top, 32)), m);
            const float f = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f;
#pragma unroll
            for (int j = 0; j < VD; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[j][r] *= f;
        }
        i32x4 w;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[b][r] = __builtin_amdgcn_exp2f(s[b][r] - m);
                if constexpr (I8) l = __builtin_fmaf(s[b][r], inv[b][r], l);
                else l += s[b][r];
            }
            w[2 * b] = pack_out16<DT>(s[b][0], s[b][1]);
            w[2 * b + 1] = pack_out16<DT>(s[b][2], s[b][3]);
        }
        // V^T: value j of the lane's, of the eight keys
#pragma unroll
        for (int j = 0; j < VD; ++j) {
            i32x4 a;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (I8) {
                    const int x = t.v[2 * e][j >> 2] >> (8 * (j & 3)), y = t.v[2 * e + 1][j >> 2] >> (8 * (j & 3));
                    a[e] = pack_out16<DT>((float)(signed char)x, (float)(signed char)y);
                } else {
                    a[e] = (int)__builtin_amdgcn_perm((unsigned)t.v[2 * e + 1][j >> 1], (unsigned)t.v[2 * e][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                }
            }
            o[j] = MMA::run(a, w, o[j]);
        }
    };

    ST t[2];
    if (n_own > 0) load(t[0], 0);
    for (int i = 0; i < n_own; i += 2) {
        if (i + 1 < n_own) load(t[1], i + 1);
        take(t[0], i);
        if (i + 2 < n_own) load(t[0], i + 2);
        if (i + 1 < n_own) take(t[1], i + 1);
    }

    // ---- the wavefronts' sums meet: row `col`, values 4 VD g + VD r + j
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) {
        out_m[wave][col] = m;
        out_l[wave][col] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; j += 4)
            *reinterpret_cast<f32x4*>(&out_o[wave][col][VD * (4 * g + r) + j]) = f32x4{o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
    __syncthreads();
    const int row = tid >> 4, d0 = (tid & 15) * VD;
    if (row >= p.group || d0 >= p.dim) return;
    const float M = __builtin_fmaxf(__builtin_fmaxf(out_m[0][row], out_m[1][row]), __builtin_fmaxf(out_m[2][row], out_m[3][row]));
    float L = 0.f, acc[VD];
#pragma unroll
    for (int j = 0; j < VD; ++j) acc[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(out_m[w][row] - M);
        L = __builtin_fmaf(f, out_l[w][row], L);
#pragma unroll
        for (int j = 0; j < VD; ++j) acc[j] = __builtin_fmaf(f, out_o[w][row][d0 + j], acc[j]);
    }
    const int qh = head * p.group + row;
    if (chunks == 1) {
        const float inv = L == 0.f ? 0.f : 1.f / L;
        char* const dst = p.O + (si.q0 * p.ldo + (long long)qh * p.dim + d0) * 2;
#pragma unroll
        for (int j = 0; j < VD; j += 4)
            *reinterpret_cast<i32x2*>(dst + 2 * j) = i32x2{pack_out16<DT>(acc[j] * inv, acc[j + 1] * inv), pack_out16<DT>(acc[j + 2] * inv, acc[j + 3] * inv)};
    } else {
        const long long at = ((long long)seq * p.heads * p.group + qh) * p.single_splits + split;
#pragma unroll
        for (int j = 0; j < VD; j += 4)
            *reinterpret_cast<f32x4*>(p.single_o + at * p.dim + d0 + j) = f32x4{acc[j], acc[j + 1], acc[j + 2], acc[j + 3]};
        if (d0 == 0) {
            p.single_ml[2 * at] = M;
            p.single_ml[2 * at + 1] = L;
        }
    }
}

// ------------------------------------------------------------------------------------------------------------------ //
// The splits of a row put together, a wavefront per row: first the rows of single tokens (by sequence), then all tokens'.
// ------------------------------------------------------------------------------------------------------------------ //
template <int DT>
__global__ __launch_bounds__(256) void attn_join_kernel(const AttnArgs p) {
    const int lane = threadIdx.x & 63;
    const int qheads = p.heads * p.group;
    long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const long long singles = p.single_splits > 1 ? (long long)p.n_seqs * qheads : 0;
    int chunks, token, qh;
    long long at;
    const float *src, *ml;
    if (row < singles) {
        const int seq = (int)(row / qheads);
        const SeqInfo si = seq_info(p, seq);
        if (si.nq != 1) return;
        qh = (int)(row - (long long)seq * qheads);
        token = si.q0;
        chunks = (si.kv + p.single_chunk - 1) / p.single_chunk;
        at = row * p.single_splits;
        src = p.single_o;
        ml = p.single_ml;
    } else {
        row -= singles;
        if (p.tile_splits <= 1 || row >= (long long)p.total_q * qheads) return;
        token = (int)(row / qheads);
        qh = (int)(row - (long long)token * qheads);
        int a = 0, b = p.n_seqs;   // the last sequence that starts at or before the token
        while (b - a > 1) {
            const int mid = (a + b) / 2;
            if (p.q_start[mid] <= token) a = mid;
            else b = mid;
        }
        const SeqInfo si = seq_info(p, a);
        if (token < si.q0 || token >= si.q0 + si.nq || (p.single && si.nq == 1)) return;
        chunks = (si.kv + p.tile_chunk - 1) / p.tile_chunk;
        at = row * p.tile_splits;
        src = p.tile_o;
        ml = p.tile_ml;
    }
    if (chunks <= 1) return;
    float M = ATTN_NONE;
    for (int i = lane; i < chunks; i += 64) M = __builtin_fmaxf(M, ml[2 * (at + i)]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) M = __builtin_fmaxf(M, __shfl_xor(M, d));
    float L = 0.f, x = 0.f, y = 0.f;
    for (int i = 0; i < chunks; ++i) {
        const float part = ml[2 * (at + i) + 1];
        if (part == 0.f) continue;   // (saw nothing)
        const float f = __builtin_amdgcn_exp2f(ml[2 * (at + i)] - M);
        L = __builtin_fmaf(f, part, L);
        if (2 * lane < p.dim) {
            x = __builtin_fmaf(f, src[(at + i) * p.dim + 2 * lane], x);
            y = __builtin_fmaf(f, src[(at + i) * p.dim + 2 * lane + 1], y);
        }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    if (2 * lane < p.dim) *reinterpret_cast<int*>(p.O + (token * p.ldo + (long long)qh * p.dim + 2 * lane) * 2) = pack_out16<DT>(x * inv, y * inv);
}

}  // namespace abft
