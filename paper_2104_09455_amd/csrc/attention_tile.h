// Many rows: a workgroup of four wavefronts takes 32 rows each of one sequence and head of the cache (rows are the new
// tokens' query heads of that head, token by token), and all keys that these rows see, 64 at a time, in 16 bits in LDS.
#pragma once
#include "attention.h"

namespace abft {

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
__device__ __forceinline__ void add_not_finite(const AttnArgs& p, f32x16 (&o)[DP / 32], float m, int k0, const SeqInfo& si, const __attribute__((address_space(4))) int* pages,
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
    // (what is the workgroup's or the wavefront's goes into scalar registers, or branches and addresses end up in vector code)
    auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    SeqInfo si = seq_info(p, seq);
    si.q0 = scalar(si.q0);
    si.nq = scalar(si.nq);
    si.kv = scalar(si.kv);
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
    const int full_from = scalar(lo_of(row_end)), full_to = scalar(hi_of(row0));            // keys that all rows of the workgroup see
    const int w_from = scalar(lo_of(wrow0)), w_to = scalar(hi_of(wrow_end)), w_full_from = scalar(lo_of(wrow_end)), w_full_to = scalar(hi_of(wrow0));
    const int t0 = scalar(from / KEYS), t1 = scalar(to > from ? (to + KEYS - 1) / KEYS : t0);   // tiles of keys

    // ---- this lane's query, as the fragments of the first product want it: values 16 s + 8 h .. + 7 of its row
    const int token = si.q0 + my_row / p.group, qh = head * p.group + my_row % p.group;
    i32x4 q[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = 16 * s + 8 * h;
        q[s] = row_on && d < p.dim ? ld16(p.Q + (token * p.ldq + (long long)qh * p.dim + d) * 2) : i32x4{0, 0, 0, 0};
    }

    // ---- copies: 16 bytes a thread, thread's chunk of rows tid / CPR + PASS i of a tile.  A wavefront's rows of a pass lie in one block
    // of sixteen keys: its place is the wavefront's, through the scalar cache, a tile ahead of the copies; a thread's offset
    // from it does not change.  No load has a condition: a chunk beyond the head's values is its row's first, a block without
    // keys the last one with some.
    constexpr int CPR = I8 ? T::PITCH / 32 : T::PITCH / 16, PASS = 256 / CPR, NP = KEYS / PASS;
    static_assert(64 / CPR <= 16, "a wavefront's rows in one block");
    const int chunk = tid % CPR, crow = tid / CPR, wrow = wave * (64 / CPR);
    const int row_bytes = p.dim * (I8 ? 1 : 2);
    const unsigned my_off = (unsigned)((crow & 15) * row_bytes + (chunk * 16 < row_bytes ? chunk * 16 : 0));
    typedef const __attribute__((address_space(4))) int ScalarInt;
    ScalarInt* const pages = (ScalarInt*)(p.table + seq * p.ld_table);
    auto block_of = [&](int kt, int i) { return (unsigned)min(kt * KEYS + wrow + i * PASS, si.kv - 1) >> 4; };
    int entries[NP];
    auto load_entries = [&](int kt) {
#pragma unroll
        for (int i = 0; i < NP; ++i) entries[i] = pages[page_of(p, block_of(kt, i))];
    };
    // 16-bit caches: straight into LDS, each lane's chunk from where its place wants it (a chunk of a key beyond the head's values:
    // zeros, since what is not finite would not vanish against the zeros of the queries).
    const int k_chunk = chunk ^ T::k_swizzle(crow), v_chunk = chunk ^ T::v_swizzle(crow);   // (a pass is a multiple of the swizzles' period)
    const unsigned k_off = (unsigned)((crow & 15) * row_bytes + k_chunk * 16), v_off = (unsigned)((crow & 15) * row_bytes + (v_chunk * 16 < row_bytes ? v_chunk * 16 : 0));
    const bool k_zero = k_chunk * 16 >= row_bytes;
    // int8: through registers, where they are widened
    i32x4 kreg[I8 ? NP : 1], vreg[I8 ? NP : 1];
    float k_scale_reg = 0.f, v_scale_reg = 0.f;
    constexpr int PER = 64 / CPR;
    auto load_tile = [&](int kt, int stage) {
        long long at[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const unsigned block = block_of(kt, i);
            at[i] = block_place(p, block, page_of(p, block), entries[i], head);
        }
        if constexpr (!I8) {
            char* const to = smem + stage * T::STAGE + wave * 1024;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const char* src = p.K + at[i] * row_bytes + k_off;
                if (p.dim < DP) src = k_zero ? g_zero_chunk : src;
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)(to + i * 4096), 16, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < NP; ++i)
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p.V + at[i] * row_bytes + v_off),
                                                 (__attribute__((address_space(3))) void*)(to + T::HALF + i * 4096), 16, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) kreg[i] = ld16g(p.K + at[i] * row_bytes + my_off);
#pragma unroll
            for (int i = 0; i < NP; ++i) vreg[i] = ld16g(p.V + at[i] * row_bytes + my_off);
            // (a wavefront's lanes in the order of its keys: PER of a pass)
            long long key = at[0] + (wrow & 15) + lane;
#pragma unroll
            for (int i = 1; i < NP; ++i)
                if (lane >= i * PER) key = at[i] + (wrow & 15) + lane - i * PER;
            if (lane < NP * PER) {
                k_scale_reg = p.ks[key];
                v_scale_reg = p.vs[key];
            }
        }
    };
    int* const special = reinterpret_cast<int*>(smem + 2 * T::STAGE);   // per stage: a tile whose V holds something not finite
    // what is left to do of a tile once its loads have come back (all wavefronts', then a barrier)
    auto finish_tile = [&](int kt, int stage) {
        char* const ks = smem + stage * T::STAGE;
        char* const vs = ks + T::HALF;
        if constexpr (I8) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int r = crow + i * PASS;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int c = 2 * chunk + e;
                    *reinterpret_cast<i32x4*>(ks + r * T::PITCH + ((c ^ T::k_swizzle(r)) * 16)) = widen8<DT>(kreg[i][2 * e], kreg[i][2 * e + 1]);
                    *reinterpret_cast<i32x4*>(vs + r * T::PITCH + ((c ^ T::v_swizzle(r)) * 16)) = widen8<DT>(vreg[i][2 * e], vreg[i][2 * e + 1]);
                }
            }
            float* const f = reinterpret_cast<float*>(vs + T::HALF);
            if (lane < NP * PER) {
                const int key = wrow + lane % PER + lane / PER * PASS;
                float l, v;
                value_scale(v_scale_reg, l, v);
                f[key] = k_scale_reg * p.c;
                f[key + KEYS] = l;
                f[key + 2 * KEYS] = v;
            }
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            // a key that some rows of the tile do not see must not reach them as 0 times infinity: zeros behind the last key, and
            // what is not finite stays out of the product and is added one by one, where it is seen.  (The thread's own chunks.)
            if (kt * KEYS < full_from || (kt + 1) * KEYS > full_to) {
                bool bad = false;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    i32x4* const at = reinterpret_cast<i32x4*>(vs + i * 4096 + tid * 16);
                    i32x4 v = *at;
                    if (kt * KEYS + crow + i * PASS >= si.kv) v = i32x4{0, 0, 0, 0};
                    if (any_not_finite<DT>(v)) {
                        bad = true;
#pragma unroll
                        for (int d = 0; d < 4; ++d) v[d] = only_finite<DT>(v[d]);
                    }
                    *at = v;
                }
                if (bad) special[stage] = kt;
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
        load_entries(t0);
        load_tile(t0, 0);
        load_entries(t0 + 1);
        finish_tile(t0, 0);
    }
    __syncthreads();
    for (int kt = t0; kt < t1; ++kt) {
        const int stage = (kt - t0) & 1;
        if (kt + 1 < t1) {
            load_tile(kt + 1, stage ^ 1);
            load_entries(kt + 2);
        }
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
                asm volatile("");   // (a branch: selects in its place would cost every tile 128 instructions)
                const int first = k0 + 4 * h - my_lo;
                const unsigned seen = (unsigned)max(my_hi - my_lo, 0);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[kb][r] = (unsigned)(first + 32 * kb + 8 * (r >> 2) + (r & 3)) < seen ? s[kb][r] : -__builtin_huge_valf();
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
        if (kt + 1 < t1) finish_tile(kt + 1, stage ^ 1);
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

// The splits of a row put together, a wavefront per row.
template <int DT>
__global__ __launch_bounds__(256) void attn_tile_join_kernel(const AttnArgs p) {
    const int qheads = p.heads * p.group;
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (row >= (long long)p.total_q * qheads) return;
    const int token = (int)(row / qheads), qh = (int)(row - (long long)token * qheads);
    int a = 0, b = p.n_seqs;   // the last sequence that starts at or before the token
    while (b - a > 1) {
        const int mid = (a + b) / 2;
        if (p.q_start[mid] <= token) a = mid;
        else b = mid;
    }
    const SeqInfo si = seq_info(p, a);
    if (token < si.q0 || token >= si.q0 + si.nq || (p.single && si.nq == 1)) return;
    const int n = (si.kv + p.tile_chunk - 1) / p.tile_chunk;
    if (n > 1) attn_join_row<DT>(p, n, [&](int i) { return row * p.tile_splits + i; }, p.tile_o, p.tile_ml, token, qh);
}

}  // namespace abft
