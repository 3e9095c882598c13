// One new token: its rows are the up to sixteen query heads of a head of the cache.  The keys of all such sequences and heads,
// put behind one another in units of 128, are divided evenly over one or two workgroups for each compute unit, so that all
// end together whatever the lengths are; a workgroup's share begins and ends anywhere, and may span several heads and
// sequences.  Its four wavefronts take 32 keys each in turn, straight from memory into fragments (nothing is read twice,
// so nothing goes through LDS); at the end of a head's keys, or of the share, their sums meet in LDS.
// Bound: the bytes of keys and values, and for few sequences the chain of loads, stores and counters behind one another.  Measured, 8 heads of
// 128 read by 4 queries each: 64 sequences of 17 to 8144 tokens, int8, 110 us (5.0 TB/s); 16 of 8192, fp16, 100 us (5.4 TB/s), int8 57 (4.8);
// one of 2048 / 32768, int8, 10.6 / 20.8 us.
#pragma once
#include "attention.h"

namespace abft {

constexpr int SINGLE_UNIT = 128;

// the first key that a single token sees (it is the last one itself), and its units: one at least, since its rows have to be written
__device__ __forceinline__ int single_lo(const AttnArgs& p, int kv) { return p.window > 0 ? max(kv - p.window, 0) : 0; }
__device__ __forceinline__ unsigned single_units(const AttnArgs& p, const SeqInfo& i) {
    const int from = single_lo(p, i.kv) & ~(SINGLE_UNIT - 1);
    return i.nq == 1 ? (unsigned)max(1, (i.kv - from + SINGLE_UNIT - 1) / SINGLE_UNIT) : 0;
}

// How the units of a launch are dealt: workgroup b has units first(b) to first(b + 1) - 1.
struct Shares {
    unsigned per, more;   // each has `per`, the first `more` one more
    __device__ __forceinline__ unsigned first(unsigned b) const { return b * per + min(b, more); }
    __device__ __forceinline__ unsigned owner(unsigned u) const {
        const unsigned big = more * (per + 1);
        return u < big ? u / (per + 1) : more + (u - big) / max(per, 1u);
    }
};
// A wavefront's look at the launch: the shares, the sequence that holds workgroup b's first unit (seq; -1: it has none), what is known of
// it, and its own first unit.
struct SingleStart {
    Shares sh;
    SeqInfo si;
    int seq;
    unsigned seq_first;
};
__device__ __forceinline__ SingleStart single_start(const AttnArgs& p, unsigned b) {
    const int lane = threadIdx.x & 63;
    // 64 sequences: what is known of them, their units, and the sums up to each of them
    SeqInfo i;
    unsigned n, sum;
    auto look = [&](int s0) {
        i = seq_info(p, min(s0 + lane, p.n_seqs - 1));   // (three loads without a condition)
        n = s0 + lane < p.n_seqs ? single_units(p, i) * (unsigned)p.heads : 0;
        sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const unsigned up = __shfl_up(sum, d);
            if (lane >= d) sum += up;
        }
    };
    unsigned total = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
        look(s0);
        total += readlane(sum, 63);
    }
    SingleStart st;
    st.sh.per = total / (unsigned)p.single_groups;
    st.sh.more = total - st.sh.per * (unsigned)p.single_groups;
    st.seq = -1;
    const unsigned unit = st.sh.first(b);
    unsigned before = 0;
    for (int s0 = 0; s0 < p.n_seqs && st.seq < 0; s0 += 64) {
        if (p.n_seqs > 64) look(s0);   // (else it has been)
        const unsigned long long at = __ballot(before + sum > unit);
        if (at != 0) {
            const int l = __builtin_ctzll(at);
            st.seq = s0 + l;
            st.si.q0 = readlane(i.q0, l);
            st.si.nq = readlane(i.nq, l);
            st.si.kv = readlane(i.kv, l);
            st.seq_first = before + readlane(sum, l) - readlane(n, l);
        }
        before += readlane(sum, 63);
    }
    return st;
}

// A head whose keys several workgroups share: its owners are owner0 and the ones behind it, whose sums lie at place0 (the first's)
// and at their first places.
struct Joint {
    unsigned owner0, owners, place0;
    int token, head;
};
// VD values of a row from d0 on, divided by the sum of weights
template <int DT, int VD>
__device__ __forceinline__ void single_store(const AttnArgs& p, int token, int qh, int d0, const float (&acc)[VD], float norm) {
    char* const dst = p.O + (token * p.ldo + (long long)qh * p.dim + d0) * 2;
#pragma unroll
    for (int j = 0; j < VD; j += 4)
        *reinterpret_cast<i32x2*>(dst + 2 * j) = i32x2{pack_out16<DT>(acc[j] * norm, acc[j + 1] * norm), pack_out16<DT>(acc[j + 2] * norm, acc[j + 3] * norm)};
}

template <int DP>
struct __attribute__((aligned(16))) SingleLds {
    float o[4][16][DP];   // the wavefronts' sums
    float m[4][16], l[4][16];
    bool last_owner[2];
};
template <int DT, bool I8, int DP>
__device__ __forceinline__ void single_tokens(const AttnArgs& p, SingleLds<DP>& lds) {
    typedef Mma<DT, 16> MMA;
    constexpr int ES = I8 ? 1 : 2, STEPS = DP / 32;
    constexpr int KB = DP / 4 * ES / 16;    // 16-byte pieces of a key in a lane: a quarter of its values
    constexpr int VD = DP / 16;             // values of a V row in a lane
    constexpr int VW = VD * ES / 4;         // registers of them
    typedef int Piece __attribute__((ext_vector_type(VW)));
    auto& out_o = lds.o;
    auto &out_m = lds.m, &out_l = lds.l;
    auto& last_owner = lds.last_owner;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int bid = blockIdx.x;
    const SingleStart start = single_start(p, bid);
    const Shares sh = start.sh;
    int seq = start.seq;
    unsigned unit = sh.first(bid), seq_first = start.seq_first;
    const unsigned share = unit, unit_end = sh.first(bid + 1);
    if (seq < 0 || unit >= unit_end) return;

    // Addresses: a block's place is the wavefront's, a lane's offsets from it do not change.  No load has a condition: a piece
    // beyond the head's values is read from the row's start (and dropped, where a 16-bit key's would reach the product;
    // the queries are zeros there), a block without keys is the last one with some.
    const int row_bytes = p.dim * ES;
    unsigned k_off[KB], v_off[4];
#pragma unroll
    for (int c = 0; c < KB; ++c) {
        const int in_row = g * (DP / 4) * ES + 16 * c;
        k_off[c] = (unsigned)(col * row_bytes + (in_row < row_bytes ? in_row : 0));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v_off[e] = (unsigned)((4 * g + e) * row_bytes + (col * VD < p.dim ? col * VD * ES : 0));

    // ---- the share, one head of a sequence after the other
    SeqInfo si = start.si;
    unsigned units = single_units(p, si);
    Joint head0 = {0, 0, 0, 0, 0}, head1 = {0, 0, 0, 0, 0};   // the heads that this share holds a part of: its first, its last
    while (unit < unit_end) {
        while (unit >= seq_first + units * p.heads) {   // (sequences of other lengths have no units)
            seq_first += units * p.heads;
            si = seq_info(p, ++seq);
            units = single_units(p, si);
        }
        const int head = (int)((unit - seq_first) / units);
        const unsigned pair_first = seq_first + head * units, pair_end = pair_first + units, here_end = min(pair_end, unit_end);
        // the keys here, from .. c_to - 1; those before lo are not seen
        const int lo = single_lo(p, si.kv), unit0 = lo & ~(SINGLE_UNIT - 1);
        const int from = unit0 + (int)(unit - pair_first) * SINGLE_UNIT, c_to = min(si.kv, unit0 + (int)(here_end - pair_first) * SINGLE_UNIT);
        const int n_tiles = c_to > from ? (c_to - from + 31) >> 5 : 0;
        const int n_own = n_tiles > wave ? (n_tiles - wave + 3) >> 2 : 0;
        const bool first_here = unit == share, whole = unit == pair_first && here_end == pair_end;
        if (!whole) {
            // (the first owner's place is its first only where its share starts with this head, the others' is their first)
            Joint j;
            j.owner0 = sh.owner(pair_first);
            j.owners = sh.owner(pair_end - 1) - j.owner0 + 1;
            j.place0 = 2 * j.owner0 + (sh.first(j.owner0) == pair_first ? 0 : 1);
            j.token = si.q0;
            j.head = head;
            if (first_here) head0 = j;
            else head1 = j;
        }
        unit = here_end;

        // the page numbers of own tile i's two blocks of sixteen keys, through the scalar cache, and the blocks' first keys as
        // indexes among a head's tokens
        const __attribute__((address_space(4))) int* const pages = (const __attribute__((address_space(4))) int*)(p.table + seq * p.ld_table);
        auto block_of = [&](int i, int b) { return (unsigned)min(from + 32 * (wave + 4 * i) + 16 * b, c_to - 1) >> 4; };
        auto entry = [&](int i, int b) { return pages[page_of(p, block_of(i, b))]; };
        long long at[2];
        auto place = [&](int i, const int (&e)[2]) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const unsigned block = block_of(i, b);
                at[b] = block_place(p, block, page_of(p, block), e[b], head);
            }
        };
        i32x4 kreg[2][KB];
        int vreg[8][VW];
        f32x4 ks[2], vs[2];
        auto load_k = [&]() {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const char* const kp = p.K + at[b] * row_bytes;
#pragma unroll
                for (int c = 0; c < KB; ++c) kreg[b][c] = ld16g(kp + k_off[c]);
                if constexpr (I8) {
                    ks[b] = bitcast<f32x4>(ld16g(reinterpret_cast<const char*>(p.ks + at[b]) + 16 * g));
                    vs[b] = bitcast<f32x4>(ld16g(reinterpret_cast<const char*>(p.vs + at[b]) + 16 * g));
                }
            }
        };
        auto load_v = [&]() {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const char* const vp = p.V + at[b] * row_bytes;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const Piece x = *(const __attribute__((address_space(1))) Piece*)(const __attribute__((address_space(1))) char*)(vp + v_off[e]);
#pragma unroll
                    for (int d = 0; d < VW; ++d) {
                        if constexpr (VW == 1) vreg[4 * b + e][d] = bitcast<int>(x);
                        else vreg[4 * b + e][d] = x[d];
                    }
                }
            }
        };

        typename MMA::Acc o[VD];
#pragma unroll
        for (int j = 0; j < VD; ++j) o[j] = typename MMA::Acc{0.f, 0.f, 0.f, 0.f};
        float m = ATTN_NONE, l = 0.f;
        int e[2] = {0, 0};
        if (n_own > 0) {
            e[0] = entry(0, 0);
            e[1] = entry(0, 1);
            place(0, e);
            load_k();
            load_v();
            e[0] = entry(1, 0);
            e[1] = entry(1, 1);
        }
        i32x4 q[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int d = g * (DP / 4) + 8 * s;
            q[s] = col < p.group && d < p.dim ? ld16(p.Q + (si.q0 * p.ldq + (long long)(head * p.group + col) * p.dim + d) * 2) : i32x4{0, 0, 0, 0};
        }
        // (waited for here: the loop's waits then count its own loads only)
#pragma unroll
        for (int s = 0; s < STEPS; ++s) asm volatile("" : "+v"(q[s]));
        for (int i = 0; i < n_own; ++i) {
            const int k0 = from + 32 * (wave + 4 * i);
            const bool masked = k0 < lo || k0 + 32 > c_to;
            // ---- S^T: row 4 g + r of block b is key k0 + 16 b + 4 g + r
            float s[2][4], inv[2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                typename MMA::Acc acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    i32x4 a;
                    if constexpr (I8) {
                        a = widen8<DT>(kreg[b][st >> 1][2 * (st & 1)], kreg[b][st >> 1][2 * (st & 1) + 1]);
                    } else {
                        a = kreg[b][st];
                        if (p.dim < DP && g * (DP / 4) + 8 * st >= p.dim) a = i32x4{0, 0, 0, 0};
                    }
                    acc = MMA::run(a, q[st], acc);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    inv[b][r] = 1.f;
                    if constexpr (I8) {
                        float lt;
                        value_scale<DT>(vs[b][r], lt, inv[b][r]);
                        s[b][r] = __builtin_fmaf(acc[r], ks[b][r] * p.c, lt);
                    } else {
                        s[b][r] = acc[r] * p.c;
                    }
                }
            }
            // (the next tile's pieces take the registers of this one's, so nothing of it may move behind their loads; behind the
            // last, its last block once more: no condition)
            place(i + 1, e);
            e[0] = entry(i + 2, 0);
            e[1] = entry(i + 2, 1);
            __builtin_amdgcn_sched_barrier(0);
            load_k();
            if (masked) {
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
            if (__any(top - m > ATTN_SLACK + ATTN_LIFT<DT>)) {
                top = __builtin_fmaxf(top, __shfl_xor(top, 16)) - ATTN_LIFT<DT>;
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
            // values of keys that are not seen: whatever lies there, zeros here (integers need none)
            if (!I8 && masked) {
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int key = k0 + 16 * (x >> 2) + 4 * g + (x & 3);
#pragma unroll
                    for (int d = 0; d < VW; ++d) vreg[x][d] = key >= lo && key < c_to ? vreg[x][d] : 0;
                }
            }
            // ---- O^T += V^T P^T: value j of the lane's, of the eight keys
#pragma unroll
            for (int j = 0; j < VD; ++j) {
                i32x4 a;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (I8) {
                        const int y = vreg[2 * x][j >> 2] >> (8 * (j & 3)), z = vreg[2 * x + 1][j >> 2] >> (8 * (j & 3));
                        a[x] = pack_out16<DT>((float)(signed char)y, (float)(signed char)z);
                    } else {
                        a[x] = (int)__builtin_amdgcn_perm((unsigned)vreg[2 * x + 1][j >> 1], (unsigned)vreg[2 * x][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
                    }
                }
                o[j] = MMA::run(a, w, o[j]);
            }
            __builtin_amdgcn_sched_barrier(0);
            load_v();
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
        if (row < p.group && d0 < p.dim) {
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
            if (whole) {
                const float norm = L == 0.f ? 0.f : 1.f / L;
                single_store<DT, VD>(p, si.q0, head * p.group + row, d0, acc, norm);
            } else {
                // a share's first head has its first place, its last the second: between them all are whole
                const int place_row = (2 * bid + (first_here ? 0 : 1)) * p.group + row;
#pragma unroll
                for (int j = 0; j < VD; j += 2) put_shared(p.single_o + (long long)place_row * p.dim + d0 + j, acc[j], acc[j + 1]);
                if (d0 == 0) put_shared(p.single_ml + 2 * place_row, M, L);
            }
        }
        __syncthreads();   // (the LDS is the next head's)
    }

    // ---- whoever is the last of a head's owners puts their sums together.  (The counter is that of the first owner, of whose heads
    // only the last can go on behind its share; it is back at zero when the launch ends.  The sums are written through to where
    // every die reads them, and waited for, before the counter moves; fences in their place, which write back and drop a die's
    // whole L2, took 64 sequences from 108 to 162 us.)
    if (head0.owners + head1.owners == 0) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (lane == 0 && wave < 2) {
        const unsigned owner0 = wave == 0 ? head0.owner0 : head1.owner0, owners = wave == 0 ? head0.owners : head1.owners;
        last_owner[wave] = owners != 0 && __hip_atomic_fetch_add(p.counters + owner0, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == owners - 1;
    }
    __syncthreads();
    // sixteen threads a row, and as many such sets as there are: each takes every set-th owner
    const int row = tid >> 4, d0 = (tid & 15) * VD, sets = 16 / p.group, set = row / p.group, r = row - set * p.group;
    for (int which = 0; which < 2; ++which) {
        if (!last_owner[which]) continue;
        const Joint j = which == 0 ? head0 : head1;
        if (tid == 0) __hip_atomic_store(p.counters + j.owner0, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        auto place_of = [&](unsigned i) { return (int)(i == 0 ? j.place0 : 2 * (j.owner0 + i)) * p.group + r; };
        float M = ATTN_NONE, L = 0.f, acc[VD];
#pragma unroll
        for (int c = 0; c < VD; ++c) acc[c] = 0.f;
        if (set < sets) {
            const int d = d0 < p.dim ? d0 : 0;
            // four owners' sums on their way at a time
            for (unsigned i0 = set; i0 < j.owners; i0 += 4 * sets) {
                float2 ml[4], x[4][VD / 2];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int at = place_of(min(i0 + u * sets, j.owners - 1));
                    ml[u] = get_shared(p.single_ml + 2 * at);
#pragma unroll
                    for (int c = 0; c < VD / 2; ++c) x[u][c] = get_shared(p.single_o + (long long)at * p.dim + d + 2 * c);
                }
                // (the last owner more than once is no harm to a maximum)
                const float top = __builtin_fmaxf(__builtin_fmaxf(__builtin_fmaxf(ml[0].x, ml[1].x), __builtin_fmaxf(ml[2].x, ml[3].x)), M);
                const float f0 = __builtin_amdgcn_exp2f(M - top);
                M = top;
                L *= f0;
#pragma unroll
                for (int c = 0; c < VD; ++c) acc[c] *= f0;
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (i0 + u * sets >= j.owners) continue;
                    const float f = __builtin_amdgcn_exp2f(ml[u].x - M);
                    L = __builtin_fmaf(f, ml[u].y, L);
#pragma unroll
                    for (int c = 0; c < VD / 2; ++c) {
                        acc[2 * c] = __builtin_fmaf(f, x[u][c].x, acc[2 * c]);
                        acc[2 * c + 1] = __builtin_fmaf(f, x[u][c].y, acc[2 * c + 1]);
                    }
                }
            }
            if ((tid & 15) == 0) {
                out_m[0][row] = M;
                out_l[0][row] = L;
            }
#pragma unroll
            for (int c = 0; c < VD; c += 4) *reinterpret_cast<f32x4*>(&out_o[0][row][d0 + c]) = f32x4{acc[c], acc[c + 1], acc[c + 2], acc[c + 3]};
        }
        __syncthreads();
        if (row < p.group && d0 < p.dim) {
            for (int i = 1; i < sets; ++i) M = __builtin_fmaxf(M, out_m[0][i * p.group + row]);
            L = 0.f;
#pragma unroll
            for (int c = 0; c < VD; ++c) acc[c] = 0.f;
            for (int i = 0; i < sets; ++i) {
                const float f = __builtin_amdgcn_exp2f(out_m[0][i * p.group + row] - M);
                L = __builtin_fmaf(f, out_l[0][i * p.group + row], L);
#pragma unroll
                for (int c = 0; c < VD; ++c) acc[c] = __builtin_fmaf(f, out_o[0][i * p.group + row][d0 + c], acc[c]);
            }
            single_store<DT, VD>(p, j.token, j.head * p.group + row, d0, acc, L == 0.f ? 0.f : 1.f / L);
        }
        __syncthreads();
    }
}

template <int DT, bool I8, int DP>
__global__ __launch_bounds__(256, 2) void attn_single_kernel(const AttnArgs p) {
    __shared__ SingleLds<DP> lds;
    single_tokens<DT, I8, DP>(p, lds);
}

}  // namespace abft
