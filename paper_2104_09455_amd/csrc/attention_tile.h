// Many rows: a workgroup of four wavefronts takes 32 rows each of one sequence and head of the cache (rows are the new
// tokens' query heads of that head, token by token), and all keys that these rows see, 64 at a time, in 16 bits in LDS.
// Bound: the softmax's vector work beside the MFMAs, and for little work what a piece costs to begin and to join, about 10 us.  Measured, 8 heads of
// 128 read by 4 queries each: 8192 of 8192 tokens, bf16, 536 to 558 us (985 to 1025 TFLOP/s); from an int8 cache, which is widened on the way, fp16 690; 2048 of
// 12000 in a window of 1000, 80 wide, 42.
#pragma once
#include "attention.h"
#include "attention_single.h"

namespace abft {

template <int DP>
struct AttnTile {
    static constexpr int PITCH = DP <= 64 ? 128 : 256;            // bytes of a key's row in LDS
    static constexpr int ROWS = 128;                              // rows of a workgroup
    static constexpr int KEYS = ATTN_BLOCK_KEYS;
    static constexpr int K_STAGE = KEYS * PITCH + 2 * KEYS * 4;   // K, and two floats a key (int8)
    static constexpr int V_STAGE = KEYS * PITCH + KEYS * 4;       // V, and one
    static constexpr int LDS_BYTES = 2 * (K_STAGE + V_STAGE) + 16;
    // 16-byte chunk c of row r lies at chunk c ^ swizzle(r): the 16 rows that a fragment of K is read from at once, and the
    // 4 (x 64 bytes) of V, lie in different banks
    static __device__ __forceinline__ int k_swizzle(int r) { return PITCH == 256 ? r & 15 : (r >> 1) & 7; }
    static __device__ __forceinline__ int v_swizzle(int r) { return PITCH == 256 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// The launch's work: row tiles of each sequence, and pieces of the keys that a row tile sees where splitting them pays.  A sequence's
// pieces are of one size, near `chunk` tiles of keys (as many as fit it, one more if more than a quarter would be left over), so large that
// the whole work makes nine tenths of a piece for each workgroup that the chip holds: a few more than that would be a second round.
// At least TILE_MIN_CHUNK (a piece's sums cost as much as three or four tiles).  The host cannot know, since lengths are on the device.
// (us, fp16, 32 heads of 128, against pieces of exactly one for each workgroup, the last of a row tile short, a row tile's pieces beside one another
// in the launch: 509 of 4605 tokens 65 / 56, 2048 of 2048 78 / 70, 3 x 700 of 5000 316 / 237, 512 of 8192 95 / 90, 1024 of 1024 level.)
constexpr int TILE_SLOTS = 464, TILE_MIN_CHUNK = 8;
// (pieces of one head beyond one for each row tile: the sum of keys / chunk over the tiles is at most twice the work in slots)
constexpr int tile_more_pieces(int heads) { return (2 * TILE_SLOTS + heads - 1) / heads; }
struct TileWork {
    int seq, tile, tiles, piece, pieces, chunk, slot, index;   // slot, index: of the piece and of the row tile among all sequences'
    int group;   // the counter of the row tile's first group of pieces, -1: they are joined all at once
};
// A workgroup that joins many pieces' sums (64 KB each) takes long over them: from TILE_MANY on they are joined in groups first, and
// then the groups.  (16 new tokens of 32768, 8 x 4 heads, 64 pieces: 99 us at once, 49.5 in groups; 128 of 8192, 16 pieces: 65 / 57.5.)
constexpr int TILE_MANY = 13, TILE_GROUP = 8;
__device__ __forceinline__ int tile_groups(int pieces) { return pieces < TILE_MANY ? 0 : (pieces + TILE_GROUP - 1) / TILE_GROUP; }
__device__ __forceinline__ int tile_rows(const AttnArgs& p, const SeqInfo& i, int rows) { return p.single && i.nq == 1 ? 0 : (i.nq * p.group + rows - 1) / rows; }
// tiles of keys that a row tile of the sequence sees, at most
__device__ __forceinline__ int tile_keys(const AttnArgs& p, const SeqInfo& i, int rows) {
    const int all = (i.kv + ATTN_BLOCK_KEYS - 1) / ATTN_BLOCK_KEYS;
    const int seen = p.window > 0 && p.causal ? (min(p.window, i.kv) + rows / p.group + 1) / ATTN_BLOCK_KEYS + 2 : all;
    return max(min(all, seen), 1);
}
// The t-th piece of the launch; false: there is none.  All of a wavefront.
__device__ __forceinline__ bool find_tile(const AttnArgs& p, int t, int rows, TileWork& w) {
    const int lane = threadIdx.x & 63;
    int n = 0, keys = 1, mean = 1, chunk = 1 << 28, all_tiles = 0;
    auto look = [&](int s0) {
        const SeqInfo i = seq_info(p, min(s0 + lane, p.n_seqs - 1));
        n = s0 + lane < p.n_seqs ? tile_rows(p, i, rows) : 0;
        keys = tile_keys(p, i, rows);
        // (causal without a window: half of the new tokens less, on the average)
        mean = p.causal && p.window <= 0 ? max(keys - min(i.nq / (2 * ATTN_BLOCK_KEYS), keys / 2), 1) : keys;
    };
    if (p.tile_split) {
        unsigned long long work = 0;
        int tiles = 0;
        for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
            look(s0);
            work += (unsigned long long)n * mean;
            tiles += n;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            work += __shfl_xor(work, d);
            tiles += __shfl_xor(tiles, d);
        }
        // (more than there are counters and room for: no pieces.  Two row tiles for each workgroup that the chip holds fill it.)
        all_tiles = tiles;
        if (tiles <= p.tile_split) chunk = (int)max((work * p.heads + TILE_SLOTS - 1) / TILE_SLOTS, (unsigned long long)TILE_MIN_CHUNK);
    }
    int before = 0, tiles_before = 0, groups_before = all_tiles;
    for (int s0 = 0; s0 < p.n_seqs; s0 += 64) {
        if (!p.tile_split || p.n_seqs > 64) look(s0);   // (else it has been)
        const int pieces = max((4 * keys + 3 * chunk) / (4 * chunk), 1), units = n * pieces, groups = n * tile_groups(pieces);
        int sum = units, tile_sum = n, group_sum = groups;   // of this lane's and all lower ones
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(sum, d), tile_up = __shfl_up(tile_sum, d), group_up = __shfl_up(group_sum, d);
            if (lane >= d) {
                sum += up;
                tile_sum += tile_up;
                group_sum += group_up;
            }
        }
        const unsigned long long at = __ballot(before + sum > t);
        if (at != 0) {
            const int first = __builtin_ctzll(at), in = t - (before + readlane(sum, first) - readlane(units, first));
            w.seq = s0 + first;
            w.tiles = readlane(n, first);
            w.pieces = readlane(pieces, first);
            w.chunk = readlane((keys + pieces - 1) / pieces, first);
            // (all first pieces, then all second ones: the long ones begin first and are spread over all compute units)
            w.piece = in / w.tiles;
            w.tile = in - w.piece * w.tiles;
            w.slot = t - in + w.tile * w.pieces + w.piece;
            w.index = tiles_before + readlane(tile_sum, first) - w.tiles + w.tile;
            // (as far as the counters reach)
            const int many = tile_groups(w.pieces);
            w.group = groups_before + readlane(group_sum, first) - (w.tiles - w.tile) * many;
            if (many == 0 || (w.group + many) * p.heads > p.tile_counters) w.group = -1;
            return true;
        }
        before += readlane(sum, 63);
        tiles_before += readlane(tile_sum, 63);
        groups_before += readlane(group_sum, 63);
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

// PAD: heads of fewer than DP values (16-bit caches; int8 ones do not care)
// MIXED: the batch has single tokens too, which the launch's first workgroups take
template <int DT, bool I8, int DP, bool PAD, bool MIXED>
__global__ __launch_bounds__(256, 2) void attn_tile_kernel(const AttnArgs p) {
    typedef AttnTile<DP> T;
    typedef Mma<DT, 32> MMA;
    constexpr int STEPS = DP / 16, BLOCKS = DP / 32, KEYS = T::KEYS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    unsigned bid = blockIdx.x;
    if constexpr (MIXED) {
        constexpr int SINGLE_DP = DP <= 64 ? 64 : 128;
        static_assert(sizeof(SingleLds<SINGLE_DP>) <= T::LDS_BYTES, "in the same place");
        if (bid < (unsigned)p.single_groups) {
            single_tokens<DT, I8, SINGLE_DP>(p, *reinterpret_cast<SingleLds<SINGLE_DP>*>(smem));
            return;
        }
        bid -= p.single_groups;
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, h = lane >> 5;   // this lane's row of the wavefront's 32, its half of the keys

    const int head = (int)(bid % (unsigned)p.heads);
    TileWork work;
    if (!find_tile(p, (int)(bid / (unsigned)p.heads), T::ROWS, work)) return;
    const int seq = work.seq, tile = work.tiles - 1 - work.tile;   // (the rows that see most first)
    // (what is the workgroup's or the wavefront's goes into scalar registers, or branches and addresses end up in vector code)
    auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    SeqInfo si = seq_info(p, seq);
    si.q0 = scalar(si.q0);
    si.nq = scalar(si.nq);
    si.kv = scalar(si.kv);
    const int rows = si.nq * p.group, before = si.kv - si.nq;

    // ---- rows: the workgroup's, the wavefront's, this lane's, and the keys that they see, lo .. hi - 1
    // (before may be negative and a window as large as an int is: no difference is taken that could wrap)
    auto lo_of = [&](int r) { return p.window > 0 ? max(before + r / p.group, p.window - 1) - (p.window - 1) : 0; };
    auto hi_of = [&](int r) { return p.causal ? min(before + r / p.group + 1, si.kv) : si.kv; };
    const int row0 = tile * T::ROWS, row_end = min(row0 + T::ROWS, rows) - 1;
    const int wrow0 = min(row0 + wave * 32, rows - 1), wrow_end = min(row0 + wave * 32 + 31, rows - 1);
    const bool wave_on = scalar(row0 + wave * 32 < rows);
    const int my_row = min(row0 + wave * 32 + col, rows - 1);
    const bool row_on = row0 + wave * 32 + col < rows;
    const int my_lo = lo_of(my_row), my_hi = hi_of(my_row);
    const int from = lo_of(row0), to = hi_of(row_end);
    const int full_from = scalar(lo_of(row_end)), full_to = scalar(hi_of(row0));            // keys that all rows of the workgroup see
    const int w_full_from = scalar(lo_of(wrow_end)), w_full_to = scalar(hi_of(wrow0));
    // tiles of keys: the row tile's, and the piece's
    const int all0 = from / KEYS, all1 = to > from ? (to + KEYS - 1) / KEYS : all0;
    // (a sequence's pieces are enough for the row tile that sees most; others may have fewer)
    const int pieces = scalar(min(work.pieces, max((all1 - all0 + work.chunk - 1) / work.chunk, 1))), piece = scalar(work.piece);
    if (piece >= pieces) return;
    const int t0 = scalar(all0 + piece * work.chunk), t1 = scalar(piece == pieces - 1 ? all1 : t0 + work.chunk);
    // ---- this lane's query, as the fragments of the first product want it: values 16 s + 8 h .. + 7 of its row
    const int token = si.q0 + my_row / p.group, qh = head * p.group + my_row % p.group;
    i32x4 q[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int d = 16 * s + 8 * h;
        q[s] = row_on && d < p.dim ? ld16(p.Q + (token * p.ldq + (long long)qh * p.dim + d) * 2) : i32x4{0, 0, 0, 0};
    }

    // ---- copies: 16 bytes a thread, thread's chunk of rows tid / CPR + PASS i of a tile.  A wavefront's rows of a pass lie in one block
    // of sixteen keys: its place is the wavefront's, its page's number loaded a tile ahead of the copies; a thread's offset
    // from it does not change.  No load has a condition: a chunk beyond the head's values is its row's first, a block without
    // keys the last one with some.
    constexpr int CPR = I8 ? T::PITCH / 32 : T::PITCH / 16, PASS = 256 / CPR, NP = KEYS / PASS, PER = 64 / CPR;
    static_assert(PER <= 16, "a wavefront's rows in one block");
    const int chunk = tid % CPR, crow = tid / CPR, wrow = wave * PER;
    const int row_bytes = p.dim * (I8 ? 1 : 2);
    const unsigned my_off = (unsigned)((crow & 15) * row_bytes + (chunk * 16 < row_bytes ? chunk * 16 : 0));
    const int* const pages = p.table + seq * p.ld_table;
    // lane i: pass i's block of a tile
    auto block_of = [&](int kt) { return (unsigned)min(kt * KEYS + wrow + min(lane, NP - 1) * PASS, si.kv - 1) >> 4; };
    int entry = 0;
    auto load_entries = [&](int kt) { entry = pages[page_of(p, block_of(kt))]; };
    // the places of the tile whose entries were loaded last but one, in bytes from the cache's start: its keys' now, its values' a
    // tile later.  Formed in lanes, a pass each, and handed to scalar registers.
    long long at[NP], key_at[I8 ? NP : 1];   // (int8: among a head's tokens, too, for the scales)
    const unsigned head_bytes = (unsigned)(p.page_size * row_bytes);
    auto place = [&](int kt) {
        const unsigned block = block_of(kt), page = min((unsigned)max(entry, 0), (unsigned)(p.pages - 1)), in_page = block - page_of(p, block) * p.page_blocks;
        const unsigned long long of_head = page * (unsigned)p.heads + (unsigned)head;
        const unsigned long long lane_at = of_head * head_bytes + in_page * (unsigned)(16 * row_bytes);
#pragma unroll
        for (int i = 0; i < NP; ++i) at[i] = (long long)readlane(lane_at, i);
        if constexpr (I8) {
            const unsigned long long lane_key = of_head * (unsigned)p.page_size + in_page * 16;
#pragma unroll
            for (int i = 0; i < NP; ++i) key_at[i] = (long long)readlane(lane_key, i);
        }
    };
    // LDS addresses: of this lane's part of a fragment of K (step st: with 32 st exclusive-ored in; rows 32 further on have the same
    // swizzle), of V's (block b: 64 b), and of the thread's widened chunks (the second: 16)
    const unsigned k_frag = (unsigned)(col * T::PITCH + (h ^ T::k_swizzle(col)) * 16);
    const int v_row = 4 * h + ((lane & 15) >> 2), v_byte = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    const unsigned v_frag = (unsigned)(v_row * T::PITCH + (((v_byte >> 4) ^ T::v_swizzle(v_row)) * 16) + (v_byte & 15));
    const unsigned k_write = (unsigned)(crow * T::PITCH + ((2 * chunk) ^ T::k_swizzle(crow)) * 16), v_write = (unsigned)(crow * T::PITCH + ((2 * chunk) ^ T::v_swizzle(crow)) * 16);
    // (a copy that the compiler takes for new each time: what is formed from it is not kept over the loop, where registers are short)
    auto fresh = [](unsigned v) {
        asm volatile("" : "+v"(v));
        return v;
    };
    // 16-bit caches: straight into LDS, each lane's chunk from where its place wants it (a chunk of a key beyond the head's values:
    // zeros, since what is not finite would not vanish against the zeros of the queries).
    const int k_chunk = chunk ^ T::k_swizzle(crow), v_chunk = chunk ^ T::v_swizzle(crow);   // (a pass is a multiple of the swizzles' period)
    const unsigned k_off = (unsigned)((crow & 15) * row_bytes + k_chunk * 16), v_off = (unsigned)((crow & 15) * row_bytes + (v_chunk * 16 < row_bytes ? v_chunk * 16 : 0));
    const bool k_zero = k_chunk * 16 >= row_bytes;
    // int8: through registers, where they are widened
    i32x4 kreg[I8 ? NP : 1], vreg[I8 ? NP : 1];
    float kc_reg = 0.f, kt_reg = 0.f, vt_reg = 0.f;
    char* const k_lds = smem;
    char* const v_lds = smem + 2 * T::K_STAGE;
    auto to_lds = [&](const char* src, char* dst) {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src, (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
    };
    // a lane's key of the wavefront's, in the order of its passes, among a head's tokens
    auto scale_place = [&]() {
        long long key = key_at[0];
        if constexpr (I8) {
#pragma unroll
            for (int i = 1; i < NP; ++i)
                if (lane >= i * PER) key = key_at[i];
        }
        return key + (wrow & 15) + lane % PER;
    };
    auto load_k = [&](int stage) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const char* src = p.K + at[i];
            if constexpr (I8) {
                kreg[i] = ld16g(src + my_off);
            } else {
                src += k_off;
                if constexpr (PAD) src = k_zero ? g_zero_chunk : src;
                to_lds(src, k_lds + stage * T::K_STAGE + wave * 1024 + i * 4096);
            }
        }
        if constexpr (I8)
            if (lane < NP * PER) {
                const long long key = scale_place();
                kc_reg = p.ks[key];
                kt_reg = p.vs[key];
            }
    };
    auto load_v = [&](int stage) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const char* const src = p.V + at[i];
            if constexpr (I8) vreg[i] = ld16g(src + my_off);
            else to_lds(src + v_off, v_lds + stage * T::V_STAGE + wave * 1024 + i * 4096);
        }
        if constexpr (I8)
            if (lane < NP * PER) vt_reg = p.vs[scale_place()];
    };
    // what is left to do of a tile's keys or values once their loads have come back (all wavefronts', then a barrier)
    const int scale_key = wrow + lane % PER + lane / PER * PASS;
    auto finish_k = [&](int stage) {
        if constexpr (I8) {
            char* const ks = k_lds + stage * T::K_STAGE;
            const unsigned to = fresh(k_write);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *reinterpret_cast<i32x4*>(ks + i * PASS * T::PITCH + (to ^ (16u * e))) = widen8<DT>(kreg[i][2 * e], kreg[i][2 * e + 1]);
            float* const f = reinterpret_cast<float*>(ks + KEYS * T::PITCH);
            if (lane < NP * PER) {
                float log2_t, inv_t;
                value_scale<DT>(kt_reg, log2_t, inv_t);
                f[scale_key] = kc_reg * p.c;
                f[scale_key + KEYS] = log2_t;
            }
        }
    };
    int* const special = reinterpret_cast<int*>(smem + 2 * (T::K_STAGE + T::V_STAGE));   // whether values that are not finite were left out
    auto partial = [&](int kt) { return kt * KEYS < full_from || (kt + 1) * KEYS > full_to; };   // (some rows do not see all of the tile)
    auto finish_v = [&](int kt, int stage) {
        char* const vs = v_lds + stage * T::V_STAGE;
        if constexpr (I8) {
            const unsigned to = fresh(v_write);
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *reinterpret_cast<i32x4*>(vs + i * PASS * T::PITCH + (to ^ (16u * e))) = widen8<DT>(vreg[i][2 * e], vreg[i][2 * e + 1]);
            if (lane < NP * PER) {
                float log2_t, inv_t;
                value_scale<DT>(vt_reg, log2_t, inv_t);
                // (a scale that is NaN makes its key's weight NaN where it is seen, and must not reach other rows as 0 times NaN)
                reinterpret_cast<float*>(vs + KEYS * T::PITCH)[scale_key] = inv_t == inv_t ? inv_t : 0.f;
            }
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            // a key that some rows of the tile do not see must not reach them as 0 times infinity: zeros behind the last key, and
            // what is not finite stays out of the product and is added at the end, where it is seen.  (The thread's own chunks.)
            if (partial(kt)) {
                bool bad = false;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    i32x4* const here = reinterpret_cast<i32x4*>(vs + i * 4096 + tid * 16);
                    i32x4 v = *here;
                    if (kt * KEYS + crow + i * PASS >= si.kv) v = i32x4{0, 0, 0, 0};
                    if (any_not_finite<DT>(v)) {
                        bad = true;
#pragma unroll
                        for (int d = 0; d < 4; ++d) v[d] = only_finite<DT>(v[d]);
                    }
                    *here = v;
                }
                if (bad) *special = 1;
            }
        }
    };

    typename MMA::Acc o[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
    float m = ATTN_NONE, l = 0.f;   // (m: as a power of two, ATTN_LIFT below the running maximum)

    // ---- the pieces of a tile's way.  S^T, two blocks of 32 keys; key of register r in block kb: k0 + 32 kb + 8 (r / 4) + 4 h + r % 4
    typedef typename MMA::Acc Scores[2];
    auto scores = [&](int stage, Scores& s) {
        const char* const ks = k_lds + stage * T::K_STAGE;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
            for (int st = 0; st < STEPS; ++st) s[kb] = MMA::run(*reinterpret_cast<const i32x4*>(ks + kb * 32 * T::PITCH + (k_frag ^ (32u * st))), q[st], s[kb]);
        }
    };
    auto scale_scores = [&](int stage, Scores& s) {
        if constexpr (I8) {
            const float* const fs = reinterpret_cast<const float*>(k_lds + stage * T::K_STAGE + KEYS * T::PITCH) + 4 * h;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const f32x4 kc = *reinterpret_cast<const f32x4*>(fs + 32 * kb + 8 * r4);
                    const f32x4 lt = *reinterpret_cast<const f32x4*>(fs + KEYS + 32 * kb + 8 * r4);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[kb][4 * r4 + r] = __builtin_fmaf(s[kb][4 * r4 + r], kc[r], lt[r]);
                    if (r4 & 1) __builtin_amdgcn_sched_barrier(0);   // (all of them read at once have no room)
                }
        }
    };
    auto mask_scores = [&](int kt, Scores& s) {
        const int k0 = kt * KEYS;
        if (k0 < w_full_from || k0 + KEYS > w_full_to) {
            asm volatile("");   // (a branch: selects in its place would cost every tile 128 instructions)
            const int first = k0 + 4 * h - my_lo;
            const unsigned seen = (unsigned)max(my_hi - my_lo, 0);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[kb][r] = (unsigned)(first + 32 * kb + 8 * (r >> 2) + (r & 3)) < seen ? s[kb][r] : -__builtin_huge_valf();
        }
    };
    auto top_of = [&](const Scores& s) {
        float top = s[0][0];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, s[kb][r]);
        return I8 ? top : top * p.c;
    };
    auto move_maximum = [&](float top) {
        if (__any(top - m > ATTN_SLACK + ATTN_LIFT<DT>)) {
            top = __builtin_fmaxf(__builtin_fmaxf(top, swap_halves(top)) - ATTN_LIFT<DT>, m);
            const float f = __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= f;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= f;
        }
    };
    // a fragment of V^T of the second product: sixteen keys, 32 kb + 16 half + {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3}, block b of its values.
    // (Transposing reads: sixteen lanes bring four keys' rows of sixteen values and get a column each.)
    auto v_fragment = [&](int stage, unsigned from, int kb, int half, int b) {
        i32x4 a;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const i32x2 v = read_transposed(v_lds + stage * T::V_STAGE + (32 * kb + 16 * half + 8 * e) * T::PITCH + (from ^ (64u * b)));
            a[2 * e] = v[0];
            a[2 * e + 1] = v[1];
        }
        return a;
    };

    // One tile: its scores (now) have been formed, masked and seen by the maximum; those of the next are formed beside its weights,
    // so that a wavefront has work for the matrix unit and for the vector unit at the same time.  The order of the instructions is
    // the one written here (sched_barrier): AHEAD fragments are on their way from LDS before the first is used, and behind each
    // matrix instruction (32 cycles) come the next read and about as many cycles of weights.  Left to itself the compiler reads
    // each fragment into the same registers and waits for it.
    auto step = [&](int kt, int stage, Scores& now, Scores& next) {
        constexpr int NS = 2 * STEPS, NV = 4 * BLOCKS, AHEAD = (I8 ? 4 : 6) < NS ? (I8 ? 4 : 6) : NS, V_AHEAD = I8 ? 3 : 4;   // (int8: no registers for more)
        constexpr int FIRST = 20;   // weights formed beside the scores: at least the first block's, 16 of 32
        const float* const inv_of = reinterpret_cast<const float*>(v_lds + stage * T::V_STAGE + KEYS * T::PITCH) + 4 * h;
        int w[4][4];
        f32x4 inv;
        float sum = 0.f;
        auto weight = [&](int e) {
            const int kb = e >> 4, r = e & 15;
            if constexpr (I8) {
                if ((e & 3) == 0) inv = *reinterpret_cast<const f32x4*>(inv_of + 32 * kb + 8 * (r >> 2));
                now[kb][r] = __builtin_amdgcn_exp2f(now[kb][r] - m);
                sum = __builtin_fmaf(now[kb][r], inv[e & 3], sum);
            } else {
                now[kb][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(now[kb][r], p.c, -m));
                sum += now[kb][r];
            }
            if (e & 1) w[e >> 3][(e & 7) >> 1] = pack_out16<DT>(now[kb][r - 1], now[kb][r]);
        };
        {
            i32x4 a[AHEAD];
            const unsigned from = fresh(k_frag);
            auto read = [&](int i) {
                a[i % AHEAD] = *reinterpret_cast<const i32x4*>(k_lds + (stage ^ 1) * T::K_STAGE + (i / STEPS) * 32 * T::PITCH + (from ^ (32u * (i % STEPS))));
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) next[kb][r] = 0.f;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                next[i / STEPS] = MMA::run(a[i % AHEAD], q[i % STEPS], next[i / STEPS]);
                if (i + AHEAD < NS) read(i + AHEAD);
#pragma unroll
                for (int e = i * FIRST / NS; e < (i + 1) * FIRST / NS; ++e) {
                    weight(e);
                    if (e & 1) asm volatile("" : "+v"(w[e >> 3][(e & 7) >> 1]), "+v"(sum));   // (here, not where they are used)
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        i32x4 a[V_AHEAD];
        const unsigned from = fresh(v_frag);
        auto read = [&](int i) { a[i % V_AHEAD] = v_fragment(stage, from, i / (2 * BLOCKS), i / BLOCKS % 2, i % BLOCKS); };
#pragma unroll
        for (int i = 0; i < V_AHEAD; ++i) read(i);
        if constexpr (!I8) mask_scores(kt + 1, next);
        __builtin_amdgcn_sched_barrier(0);
        float top = next[0][0];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            o[i % BLOCKS] = MMA::run(a[i % V_AHEAD], i32x4{w[i / BLOCKS][0], w[i / BLOCKS][1], w[i / BLOCKS][2], w[i / BLOCKS][3]}, o[i % BLOCKS]);
            if (i + V_AHEAD < NV) read(i + V_AHEAD);
            if (i < NV / 2) {
#pragma unroll
                for (int e = FIRST + i * (32 - FIRST) / (NV / 2); e < FIRST + (i + 1) * (32 - FIRST) / (NV / 2); ++e) weight(e);
            } else if constexpr (!I8) {
                const int j = i - NV / 2;
#pragma unroll
                for (int e = j * 32 / (NV / 2); e < (j + 1) * 32 / (NV / 2); ++e) top = __builtin_fmaxf(top, next[e >> 4][e & 15]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
        if constexpr (I8) {
            scale_scores(stage ^ 1, next);
            mask_scores(kt + 1, next);
            top = top_of(next);
        } else {
            top *= p.c;
        }
        move_maximum(top);
    };

    if (tid == 0) *special = 0;
    __syncthreads();
    Scores s0, s1;
    if (t1 > t0) {
        load_entries(t0);
        place(t0);
        load_entries(t0 + 1);
        load_k(0);
        load_v(0);
        finish_k(0);
        finish_v(t0, 0);
        place(t0 + 1);
        load_entries(t0 + 2);
        load_k(1);
        finish_k(1);
        if constexpr (!I8) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        scores(0, s0);
        scale_scores(0, s0);
        mask_scores(t0, s0);
        move_maximum(top_of(s0));
        __syncthreads();   // (the first keys' place is the third's)
    }
    // tile kt + 2's keys and kt + 1's values come in while kt + 1's keys and kt's values are used (beyond the last tile: whatever
    // block_of gives, unused)
    auto turn = [&](int kt, auto stage_c, Scores& now, Scores& next) {
        constexpr int stage = decltype(stage_c)::value;
        load_v(stage ^ 1);
        place(kt + 2);
        load_entries(kt + 3);
        load_k(stage);
        if (wave_on) step(kt, stage, now, next);
        finish_k(stage);
        finish_v(kt + 1, stage ^ 1);
        __syncthreads();
    };
    for (int kt = t0; kt < t1; kt += 2) {
        turn(kt, std::integral_constant<int, 0>(), s0, s1);
        if (kt + 1 < t1) turn(kt + 1, std::integral_constant<int, 1>(), s1, s0);
    }
    if constexpr (!I8) {
        if (__builtin_expect(*special != 0, 0)) {
            for (int kt = t0; kt < t1; ++kt)
                if (partial(kt)) add_not_finite<DT, DP>(p, o, m, kt * KEYS, si, pages, head, token, qh, my_lo, row_on ? my_hi : 0, h);
        }
    }

    l += swap_halves(l);
    if (pieces > 1) {
        // ---- whoever is the last of a row tile's pieces puts their sums together, in the order of the pieces.  (They are written through
        // to where every die reads them, as they lie in the registers, and waited for, before the counter moves.  A second kernel
        // for it took 8 to 10 us, and 6 where no row tile was in pieces.)
        constexpr int PAIRS = 8 * BLOCKS;
        const long long first_place = (long long)(work.slot - piece) * p.heads + head;
        auto place_of = [&](int i) { return ((first_place + (long long)i * p.heads) * 4 + wave) * 64 + lane; };   // (in twos of floats; of sums, PAIRS times that)
        auto sums_of = [&](int i) { return p.tile_o + ((place_of(i) - lane) * PAIRS + lane) * 2; };
        auto fetch = [&](int i, float2& ml, float2 (&x)[PAIRS]) {
            const float* const from = sums_of(i);
            ml = get_shared(p.tile_ml + place_of(i) * 2);
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) x[k] = get_shared(from + k * 128);
        };
        auto add = [&](const float2& ml, const float2 (&x)[PAIRS]) {
            const float top = __builtin_fmaxf(m, ml.x), f0 = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(ml.x - top);
            m = top;
            l = __builtin_fmaf(f, ml.y, l * f0);
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) {
                o[k / 8][2 * (k % 8)] = __builtin_fmaf(f, x[k].x, o[k / 8][2 * (k % 8)] * f0);
                o[k / 8][2 * (k % 8) + 1] = __builtin_fmaf(f, x[k].y, o[k / 8][2 * (k % 8) + 1] * f0);
            }
        };
        // who meets here: `count` pieces from `first` on, every step-th; the sums so far are those of piece `mine`
        unsigned* const counters = p.counters + (MIXED ? p.single_groups : 0);
        unsigned* counter = counters + work.index * p.heads + head;
        int mine = piece, first = 0, step = 1, count = pieces;
        const bool grouped = scalar(work.group) >= 0 && pieces > TILE_GROUP;
        if (grouped) {
            first = piece / TILE_GROUP * TILE_GROUP;
            count = min(TILE_GROUP, pieces - first);
            counter = counters + (work.group + piece / TILE_GROUP) * p.heads + head;
        }
        for (bool last = !grouped;; last = true) {
            if (wave_on) {
                float* const to = sums_of(mine);
#pragma unroll
                for (int k = 0; k < PAIRS; ++k) put_shared(to + k * 128, o[k / 8][2 * (k % 8)], o[k / 8][2 * (k % 8) + 1]);
                put_shared(p.tile_ml + place_of(mine) * 2, m, l);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (tid == 0) *special = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)count - 1;
            __syncthreads();
            if (*special == 0) return;
            if (tid == 0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // (zero again when the launch ends)
            if (wave_on) {
                m = ATTN_NONE;
                l = 0.f;
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
                float2 ml0, ml1, x0[PAIRS], x1[PAIRS];   // two pieces on their way
                fetch(first, ml0, x0);
                for (int i = 0; i < count; i += 2) {
                    fetch(first + min(i + 1, count - 1) * step, ml1, x1);
                    add(ml0, x0);
                    if (i + 1 < count) {
                        fetch(first + min(i + 2, count - 1) * step, ml0, x0);
                        add(ml1, x1);
                    }
                }
            }
            if (last) break;
            mine = first;
            first = 0;
            step = TILE_GROUP;
            count = (pieces + TILE_GROUP - 1) / TILE_GROUP;
            counter = counters + work.index * p.heads + head;
        }
    }
    // ---- out: this lane's row, values 32 b + 8 (r / 4) + 4 h + r % 4
    if (!row_on) return;
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
}

}  // namespace abft
