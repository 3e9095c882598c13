// Attention over a paged cache: the checks and the division of the work (see include/abft.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "attention_single.h"
#include "attention_tile.h"

namespace abft {
hipError_t launch_attention_f16(const AttnArgs& a, bool i8, hipStream_t stream);
hipError_t launch_attention_bf16(const AttnArgs& a, bool i8, hipStream_t stream);
}  // namespace abft

using namespace abft;

namespace {

long long cdiv(long long a, long long b) { return (a + b - 1) / b; }
size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int MAX_KV = 1 << 24;
constexpr int COMPUTE_UNITS = 256, COUNTERS = COMPUTE_UNITS * 4;
// Workgroups of single tokens in a launch that has chunks too: beside each of them a compute unit has room for one of a chunk, which
// multiplies while this one waits for memory.  (Batch of 3 chunks and 5 single tokens over 8000, 28 heads, fp16 cache: 100 us in two
// launches, 75 in one; 48 single tokens and 512 new ones, 32 heads, int8: 123 / 117, and 127 with twice as many.)
constexpr int MIXED_GROUPS = COMPUTE_UNITS;

constexpr long long MAX_BLOCKS = (1 << 24) - 1;   // of 256 threads: a launch of 2^32 threads or more wraps, without an error

// How a call's work is divided, from what the host knows of it.
struct Division {
    int single, single_groups;
    int tiles, tile_split;      // tiles: an upper bound of the row tiles, 0: none can be there; up to how many of them their keys may be divided
    size_t off_single_o, off_single_ml, off_tile_o, off_tile_ml, bytes;
    long long blocks(int heads) const { return single_groups + ((long long)tiles + (tile_split ? tile_more_pieces(heads) : 0)) * heads; }
};
Division divide(const abft_kv_cache_t* c, int n, int total_q, int max_q, int max_kv, int q_heads) {
    Division d;
    std::memset(&d, 0, sizeof d);
    const int group = q_heads / c->heads;
    // sequences of one token have a kernel; where all have the same number of tokens, and more than one, there are none
    d.single = group <= ATTN_GROUP_MAX && (max_q == 1 || (long long)n * max_q != total_q);
    const bool tiled = !d.single || max_q > 1;
    if (d.single) {
        // Workgroups: one a unit up to 128, and more, up to one a compute unit, for four units each; two a compute unit with 256 heads of
        // sequences, and as many as there are heads in any case, so that fewer of them are shared.  (One token of 2048, int8, 128
        // wide: 64 / 128 workgroups 11.3 / 10.7 us; of 4096 128 / 256 11.7 / 12.5; of 32768 256 / 512 21.1 / 26.4; 16 of 8192 57.6 / 59.7; 64
        // of 4096 120.6 / 105.2 and with three a compute unit 117, where shares end inside more heads; 64 of 300 16.7 / 13.0 / 20.3.)
        const long long heads = (long long)n * c->heads, units = cdiv(max_kv, SINGLE_UNIT) * heads;
        const long long most = tiled ? MIXED_GROUPS : heads < COMPUTE_UNITS ? COMPUTE_UNITS : 2 * COMPUTE_UNITS;
        d.single_groups = (int)std::min(most, std::max({heads, std::min(units, 128ll), cdiv(units, 4)}));
    }
    if (tiled) {
        // Row tiles: at most one more for each sequence that has any than the rows fill (single tokens have none where they have a kernel), at least
        // what the tokens fill that are not such.
        const long long rows = (long long)total_q * group, at_most = d.single ? std::min(n, total_q / 2) : n, others = d.single ? std::max(total_q - n, 0) : total_q;
        d.tiles = (int)std::min(at_most + rows / AttnTile<128>::ROWS, MAX_BLOCKS + 1);
        const long long least = d.single || (long long)n * max_q != total_q ? cdiv(others * group, AttnTile<128>::ROWS) : n * cdiv((long long)max_q * group, AttnTile<128>::ROWS);
        // Their keys may be divided as long as there is a counter for each: beyond that two of them for each workgroup that the chip holds fill
        // it.  How many there are, and so whether, is for the device to see.  (us, 8 heads of 128 read by 4 queries each, int8, as if every
        // sequence had row tiles of its own / so: 127 single tokens and 512 of 32768 895 / 419, 129 and 16 of 32768 926 / 96, 63 and 1024 of
        // 8192 250 / 220, 100 and 3 x 300 of 5000 178 / 155; 150 x 2 of 2000, undivided both ways, level.)
        const int counted = (COUNTERS - d.single_groups) / c->heads;
        if (least <= counted && max_kv > TILE_MIN_CHUNK * ATTN_BLOCK_KEYS) d.tile_split = std::min(d.tiles, counted);
    }
    size_t at = 0;
    auto take = [&](size_t floats) {
        const size_t here = at;
        at = align_up(at + floats * 4, 256);
        return here;
    };
    const size_t places = (size_t)2 * d.single_groups * group, rows = d.tile_split ? (size_t)(d.tile_split + tile_more_pieces(c->heads)) * c->heads * AttnTile<128>::ROWS : 0;
    if (places + rows == 0) return d;
    // (the counters first, always of one size: calls of different shapes share a workspace)
    take(COUNTERS);
    d.off_single_o = take(places * c->head_dim);
    d.off_single_ml = take(places * 2);
    // (a row's sums as they lie in two lanes' registers)
    d.off_tile_o = take(rows * align_up(c->head_dim, 32));
    d.off_tile_ml = take(rows * 4);
    d.bytes = at;
    return d;
}

int validate(const abft_kv_cache_t* c, int n, int total_q, int max_q, int max_kv, int q_heads, int dtype) {
    const int rc = kv_validate(c, dtype);
    if (rc != ABFT_OK) return rc;
    if (n <= 0 || total_q < 0 || max_q < 0 || max_q > total_q || max_kv < 0 || max_kv > MAX_KV) return ABFT_E_SHAPE;
    if (q_heads <= 0 || q_heads % c->heads != 0) return ABFT_E_SHAPE;
    if ((long long)total_q * q_heads > 0x7fffffffll || (long long)n * q_heads > 0x7fffffffll / (max_kv / SINGLE_UNIT + 1)) return ABFT_E_SHAPE;
    return divide(c, n, total_q, max_q, max_kv, q_heads).blocks(c->heads) > MAX_BLOCKS ? ABFT_E_SHAPE : ABFT_OK;
}

}  // namespace

extern "C" {

size_t abft_attention_workspace_bytes(const abft_kv_cache_t* cache, int n_seqs, int total_q, int max_q, int max_kv, int q_heads, int dtype) {
    if (validate(cache, n_seqs, total_q, max_q, max_kv, q_heads, dtype) != ABFT_OK || total_q == 0) return 0;
    return divide(cache, n_seqs, total_q, max_q, max_kv, q_heads).bytes;
}

int abft_attention(const abft_kv_cache_t* cache, int n_seqs, const int32_t* q_start, const int32_t* kv_len, const int32_t* block_table,
                   int64_t ld_table, int total_q, int max_q, int max_kv, const void* Q, int64_t ldq, int q_heads, int dtype, float scale,
                   int causal, int window, void* O, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = validate(cache, n_seqs, total_q, max_q, max_kv, q_heads, dtype);
    if (rc != ABFT_OK) return rc;
    if (!(scale > 0.f) || !std::isfinite(scale) || window < 0) return ABFT_E_VALUE;
    if (total_q == 0 || max_q == 0) return ABFT_OK;
    if (!q_start || !kv_len || !block_table || !Q || !O) return ABFT_E_NULL;
    const long long row = (long long)q_heads * cache->head_dim;
    if (ldq < row || ldo < row || ld_table < 0 || ld_table * cache->page_size < max_kv) return ABFT_E_LD;
    if (ldq % 8 != 0 || ldo % 4 != 0 || (reinterpret_cast<uintptr_t>(Q) & 15u) || (reinterpret_cast<uintptr_t>(O) & 7u)) return ABFT_E_LD;
    const Division d = divide(cache, n_seqs, total_q, max_q, max_kv, q_heads);
    char* const ws = reinterpret_cast<char*>(workspace);
    if (d.bytes > 0 && (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || workspace_bytes < d.bytes)) return ABFT_E_WORKSPACE;
    AttnArgs a;
    std::memset(&a, 0, sizeof a);
    a.K = reinterpret_cast<const char*>(cache->k); a.V = reinterpret_cast<const char*>(cache->v);
    a.ks = cache->k_scale; a.vs = cache->v_scale;
    a.pages = cache->pages; a.page_size = cache->page_size; a.heads = cache->heads; a.dim = cache->head_dim;
    a.page_blocks = (unsigned)cache->page_size / 16;
    a.page_magic = (unsigned)cdiv(1ll << 31, a.page_blocks);
    a.q_start = q_start; a.kv_len = kv_len; a.table = block_table; a.ld_table = ld_table;
    a.n_seqs = n_seqs; a.total_q = total_q; a.max_q = max_q; a.max_kv = max_kv;
    a.Q = reinterpret_cast<const char*>(Q); a.O = reinterpret_cast<char*>(O); a.ldq = ldq; a.ldo = ldo;
    a.group = q_heads / cache->heads;
    a.c = scale * 1.44269504f;
    a.causal = causal != 0; a.window = window;
    a.single = d.single;
    a.single_groups = d.single_groups; a.tiles = d.tiles; a.tile_split = d.tile_split; a.tile_counters = COUNTERS - d.single_groups;
    a.counters = reinterpret_cast<unsigned*>(ws);
    a.single_o = reinterpret_cast<float*>(ws + d.off_single_o); a.single_ml = reinterpret_cast<float*>(ws + d.off_single_ml);
    a.tile_o = reinterpret_cast<float*>(ws + d.off_tile_o); a.tile_ml = reinterpret_cast<float*>(ws + d.off_tile_ml);
    const hipError_t e = (dtype == ABFT_F16 ? launch_attention_f16 : launch_attention_bf16)(a, cache->dtype == ABFT_I8, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? ABFT_OK : ABFT_E_HIP;
}

}  // extern "C"
