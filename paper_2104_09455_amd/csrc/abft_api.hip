// C-ABI entry points of the ABFT GEMM library (see include/abft.h) and the small
// kernels around the GEMM: weight checksum (offline, paper Sec. 2.5), activation
// checksum fused with the checksum dot product (Sec. 2.4 steps 1-2) and the final
// reduction + comparison (Sec. 2.4 steps 3-4, Sec. 2.5 step 5).
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>
#include <cstdio>
#include <cstdlib>
#include <algorithm>
#include <cstring>
#include <atomic>
#include <mutex>
#include <new>
#include <vector>

#include "../../include/abft.h"
#include "gemm_configs.h"
#include "mlp_chain.h"
#include "gemm_group.h"
#include "quantize.h"

using namespace abft;

namespace {

// ------------------------------------------------------------------------- //
// constants of the method as built here
// ------------------------------------------------------------------------- //
// Tolerance: tau = C_TOL * (2^-24 * sqrt(K) + u_chi) * ||C_S||_F + C_BIAS * 2^-24 * K * ||C_S||_1
// (the last term for the global scheme only).  2^-24 is the unit
// roundoff of the fp32 accumulators; an accumulator that takes K products carries a
// random-walk error ~ 2^-24 sqrt(K) |C_ij| / 2.4 and the errors of the entries add in
// quadrature under the output summation.  The ||.||_1 term covers a small coherent bias of the
// matrix unit's accumulation (measured: up to 2e-4 * 2^-24 * K per entry, same sign for all
// entries of a tile with same-sign operands).  Under ABFT_THREAD (fp16, bf16) every checksum
// accumulator goes through the MFMAs of a product accumulator in their order, so both sides carry the
// same errors, bias and all, and differ only where a tile is the sum of several wavefronts'
// partial tiles, by the roundings of that addition.  (ABFT_REPLICA's blocks take the products of
// several fragments, twice to four times as many at as many times the magnitude, and neither walk nor
// bias cancels: 0.43 tau on 2048 x 2048 x 65536 operands of one sign.)  u_chi (thread-level schemes) is
// the error of a tile checksum cut into two fp16 / three bf16 pieces, which no scheme here forms: headroom.
constexpr double C_TOL = 8.0;
constexpr double C_BIAS = 1.0e-3;
constexpr double U_ACC = 5.9604644775390625e-08;  // 2^-24
constexpr double U_CHI_F16 = 2.384185791015625e-07;  // 2^-22
constexpr double U_CHI_BF16 = 1.1920928955078125e-07;  // 2^-23
// ABFT_THREAD_HALF / ABFT_TWOSIDED add checksums in the operand type: every such add rounds to
// u_half = 2^-11 (fp16) / 2^-8 (bf16).  The errors of the B-side sums enter the comparison
// weighted with the column sums of the A tile, which are at most sqrt(tile rows) times the
// columns' norms (and the other way round for the A-side sums of the two-sided scheme):
//   tau += C_HALF * u_half * sqrt(n_B * tile_m + n_A * tile_n) * ||C_S||_F
// with n_B / n_A the number of adds per checksum element (fragments per wavefront tile - 1).
constexpr double C_HALF = 4.0;
constexpr double U_HALF_F16 = 4.8828125e-04, U_HALF_BF16 = 3.90625e-03;


// MI355X spec-sheet peaks (dense) and HBM3E bandwidth
constexpr double PEAK_F16 = 2516.6e12, PEAK_I8 = 5033.2e12, HBM_BW = 8.0e12;
double g_cmr_override[3] = {0.0, 0.0, 0.0};

// optional events recorded around the GEMM kernel launch (abft_set_kernel_events)
thread_local hipEvent_t g_ev_start = nullptr, g_ev_stop = nullptr;

// Scratch of abft_gemm_static: one array per GPU the library runs on, held until the process
// ends.  The name below is only a host-side stand-in for the array; its device address is asked
// for once per device (scratch_of_current_device) and that pointer is what kernels are given.
constexpr size_t STATIC_SCRATCH_BYTES = 8u << 20;
__device__ __align__(256) unsigned char g_static_scratch[STATIC_SCRATCH_BYTES];
// product launches so far that took their activation checksums from the layer before (diagnostics)
std::atomic<long long> g_handover_launches{0};
// chains of layers so far that went out as one launch (diagnostics)
std::atomic<long long> g_chain_launches{0};
constexpr int MAX_DEVICES = 64;
void* g_scratch_ptr[MAX_DEVICES] = {nullptr};
std::mutex g_scratch_mutex;

// device address of this GPU's copy of the scratch array (null: the runtime refused)
void* scratch_of_current_device() {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return nullptr;
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void* ptr = nullptr;
        if (hipGetSymbolAddress(&ptr, HIP_SYMBOL(g_static_scratch)) != hipSuccess) return nullptr;
        g_scratch_ptr[dev] = ptr;
    }
    return g_scratch_ptr[dev];
}

inline int esize(int dt) { return dt == ABFT_I8 ? 1 : 2; }
inline int csize(int dt) { return dt == ABFT_I8 ? 4 : 2; }
inline bool valid_dtype(int dt) { return dt == ABFT_F16 || dt == ABFT_BF16 || dt == ABFT_I8; }
inline long long cdiv(long long a, long long b) { return (a + b - 1) / b; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

// ------------------------------------------------------------------------- //
// tile configuration choice (host logic)
// ------------------------------------------------------------------------- //
// mode: the scheme the product will run with; force >= 0 pins a configuration (tuning aid,
// environment variable ABFT_FORCE_CFG).  conv: the product of a convolution read as an implicit
// matrix (unprotected products only: what is reported of the other schemes' tiles has no such word).
int pick_cfg(int M, int N, int K, int dt, bool aligned16, int mode, bool conv = false) {
    // (every wavefront-level scheme is checked per wavefront tile: the same tiles)
    if (mode == ABFT_REPLICA || mode == ABFT_THREAD_HALF || mode == ABFT_TWOSIDED) mode = ABFT_THREAD;
    if (mode == ABFT_GLOBAL_WEIGHTED) mode = ABFT_GLOBAL;
    static const int force = [] {
        const char* e = std::getenv("ABFT_FORCE_CFG");
        return e ? std::atoi(e) : -1;
    }();
    // the direct-to-LDS kernel needs whole k tiles of 128 bytes; the streaming kernel takes any whole
    // number of 16-byte chunks (a variant of it fills a short last tile up with zeros)
    const bool fast_ok = aligned16 && ((long long)K * esize(dt)) % 128 == 0;
    const bool force_fits = force >= 0 && force < CFG_COUNT &&
                            (fast_ok || !cfg_info_host(force).fast || (aligned16 && cfg_is_stream(force)));
    // (the 256 x 256 tile carries no wavefront-level scheme: a forced choice of it does not apply to those)
    // the row-streaming kernel: 16-bit types, no scheme that compares across wavefronts, the weights within
    // LDS (one column block of 64 and up to twenty k tiles, or a single k tile and up to twenty column blocks)
    const bool rows_fit = fast_ok && dt != ABFT_I8 && mode != ABFT_GLOBAL &&
                          (N <= 64 || (long long)K * esize(dt) == 128) && cdiv(N, 64) * cdiv((long long)K * esize(dt), 128) <= 20;
    if (force == CFG_R64 && rows_fit) return force;
    if (force_fits && force != CFG_R64 && !((force == CFG_F256W || force == CFG_F256N || force == CFG_F256S || force == CFG_F128E) && mode == ABFT_THREAD)) return force;
    const long long nkt_gen = cdiv((long long)K * esize(dt), 128);
    auto tiles = [&](int id) {
        CfgInfo ci = cfg_info_host(id);
        return cdiv(M, ci.bm) * cdiv(N, ci.bn);
    };
    // (few rows, a long k loop, at most one 64 x 64 tile per compute unit: the groups that share the tile's k
    // loop outweigh its rows of zeros: 16 x 4096 x 4095 27 against 45 us, 16 x 16384 x 2049 18 / 26, 16384 x 4096 K
    // x N 35 / 53; near level at half to a quarter of that k loop, 16 x 512 x 1023 9.9 / 10.7; 16 x 512 x 300
    // 6.4 / 5.5.  A second round of workgroups that fill a compute unit each costs more than it gives: 1 x 32000
    // x 4095 71 / 59, 8 x 128000 x 2049 153 / 121)
    if (M <= 16 && !aligned16) return nkt_gen >= 32 && tiles(CFG_G64K) <= 256 ? CFG_G64K : CFG_G16;
    if (aligned16) {
        // fill the 256 compute units before growing the tile
        // (wavefront-level: the 128 x 128 tile of wide wavefront tiles; the 256 x 256 one would spill)
        // (a single k tile: the 128 x 128 tile, of which several fit a compute unit at once)
        const long long nkt_all = cdiv((long long)K * esize(dt), 128);
        // The 256 x 256 tile runs one workgroup per compute unit, in rounds of 256: it is taken when
        // the rounds are at least 70 % full (288 tiles would leave the second round of 6000 x 3072 x
        // 768 almost empty: 58 us against 48 us on 128 x 128 tiles), from 192 tiles on when the k loop
        // is eight tiles long or more (50176 x 256 x 512, 12544 x 1024 x 512: 196 tiles each), else from 224.
        const long long t256 = tiles(CFG_F256W);
        const bool rounds_full = t256 * 10 >= cdiv(t256, 256) * 256 * 7;
        if (fast_ok && N > 128 && nkt_all > 1 && rounds_full && (t256 >= 224 || (t256 >= 192 && nkt_all >= 8)))
            return mode == ABFT_THREAD ? CFG_F128T : CFG_F256W;
        // About one 256 x 128 tile per compute unit (one round, more than half full) with a k loop
        // of six tiles or more: that tile keeps three stages in LDS and asks the vector memory
        // path for three quarters of what 128 x 128 tiles ask per MFMA (2048 x 4096 x 4096: 70 us
        // against 77 us; 1536 x 4096 x 4096: 59 against 65; 2048 x 3072 x 4096: 56 against 63;
        // 144 tiles, 1152 x 4096 x 4096: 52 against 57; 128 tiles, 1024 x 4096 x 4096: 53 against 48;
        // k loop of four tiles: level).  Its wavefront tiles carry no wavefront-level scheme.
        const long long t256n = tiles(CFG_F256N);
        if (fast_ok && mode != ABFT_THREAD && N >= 128 && nkt_all >= 6 && t256n >= 144 && t256n <= 256) return CFG_F256N;
        // Very many rows whose weights fit in LDS: the row-streaming kernel, from two 32-row tiles per wavefront
        // of the chip on (below, the loads into an empty pipeline lose: 50176 x 64 x 256 18.6 / 16.9 us thread-level
        // / unprotected against 18 / 13.5 on 128 x 128 tiles, 70000 rows 19 / 13 against 18 / 15).
        // Unprotected: every convolution, whose neighbouring rows share their input (against the better of 128
        // x 128 and 256 x 64 tiles: 3 x 3 64 -> 64 on 131712 rows 27 / 30, on 200704 bf16 35 / 39; 128 -> 64 44 /
        // 47; stem on 802816 rows 71 / 90; 1 x 1, stride 2, 64 -> 64 16 / 17); products of two to four k tiles
        // (180000 x 64 x 128 18 / 19, 262144 x 16 x 192 28 / 31; five k tiles level, 180000 x 16 x 320 32 / 31, twenty
        // 82 / 75) and of one with more than 128 columns (262144 x 192 x 64 35 / 43, 131072 x 1280 x 64 90 / 112; 128
        // columns 17 / 16, 64 columns 12 / 11).
        // Wavefront-level: whatever fits (thread-level 131072 x 64 x 1280 85 / 87, 200000 x 64 x 256 35 / 41; 3 x 3
        // 64 -> 64 on 200704 rows 39 / 56) but for one k tile with 65 to 128 columns (400000 x 128 x 64 50 / 47) and
        // more than eighteen k tiles with at most 32 columns (131072 x 32 x 1280 81 / 77).
        const bool rows_pay = mode == ABFT_THREAD ? (nkt_all == 1 ? N <= 64 || N > 128 : nkt_all <= 18 || N > 32)
                                                  : conv || (nkt_all == 1 ? N > 128 : nkt_all <= 4);
        if (rows_fit && M >= 131072 && rows_pay) return CFG_R64;
        // Outputs of at most 64 columns and very many rows (ResNet-50's first stage at batch 64: 200704
        // rows) otherwise: 256 x 64 tiles with three stages.  3 x 3 convolution 64 -> 64: 52 us against 63 on 128 x 128
        // tiles, global; K = 64: 17 against 23 us global, level unprotected; k loops of two to five
        // tiles: slower unprotected (33 against 30 us at K = 256).
        if (fast_ok && mode != ABFT_THREAD && N <= 64 && N > 32 && M >= 65536 &&
            (nkt_all >= 6 || (nkt_all == 1 && mode == ABFT_GLOBAL)))
            return CFG_F256S;
        const bool fills128 = tiles(CFG_F128) >= 128;
        if (fast_ok && fills128 && N < 128) return CFG_F128T;  // narrow outputs: every wavefront spans all columns
        // Few tiles: the time is the latency of a workgroup's k loop and the rate at which one
        // compute unit can stream its operands, so the streaming configurations take over (no
        // barriers in the k loop, four wavefronts sharing the k tiles): the smallest tile that
        // still fits the chip in one round of workgroups, 64 x 64 for up to two rounds (that one
        // only with a k loop of at least one tile per wavefront, sixteen tiles for a second round:
        // the idle wavefronts of a short loop cost more than the barriers they save; 3000 x 384 x
        // 384 takes 9.9 us on 282 such tiles, 8.2 us on 64 x 128 tiles; thread-level, fp16, 2048 x 1024 x 512 12.3
        // against 10.5, K = 768 14.7 / 13.5, K = 1024 16.7 / 16.3, K = 2048 23.3 / 25.6).  Wavefront-level bf16 and
        // int8 from eight: their checksums cost vector work, more of it on the 64 x 128 tile's wide wavefront
        // tiles (K = 512 bf16, half-precision sums, 11.9 / 13.3, exact 12.8 / 10.8; int8 K = 1024 14.6 / 17.5).
        // Fewer than a quarter of the compute units in use and a long k loop: eight wavefronts per tile, two per
        // SIMD, so that one's copies and address work run under the other's products (3 x 3 convolutions at batch
        // 1: 512 -> 512 on 49 rows, 32 tiles of 72 k tiles, 10.3 against 11.7 us thread-level, 256 -> 256 on 196
        // rows 7.6 / 8.2; 16 x 512 x 8192 10.9 / 11.9; global 16 x 2016 x 8192 13.8 / 16.9).  More tiles: level for
        // products (256 x 512 x 2048 5.9 / 5.9, 16 x 4096 x 4096 8.9 / 8.7).  Unprotected there is little to run
        // under, and four wavefronts with twice the stages each stream long loops better: eight up to 128 k
        // tiles (4 tiles of 128: 9.8 / 10.2, of 256: 18.8 / 18.0) and nine of them per compute unit of the chip (49 x
        // 512 x 4608 6.9 / 7.2, 16 x 1024 x 4096 6.5 / 6.7; 16 x 1280 x 4096 7.4 / 7.2, 16 x 2016 x 16384 20.6 / 19.0).
        if (tiles(CFG_S32) <= 256) {
            const bool eight = nkt_all >= 32 && tiles(CFG_S32) < 64 &&
                               (mode != ABFT_NONE || (nkt_all <= 128 && tiles(CFG_S32) * nkt_all <= 9 * 256));
            return eight ? CFG_S32W : CFG_S32;
        }
        if (tiles(CFG_S64) <= 256) return CFG_S64;
        if (tiles(CFG_S128) <= 256 ? nkt_all >= 4 : (tiles(CFG_S128) <= 512 && nkt_all >= (mode == ABFT_THREAD && dt != ABFT_F16 ? 8 : 16))) return CFG_S128;
        if (fast_ok) {
            // (wavefront-level: 64 x 64 wavefront tiles with at most one workgroup per compute unit, 32 x 128 ones once
            // two share it.  The exact scheme issues the same MFMAs on both and is level, the wide tiles 0 to 3 %
            // behind: 1536 x 2048 x 2048 33.1 / 33.8 us, 4096^3 222 / 226; fp16 half-precision sums take an extra MFMA
            // per A fragment, of which the wide tiles have half: 3072 x 2048 x 2048 49.2 / 45.8, 4096^3 193 / 183)
            // At most one 128 x 128 tile per compute unit (one round): eight wavefronts of 32 x 64 on the
            // 16x16x32 shapes with three stages instead of four wavefronts of 64 x 64 with two: the second
            // wavefront per SIMD and the deeper pipeline hide what a second workgroup would (1024 x 4096 x
            // 4096: 40-43 us against 46-48; 2048^3: 22 against 26; 12544 x 256 x 2304: 25 against 28;
            // global the same tenth).  Two rounds: slower (3072 x 4096 x 4096: 115 against 91 us on two
            // workgroups per unit).  No wavefront-level scheme on it.
            if (fills128 && mode != ABFT_THREAD && tiles(CFG_F128) <= 256 && nkt_all >= 4) return CFG_F128E;
            if (fills128) return (nkt_all <= 1 || (mode == ABFT_THREAD && tiles(CFG_F128) > 256)) ? CFG_F128T : CFG_F128;
            return CFG_F64T;
        }
    }
    if (tiles(CFG_G128) >= 192) return CFG_G128;
    if (tiles(CFG_G64) >= 1024) return CFG_G128;
    // Four groups sharing the k loop where at most one such tile per compute unit is there (one tile in
    // flight per group, so four times the loads): from five k tiles on (300 x 1000 x 257 thread-level 7.0
    // against 7.3 us, K = 400 7.1 / 8.3, 1000 x 1000 x 1000 12.9 / 21.0; three tiles 6.3 / 5.9); with two
    // rounds of them only for long loops (400 x 4096 x 2048 38 / 40, 512 x 4096 x 4096 69 / 75; 1024 x
    // 2048 x 1024 23.5 / 22.3).
    if (tiles(CFG_G64) <= 256 ? nkt_gen >= 5 : (tiles(CFG_G64) <= 512 && nkt_gen >= 32)) return CFG_G64K;
    return CFG_G64;
}

// ------------------------------------------------------------------------- //
// auxiliary kernels
// ------------------------------------------------------------------------- //
struct PreArgs {
    const char* A;
    int M, K;
    long long lda;
    int vec;
    int conv, H, W, Cin, KH, KW, stride, pad, OH, OW;
    long long imgpitch, rowpitch;  // as in GemmArgs
    int pix;
    void* alpha_out;      // K doubles / int64: the plain checksum (single-slab launches only), or null
    int rows_per_slab;    // rows of one row block of the product's tiling
    int rows_per_block;   // rows one workgroup sums; divides rows_per_slab
    const void* beta;     // K x nb (k-major) weight checksums per column block, or null
    void* partial_dots;   // [slab][nb][subs * gridDim.x] partial checksum dot products, or null
    int nb;
};

// Activation checksum alpha_s[k] = sum over the rows m of slab s of A[m][k] (Sec. 2.4
// step 1), one slab per row block of the product's workgroup tiling: convolutions, and matrices whose rows are shorter
// than a 16-byte chunk (the others have the kernel below).
// Block = 32 chunk columns x 8 row lanes.
template <int DT>
__global__ __launch_bounds__(256) void act_checksum_kernel(const PreArgs p) {
    constexpr int ESIZE = DT == DT_I8 ? 1 : 2;
    constexpr int EPC = 16 / ESIZE;
    typedef typename std::conditional<DT == DT_I8, long long, double>::type Wide;
    __shared__ Wide red[8][32][EPC];
    __shared__ Wide alpha_s[32 * EPC];

    const int tid = threadIdx.x, tx = tid & 31, ty = tid >> 5;
    const int k0 = (blockIdx.x * 32 + tx) * EPC;
    const int subs = p.rows_per_slab / p.rows_per_block;
    const int slab = blockIdx.y / subs, sub = blockIdx.y - slab * subs;
    const int row_begin = slab * p.rows_per_slab + sub * p.rows_per_block;
    const int row_end = min(p.M, row_begin + p.rows_per_block);
    Wide* out = reinterpret_cast<Wide*>(p.alpha_out);

    if (!p.conv) {
        // one element per thread and row: thread t takes column t % K and every nrg-th row, so that adjacent lanes
        // read adjacent elements and the loads of one thread do not wait for each other
        const int kb = p.K, nrg = 256 / kb, col = tid % kb, rg = tid / kb;
        Wide* part = &red[0][0][0];
        Wide acc = 0;
        if (rg < nrg) {
            const char* src = p.A + (long long)col * ESIZE;
            for (int m0 = row_begin + rg; m0 < row_end; m0 += 8 * nrg) {
                Wide v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int m = m0 + u * nrg;
                    const int mc = m < row_end ? m : m0;   // a valid row; its value is dropped below
                    const char* q = src + (long long)mc * p.lda * ESIZE;
                    Wide x;
                    if constexpr (DT == DT_F16) x = (double)(float)*reinterpret_cast<const _Float16*>(q);
                    else if constexpr (DT == DT_BF16) x = (double)(float)*reinterpret_cast<const __bf16*>(q);
                    else x = (long long)*reinterpret_cast<const signed char*>(q);
                    v[u] = m < row_end ? x : (Wide)0;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) acc += v[u];
            }
        }
        part[tid] = acc;
        __syncthreads();
        for (int k = tid; k < 32 * EPC; k += 256) {
            Wide a = 0;
            if (k < kb) {
                for (int g = 0; g < nrg; ++g) a += part[g * kb + k];
                if (out) out[k] = a;
            }
            alpha_s[k] = a;
        }
    } else {
        // per-element filter tap for the implicit-GEMM view (k is fixed per thread)
        int e_off[EPC], e_kh[EPC], e_kw[EPC];
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            int k = k0 + e;
            int tap = k / p.Cin;
            e_off[e] = k - tap * p.Cin;
            e_kh[e] = tap / p.KW;
            e_kw[e] = tap - e_kh[e] * p.KW;
        }
        Wide s[EPC];
#pragma unroll
        for (int e = 0; e < EPC; ++e) s[e] = 0;
        for (int m0 = row_begin + ty; m0 < row_end; m0 += 64) {
            // int8: up to eight rows are summed in int32 first (exact); fp16 / bf16 values are
            // widened and added in fp64 one by one, so the checksum side carries no rounding
            // that could show up in the comparison
            typename std::conditional<DT == DT_I8, int, double>::type f[EPC];
#pragma unroll
            for (int e = 0; e < EPC; ++e) f[e] = 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int m = m0 + 8 * u;
                if (m >= row_end || k0 >= p.K) continue;
                i32x4 v = {0, 0, 0, 0};
                int img = m / (p.OH * p.OW);
                int rem = m - img * (p.OH * p.OW);
                int oh = rem / p.OW, ow = rem - oh * p.OW;
                int ih0 = oh * p.stride - p.pad, iw0 = ow * p.stride - p.pad;
                const char* base = p.A + (long long)img * p.imgpitch * ESIZE;
                if (p.vec) {
                    int ih = ih0 + e_kh[0], iw = iw0 + e_kw[0];
                    if (ih >= 0 && ih < p.H && iw >= 0 && iw < p.W)
                        v = ld16(base + ((long long)ih * p.rowpitch + (long long)iw * p.pix + e_off[0]) * ESIZE);
                } else {
#pragma unroll
                    for (int e = 0; e < EPC; ++e) {
                        int ih = ih0 + e_kh[e], iw = iw0 + e_kw[e];
                        unsigned x = 0;
                        if (k0 + e < p.K && ih >= 0 && ih < p.H && iw >= 0 && iw < p.W) {
                            const char* src = base + ((long long)ih * p.rowpitch + (long long)iw * p.pix + e_off[e]) * ESIZE;
                            x = ESIZE == 2 ? (unsigned)*reinterpret_cast<const unsigned short*>(src)
                                           : (unsigned)*reinterpret_cast<const unsigned char*>(src);
                        }
                        if (ESIZE == 2) v[e >> 1] |= (int)(x << (16 * (e & 1)));
                        else v[e >> 2] |= (int)(x << (8 * (e & 3)));
                    }
                }
                if constexpr (DT == DT_F16) {
                    f16x8 h = bitcast<f16x8>(v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] += (double)(float)h[e];
                } else if constexpr (DT == DT_BF16) {
                    bf16x8 h = bitcast<bf16x8>(v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] += (double)(float)h[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] += (int)(signed char)(v[e >> 2] >> (8 * (e & 3)));
                }
            }
#pragma unroll
            for (int e = 0; e < EPC; ++e) s[e] += (Wide)f[e];
        }
#pragma unroll
        for (int e = 0; e < EPC; ++e) red[ty][tx][e] = s[e];
        __syncthreads();
        if (ty == 0) {
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                Wide a = 0;
                for (int y = 0; y < 8; ++y) a += red[y][tx][e];
                alpha_s[tx * EPC + e] = (k0 + e < p.K) ? a : (Wide)0;
                if (out && k0 + e < p.K) out[k0 + e] = a;
            }
        }
    }
    if (!p.partial_dots) return;
    // Sec. 2.4 step 2, fused: this block's share of the checksum dot products
    //   P[slab][j][sub, chunk] = sum over the block's rows and k range of A[m][k] * beta_j[k]
    // lanes run over the column blocks j (beta is k-major, so these reads are contiguous),
    // the 8 lane groups split the k range
    __syncthreads();
    const int kbase = blockIdx.x * 32 * EPC;
    const int kcount = min(32 * EPC, p.K - kbase);
    const Wide* beta = reinterpret_cast<const Wide*>(p.beta);
    Wide* red2 = &red[0][0][0];  // reuse: 8 x 32 values
    const int n_parts = subs * gridDim.x;
    Wide* pout = reinterpret_cast<Wide*>(p.partial_dots) + (long long)slab * p.nb * n_parts + sub * gridDim.x + blockIdx.x;
    for (int jb = 0; jb < p.nb; jb += 32) {
        const int j = jb + tx;
        Wide acc = 0;
        if (j < p.nb) {
            // 32 * EPC / 8 values of k per thread, loaded in independent batches of eight
            const Wide* bj = beta + (long long)kbase * p.nb + j;
            for (int k0b = ty; k0b < 32 * EPC; k0b += 64) {
                Wide bv[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int k = k0b + 8 * u;
                    bv[u] = k < kcount ? bj[(long long)k * p.nb] : (Wide)0;
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) acc += alpha_s[k0b + 8 * u] * bv[u];
            }
        }
        __syncthreads();
        red2[ty * 32 + tx] = acc;
        __syncthreads();
        if (ty == 0 && j < p.nb) {
            Wide tot = 0;
            for (int y = 0; y < 8; ++y) tot += red2[y * 32 + tx];
            pout[(long long)j * n_parts] = tot;
        }
    }
}

// The same for matrices whose rows are contiguous (at any alignment): the pass over A of the global scheme.  A chunk
// that K cuts short is read as the last 16 bytes of its row and shifted down.  Four rows per thread are on their
// way while four are added, and the first weight checksums of the block's k range before any of them; registers for
// four workgroups per compute unit.  Bound: HBM (A once); with few row blocks, the trip for A.
// With the weight checksums / this pass of the kernel above, global over unprotected: 511 x 1000 x 2047 fp16 +9.2 / +6.4 us,
// 2048 x 2048 x 2047 int8 +15.7 / +8, 700 x 128 x 1000 int8, K x N, +14.4 / +7.7 (rows that are no whole chunks went by
// the element there), 256 x 4096 x 4096, K x N, +10.2 / +6.9, 8192 x 4096 x 4096 bf16 +18 / +14; 8192^3 level (+28).
template <int DT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(DT == DT_I8 ? 2 : 4)))
void act_checksum_rows_kernel(const PreArgs p) {
    constexpr int ESIZE = DT == DT_I8 ? 1 : 2;
    constexpr int EPC = 16 / ESIZE;
    constexpr int KB = 32 * EPC;   // values of k per workgroup
    constexpr int NR = 4;          // rows per set of loads
    constexpr int NBV = 16;        // weight checksums per batch
    typedef typename std::conditional<DT == DT_I8, long long, double>::type Wide;
    __shared__ Wide red[8][32][EPC];
    __shared__ Wide alpha_s[KB];
    const int tid = threadIdx.x, tx = tid & 31, ty = tid >> 5;
    const int kbase = blockIdx.x * KB, k0 = kbase + tx * EPC;
    const int subs = p.rows_per_slab / p.rows_per_block;
    const int slab = blockIdx.y / subs, sub = blockIdx.y - slab * subs;
    const int row_begin = slab * p.rows_per_slab + sub * p.rows_per_block;
    const int row_end = min(p.M, row_begin + p.rows_per_block);
    const int kcount = min(KB, p.K - kbase);

    // this lane's column block, sixteen values of k at a time (out of range: a valid value, multiplied with a
    // zero or dropped)
    Wide bv[NBV];
    auto load_beta = [&](int jb, int batch) {
        const Wide* bj = reinterpret_cast<const Wide*>(p.beta) + (long long)kbase * p.nb + (jb + tx < p.nb ? jb + tx : p.nb - 1);
#pragma unroll
        for (int u = 0; u < NBV; ++u) {
            const int k = ty + 8 * (batch * NBV + u);
            bv[u] = bj[(long long)(k < kcount ? k : 0) * p.nb];
        }
    };
    if (p.partial_dots) load_beta(0, 0);

    Wide s[EPC];
#pragma unroll
    for (int e = 0; e < EPC; ++e) s[e] = 0;
    if (row_begin < row_end) {
        const int early = k0 < p.K && k0 + EPC > p.K ? (k0 + EPC - p.K) * ESIZE : 0;
        const char* const src = p.A + (long long)(k0 + EPC <= p.K ? k0 : p.K - EPC) * ESIZE;
        // set `it`: rows ty, ty + 8, .. of 8 NR rows
        auto load = [&](int it, i32x4(&v)[NR]) {
#pragma unroll
            for (int u = 0; u < NR; ++u) {
                const int m = row_begin + ty + 8 * (NR * it + u);
                v[u] = ld16u(src + (long long)(m < row_end ? m : row_end - 1) * p.lda * ESIZE);
            }
        };
        // values are widened and added in fp64 one by one (int8: a set in int32 first, exactly), so that the
        // checksum side carries no rounding that could show up in the comparison
        auto add = [&](int it, const i32x4(&v)[NR]) {
            int f[DT == DT_I8 ? EPC : 1] = {0};
#pragma unroll
            for (int u = 0; u < NR; ++u) {
                i32x4 x = v[u];
                if (early) x = shift_down(x, early);
                if (row_begin + ty + 8 * (NR * it + u) >= row_end || k0 >= p.K) x = i32x4{0, 0, 0, 0};
                if constexpr (DT == DT_F16) {
                    const f16x8 h = bitcast<f16x8>(x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += (double)(float)h[e];
                } else if constexpr (DT == DT_BF16) {
                    const bf16x8 h = bitcast<bf16x8>(x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] += (double)(float)h[e];
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] += (int)(signed char)(x[e >> 2] >> (8 * (e & 3)));
                }
            }
            if constexpr (DT == DT_I8) {
#pragma unroll
                for (int e = 0; e < EPC; ++e) s[e] += (Wide)f[e];
            }
        };
        const int n_it = (row_end - row_begin + 8 * NR - 1) / (8 * NR);
        i32x4 va[NR], vb[NR];
        load(0, va);
#pragma nounroll
        for (int it = 0; it < n_it; it += 2) {
            if (it + 1 < n_it) load(it + 1, vb);
            add(it, va);
            if (it + 2 < n_it) load(it + 2, va);
            if (it + 1 < n_it) add(it + 1, vb);
        }
    }
#pragma unroll
    for (int e = 0; e < EPC; ++e) red[ty][tx][e] = s[e];
    __syncthreads();
    Wide* out = reinterpret_cast<Wide*>(p.alpha_out);
    for (int k = tid; k < KB; k += 256) {
        Wide a = 0;
#pragma unroll
        for (int y = 0; y < 8; ++y) a += (&red[y][0][0])[k];
        alpha_s[k] = a;                                   // (zero beyond K)
        if (out && kbase + k < p.K) out[kbase + k] = a;
    }
    if (!p.partial_dots) return;
    // Sec. 2.4 step 2: this block's share of the checksum dot products, as in the kernel above
    __syncthreads();
    Wide* red2 = &red[0][0][0];  // reuse: 8 x 32 values
    const int n_parts = subs * gridDim.x;
    Wide* pout = reinterpret_cast<Wide*>(p.partial_dots) + (long long)slab * p.nb * n_parts + sub * gridDim.x + blockIdx.x;
    for (int jb = 0; jb < p.nb; jb += 32) {
        Wide acc = 0;
#pragma nounroll
        for (int batch = 0; batch < KB / 8 / NBV; ++batch) {
            if (batch > 0 || jb > 0) load_beta(jb, batch);
#pragma unroll
            for (int u = 0; u < NBV; ++u) acc += alpha_s[ty + 8 * (batch * NBV + u)] * bv[u];
        }
        __syncthreads();
        red2[ty * 32 + tx] = acc;
        __syncthreads();
        if (ty == 0 && jb + tx < p.nb) {
            Wide tot = 0;
            for (int y = 0; y < 8; ++y) tot += red2[y * 32 + tx];
            pout[(long long)(jb + tx) * n_parts] = tot;
        }
    }
}

// Weight checksum per block of columns: beta_b[k] = sum over the columns n of block b of
// B[k][n] (Sec. 2.5, offline), for any storage order (element strides).
// Block = 32 values of k x 8 lanes over n; blockIdx.y = column block.  Not tuned: offline.
template <int DT>
__global__ __launch_bounds__(256) void weight_checksum_kernel(const char* B, int K, int N, long long sn,
                                                              long long sk, int block_n, int wnorm, void* beta,
                                                              char* beta_k, char* beta_p, char* beta_r) {
    constexpr int ESIZE = DT == DT_I8 ? 1 : 2;
    typedef typename std::conditional<DT == DT_I8, long long, double>::type Wide;
    __shared__ Wide red[2][8][32];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int k = blockIdx.x * 32 + tx;
    const int n_begin = blockIdx.y * block_n, n_end = min(N, n_begin + block_n);
    // s: the plain checksum of the block's columns; sv: the same with column j of the block
    // weighted j + 1 (int8) or (j + 1) / wnorm (floating point; wnorm: the nominal block width, also
    // where N cuts the block short), the second of the independent linear combinations of Sec. 2.4's
    // last paragraph
    Wide s = 0, sv = 0;
    if (k < K) {
        for (int n = n_begin + ty; n < n_end; n += 8) {
            const char* src = B + ((long long)n * sn + (long long)k * sk) * ESIZE;
            Wide x;
            if constexpr (DT == DT_F16) x = (double)(float)*reinterpret_cast<const _Float16*>(src);
            else if constexpr (DT == DT_BF16) x = (double)(float)*reinterpret_cast<const __bf16*>(src);
            else x = (long long)*reinterpret_cast<const signed char*>(src);
            s += x;
            if constexpr (DT == DT_I8) sv += x * (n - n_begin + 1);
            else sv += x * ((double)(n - n_begin + 1) / (double)wnorm);
        }
    }
    red[0][ty][tx] = s;
    red[1][ty][tx] = sv;
    __syncthreads();
    if (ty == 0 && k < K) {
        Wide a = 0, av = 0;
        for (int y = 0; y < 8; ++y) {
            a += red[0][y][tx];
            av += red[1][y][tx];
        }
        reinterpret_cast<Wide*>(beta)[(long long)k * gridDim.y + blockIdx.y] = a;
        // second copy, per column block along k, for the in-kernel checksum dot product of the
        // direct-to-LDS kernel: floats, or (int8) balanced base-256 digits, K low then K high;
        // third copy (8 bytes per k and block) for the streaming kernel's matrix-unit form: fp16:
        // four planes of K halves, hi = fl16(beta), lo = fl16((beta - hi) 2^11), and the same two
        // pieces of the column-weighted checksum; int8: four planes of K digits of the
        // column-weighted checksum (balanced base 256, least significant first)
        // fourth copy, for the direct-to-LDS kernel: per block and k tile of that kernel (64 values of k;
        // int8: 128) a record of 1 KB -- fp16: 64 halves fl16(beta), 64 halves fl16((beta - hi) 2^11), then
        // (at byte 256) 64 floats; bf16: the 64 floats; int8: 128 low digits, 128 high digits
        constexpr int KT = DT == DT_I8 ? 128 : 64;
        char* rec = beta_r + ((long long)blockIdx.y * ((K + KT - 1) / KT) + k / KT) * 1024;
        const int kin = k % KT;
        if constexpr (DT == DT_I8) {
            const long long lo = (long long)(signed char)(a & 0xff);
            const long long hi = (a - lo) >> 8;
            signed char* d = reinterpret_cast<signed char*>(beta_k) + (long long)blockIdx.y * 2 * K;
            d[k] = (signed char)lo;
            d[K + k] = (signed char)(hi < -128 ? -128 : (hi > 127 ? 127 : hi));
            reinterpret_cast<signed char*>(rec)[kin] = d[k];
            reinterpret_cast<signed char*>(rec)[128 + kin] = d[K + k];
            signed char* dv = reinterpret_cast<signed char*>(beta_p) + (long long)blockIdx.y * 8 * K;
            long long rest = av;
            for (int q = 0; q < 4; ++q) {
                const long long digit = (long long)(signed char)(rest & 0xff);
                dv[(long long)q * K + k] = (signed char)digit;
                rest = (rest - digit) >> 8;
            }
        } else {
            reinterpret_cast<float*>(beta_k)[(long long)blockIdx.y * K + k] = (float)a;
            reinterpret_cast<float*>(rec + 256)[kin] = (float)a;
            if constexpr (DT == DT_F16) {
                _Float16* pl = reinterpret_cast<_Float16*>(beta_p) + (long long)blockIdx.y * 4 * K;
                const _Float16 hi = (_Float16)(float)a;
                pl[k] = hi;
                pl[K + k] = (_Float16)(((float)a - (float)hi) * 2048.f);
                reinterpret_cast<_Float16*>(rec)[kin] = pl[k];
                reinterpret_cast<_Float16*>(rec + 128)[kin] = pl[K + k];
                const _Float16 vhi = (_Float16)(float)av;
                pl[2 * K + k] = vhi;
                pl[3 * K + k] = (_Float16)(((float)av - (float)vhi) * 2048.f);
            }
        }
    }
}

// ------------------------------------------------------------------------- //
// Convolutions with few input channels (ResNet's first layer: Cin = 3), lowered to row
// segments.  For a filter row kh the KW taps x Cin channels are one contiguous run of the
// input row, so k is re-ordered as (kh, run position) with every run padded to whole 16-byte
// chunks, the input is copied once with its zero border (so no chunk needs masking) and the
// product reads whole chunks instead of gathering single elements.
// ------------------------------------------------------------------------- //
// padded copy of the NHWC input: out[img][r][x] (row pitch rowp elements), r over H + 2 pad rows,
// x over the padded row; one 16-byte chunk per thread
template <int ESIZE>
__global__ __launch_bounds__(256) void conv_pad_kernel(const char* x, char* out, int H, int WC, int pad, int padC,
                                                      int Hp, long long rowp, long long chunks_per_row,
                                                      long long total_chunks) {
    constexpr int EPC = 16 / ESIZE;
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    if (t >= total_chunks) return;
    // (32-bit divisions where they do: the 64-bit ones cost more than the copy)
    const bool small = total_chunks <= 0x7fffffffLL;
    const long long row = small ? (long long)((unsigned)t / (unsigned)chunks_per_row) : t / chunks_per_row;
    const long long e0 = (t - row * chunks_per_row) * EPC;
    const long long img = small ? (long long)((unsigned)row / (unsigned)Hp) : row / Hp;
    const int ih = (int)(row - img * Hp) - pad;
    i32x4 v = {0, 0, 0, 0};
    if (ih >= 0 && ih < H) {
        const char* src = x + ((img * H + ih) * (long long)WC) * ESIZE;
        // chunks inside the input row in one read at whatever alignment, those at its ends by the element
        if (e0 >= padC && e0 + EPC - padC <= WC) v = ld16u(src + (e0 - padC) * ESIZE);
        else
#pragma unroll
        for (int e = 0; e < EPC; ++e) {
            const long long xe = e0 + e - padC;
            unsigned val = 0;
            if (xe >= 0 && xe < WC)
                val = ESIZE == 2 ? (unsigned)*reinterpret_cast<const unsigned short*>(src + xe * 2)
                                 : (unsigned)*reinterpret_cast<const unsigned char*>(src + xe);
            if (ESIZE == 2) v[e >> 1] |= (int)(val << (16 * (e & 1)));
            else v[e >> 2] |= (int)(val << (8 * (e & 3)));
        }
    }
    *reinterpret_cast<i32x4*>(out + (row * rowp + e0) * ESIZE) = v;
}

// weights in the lowered order: out[n][kh * segp + r] = B[k = (kh KW + r / Cin) Cin + r % Cin][n] for
// r < KW Cin and kh < KH, else 0
template <int ESIZE>
__global__ __launch_bounds__(256) void conv_weights_kernel(const char* B, long long sn, long long sk, char* out, int N,
                                                          int Kp, int segp, int seg, int KH) {
    const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
    if (t >= (long long)N * Kp) return;
    const int n = (int)(t / Kp), kp = (int)(t - (long long)n * Kp);
    const int kh = kp / segp, r = kp - kh * segp;
    if (ESIZE == 2) {
        unsigned short v = 0;
        if (r < seg && kh < KH) v = *reinterpret_cast<const unsigned short*>(B + ((long long)n * sn + (long long)(kh * seg + r) * sk) * 2);
        reinterpret_cast<unsigned short*>(out)[t] = v;
    } else {
        unsigned char v = 0;
        if (r < seg && kh < KH) v = *reinterpret_cast<const unsigned char*>(B + ((long long)n * sn + (long long)(kh * seg + r) * sk));
        reinterpret_cast<unsigned char*>(out)[t] = v;
    }
}

// ------------------------------------------------------------------------- //
// host helpers
// ------------------------------------------------------------------------- //
struct Problem {
    int M, N, K, dtype, b_layout;
    const void* A;
    long long lda;
    const void* B;
    long long ldb;
    void* C;
    long long ldc;
    bool conv;
    abft_conv_t cg;
    int OH, OW;
    long long imgpitch, rowpitch;  // conv: input element (img, ih, iw, c) at img*imgpitch + ih*rowpitch + iw*pix + c
    int pix;
    int tol_K;                     // K the tolerance is taken for (differs from K for a lowered convolution)
    int run_seg;                   // lowered weights on the input as it is (strip kernel): elements of a filter row's run, else 0
    int act;                       // abft_act_t applied to the stored values
    // chains of layers (Sec. 2.4 step 4): where this layer's epilogue leaves the activation checksums
    // of the NEXT layer (per 32-row block, leading dimension ld_alpha_out; see GemmArgs), whether it
    // did (not every kernel can), and the ones the layer before left for this layer's A
    float* alpha_out;
    long long ld_alpha_out;
    bool* alpha_emitted;
    const float* alpha_in;
    // scaled int8 product (row_scale not null): the type C is stored in, its scales, a bias or null
    int out_dtype;
    const float *row_scale, *col_scale, *bias;
};

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool a_vectorisable(const Problem& pr) {
    const int es = esize(pr.dtype);
    if (pr.run_seg) return true;
    if (!aligned16(pr.A)) return false;
    // (a lowered convolution reads chunks at 4-byte aligned addresses: 16-byte loads still apply)
    if (pr.conv) return (pr.cg.Cin * es) % 16 == 0;
    return (pr.K * es) % 16 == 0 && (pr.lda * es) % 16 == 0;
}
bool b_vectorisable(const Problem& pr) {
    const int es = esize(pr.dtype);
    return pr.b_layout == ABFT_B_NK && aligned16(pr.B) && (pr.K * es) % 16 == 0 && (pr.ldb * es) % 16 == 0;
}

int conv_out(int in, int k, int stride, int pad) { return (in + 2 * pad - k) / stride + 1; }

struct WsLayout {
    size_t off_pd, off_beta, total;
};

int pre_grid_x(int K, int dt) { return (int)cdiv(K, 32 * (16 / esize(dt))); }
// rows one workgroup of the activation-checksum kernel sums: a whole row block of the tiling
// when that still gives a few workgroups per compute unit, else 64 rows
int pre_rows_per_block(int bm, int M, int K) {
    if (bm <= 64) return bm;
    return cdiv(M, bm) * cdiv(K, 256) >= 512 ? bm : 64;
}

// Workspace of the global scheme for the tile configuration `cfg`: per-tile partial
// checksum dot products, per-column-block weight checksums
// (the last only used when the caller passes no precomputed ones).  Sized for any dtype.
// The weight-checksum buffer holds two copies: K x nb wide values (double / int64, k-major) for
// the activation-checksum kernel's dot products, then, 256-byte aligned, the per-block copy
// along k for the in-kernel dot product (4 bytes per k and block reserved).
size_t beta_k_offset(int K, int nb) { return align_up((size_t)K * nb * 8, 256); }
// third copy, 8 bytes per k and block: the columns of the extra operand with which the streaming
// kernel forms its dot products on the matrix unit (see weight_checksum_kernel)
size_t beta_p_offset(int K, int nb) { return beta_k_offset(K, nb) + align_up((size_t)K * nb * 4, 256); }
// fourth copy: one 1 KB record per block and k tile of the direct-to-LDS kernel (64 values of k; int8:
// 128), which one 16-byte-per-lane copy brings in with the operand tiles (see weight_checksum_kernel);
// sized for the shorter k tile
size_t beta_r_offset(int K, int nb) { return beta_p_offset(K, nb) + align_up((size_t)K * nb * 8, 256); }
size_t beta_total_bytes(int K, int nb) { return beta_r_offset(K, nb) + (size_t)nb * cdiv(K, 64) * 1024; }

WsLayout ws_layout(int M, int N, int K, int cfg) {
    CfgInfo ci = cfg_info_host(cfg);
    const size_t tm = (size_t)cdiv(M, ci.bm), tn = (size_t)cdiv(N, ci.bn);
    const size_t n_parts = (size_t)(ci.bm / (ci.bm < 64 ? ci.bm : 64)) * (size_t)cdiv(K, 256);  // upper bound
    WsLayout w;
    w.off_pd = 0;
    w.off_beta = align_up(w.off_pd + tm * tn * n_parts * 8, 256);
    w.total = align_up(w.off_beta + beta_total_bytes(K, (int)tn), 256);
    return w;
}

size_t ws_bytes_any_cfg(int M, int N, int K) {
    size_t best = 0;
    for (int id = 0; id < CFG_COUNT; ++id) {
        size_t t = ws_layout(M, N, K, id).total;
        if (t > best) best = t;
    }
    return best;
}

// extra coefficient of ||C_S||_F for the schemes that add checksums in the operand type, on
// wavefront tiles of tile_m x tile_n (MFMA blocks of mi rows / columns)
double tol_half_coeff(int dt, int mode, int tile_m, int tile_n, int mi) {
    if (dt == ABFT_I8 || (mode != ABFT_THREAD_HALF && mode != ABFT_TWOSIDED)) return 0.0;
    const double n_b = tile_n / mi - 1, n_a = mode == ABFT_TWOSIDED ? tile_m / mi - 1 : 0;
    return C_HALF * (dt == ABFT_F16 ? U_HALF_F16 : U_HALF_BF16) * std::sqrt(n_b * tile_m + n_a * tile_n);
}

double tol_coeff(int K, int dt, int mode) {
    if (dt == ABFT_I8) return 0.0;
    // (two fp32 accumulations compared, as in the thread-level scheme)
    if (mode == ABFT_REPLICA || mode == ABFT_THREAD_HALF || mode == ABFT_TWOSIDED) mode = ABFT_THREAD;
    double u_chi = 0.0;
    if (mode == ABFT_THREAD) u_chi = dt == ABFT_F16 ? U_CHI_F16 : U_CHI_BF16;
    return C_TOL * (U_ACC * std::sqrt((double)K) + u_chi);
}

// coefficient of the sum of magnitudes (global scheme only): covers the coherent bias of
// the matrix unit's accumulation, which grows like K per entry instead of sqrt(K)
double tol_bias_coeff(int K, int dt, int mode) {
    if (dt == ABFT_I8 || mode != ABFT_GLOBAL) return 0.0;
    return C_BIAS * U_ACC * (double)K;
}

double cmr_of(int dt) {
    if (g_cmr_override[dt] > 0.0) return g_cmr_override[dt];
    return (dt == ABFT_I8 ? PEAK_I8 : PEAK_F16) / HBM_BW;
}

double intensity(int M, int N, int K, int dt) {
    const double sa = esize(dt), sb = esize(dt), sc = csize(dt);
    const double m = M, n = N, k = K;
    return 2.0 * m * n * k / (sa * m * k + sb * k * n + sc * m * n);
}

int select_mode(int M, int N, int K, int dt) {
    return intensity(M, N, K, dt) > cmr_of(dt) ? ABFT_GLOBAL : ABFT_THREAD;
}
// The faster protected scheme of a scaled product.  Aligned, the global one wherever 32 x 32 tiles are more than one per compute unit:
// beyond that the thread-level one forms its checksums on the vector unit of every wavefront (bf16 out, thread-level / global,
// us: 64 x 4096 x 4096 7.7 / 8.2, 96 rows 13.1 / 9.4, 256 rows 17.3 / 12.4, 1024 46 / 26; 128 x 2048 x 8192 9.9 / 10.7, 192 rows
// 20.3 / 13.2; 512 x 512 x 512 4.3 / 4.5, 1024 rows 5.7 / 5.1).  Few rows, whole calls with the quantisation, weights from memory: 1 x 8192 x
// 4096 11.5 / 12.2, 1 x 8224 x 4096 15.3 / 13.7, 4 x 11008 x 4096 16.7 / 15.7, 16 x 14336 x 8192 30.8 / 29.1, 32 x 32000 x 1024 20.0 / 17.2; only
// where the checksums of very many weights are read for few rows is it the wrong way round: 1 x 32000 x 4096 40.0 / 42.3, 4 x 32000 x
// 8192 64.8 / 74.0, 64 rows 68.4 / 77.5.  Else the global one takes a pass over A, and the intensity decides as ever (511 x 1000 x 2047
// 9.7 / 17.8).
int scaled_select(int M, int N, int K, bool aligned) {
    if (aligned) return cdiv(M, 32) * cdiv(N, 32) > 256 ? ABFT_GLOBAL : ABFT_THREAD;
    return select_mode(M, N, K, ABFT_I8);
}

hipError_t launch_weight_checksum(int K, int N, const void* B, long long ldb, int layout, int dt, int block_n,
                                  void* beta_buf, hipStream_t st) {
    long long sn = layout == ABFT_B_NK ? ldb : 1, sk = layout == ABFT_B_NK ? 1 : ldb;
    const int wnorm = block_n > 0 ? block_n : N;
    if (block_n <= 0 || block_n > N) block_n = N;
    void* beta = beta_buf;
    char* beta_k = reinterpret_cast<char*>(beta_buf) + beta_k_offset(K, (int)cdiv(N, block_n));
    char* beta_p = reinterpret_cast<char*>(beta_buf) + beta_p_offset(K, (int)cdiv(N, block_n));
    char* beta_r = reinterpret_cast<char*>(beta_buf) + beta_r_offset(K, (int)cdiv(N, block_n));
    dim3 grid((unsigned)cdiv(K, 32), (unsigned)cdiv(N, block_n)), block(256);
    const char* b = reinterpret_cast<const char*>(B);
    if (dt == ABFT_F16)
        hipLaunchKernelGGL(weight_checksum_kernel<DT_F16>, grid, block, 0, st, b, K, N, sn, sk, block_n, wnorm, beta, beta_k, beta_p, beta_r);
    else if (dt == ABFT_BF16)
        hipLaunchKernelGGL(weight_checksum_kernel<DT_BF16>, grid, block, 0, st, b, K, N, sn, sk, block_n, wnorm, beta, beta_k, beta_p, beta_r);
    else
        hipLaunchKernelGGL(weight_checksum_kernel<DT_I8>, grid, block, 0, st, b, K, N, sn, sk, block_n, wnorm, beta, beta_k, beta_p, beta_r);
    return hipGetLastError();
}

hipError_t launch_act_checksum(const Problem& pr, void* alpha_out, int rows_per_slab, const void* beta, int nb,
                               void* partial_dots, hipStream_t st) {
    PreArgs a;
    std::memset(&a, 0, sizeof a);
    a.A = reinterpret_cast<const char*>(pr.A);
    a.M = pr.M;
    a.K = pr.K;
    a.lda = pr.lda;
    a.vec = a_vectorisable(pr) ? 1 : 0;
    a.conv = pr.conv ? 1 : 0;
    if (pr.conv) {
        a.imgpitch = pr.imgpitch; a.rowpitch = pr.rowpitch; a.pix = pr.pix;
        a.H = pr.cg.H; a.W = pr.cg.W; a.Cin = pr.cg.Cin; a.KH = pr.cg.KH; a.KW = pr.cg.KW;
        a.stride = pr.cg.stride; a.pad = pr.cg.pad; a.OH = pr.OH; a.OW = pr.OW;
    }
    a.alpha_out = alpha_out;
    a.rows_per_slab = rows_per_slab;
    // the plain checksum is one slab summed by one row of blocks; the fused form splits each
    // row block of the tiling over several blocks to have enough loads in flight
    a.rows_per_block = alpha_out ? rows_per_slab : pre_rows_per_block(rows_per_slab, pr.M, pr.K);
    a.beta = beta;
    a.nb = nb;
    a.partial_dots = partial_dots;
    const int subs = a.rows_per_slab / a.rows_per_block;
    dim3 grid((unsigned)pre_grid_x(pr.K, pr.dtype), (unsigned)(cdiv(pr.M, rows_per_slab) * subs)), block(256);
    if (!pr.conv && pr.K >= 16 / esize(pr.dtype)) {
        if (pr.dtype == ABFT_F16) hipLaunchKernelGGL(act_checksum_rows_kernel<DT_F16>, grid, block, 0, st, a);
        else if (pr.dtype == ABFT_BF16) hipLaunchKernelGGL(act_checksum_rows_kernel<DT_BF16>, grid, block, 0, st, a);
        else hipLaunchKernelGGL(act_checksum_rows_kernel<DT_I8>, grid, block, 0, st, a);
        return hipGetLastError();
    }
    if (pr.dtype == ABFT_F16) hipLaunchKernelGGL(act_checksum_kernel<DT_F16>, grid, block, 0, st, a);
    else if (pr.dtype == ABFT_BF16) hipLaunchKernelGGL(act_checksum_kernel<DT_BF16>, grid, block, 0, st, a);
    else hipLaunchKernelGGL(act_checksum_kernel<DT_I8>, grid, block, 0, st, a);
    return hipGetLastError();
}

int validate_common(const Problem& pr, int mode, const uint32_t* flag) {
    if (!valid_dtype(pr.dtype)) return ABFT_E_ENUM;
    if (mode < ABFT_NONE || mode > ABFT_GLOBAL_WEIGHTED) return ABFT_E_ENUM;
    if (pr.b_layout != ABFT_B_NK && pr.b_layout != ABFT_B_KN) return ABFT_E_ENUM;
    if (pr.M <= 0 || pr.N <= 0 || pr.K <= 0) return ABFT_E_SHAPE;
    if (!pr.A || !pr.B || !pr.C) return ABFT_E_NULL;
    if (mode != ABFT_NONE && !flag) return ABFT_E_NULL;
    if (!pr.conv && pr.lda < pr.K) return ABFT_E_LD;
    if (pr.b_layout == ABFT_B_NK ? pr.ldb < pr.K : pr.ldb < pr.N) return ABFT_E_LD;
    if (pr.ldc < pr.N) return ABFT_E_LD;
    return ABFT_OK;
}

// Global scheme: where the activation checksum's dot products are formed.  Inside the product
// kernel (direct-to-LDS configurations) it costs about a tenth of the kernel's time; as a
// pass of its own over A it costs a launch plus reading A once.  Take the cheaper by estimate
// (environment variable ABFT_GLOBAL_DOT = fused | pre pins the choice: tuning aid).
// Unprotected / in the loop / with the pass, us (the estimate takes the faster or one within 3 % of it): 2048 x 4096 x 4096
// fp16 72 / 80 / 75, bf16 69 / 79 / 72, int8 41 / 45 / 47; 4096 x 4096 x 1024 33 / 37 / 40, 31 / 40 / 39, 26 / 28.5 / 34.7; 4096^3
// 107 / 119 / 118, 100 / 134 / 114, 60 / 67 / 72; 8192 x 4096 x 4096 int8 117 / 130 / 132; 8192^3 825 / 926 / 852, 787 / 1013 /
// 814, 443 / 490 / 459; 12544 x 1024 x 512 18.5 / 21.6 / 27, 18 / 22.6 / 26, 22 / 21.5 / 29.
bool fused_global(const Problem& pr, const CfgInfo& ci) {
    if (!ci.fast) return false;
    if (ci.kways > 1) return true;  // streaming configurations have no other variant
    static const int force = [] {
        const char* e = std::getenv("ABFT_GLOBAL_DOT");
        return !e ? 0 : (e[0] == 'f' ? 1 : 2);
    }();
    if (force) return force == 1;
    const double t_gemm = 2.0 * pr.M * pr.N * pr.K / (pr.dtype == ABFT_I8 ? 2.0e15 : 1.0e15);
    const double t_pre = 8.0e-6 + (double)pr.M * pr.K * esize(pr.dtype) / 4.5e12;
    // share of the product's time that the in-loop form costs: about a tenth on the 32x32-shape tiles
    // (matrix-unit form, or vector form on 64 x 64 wavefront tiles) and for int8 everywhere (9 to 12 %); the vector
    // form of fp16 / bf16 on the 16x16-shape tiles: a tenth for fp16 on the 256 x 256 tile, a quarter for
    // bf16 there (three-piece products), a fifth on the smaller tiles (less work per wavefront to hide it in)
    double in_loop = 0.09;
    if (pr.dtype != ABFT_I8 && ci.mi == 16) in_loop = ci.bm == 256 && ci.bn == 256 ? (pr.dtype == ABFT_BF16 ? 0.25 : 0.09) : 0.2;
    return in_loop * t_gemm < t_pre;
}

// The strip kernel's share of LDS for a convolution on its input as it is (see gemm_strip.h): the
// input rows under them beside the weights.  Kp: k as the weights hold it; segp: elements of a filter row's run in
// them, 0: a pixel's channels are one k tile.  Whether it fits.
bool strip_fits(const Problem& pr, int Kp, int segp, int& rows, int& pitch) {
    if (!pr.conv || esize(pr.dtype) != 2 || pr.N > 64) return false;
    const abft_conv_t& c = pr.cg;
    // (the padded copy of a lowered convolution has pitches of its own, also where a run is a whole k tile)
    if (pr.pix != c.Cin || pr.rowpitch != (long long)c.W * c.Cin || pr.imgpitch != pr.rowpitch * c.H) return false;
    const long long pixB = 2ll * c.Cin, WB = c.W * pixB;
    if (segp == 0 && pixB != 128) return false;
    if (segp != 0 && (pixB * c.stride % 4 != 0 || WB < 16)) return false;
    const long long Hv = (long long)(pr.OH - 1) * c.stride + c.KH;
    // output rows that a strip's consecutive rows of C can meet, ends of images among them, and their input rows
    const int form = segp ? STRIP_RUNS : STRIP_TAPS;
    const long long nr = cdiv(32 * strip_waves(form) - 1, pr.OW) + 1, ends = cdiv(nr - 1, pr.OH);
    const long long r = (nr - 1) * c.stride + c.KH + ends * std::max(0, c.KH - c.stride);
    const long long w = segp ? std::max(WB + 2 * c.pad * pixB, (pr.OW - 1) * c.stride * pixB + 2ll * segp) : WB + 2 * c.pad * pixB;
    if (w > 65536 || r > STRIP_ROWS_MAX || r > Hv || pr.OW < 2 || (long long)r * WB > 0x3fffffff || std::llabs(Hv - c.H) * WB > 0x3fffffff) return false;
    const long long nkt = cdiv(2ll * Kp, 128), p16 = (long long)align_up((size_t)w, 16);
    if (nkt > 20 || r * p16 > strip_max_bytes(form) || strip_lds_bytes(form, (int)nkt, (int)r, (int)p16) > 160 * 1024)
        return false;
    if ((c.batch + 1) * Hv > 0x3fffffff) return false;
    rows = (int)r;
    pitch = (int)p16;
    return true;
}

// Can the skinny kernel run a product that the tiling `cfg` would take?  At most sixteen rows of 32 x 32 streaming tiles or of
// the generic kernel's tiles for few rows, both operands contiguous along k in rows of a chunk or more, and at most two
// workgroups of 16 columns per compute unit; only the global scheme needs the tiling's column blocks.
bool skinny_fits(const Problem& pr, int cfg, int mode) {
    if (cfg != CFG_S32 && cfg != CFG_S32W && cfg != CFG_G16 && cfg != CFG_G64K) return false;
    const long long kb = (long long)pr.K * esize(pr.dtype);
    return pr.M <= SKINNY_ROWS && !pr.conv && pr.b_layout == ABFT_B_NK && mode != ABFT_GLOBAL && mode != ABFT_GLOBAL_WEIGHTED &&
           kb >= 16 && kb < (1 << 30) && pr.N <= 16 * 512;
}

// Does it?  Thread-level, the tiling's kernel / skinny (us a call of many in a graph; the first three alone):
// 16 x 4096 x 4096 bf16 8.3 / 8.0, 16 x 4096 x 8192 13.1 / 12.8, 12 x 2048 x 8192 11.8 / 9.7; 16 x 5120 x 1024 fp16 4.60 / 4.20, 16 x
// 8192 x 1024 4.65 / 4.28, 8 x 8192 x 2048 int8 4.50 / 4.18; unaligned 16 x 1000 x 2047 14.9 / 7.1, 16 x 8000 x 4003 25.6 / 16.8.
// Aligned with more than one workgroup per compute unit and many weights the tiles of 32 columns, which read A half
// as often, are ahead: 16 x 6144 x 2560 8.2 / 8.6, 16 x 8192 x 4096 12.7 / 13.1, 1 x 8192 x 8192 27.7 / 32; unprotected they are with
// few, too: 16 x 8192 x 256 bytes 2.79 / 3.05, 1 KB 3.24 / 3.36, 16 x 5120 x 1024 fp16 level.  So is, unaligned, the 16 x 64 tile on one of
// its k tiles (256 bytes): 1 x 5760 x 61 fp16 unprotected 2.83 / 3.13, thread-level 3.20 / 3.46, on two 1 x 5760 x 189 thread-level 3.79 / 3.46; with at
// most one workgroup per compute unit it is not (unprotected 1 x 2048 x 253 int8 2.82 / 2.65; thread-level 16 x 512 x 61 fp16 3.21 / 3.01).
bool skinny_takes(const Problem& pr, int cfg, int mode) {
    if (!skinny_fits(pr, cfg, mode)) return false;
    const long long kb = (long long)pr.K * esize(pr.dtype);
    const bool one_round = pr.N <= 16 * 256, checked = mode != ABFT_NONE;
    if (cfg_is_generic(cfg)) return kb > 256 || one_round;
    return one_round || (checked && pr.N * kb <= (16 << 20));
}

// rows of A or B that do not start at multiples of four bytes
bool rows_off_dwords(const GemmArgs& g, int dt) {
    return ((reinterpret_cast<uintptr_t>(g.A) | reinterpret_cast<uintptr_t>(g.B) | (uintptr_t)(g.lda * esize(dt)) | (uintptr_t)(g.ldb * esize(dt))) & 3u) != 0;
}

// Does shallow_tile take a product that the tiling `cfg` would take?  One 64 x 64 generic tile's k: rows contiguous along k, of 16 to 128
// bytes, at any address; results and comparisons are that tile's.  By itself: up to 96 bytes and two rounds of workgroups, off dwords one
// round beyond 64 bytes.  Fp16, N x K, in LDS / so, us: 250 x 1000 rows of 26 bytes unprotected 3.5 / 2.9, 62 bytes thread-level 4.0 / 3.6, 92
// 3.9 / 3.5, 94 4.0 / 3.8, 110 4.0 / 4.1, 124 3.8 / 4.1; 1000 x 2040 62 bytes 4.8 / 4.5, 92 4.6 / 4.2, 74 4.7 / 4.9; 2000 x 2040 60 bytes 7.2 / 7.3.
bool shallow_takes(const Problem& pr, int cfg, int mode) {
    const long long kb = (long long)pr.K * esize(pr.dtype);
    return cfg == CFG_G64 && (mode == ABFT_NONE || mode == ABFT_THREAD) && !pr.conv && pr.b_layout == ABFT_B_NK && kb >= 16 && kb <= 128;
}

size_t plain_workspace_bytes(int M, int N, int K, int dtype, int mode);

// ---- int8 products of 16-bit activations ----
constexpr int SCALED_MAX_K = (1 << 17) - 1;
int validate_quantize(int M, int K, const void* X, long long ldx, int dtype) {
    if (dtype != ABFT_F16 && dtype != ABFT_BF16) return ABFT_E_ENUM;
    if (M <= 0 || K <= 0) return ABFT_E_SHAPE;
    if (!X) return ABFT_E_NULL;
    if (ldx < K) return ABFT_E_LD;
    return ABFT_OK;
}
hipError_t quantize_rows(int M, int K, const void* X, long long ldx, int dtype, void* Q, long long ldq, float* scale, hipStream_t st) {
    QuantizeArgs a;
    a.X = reinterpret_cast<const char*>(X);
    a.Q = reinterpret_cast<signed char*>(Q);
    a.scale = scale;
    a.M = M; a.K = K; a.ldx = ldx; a.ldq = ldq;
    return dtype == ABFT_F16 ? launch_quantize_rows<DT_F16>(a, st) : launch_quantize_rows<DT_BF16>(a, st);
}
// A scaled product as a problem, checked as far as it is more than one in int8; AUTO becomes a scheme.  K: beyond it 128 * 128 * K passes an int32.
int scaled_problem(int M, int N, int K, const void* A, long long lda, const float* row_scale, const void* B, long long ldb, int b_layout,
                   const float* col_scale, const float* bias, int act, void* C, long long ldc, int out_dtype, int& mode, const uint32_t* flag,
                   Problem& pr) {
    std::memset(&pr, 0, sizeof pr);
    pr.M = M; pr.N = N; pr.K = K; pr.dtype = ABFT_I8; pr.b_layout = b_layout;
    pr.A = A; pr.lda = lda; pr.B = B; pr.ldb = ldb; pr.C = C; pr.ldc = ldc;
    pr.act = act; pr.out_dtype = out_dtype;
    pr.row_scale = row_scale; pr.col_scale = col_scale; pr.bias = bias;
    if (out_dtype != ABFT_F16 && out_dtype != ABFT_BF16) return ABFT_E_ENUM;
    if (act != ABFT_ACT_NONE && act != ABFT_ACT_RELU) return ABFT_E_ENUM;
    if (!row_scale || !col_scale) return ABFT_E_NULL;
    if (K > SCALED_MAX_K) return ABFT_E_SHAPE;
    const int rc = validate_common(pr, mode, flag);
    if (rc != ABFT_OK) return rc;
    if (mode == ABFT_AUTO) mode = scaled_select(M, N, K, a_vectorisable(pr) && b_vectorisable(pr));
    return mode == ABFT_NONE || mode == ABFT_GLOBAL || mode == ABFT_THREAD ? ABFT_OK : ABFT_E_UNSUPPORTED;
}
// where a linear layer's workspace holds the quantised activations (rows of whole 16-byte chunks, at its start), their scales, and
// what the product wants
long long linear_ld(int K) { return (long long)align_up((size_t)K, 16); }
size_t linear_scale_offset(int M, int K) { return align_up((size_t)M * linear_ld(K), 256); }
size_t linear_product_offset(int M, int K) { return linear_scale_offset(M, K) + align_up((size_t)M * 4, 256); }

// the k granularity of a fault that is planted in the loop, and whether a fault lies inside the product
bool inject_in_range(const Problem& pr, int mode, const abft_fault_t& f) {
    if (mode == ABFT_AUTO) mode = select_mode(pr.M, pr.N, pr.K, pr.dtype);
    const int cfg = pick_cfg(pr.M, pr.N, pr.K, pr.dtype, a_vectorisable(pr) && b_vectorisable(pr), mode, pr.conv);
    const int bk = cfg_info_host(cfg).bk_bytes / esize(pr.dtype);
    if (f.row < 0 || f.row >= pr.M || f.col < 0 || f.col >= pr.N || f.bit < 0 || f.bit > 31 || f.k_after < -2) return false;
    return f.k_after < 0 || (f.k_after != 0 && f.k_after % bk == 0 && f.k_after < pr.K);
}

// A product ready to be launched
struct Prepared {
    GemmArgs g;
    int cfg, kmode, dtype;   // kmode: the kernels' scheme index
    bool inj, skinny, shallow;
};

// Everything of a product up to its kernel's launch: checks, tiling, kernel arguments, and the launches that
// come before it (weight checksums that were not handed in, a pass over A of its own).
int prepare_problem(const Problem& pr, int mode, const void* beta, void* workspace, size_t ws_bytes, uint32_t* flag,
                    abft_report_t* report, const abft_fault_t* inject, hipStream_t st, Prepared& out) {
    int rc = validate_common(pr, mode, flag);
    if (rc != ABFT_OK) return rc;
    if (mode == ABFT_AUTO) mode = select_mode(pr.M, pr.N, pr.K, pr.dtype);
    // the weighted checks are the global scheme with two more checksum pairs
    const bool weighted = mode == ABFT_GLOBAL_WEIGHTED;
    if (weighted) mode = ABFT_GLOBAL;

    const bool avec = a_vectorisable(pr), bvec = b_vectorisable(pr);
    const bool all16 = avec && bvec;
    const int cfg = pr.run_seg ? (int)CFG_R64 : pick_cfg(pr.M, pr.N, pr.K, pr.dtype, all16, mode, pr.conv);
    const CfgInfo ci = cfg_info_host(cfg);
    const int bk = ci.bk_bytes / esize(pr.dtype);

    GemmArgs& g = out.g;
    std::memset(&g, 0, sizeof g);
    g.A = reinterpret_cast<const char*>(pr.A);
    g.B = reinterpret_cast<const char*>(pr.B);
    g.C = reinterpret_cast<char*>(pr.C);
    g.M = pr.M; g.N = pr.N; g.K = pr.K;
    g.lda = pr.lda; g.ldb = pr.ldb; g.ldc = pr.ldc;
    g.b_sn = pr.b_layout == ABFT_B_NK ? pr.ldb : 1;
    g.b_sk = pr.b_layout == ABFT_B_NK ? 1 : pr.ldb;
    g.a_vec = avec; g.b_vec = bvec;
    g.conv = pr.conv ? 1 : 0;
    if (pr.conv) {
        g.imgpitch = pr.imgpitch; g.rowpitch = pr.rowpitch; g.pix = pr.pix;
        g.H = pr.cg.H; g.W = pr.cg.W; g.Cin = pr.cg.Cin; g.KH = pr.cg.KH; g.KW = pr.cg.KW;
        g.stride = pr.cg.stride; g.pad = pr.cg.pad; g.OH = pr.OH; g.OW = pr.OW;
    }
    // (they ride in spare columns of the streaming kernel's extra matrix operand: latency-bound
    // products with fp16 or int8 operands)
    if (weighted && (!cfg_is_stream(cfg) || pr.dtype == ABFT_BF16)) return ABFT_E_UNSUPPORTED;
    if (cfg == CFG_R64 && strip_fits(pr, pr.K, pr.run_seg, g.strip_rows, g.strip_pitch)) g.strip_seg = pr.run_seg;
    g.tiles_m = (int)cdiv(pr.M, ci.bm);
    g.tiles_n = (int)cdiv(pr.N, ci.bn);
    g.flag = flag;
    g.act = pr.act;
    g.row_scale = pr.row_scale; g.col_scale = pr.col_scale; g.bias = pr.bias;
    g.report = reinterpret_cast<Report*>(report);
    const int tol_K = pr.tol_K > 0 ? pr.tol_K : pr.K;
    g.tol_coeff = tol_coeff(tol_K, pr.dtype, mode) + tol_half_coeff(pr.dtype, mode, ci.wm, ci.wn, cfg == CFG_G16 ? 16 : 32);
    g.f_row = g.f_col = -1; g.f_bit = 0; g.f_kt = -1;
    // (the streaming kernel stores through an epilogue of its own, the 16-row shapes hold other rows per lane)
    if (pr.alpha_out && pr.dtype != ABFT_I8 && !cfg_is_stream(cfg) && cfg != CFG_G16) {
        g.alpha_out = pr.alpha_out;
        g.ld_alpha_out = pr.ld_alpha_out;
        if (pr.alpha_emitted) *pr.alpha_emitted = true;
    }

    bool inj = false;
    if (inject) {
        if (inject->row < 0 || inject->row >= pr.M || inject->col < 0 || inject->col >= pr.N) return ABFT_E_INJECT;
        if (inject->bit < 0 || inject->bit > 31) return ABFT_E_INJECT;
        if (inject->k_after < -2) return ABFT_E_INJECT;
        if (inject->k_after >= 0) {
            if (inject->k_after == 0 || inject->k_after % bk != 0 || inject->k_after >= pr.K) return ABFT_E_INJECT;
            g.f_kt = inject->k_after / bk - 1;
        }
        // -2: the finished value after the partial tiles of several wavefronts have been added (the
        // streaming configurations); the same as -1 where one wavefront forms the whole sum
        if (inject->k_after == -2 && ci.kways > 1) g.f_kt = -2;
        g.f_row = (int)inject->row; g.f_col = (int)inject->col; g.f_bit = inject->bit;
        inj = true;
    }

    WsLayout w;
    std::memset(&w, 0, sizeof w);
    int kmode = mode;  // the kernels' scheme index
    char* ws = reinterpret_cast<char*>(workspace);
    const void* beta_used = beta;
    if (mode == ABFT_GLOBAL) {
        w = ws_layout(pr.M, pr.N, pr.K, cfg);
        if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < w.total) return ABFT_E_WORKSPACE;
        g.tol_l1 = tol_bias_coeff(tol_K, pr.dtype, mode);
        if (!beta_used) {
            if (launch_weight_checksum(pr.K, pr.N, pr.B, pr.ldb, pr.b_layout, pr.dtype, ci.bn, ws + w.off_beta,
                                       st) != hipSuccess)
                return ABFT_E_HIP;
            beta_used = ws + w.off_beta;
        }
        if (weighted) kmode = MODE_GLOBAL_W;
        // (not on the eight-wavefront 128 x 128 tile: its wavefront tiles are so small that the sums' ring
        // costs more than the in-loop form: 46 against 44.5 us at 1024 x 4096 x 4096)
        if (pr.alpha_in && !weighted && !pr.conv && pr.dtype != ABFT_I8 && ci.fast && ci.kways == 1 && cfg != CFG_F128E) {
            // steps 1-2 were the previous layer's: its epilogue left the column sums of this
            // layer's A per 32-row block; one multiplication per lane and k tile is all that is left
            kmode = MODE_GLOBAL_FED;
            g_handover_launches.fetch_add(1, std::memory_order_relaxed);
            g.alpha_in = pr.alpha_in;
            g.beta_k = reinterpret_cast<const char*>(beta_used) + beta_k_offset(pr.K, g.tiles_n);
        } else if (fused_global(pr, ci)) {
            // the direct-to-LDS kernel forms the activation checksum's dot product with the weight
            // checksums itself, from the A tiles it multiplies (steps 1-3 inside the product's loop)
            g.beta_k = reinterpret_cast<const char*>(beta_used) + beta_k_offset(pr.K, g.tiles_n);
            g.beta_p = reinterpret_cast<const char*>(beta_used) + beta_p_offset(pr.K, g.tiles_n);
            g.beta_r = reinterpret_cast<const char*>(beta_used) + beta_r_offset(pr.K, g.tiles_n);
        } else {
            kmode = MODE_GLOBAL_PRE;
            g.partial_dots = ws + w.off_pd;
            g.n_parts = pre_grid_x(pr.K, pr.dtype) * (ci.bm / pre_rows_per_block(ci.bm, pr.M, pr.K));
            // steps 1-2: activation checksum of every row block of the tiling and its partial dot
            // products with the weight checksums
            if (launch_act_checksum(pr, nullptr, ci.bm, beta_used, g.tiles_n, ws + w.off_pd, st) != hipSuccess)
                return ABFT_E_HIP;
        }
    }

    out.cfg = cfg;
    out.kmode = kmode;
    out.dtype = pr.dtype;
    out.inj = inj;
    const long long blocks = (long long)g.tiles_m * g.tiles_n;
    out.shallow = !inj && !g.alpha_out && !pr.row_scale && shallow_takes(pr, cfg, mode) && blocks <= 512 &&
                  (long long)pr.K * esize(pr.dtype) <= (blocks > 256 && rows_off_dwords(g, pr.dtype) ? 64 : 96);
    out.skinny = !g.alpha_out && skinny_takes(pr, cfg, mode);
    if (out.skinny) {
        // (its k tiles are of 128 bytes; a planted fault lands in the share of the tiling's shares that it names)
        if (g.f_kt >= 0) g.f_kt = (g.f_kt + 1) * (ci.bk_bytes / 128) - 1;
        if (g.f_kt == -1 && ci.kways == 1) g.f_kt = -2;
        g.n_parts = ci.kways;
    }
    return ABFT_OK;
}

int run_problem(const Problem& pr, int mode, const void* beta, void* workspace, size_t ws_bytes, uint32_t* flag,
                abft_report_t* report, const abft_fault_t* inject, hipStream_t st) {
    Prepared w;
    const int rc = prepare_problem(pr, mode, beta, workspace, ws_bytes, flag, report, inject, st, w);
    if (rc != ABFT_OK) return rc;
    hipError_t e;
    if (g_ev_start && hipEventRecord(g_ev_start, st) != hipSuccess) return ABFT_E_HIP;
    if (pr.row_scale) {
        const bool f16 = pr.out_dtype == ABFT_F16;
        if (w.skinny) e = (f16 ? launch_scaled_skinny_f16 : launch_scaled_skinny_bf16)(w.kmode, rows_off_dwords(w.g, w.dtype), cfg_info_host(w.cfg).wn, w.g, st);
        else e = f16 ? launch_scaled_f16(w.cfg, w.kmode, w.inj, w.g, st) : launch_scaled_bf16(w.cfg, w.kmode, w.inj, w.g, st);
    } else if (w.skinny) {
        const int columns = cfg_info_host(w.cfg).wn;
        e = w.dtype == ABFT_F16    ? launch_skinny_f16(w.kmode, rows_off_dwords(w.g, w.dtype), columns, w.g, st)
            : w.dtype == ABFT_BF16 ? launch_skinny_bf16(w.kmode, rows_off_dwords(w.g, w.dtype), columns, w.g, st)
                                   : launch_skinny_i8(w.kmode, rows_off_dwords(w.g, w.dtype), columns, w.g, st);
    } else if (w.shallow) {
        e = w.dtype == ABFT_F16    ? launch_shallow_f16(w.kmode, rows_off_dwords(w.g, w.dtype), w.g, st)
            : w.dtype == ABFT_BF16 ? launch_shallow_bf16(w.kmode, rows_off_dwords(w.g, w.dtype), w.g, st)
                                   : launch_shallow_i8(w.kmode, rows_off_dwords(w.g, w.dtype), w.g, st);
    } else if (w.dtype == ABFT_F16) e = launch_gemm_f16(w.cfg, w.kmode, w.inj, w.g, st);
    else if (w.dtype == ABFT_BF16) e = launch_gemm_bf16(w.cfg, w.kmode, w.inj, w.g, st);
    else e = launch_gemm_i8(w.cfg, w.kmode, w.inj, w.g, st);
    if (e != hipSuccess) return ABFT_E_HIP;
    if (g_ev_stop && hipEventRecord(g_ev_stop, st) != hipSuccess) return ABFT_E_HIP;

    return ABFT_OK;
}

int conv_problem(const abft_conv_t* conv, int N, Problem& pr) {
    if (!conv) return ABFT_E_NULL;
    if (conv->batch <= 0 || conv->H <= 0 || conv->W <= 0 || conv->Cin <= 0 || conv->KH <= 0 || conv->KW <= 0 ||
        conv->stride <= 0 || conv->pad < 0)
        return ABFT_E_SHAPE;
    if (conv->H + 2 * conv->pad < conv->KH || conv->W + 2 * conv->pad < conv->KW) return ABFT_E_SHAPE;
    pr.conv = true;
    pr.cg = *conv;
    pr.OH = conv_out(conv->H, conv->KH, conv->stride, conv->pad);
    pr.OW = conv_out(conv->W, conv->KW, conv->stride, conv->pad);
    long long M = (long long)conv->batch * pr.OH * pr.OW;
    long long K = (long long)conv->KH * conv->KW * conv->Cin;
    if (M <= 0 || M > 0x7fffffffLL || K > 0x7fffffffLL) return ABFT_E_SHAPE;
    pr.M = (int)M;
    pr.K = (int)K;
    pr.N = N;
    pr.lda = pr.K;
    pr.pix = conv->Cin;
    pr.rowpitch = (long long)conv->W * conv->Cin;
    pr.imgpitch = pr.rowpitch * conv->H;
    // a 1 x 1 filter at stride 1 without padding is the plain product on the NHWC tensor read as
    // an M x Cin matrix
    if (conv->KH == 1 && conv->KW == 1 && conv->stride == 1 && conv->pad == 0) {
        pr.conv = false;
        pr.lda = conv->Cin;
    }
    return ABFT_OK;
}

// Lowering of a convolution with few input channels to row segments (see conv_pad_kernel).
struct ConvLowering {
    bool ok;
    int seg, segp, Kp, Hp;
    long long rowp;
    size_t xp_bytes, bp_bytes;
};
ConvLowering conv_lowering(const Problem& pr) {
    ConvLowering lw;
    std::memset(&lw, 0, sizeof lw);
    if (!pr.conv) return lw;
    const abft_conv_t& c = pr.cg;
    const int es = esize(pr.dtype), epc = 16 / es;
    if ((c.Cin * es) % 16 == 0) return lw;                      // chunks already line up with the channels
    if ((long long)c.KW * c.Cin > 64) return lw;                // long runs gain little
    if (((long long)c.stride * c.Cin * es) % 4 != 0) return lw;  // chunk addresses must be 4-byte aligned
    lw.seg = c.KW * c.Cin;
    lw.segp = (int)align_up((size_t)lw.seg, (size_t)epc);
    // whole k tiles of 128 bytes, so that the direct-to-LDS kernel applies (the tail multiplies
    // input rows below the window, or zeros, with zero weights)
    lw.Kp = (int)align_up((size_t)c.KH * lw.segp, (size_t)(128 / es));
    lw.Hp = c.H + 2 * c.pad;
    const long long need = std::max((long long)(c.W + 2 * c.pad) * c.Cin,
                                    (long long)(pr.OW - 1) * c.stride * c.Cin + lw.segp);
    lw.rowp = (long long)align_up((size_t)need, (size_t)epc);
    lw.xp_bytes = align_up((size_t)c.batch * lw.Hp * lw.rowp * es, 256);
    lw.bp_bytes = align_up((size_t)pr.N * lw.Kp * es, 256);
    lw.ok = true;
    return lw;
}


// bytes of workspace that let a convolution run lowered: the lowered product's own scratch, the
// padded input, the re-ordered weights
size_t lowered_workspace_bytes(const Problem& pr, const ConvLowering& lw, int mode) {
    return align_up(plain_workspace_bytes(pr.M, pr.N, lw.Kp, pr.dtype, mode), 256) + lw.xp_bytes + lw.bp_bytes;
}

// Weights of a lowered convolution prepared ahead of the call (a plan does this once, offline:
// the weights are known before inference, Sec. 2.1): the re-ordered N x Kp matrix and, for the
// global scheme, its weight checksums per block of beta_block_n columns.
struct LoweredWeights {
    const void* bp;
    const void* beta;
    int beta_block_n;
};

hipError_t launch_conv_weights(const Problem& pr, const ConvLowering& lw, char* bp, hipStream_t st) {
    const long long sn = pr.b_layout == ABFT_B_NK ? pr.ldb : 1, sk = pr.b_layout == ABFT_B_NK ? 1 : pr.ldb;
    dim3 grid((unsigned)cdiv((long long)pr.N * lw.Kp, 256)), block(256);
    if (esize(pr.dtype) == 2)
        hipLaunchKernelGGL(conv_weights_kernel<2>, grid, block, 0, st, reinterpret_cast<const char*>(pr.B), sn, sk, bp,
                           pr.N, lw.Kp, lw.segp, lw.seg, pr.cg.KH);
    else
        hipLaunchKernelGGL(conv_weights_kernel<1>, grid, block, 0, st, reinterpret_cast<const char*>(pr.B), sn, sk, bp,
                           pr.N, lw.Kp, lw.segp, lw.seg, pr.cg.KH);
    return hipGetLastError();
}

// the lowered product of a convolution: same C, k re-ordered as (filter row, padded run)
Problem lowered_problem(const Problem& pr, const ConvLowering& lw, const void* xp, const void* bp) {
    const abft_conv_t& c = pr.cg;
    Problem q = pr;
    q.A = xp;
    q.B = bp;
    q.b_layout = ABFT_B_NK;
    q.ldb = lw.Kp;
    q.K = lw.Kp;
    q.lda = lw.Kp;
    q.tol_K = pr.K;
    q.cg.H = lw.Hp;
    q.cg.W = (pr.OW - 1) * c.stride + 1;  // every window start lies inside the padded row
    q.cg.Cin = lw.segp;
    q.cg.KW = 1;
    q.cg.pad = 0;
    q.pix = c.Cin;
    q.rowpitch = lw.rowp;
    q.imgpitch = lw.rowp * lw.Hp;
    return q;
}

// Does the strip kernel take a lowered convolution?  Where its input rows fit LDS: under the schemes whose other tiles
// check C in the same pieces, so that what is reported of them stays (32 rows by all of at most 64 columns: the row-streaming
// kernel, and the 64 x 128 and 128 x 128 tiles of 32 x 128 per wavefront; sums in the operand type have a tolerance by
// the nominal tile and stay on those), and unprotected wherever the product fills more than streaming tiles.
bool lowered_on_strips(const Problem& pr, const ConvLowering& lw, int mode) {
    int rows, pitch;
    if (mode == ABFT_GLOBAL || mode == ABFT_GLOBAL_WEIGHTED || !strip_fits(pr, lw.Kp, lw.segp, rows, pitch)) return false;
    const int cfg = pick_cfg(pr.M, pr.N, lw.Kp, pr.dtype, true, mode, true);
    if (cfg == CFG_R64) return true;
    if (mode == ABFT_NONE) return !cfg_is_stream(cfg) && !cfg_is_generic(cfg);
    return (mode == ABFT_THREAD || mode == ABFT_REPLICA) && (cfg == CFG_F64T || cfg == CFG_F128T);
}

// a convolution: lowered to row segments when it qualifies and the workspace has the room.
// A fault planted in a running accumulator (k_after >= 0) counts k in the order of abft_conv_t,
// which the lowered product does not keep: such a call runs unlowered.
int run_conv(const Problem& pr, int mode, const void* beta, void* workspace, size_t ws_bytes, uint32_t* flag,
             abft_report_t* report, const abft_fault_t* inject, hipStream_t st, const LoweredWeights* pre = nullptr) {
    const int rc = validate_common(pr, mode, flag);
    if (rc != ABFT_OK) return rc;
    if (mode == ABFT_AUTO) mode = select_mode(pr.M, pr.N, pr.K, pr.dtype);
    const ConvLowering lw = conv_lowering(pr);
    const size_t own_weights = pre ? 0 : lw.bp_bytes;
    if (!lw.ok || (inject && inject->k_after >= 0) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
        ws_bytes < lowered_workspace_bytes(pr, lw, mode) - (lw.bp_bytes - own_weights))
        return run_problem(pr, mode, beta, workspace, ws_bytes, flag, report, inject, st);
    const abft_conv_t& c = pr.cg;
    const int es = esize(pr.dtype);
    const size_t inner = align_up(plain_workspace_bytes(pr.M, pr.N, lw.Kp, pr.dtype, mode), 256);
    char* xp = reinterpret_cast<char*>(workspace) + inner;
    char* bp = xp + lw.xp_bytes;
    if (lowered_on_strips(pr, lw, mode)) {
        // the lowered weights on the input as it is, without the padded copy
        if (!pre && launch_conv_weights(pr, lw, bp, st) != hipSuccess) return ABFT_E_HIP;
        Problem q = pr;
        q.B = pre ? pre->bp : bp;
        q.b_layout = ABFT_B_NK;
        q.ldb = q.K = q.lda = lw.Kp;
        q.tol_K = pr.K;
        q.run_seg = lw.segp;
        return run_problem(q, mode, nullptr, workspace, inner, flag, report, inject, st);
    }
    {
        const long long chunks_per_row = lw.rowp / (16 / es);
        const long long total = (long long)c.batch * lw.Hp * chunks_per_row;
        dim3 grid((unsigned)cdiv(total, 256)), block(256);
        if (es == 2)
            hipLaunchKernelGGL(conv_pad_kernel<2>, grid, block, 0, st, reinterpret_cast<const char*>(pr.A), xp, c.H,
                               c.W * c.Cin, c.pad, c.pad * c.Cin, lw.Hp, lw.rowp, chunks_per_row, total);
        else
            hipLaunchKernelGGL(conv_pad_kernel<1>, grid, block, 0, st, reinterpret_cast<const char*>(pr.A), xp, c.H,
                               c.W * c.Cin, c.pad, c.pad * c.Cin, lw.Hp, lw.rowp, chunks_per_row, total);
        if (hipGetLastError() != hipSuccess) return ABFT_E_HIP;
        if (!pre && launch_conv_weights(pr, lw, bp, st) != hipSuccess) return ABFT_E_HIP;
    }
    const Problem q = lowered_problem(pr, lw, xp, pre ? pre->bp : bp);
    // offline weight checksums of the lowered weights fit only the tiling they were made for
    const void* qbeta = nullptr;
    if (pre && pre->beta && mode == ABFT_GLOBAL) {
        const int bn_now = cfg_info_host(pick_cfg(q.M, q.N, q.K, q.dtype, a_vectorisable(q) && b_vectorisable(q), ABFT_GLOBAL)).bn;
        if (bn_now == pre->beta_block_n) qbeta = pre->beta;
    }
    return run_problem(q, mode, qbeta, workspace, inner, flag, report, inject, st);
}

size_t plain_workspace_bytes(int M, int N, int K, int dtype, int mode) {
    if (mode == ABFT_AUTO) mode = select_mode(M, N, K, dtype);
    // only the global scheme keeps anything outside the operands
    return (mode == ABFT_GLOBAL || mode == ABFT_GLOBAL_WEIGHTED) ? ws_bytes_any_cfg(M, N, K) : 0;
}

}  // namespace

// ------------------------------------------------------------------------- //
// plans
// ------------------------------------------------------------------------- //
struct abft_plan {
    struct Layer {
        abft_layer_t desc;
        int mode;
        void* beta;       // per-column-block weight checksums, blocks of beta_block_n columns
        int beta_block_n;
        void* workspace;
        size_t ws_bytes;
        double t_us[3];
        int act;          // abft_act_t applied to the stored output
        // a convolution that runs lowered to row segments: its re-ordered weights and their
        // checksums, made once at creation
        void* lowered_B;
        void* lowered_beta;
        int lowered_block_n;
        // a fully-connected layer that can run inside a chain of layers in one launch
        // (abft_plan_run_chain): weight checksums per block of 32 columns, its tiling there
        void* chain_beta;
        // activation checksums of this layer's input, left by the layer before it in a chain run
        // layer by layer: ceil(M / 32) x K floats (fully-connected fp16 / bf16 layers)
        float* alpha32;
        // diagnostics block and planted fault (test hook) handed to every run of the layer
        abft_report_t* report;
        abft_fault_t fault;
        bool has_fault;
    };
    std::vector<Layer> layers;
    // completion flags and status word of the chain kernel (zero at creation; see mlp_chain.h)
    unsigned* chain_flags = nullptr;
    int chain_spin_limit = 1 << 20;

};

namespace {

// Can this layer run inside the chain kernel?  Fully connected, fp16 / bf16, weights with k
// contiguous and 16-byte aligned rows, K whole k tiles of 128 bytes.
bool chain_layer_ok(const abft_layer_t& d) {
    if (d.has_conv || d.dtype == ABFT_I8 || d.b_layout != ABFT_B_NK) return false;
    return ((long long)d.K * 2) % 128 == 0 && (d.ldb * 2) % 16 == 0 && aligned16(d.B);
}

}  // namespace

// ------------------------------------------------------------------------- //
// exported functions
// ------------------------------------------------------------------------- //
extern "C" {

int abft_gemm(int M, int N, int K, const void* A, int64_t lda, const void* B, int64_t ldb, int b_layout, void* C,
              int64_t ldc, int dtype, int mode, const void* beta, void* workspace, size_t workspace_bytes,
              uint32_t* fault_flag, abft_report_t* report, const abft_fault_t* inject, void* stream) {
    Problem pr;
    std::memset(&pr, 0, sizeof pr);
    pr.M = M; pr.N = N; pr.K = K; pr.dtype = dtype; pr.b_layout = b_layout;
    pr.A = A; pr.lda = lda; pr.B = B; pr.ldb = ldb; pr.C = C; pr.ldc = ldc;
    pr.conv = false;
    return run_problem(pr, mode, beta, workspace, workspace_bytes, fault_flag, report, inject,
                       reinterpret_cast<hipStream_t>(stream));
}

int abft_gemm_static(int M, int N, int K, const void* A, int64_t lda, const void* B, int64_t ldb, int b_layout,
                     void* C, int64_t ldc, int dtype, int mode, const void* beta, uint32_t* fault_flag,
                     abft_report_t* report, const abft_fault_t* inject, void* stream) {
    Problem pr;
    std::memset(&pr, 0, sizeof pr);
    pr.M = M; pr.N = N; pr.K = K; pr.dtype = dtype; pr.b_layout = b_layout;
    pr.A = A; pr.lda = lda; pr.B = B; pr.ldb = ldb; pr.C = C; pr.ldc = ldc;
    pr.conv = false;
    void* scratch = scratch_of_current_device();
    if (!scratch) return ABFT_E_HIP;
    // (a product whose scratch does not fit comes back as ABFT_E_WORKSPACE before anything is launched)
    return run_problem(pr, mode, beta, scratch, STATIC_SCRATCH_BYTES, fault_flag, report, inject,
                       reinterpret_cast<hipStream_t>(stream));
}

int abft_quantize_rows(int M, int K, const void* X, int64_t ldx, int dtype, void* Q, int64_t ldq, float* scale, void* stream) {
    const int rc = validate_quantize(M, K, X, ldx, dtype);
    if (rc != ABFT_OK) return rc;
    if (!Q || !scale) return ABFT_E_NULL;
    if (ldq < K) return ABFT_E_LD;
    return quantize_rows(M, K, X, ldx, dtype, Q, ldq, scale, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? ABFT_OK : ABFT_E_HIP;
}

int abft_gemm_scaled(int M, int N, int K, const void* A, int64_t lda, const float* row_scale, const void* B, int64_t ldb, int b_layout,
                     const float* col_scale, const float* bias, int act, void* C, int64_t ldc, int out_dtype, int mode, const void* beta,
                     void* workspace, size_t workspace_bytes, uint32_t* fault_flag, abft_report_t* report, const abft_fault_t* inject,
                     void* stream) {
    Problem pr;
    const int rc = scaled_problem(M, N, K, A, lda, row_scale, B, ldb, b_layout, col_scale, bias, act, C, ldc, out_dtype, mode, fault_flag, pr);
    if (rc != ABFT_OK) return rc;
    return run_problem(pr, mode, beta, workspace, workspace_bytes, fault_flag, report, inject, reinterpret_cast<hipStream_t>(stream));
}

int abft_scaled_select(int M, int N, int K, int aligned) {
    if (M <= 0 || N <= 0 || K <= 0) return ABFT_E_SHAPE;
    return scaled_select(M, N, K, aligned != 0);
}

size_t abft_linear_scaled_workspace_bytes(int M, int N, int K, int mode) {
    if (M <= 0 || N <= 0 || K <= 0) return 0;
    // (whatever the alignment will be)
    if (mode == ABFT_AUTO) mode = scaled_select(M, N, K, true) == ABFT_GLOBAL ? ABFT_GLOBAL : scaled_select(M, N, K, false);
    return linear_product_offset(M, K) + plain_workspace_bytes(M, N, K, ABFT_I8, mode);
}

int abft_linear_scaled(int M, int N, int K, const void* X, int64_t ldx, int dtype, const void* B, int64_t ldb, int b_layout,
                       const float* col_scale, const float* bias, int act, void* C, int64_t ldc, int mode, const void* beta,
                       void* workspace, size_t workspace_bytes, uint32_t* fault_flag, abft_report_t* report, const abft_fault_t* inject,
                       void* stream) {
    int rc = validate_quantize(M, K, X, ldx, dtype);
    if (rc != ABFT_OK) return rc;
    const hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    char* const ws = reinterpret_cast<char*>(workspace);
    const size_t product = linear_product_offset(M, K);
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || workspace_bytes < product) return ABFT_E_WORKSPACE;
    float* const row_scale = reinterpret_cast<float*>(ws + linear_scale_offset(M, K));
    Problem pr;
    rc = scaled_problem(M, N, K, ws, linear_ld(K), row_scale, B, ldb, b_layout, col_scale, bias, act, C, ldc, dtype, mode, fault_flag, pr);
    if (rc != ABFT_OK) return rc;
    // (everything that can be refused is, before the first launch)
    const size_t left = workspace_bytes - product;
    if (left < plain_workspace_bytes(M, N, K, ABFT_I8, mode)) return ABFT_E_WORKSPACE;
    if (inject && !inject_in_range(pr, mode, *inject)) return ABFT_E_INJECT;
    if (skinny_few_fits(M, K) && mode != ABFT_GLOBAL && !report && !inject) {
        // one launch where the product's kernel can quantise the few rows itself
        Prepared w;
        rc = prepare_problem(pr, mode, nullptr, nullptr, 0, fault_flag, nullptr, nullptr, st, w);
        if (rc != ABFT_OK) return rc;
        if (w.skinny) {
            const bool bytes = rows_off_dwords(w.g, ABFT_I8);
            w.g.A = reinterpret_cast<const char*>(X);
            w.g.lda = ldx;
            if (g_ev_start && hipEventRecord(g_ev_start, st) != hipSuccess) return ABFT_E_HIP;
            if ((dtype == ABFT_F16 ? launch_scaled_few_f16 : launch_scaled_few_bf16)(w.kmode, bytes, w.g, st) != hipSuccess) return ABFT_E_HIP;
            if (g_ev_stop && hipEventRecord(g_ev_stop, st) != hipSuccess) return ABFT_E_HIP;
            return ABFT_OK;
        }
    }
    if (quantize_rows(M, K, X, ldx, dtype, ws, linear_ld(K), row_scale, st) != hipSuccess) return ABFT_E_HIP;
    return run_problem(pr, mode, beta, left ? ws + product : nullptr, left, fault_flag, report, inject, st);
}

size_t abft_static_scratch_bytes(void) { return STATIC_SCRATCH_BYTES; }

int abft_conv(const abft_conv_t* conv, int N, const void* x, const void* B, int64_t ldb, int b_layout, void* C,
              int64_t ldc, int dtype, int mode, const void* beta, void* workspace, size_t workspace_bytes,
              uint32_t* fault_flag, abft_report_t* report, const abft_fault_t* inject, void* stream) {
    Problem pr;
    std::memset(&pr, 0, sizeof pr);
    if (N <= 0) return ABFT_E_SHAPE;
    int rc = conv_problem(conv, N, pr);
    if (rc != ABFT_OK) return rc;
    pr.dtype = dtype; pr.b_layout = b_layout;
    pr.A = x; pr.B = B; pr.ldb = ldb; pr.C = C; pr.ldc = ldc;
    return run_conv(pr, mode, beta, workspace, workspace_bytes, fault_flag, report, inject,
                    reinterpret_cast<hipStream_t>(stream));
}

size_t abft_workspace_bytes(int M, int N, int K, int dtype, int mode) {
    if (M <= 0 || N <= 0 || K <= 0 || !valid_dtype(dtype)) return 0;
    return plain_workspace_bytes(M, N, K, dtype, mode);
}

size_t abft_conv_workspace_bytes(const abft_conv_t* conv, int N, int dtype, int mode) {
    Problem pr;
    std::memset(&pr, 0, sizeof pr);
    if (N <= 0 || !valid_dtype(dtype) || conv_problem(conv, N, pr) != ABFT_OK) return 0;
    pr.dtype = dtype;
    if (mode == ABFT_AUTO) mode = select_mode(pr.M, pr.N, pr.K, dtype);
    const ConvLowering lw = conv_lowering(pr);
    const size_t plain = plain_workspace_bytes(pr.M, pr.N, pr.K, dtype, mode);
    return lw.ok ? std::max(plain, lowered_workspace_bytes(pr, lw, mode)) : plain;
}

size_t abft_beta_bytes(int K, int N, int block_n) {
    if (K <= 0 || N <= 0) return 0;
    if (block_n <= 0 || block_n > N) block_n = N;
    return beta_total_bytes(K, (int)cdiv(N, block_n));
}

int abft_weight_checksum(int K, int N, const void* B, int64_t ldb, int b_layout, int dtype, int block_n,
                         void* beta, void* stream) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (b_layout != ABFT_B_NK && b_layout != ABFT_B_KN) return ABFT_E_ENUM;
    if (K <= 0 || N <= 0) return ABFT_E_SHAPE;
    if (!B || !beta) return ABFT_E_NULL;
    if (b_layout == ABFT_B_NK ? ldb < K : ldb < N) return ABFT_E_LD;
    return launch_weight_checksum(K, N, B, ldb, b_layout, dtype, block_n, beta,
                                  reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? ABFT_OK
               : ABFT_E_HIP;
}

int abft_activation_checksum(int M, int K, const void* A, int64_t lda, const abft_conv_t* conv, int dtype,
                             void* alpha, void* stream) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (!A || !alpha) return ABFT_E_NULL;
    Problem pr;
    std::memset(&pr, 0, sizeof pr);
    pr.dtype = dtype;
    if (conv) {
        int rc = conv_problem(conv, 1, pr);
        if (rc != ABFT_OK) return rc;
        if (pr.M != M || pr.K != K) return ABFT_E_SHAPE;
    } else {
        if (M <= 0 || K <= 0) return ABFT_E_SHAPE;
        if (lda < K) return ABFT_E_LD;
        pr.M = M; pr.K = K; pr.lda = lda;
    }
    pr.A = A;
    // one slab covering every row: the plain 1 x K checksum
    return launch_act_checksum(pr, alpha, M, nullptr, 0, nullptr, reinterpret_cast<hipStream_t>(stream)) == hipSuccess
               ? ABFT_OK
               : ABFT_E_HIP;
}

int abft_k_ways(int M, int N, int K, int dtype, int aligned, int mode, int* ways, int* step) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (M <= 0 || N <= 0 || K <= 0) return ABFT_E_SHAPE;
    if (mode == ABFT_AUTO) mode = select_mode(M, N, K, dtype);
    const CfgInfo ci = cfg_info_host(pick_cfg(M, N, K, dtype, aligned != 0, mode));
    if (ways) *ways = ci.kways;
    if (step) *step = ci.kway_bytes / esize(dtype);
    return ABFT_OK;
}

const char* abft_kernel_name(int M, int N, int K, int dtype, int aligned, int mode, int conv) {
    if (!valid_dtype(dtype) || M <= 0 || N <= 0 || K <= 0 || mode < ABFT_NONE || mode > ABFT_GLOBAL_WEIGHTED) return nullptr;
    if (mode == ABFT_AUTO) mode = select_mode(M, N, K, dtype);
    return cfg_name(pick_cfg(M, N, K, dtype, aligned != 0, mode, conv != 0));
}

double abft_arithmetic_intensity(int M, int N, int K, int dtype) {
    if (M <= 0 || N <= 0 || K <= 0 || !valid_dtype(dtype)) return 0.0;
    return intensity(M, N, K, dtype);
}

double abft_cmr(int dtype) { return valid_dtype(dtype) ? cmr_of(dtype) : 0.0; }

void abft_set_cmr(int dtype, double value) {
    if (valid_dtype(dtype)) g_cmr_override[dtype] = value > 0.0 ? value : 0.0;
}

int abft_select(int M, int N, int K, int dtype) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (M <= 0 || N <= 0 || K <= 0) return ABFT_E_SHAPE;
    return select_mode(M, N, K, dtype);
}

int abft_tile_shape(int M, int N, int K, int dtype, int aligned, int* tile_m, int* tile_n, int* k_step) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (M <= 0 || N <= 0 || K <= 0) return ABFT_E_SHAPE;
    CfgInfo ci = cfg_info_host(pick_cfg(M, N, K, dtype, aligned != 0, ABFT_THREAD));
    if (tile_m) *tile_m = ci.wm;
    if (tile_n) *tile_n = ci.wn;
    if (k_step) *k_step = ci.bk_bytes / esize(dtype);
    return ABFT_OK;
}

int abft_region_shape(int M, int N, int K, int dtype, int aligned, int* region_m, int* region_n) {
    if (!valid_dtype(dtype)) return ABFT_E_ENUM;
    if (M <= 0 || N <= 0 || K <= 0) return ABFT_E_SHAPE;
    CfgInfo ci = cfg_info_host(pick_cfg(M, N, K, dtype, aligned != 0, ABFT_GLOBAL));
    if (region_m) *region_m = ci.bm;
    if (region_n) *region_n = ci.bn;
    return ABFT_OK;
}

double abft_tolerance_coeff(int K, int dtype, int mode) {
    if (!valid_dtype(dtype) || K <= 0) return 0.0;
    return tol_coeff(K, dtype, mode);
}

double abft_tolerance_half_coeff(int dtype, int mode, int tile_m, int tile_n) {
    if (!valid_dtype(dtype) || tile_m <= 0 || tile_n <= 0) return 0.0;
    return tol_half_coeff(dtype, mode, tile_m, tile_n, tile_m < 32 ? 16 : 32);
}

double abft_tolerance_bias_coeff(int K, int dtype, int mode) {
    if (!valid_dtype(dtype) || K <= 0) return 0.0;
    return tol_bias_coeff(K, dtype, mode);
}

int abft_plan_create(abft_plan_t** plan, const abft_layer_t* layers, int n_layers, int profile, void* stream) {
    if (!plan || !layers) return ABFT_E_NULL;
    if (n_layers <= 0) return ABFT_E_SHAPE;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    abft_plan* p = new (std::nothrow) abft_plan;
    if (!p) return ABFT_E_HIP;
    int rc = ABFT_OK;
    for (int i = 0; i < n_layers && rc == ABFT_OK; ++i) {
        abft_plan::Layer L;
        std::memset(&L, 0, sizeof L);
        L.desc = layers[i];
        const abft_layer_t& d = L.desc;
        if (!valid_dtype(d.dtype)) { rc = ABFT_E_ENUM; break; }
        if (d.b_layout != ABFT_B_NK && d.b_layout != ABFT_B_KN) { rc = ABFT_E_ENUM; break; }
        if (d.M <= 0 || d.N <= 0 || d.K <= 0) { rc = ABFT_E_SHAPE; break; }
        if (!d.B) { rc = ABFT_E_NULL; break; }
        if (d.has_conv) {
            Problem pr;
            std::memset(&pr, 0, sizeof pr);
            rc = conv_problem(&d.conv, d.N, pr);
            if (rc != ABFT_OK) break;
            if (pr.M != d.M || pr.K != d.K) { rc = ABFT_E_SHAPE; break; }
        }
        L.mode = select_mode(d.M, d.N, d.K, d.dtype);
        // offline weight checksum and workspace for the global scheme (kept for either
        // choice so that profiling can time both)
        L.ws_bytes = ws_bytes_any_cfg(d.M, d.N, d.K);
        for (int md = ABFT_NONE; md <= ABFT_THREAD; ++md) {
            const size_t need = d.has_conv ? abft_conv_workspace_bytes(&d.conv, d.N, d.dtype, md)
                                           : abft_workspace_bytes(d.M, d.N, d.K, d.dtype, md);
            if (need > L.ws_bytes) L.ws_bytes = need;
        }
        {
            // the tiling the layer will run with when its activations are 16-byte aligned
            const int es = esize(d.dtype);
            const bool b16 = d.b_layout == ABFT_B_NK && aligned16(d.B) && (d.K * es) % 16 == 0 && (d.ldb * es) % 16 == 0;
            const bool a16 = d.has_conv ? (d.conv.Cin * es) % 16 == 0 : (d.K * es) % 16 == 0;
            L.beta_block_n = cfg_info_host(pick_cfg(d.M, d.N, d.K, d.dtype, a16 && b16, ABFT_GLOBAL)).bn;
        }
        if (hipMalloc(&L.beta, beta_total_bytes(d.K, (int)cdiv(d.N, L.beta_block_n))) != hipSuccess) { rc = ABFT_E_HIP; break; }
        if (hipMalloc(&L.workspace, L.ws_bytes) != hipSuccess) { (void)hipFree(L.beta); rc = ABFT_E_HIP; break; }
        p->layers.push_back(L);
        if (d.dtype != ABFT_I8 && (!d.has_conv || (d.conv.KH == 1 && d.conv.KW == 1 && d.conv.stride == 1 && d.conv.pad == 0))) {
            // (a layer that reads a plain M x K matrix can take its activation checksums from the layer before)
            abft_plan::Layer& PL = p->layers.back();
            if (hipMalloc(reinterpret_cast<void**>(&PL.alpha32), (size_t)cdiv(d.M, 32) * d.K * sizeof(float)) != hipSuccess) {
                rc = ABFT_E_HIP;
                break;
            }
        }
        if (chain_layer_ok(d)) {
            abft_plan::Layer& PL = p->layers.back();
            if (hipMalloc(&PL.chain_beta, beta_total_bytes(d.K, (int)cdiv(d.N, 32))) != hipSuccess ||
                launch_weight_checksum(d.K, d.N, d.B, d.ldb, d.b_layout, d.dtype, 32, PL.chain_beta, st) != hipSuccess) {
                rc = ABFT_E_HIP;
                break;
            }
        }
        if (d.has_conv) {
            // few input channels: the layer will run lowered to row segments; its weights are
            // re-ordered, and their checksums formed, here and now (offline, Sec. 2.5)
            Problem pr;
            std::memset(&pr, 0, sizeof pr);
            (void)conv_problem(&d.conv, d.N, pr);
            pr.dtype = d.dtype; pr.b_layout = d.b_layout; pr.B = d.B; pr.ldb = d.ldb;
            const ConvLowering lw = conv_lowering(pr);
            if (lw.ok) {
                abft_plan::Layer& PL = p->layers.back();
                PL.lowered_block_n = cfg_info_host(pick_cfg(d.M, d.N, lw.Kp, d.dtype, true, ABFT_GLOBAL)).bn;
                if (hipMalloc(&PL.lowered_B, lw.bp_bytes) != hipSuccess ||
                    hipMalloc(&PL.lowered_beta, beta_total_bytes(lw.Kp, (int)cdiv(d.N, PL.lowered_block_n))) != hipSuccess ||
                    launch_conv_weights(pr, lw, reinterpret_cast<char*>(PL.lowered_B), st) != hipSuccess ||
                    launch_weight_checksum(lw.Kp, d.N, PL.lowered_B, lw.Kp, ABFT_B_NK, d.dtype, PL.lowered_block_n,
                                           PL.lowered_beta, st) != hipSuccess) {
                    rc = ABFT_E_HIP;
                    break;
                }
            }
        }
        if (launch_weight_checksum(d.K, d.N, d.B, d.ldb, d.b_layout, d.dtype, L.beta_block_n, L.beta, st) !=
            hipSuccess) {
            rc = ABFT_E_HIP;
            break;
        }
    }
    if (rc == ABFT_OK) {
        const size_t bytes = (size_t)(CHAIN_FLAG_WORDS + 64) * sizeof(unsigned);
        if (hipMalloc(reinterpret_cast<void**>(&p->chain_flags), bytes) != hipSuccess ||
            hipMemsetAsync(p->chain_flags, 0, bytes, st) != hipSuccess)
            rc = ABFT_E_HIP;
    }
    if (rc == ABFT_OK && profile) {
        // pre-deployment profiling (Sec. 5.3): time each scheme on scratch inputs, keep the faster
        hipEvent_t e0, e1;
        uint32_t* d_flag = nullptr;
        if (hipEventCreate(&e0) != hipSuccess || hipEventCreate(&e1) != hipSuccess ||
            hipMalloc(&d_flag, 4) != hipSuccess)
            rc = ABFT_E_HIP;
        for (size_t i = 0; i < p->layers.size() && rc == ABFT_OK; ++i) {
            abft_plan::Layer& L = p->layers[i];
            const abft_layer_t& d = L.desc;
            size_t a_elems = d.has_conv ? (size_t)d.conv.batch * d.conv.H * d.conv.W * d.conv.Cin
                                        : (size_t)d.M * d.K;
            void *A = nullptr, *C = nullptr;
            if (hipMalloc(&A, a_elems * esize(d.dtype)) != hipSuccess) { rc = ABFT_E_HIP; break; }
            if (hipMalloc(&C, (size_t)d.M * d.N * csize(d.dtype)) != hipSuccess) { (void)hipFree(A); rc = ABFT_E_HIP; break; }
            (void)hipMemsetAsync(A, 0, a_elems * esize(d.dtype), st);
            (void)hipMemsetAsync(d_flag, 0, 4, st);
            const int modes[3] = {ABFT_NONE, ABFT_GLOBAL, ABFT_THREAD};
            for (int mi = 0; mi < 3 && rc == ABFT_OK; ++mi) {
                const int reps = 20;
                for (int r = -3; r < reps && rc == ABFT_OK; ++r) {
                    if (r == 0) (void)hipEventRecord(e0, st);
                    int saved = L.mode;
                    L.mode = modes[mi];
                    rc = abft_plan_run(p, (int)i, A, d.K, C, d.N, d_flag, stream);
                    L.mode = saved;
                }
                (void)hipEventRecord(e1, st);
                if (hipEventSynchronize(e1) != hipSuccess) rc = ABFT_E_HIP;
                float ms = 0.f;
                (void)hipEventElapsedTime(&ms, e0, e1);
                L.t_us[mi] = 1000.0 * ms / reps;
            }
            if (rc == ABFT_OK) L.mode = L.t_us[1] <= L.t_us[2] ? ABFT_GLOBAL : ABFT_THREAD;
            (void)hipFree(A);
            (void)hipFree(C);
        }
        if (d_flag) (void)hipFree(d_flag);
        (void)hipEventDestroy(e0);
        (void)hipEventDestroy(e1);
    }
    if (rc != ABFT_OK) {
        abft_plan_destroy(p);
        return rc;
    }
    *plan = p;
    return ABFT_OK;
}

}  // extern "C"

namespace {

// Does layer `next` of the plan, reading the M x K matrix at (a_next, lda_next) that layer `next - 1`
// is about to store, want that layer's epilogue to leave the column sums of what it stores?  Under
// the global scheme, same M, dtype and K = the producer's N, and when it will run on the kernel that
// takes them.  Returns where they go (the consumer's buffer), or null.
float* handover_target(const abft_plan_t* plan, int next, const void* a_next, int64_t lda_next) {
    const abft_plan::Layer& nx = plan->layers[next];
    const abft_layer_t& d = plan->layers[next - 1].desc;
    const abft_layer_t& e = nx.desc;
    if (nx.mode != ABFT_GLOBAL || !nx.alpha32 || e.M != d.M || e.K != d.N || e.dtype != d.dtype) return nullptr;
    const int es = esize(e.dtype);
    const bool a16 = aligned16(a_next) && (lda_next * es) % 16 == 0 && (e.K * es) % 16 == 0;
    const bool b16 = e.b_layout == ABFT_B_NK && aligned16(e.B) && (e.K * es) % 16 == 0 && (e.ldb * es) % 16 == 0;
    const int cfg = pick_cfg(e.M, e.N, e.K, e.dtype, a16 && b16, ABFT_GLOBAL);
    const CfgInfo ci = cfg_info_host(cfg);
    return (ci.fast && ci.kways == 1 && cfg != CFG_F128E) ? nx.alpha32 : nullptr;
}

// The product a layer stands for on these buffers.
int layer_problem(const abft_plan::Layer& L, const void* A, int64_t lda, void* C, int64_t ldc, Problem& pr) {
    const abft_layer_t& d = L.desc;
    std::memset(&pr, 0, sizeof pr);
    if (d.has_conv) {
        int rc = conv_problem(&d.conv, d.N, pr);
        if (rc != ABFT_OK) return rc;
    } else {
        pr.M = d.M; pr.N = d.N; pr.K = d.K; pr.lda = lda;
    }
    pr.dtype = d.dtype; pr.b_layout = d.b_layout;
    pr.A = A; pr.B = d.B; pr.ldb = d.ldb; pr.C = C; pr.ldc = ldc;
    pr.act = L.act;
    return ABFT_OK;
}
// the layer's offline weight checksums where they fit the tiling chosen for this input (an input that
// forces another tiling gets them recomputed into the workspace), else null
const void* layer_beta(const abft_plan::Layer& L, const Problem& pr) {
    const int bn_now = cfg_info_host(pick_cfg(pr.M, pr.N, pr.K, pr.dtype, a_vectorisable(pr) && b_vectorisable(pr), ABFT_GLOBAL)).bn;
    return bn_now == L.beta_block_n ? L.beta : nullptr;
}

// One layer of a plan.  alpha_out (may be null): where to leave the activation checksums of the
// layer that follows (leading dimension ld_alpha_out), *alpha_emitted set when the kernel that ran
// could; alpha_in (may be null): those the layer before left for this layer's input.
int plan_run_layer(abft_plan_t* plan, int layer, const void* A, int64_t lda, void* C, int64_t ldc, uint32_t* fault_flag,
                   void* stream, float* alpha_out, long long ld_alpha_out, bool* alpha_emitted, const float* alpha_in) {
    abft_plan::Layer& L = plan->layers[layer];
    Problem pr;
    const int rc = layer_problem(L, A, lda, C, ldc, pr);
    if (rc != ABFT_OK) return rc;
    pr.alpha_out = alpha_out; pr.ld_alpha_out = ld_alpha_out; pr.alpha_emitted = alpha_emitted; pr.alpha_in = alpha_in;
    const void* beta = layer_beta(L, pr);
    const abft_fault_t* fault = L.has_fault ? &L.fault : nullptr;
    if (pr.conv) {
        const LoweredWeights pre = {L.lowered_B, L.lowered_beta, L.lowered_block_n};
        return run_conv(pr, L.mode, beta, L.workspace, L.ws_bytes, fault_flag, L.report, fault,
                        reinterpret_cast<hipStream_t>(stream), L.lowered_B ? &pre : nullptr);
    }
    return run_problem(pr, L.mode, beta, L.workspace, L.ws_bytes, fault_flag, L.report, fault,
                       reinterpret_cast<hipStream_t>(stream));
}

// ------------------------------------------------------------------------- //
// A pass over a plan's layers (abft_plan_run_all).  Layers that do not wait for one another may share a
// launch: the pass is looked at in windows of up to 64 layers; a layer's depth is one more than that of the
// deepest earlier layer it has to wait for (that one writes what it reads, or either writes what the
// other touches), layers of one depth and kind share a launch, and the launches go out by depth.
// Results are those of the layers one behind the other.
// ------------------------------------------------------------------------- //
// product launches so far that carried several layers of a pass (diagnostics)
std::atomic<long long> g_shared_launches{0};

struct PassWindow {
    static constexpr int MAX_LAYERS = 64;
    struct Range {
        uintptr_t lo, hi;
        bool meets(const Range& o) const { return lo < o.hi && o.lo < hi; }
    };
    struct Entry {
        int layer, depth;
        Range in, weights, out;
    };
    struct Slot {
        int depth;
        int cfg, kmode, dtype;    // of a launch that can take more layers; cfg < 0: one layer, by itself
        int stages;               // direct-to-LDS kernel: the k tiles that LDS holds at a time
        int count;
        int entry[GROUP_MAX];
    };
    abft_plan_t* plan;
    const void* const* A;
    const int64_t* lda;
    void* const* C;
    const int64_t* ldc;
    uint32_t* flag;
    void* stream;
    int n_entries = 0, n_slots = 0;
    Entry entries[MAX_LAYERS];
    Slot slots[MAX_LAYERS];
    // activation checksums that a layer's epilogue left for the layer behind it (alpha[i - base] for layer i; the
    // window's layers are base, base + 1, ...)
    int base = 0;
    const float* alpha[MAX_LAYERS + 1] = {nullptr};

    PassWindow(abft_plan_t* p, const void* const* A_, const int64_t* lda_, void* const* C_, const int64_t* ldc_, uint32_t* f, void* s)
        : plan(p), A(A_), lda(lda_), C(C_), ldc(ldc_), flag(f), stream(s) {}

    // layer i by itself, here and now
    int run_now(int i) {
        // a layer whose input IS the output of the layer before it (same pointer and leading
        // dimension) is chained to it: it can take its activation checksums from that layer's epilogue
        const bool next_chained = i + 1 < (int)plan->layers.size() && A[i + 1] == C[i] && lda[i + 1] == ldc[i];
        float* alpha_out = next_chained ? handover_target(plan, i + 1, C[i], ldc[i]) : nullptr;
        bool emitted = false;
        const int rc = plan_run_layer(plan, i, A[i], lda[i], C[i], ldc[i], flag, stream, alpha_out,
                                      alpha_out ? plan->layers[i + 1].desc.K : 0, &emitted, alpha[i - base]);
        alpha[i - base + 1] = emitted ? alpha_out : nullptr;
        return rc;
    }

    int add(int i) {
        const abft_plan::Layer& L = plan->layers[i];
        const abft_layer_t& d = L.desc;
        Problem pr;
        int rc = layer_problem(L, A[i], lda[i], C[i], ldc[i], pr);
        if (rc == ABFT_OK) rc = validate_common(pr, L.mode, flag);
        if (rc != ABFT_OK) return rc;
        int mode = L.mode;
        if (mode == ABFT_AUTO) mode = select_mode(pr.M, pr.N, pr.K, pr.dtype);
        // (diagnostics, planted faults and the schemes that are never chosen: in order, by themselves)
        if (L.report || L.has_fault || (mode != ABFT_NONE && mode != ABFT_GLOBAL && mode != ABFT_THREAD)) {
            return in_place(i);
        }
        if (n_entries == MAX_LAYERS) {
            rc = flush();
            if (rc != ABFT_OK) return rc;
        }
        const long long es = esize(d.dtype), cs = csize(d.dtype);
        Entry& e = entries[n_entries];
        e.layer = i;
        auto range = [](const void* p, long long bytes) { return Range{reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)bytes}; };
        e.in = range(pr.A, es * (d.has_conv ? (long long)d.conv.batch * d.conv.H * d.conv.W * d.conv.Cin : (pr.M - 1) * pr.lda + pr.K));
        e.weights = range(pr.B, es * (pr.b_layout == ABFT_B_NK ? (pr.N - 1) * pr.ldb + pr.K : (pr.K - 1) * pr.ldb + pr.N));
        e.out = range(pr.C, cs * ((pr.M - 1) * pr.ldc + pr.N));
        e.depth = 0;
        for (int j = 0; j < n_entries; ++j) {
            const Entry& o = entries[j];
            if (o.depth >= e.depth && ordered(e, o)) e.depth = o.depth + 1;
        }
        const int cfg = shared_cfg(i, pr, mode);
        const int stages = cfg >= 0 && cfg < CFG_COUNT && !cfg_is_stream(cfg) ? (int)std::min(cdiv(pr.K * es, 128), 3LL) : 0;
        int s = n_slots;
        if (cfg >= 0) {
            s = 0;
            while (s < n_slots && !(slots[s].depth == e.depth && slots[s].cfg == cfg && slots[s].kmode == mode && slots[s].dtype == d.dtype &&
                                    slots[s].stages == stages && slots[s].count < GROUP_MAX))
                ++s;
        }
        if (s == n_slots) slots[n_slots++] = Slot{e.depth, cfg, mode, d.dtype, stages, 0, {}};
        slots[s].entry[slots[s].count++] = n_entries;
        ++n_entries;
        return ABFT_OK;
    }

    // does one of two layers have to wait for the other?
    static bool ordered(const Entry& e, const Entry& o) {
        return e.in.meets(o.out) || e.out.meets(o.out) || e.out.meets(o.in) || e.weights.meets(o.out) || e.out.meets(o.weights);
    }

    // the configuration under which layer i can share a launch, or -1: the streaming kernel on whole
    // k tiles, with nothing to launch ahead of it; the skinny kernel; or the direct-to-LDS kernel's tiles of 32 x 128 per
    // wavefront, unprotected or thread-level, for matrices of at most 512 tiles (beyond two rounds of workgroups a launch
    // of its own is full) that leave no activation checksums to the layer behind them
    static constexpr int SKINNY = CFG_COUNT, SHALLOW = CFG_COUNT + 1;
    // ... or, in a launch of the streaming kernel with four wavefronts, a product for shallow_tile
    static bool takes_shallow(int cfg) { return cfg == CFG_S32 || cfg == CFG_S64 || cfg == CFG_S128; }
    int shared_cfg(int i, const Problem& pr, int mode) const {
        const abft_plan::Layer& L = plan->layers[i];
        if (pr.M <= SKINNY_ROWS) {
            // (also where it would be slower alone, if its results are the tiling's bit by bit: the 16 x 64 tile's on one k tile, whose sums nobody shares)
            const int alone = pick_cfg(pr.M, pr.N, pr.K, pr.dtype, a_vectorisable(pr) && b_vectorisable(pr), mode, pr.conv);
            if (skinny_takes(pr, alone, mode) || (alone == CFG_G16 && skinny_fits(pr, alone, mode) && (long long)pr.K * esize(pr.dtype) <= 128)) return SKINNY;
        }
        const bool hands_over = i + 1 < (int)plan->layers.size() && A[i + 1] == C[i] && lda[i + 1] == ldc[i] && handover_target(plan, i + 1, C[i], ldc[i]);
        if (shallow_takes(pr, pick_cfg(pr.M, pr.N, pr.K, pr.dtype, a_vectorisable(pr) && b_vectorisable(pr), mode, pr.conv), mode))
            return hands_over ? -1 : (int)SHALLOW;
        if (!a_vectorisable(pr) || !b_vectorisable(pr) || ((long long)pr.K * esize(pr.dtype)) % 128 != 0) return -1;
        if (pr.conv && conv_lowering(pr).ok) return -1;
        const int cfg = pick_cfg(pr.M, pr.N, pr.K, pr.dtype, true, mode, pr.conv);
        if (cfg == CFG_F64T || cfg == CFG_F128T) {
            const CfgInfo ci = cfg_info_host(cfg);
            return mode == ABFT_GLOBAL || pr.conv || hands_over || cdiv(pr.M, ci.bm) * cdiv(pr.N, ci.bn) > 512 ? -1 : cfg;
        }
        if (!cfg_is_stream(cfg) || (mode == ABFT_GLOBAL && !layer_beta(L, pr))) return -1;
        return cfg;
    }

    int launch_shared(const Slot& slot) {
        // longest k loops first, so that the last workgroups to start are short ones
        int order[GROUP_MAX];
        for (int q = 0; q < slot.count; ++q) {
            int at = q;
            while (at > 0 && plan->layers[entries[order[at - 1]].layer].desc.K < plan->layers[entries[slot.entry[q]].layer].desc.K) {
                order[at] = order[at - 1];
                --at;
            }
            order[at] = slot.entry[q];
        }
        GroupArgs a;
        std::memset(&a, 0, sizeof a);
        int blocks = 0;
        for (int q = 0; q < slot.count; ++q) {
            const int i = entries[order[q]].layer;
            abft_plan::Layer& L = plan->layers[i];
            Problem pr;
            Prepared w;
            int rc = layer_problem(L, A[i], lda[i], C[i], ldc[i], pr);
            if (rc == ABFT_OK)
                rc = prepare_problem(pr, L.mode, slot.kmode == ABFT_GLOBAL ? layer_beta(L, pr) : nullptr, L.workspace, L.ws_bytes, flag, nullptr, nullptr,
                                     reinterpret_cast<hipStream_t>(stream), w);
            if (rc != ABFT_OK) return rc;
            const GemmArgs& g = w.g;
            GroupItem& it = a.item[q];
            it.A = g.A; it.B = g.B; it.C = g.C; it.beta_k = g.beta_k; it.beta_p = g.beta_p;
            it.lda = g.lda; it.ldb = g.ldb; it.ldc = g.ldc; it.imgpitch = g.imgpitch; it.rowpitch = g.rowpitch;
            it.tol_coeff = g.tol_coeff; it.tol_l1 = g.tol_l1;
            it.M = g.M; it.N = g.N; it.K = g.K; it.tiles_m = g.tiles_m; it.tiles_n = g.tiles_n; it.act = g.act;
            it.conv = g.conv; it.H = g.H; it.W = g.W; it.Cin = g.Cin; it.KH = g.KH; it.KW = g.KW;
            it.stride = g.stride; it.pad = g.pad; it.OH = g.OH; it.OW = g.OW; it.pix = g.pix;
            it.shallow = w.cfg == CFG_G64;
            if (slot.cfg == SKINNY) {
                it.tiles_n = (int)cdiv(g.N, 16);
                it.bytes = rows_off_dwords(g, slot.dtype);
            }
            a.first[q] = blocks;
            blocks += it.tiles_m * it.tiles_n;
        }
        for (int q = slot.count; q < GROUP_MAX; ++q) a.first[q] = 0x7fffffff;
        a.flag = flag;
        g_shared_launches.fetch_add(1, std::memory_order_relaxed);
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        if (slot.cfg == SKINNY) {
            const hipError_t e = slot.dtype == ABFT_F16    ? launch_skinny_group_f16(slot.kmode, blocks, a, st)
                                 : slot.dtype == ABFT_BF16 ? launch_skinny_group_bf16(slot.kmode, blocks, a, st)
                                                           : launch_skinny_group_i8(slot.kmode, blocks, a, st);
            return e == hipSuccess ? ABFT_OK : ABFT_E_HIP;
        }
        const hipError_t e = slot.dtype == ABFT_F16    ? launch_group_f16(slot.cfg, slot.kmode, blocks, a, st)
                             : slot.dtype == ABFT_BF16 ? launch_group_bf16(slot.cfg, slot.kmode, blocks, a, st)
                                                       : launch_group_i8(slot.cfg, slot.kmode, blocks, a, st);
        return e == hipSuccess ? ABFT_OK : ABFT_E_HIP;
    }

    // A layer that would go out alone joins a launch that takes it, now or a later one of its kind, if nothing that goes out until then waits for it
    // (ResNet-50 at batch 1: a downsampling of 64 -> 256 channels, 4 to 5 us by itself, with the three expansions of its stage)
    void join(Slot& lone) {
        Entry& e = entries[lone.entry[0]];
        for (int s = 0; s < n_slots; ++s) {
            Slot& to = slots[s];
            if (&to == &lone || to.depth < lone.depth || to.count == 0 || to.count == GROUP_MAX || to.kmode != lone.kmode || to.dtype != lone.dtype ||
                !(lone.cfg == SHALLOW ? takes_shallow(to.cfg) : to.cfg == lone.cfg && to.stages == lone.stages))
                continue;
            bool free = true;
            for (int j = 0; j < n_entries && free; ++j)
                free = entries[j].depth <= lone.depth || entries[j].depth > to.depth || !ordered(e, entries[j]);
            if (!free) continue;
            e.depth = to.depth;
            to.entry[to.count++] = lone.entry[0];
            lone.count = 0;
            return;
        }
    }

    // what has been added so far goes out; the window is empty again and starts behind it
    int flush() {
        int rc = ABFT_OK;
        for (int s = 0; s < n_slots; ++s)
            if (slots[s].count == 1 && slots[s].cfg >= 0) join(slots[s]);
        for (int depth = 0, left = n_slots; left > 0 && rc == ABFT_OK; ++depth)
            for (int s = 0; s < n_slots && rc == ABFT_OK; ++s)
                if (slots[s].depth == depth) {
                    --left;
                    if (slots[s].count == 0) continue;
                    if (slots[s].count == 1 || slots[s].cfg == SHALLOW) {
                        for (int q = 0; q < slots[s].count && rc == ABFT_OK; ++q) rc = run_now(entries[slots[s].entry[q]].layer);
                    } else {
                        rc = launch_shared(slots[s]);
                    }
                }
        advance(n_entries);
        n_entries = n_slots = 0;
        return rc;
    }
    // a layer that keeps to its place: behind everything before it, ahead of everything after it
    int in_place(int i) {
        int rc = flush();
        if (rc == ABFT_OK) rc = run_now(i);
        advance(1);
        return rc;
    }
    void advance(int layers) {
        const float* carried = alpha[layers];
        for (int q = 0; q <= layers; ++q) alpha[q] = nullptr;
        alpha[0] = carried;
        base += layers;
    }
};

}  // namespace

extern "C" {

int abft_plan_run(abft_plan_t* plan, int layer, const void* A, int64_t lda, void* C, int64_t ldc,
                  uint32_t* fault_flag, void* stream) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    return plan_run_layer(plan, layer, A, lda, C, ldc, fault_flag, stream, nullptr, 0, nullptr, nullptr);
}

int abft_plan_run_all(abft_plan_t* plan, const void* const* A, const int64_t* lda, void* const* C,
                      const int64_t* ldc, uint32_t* fault_flag, int event_layer, void* stream) {
    if (!plan) return ABFT_E_PLAN;
    if (!A || !lda || !C || !ldc) return ABFT_E_NULL;
    const hipEvent_t ev0 = g_ev_start, ev1 = g_ev_stop;
    const int n = (int)plan->layers.size();
    PassWindow w(plan, A, lda, C, ldc, fault_flag, stream);
    g_ev_start = g_ev_stop = nullptr;
    int rc = ABFT_OK;
    for (int i = 0; i < n && rc == ABFT_OK; ++i) {
        // the measurement hook, if set, brackets the product kernel of one layer only
        const bool hooked = i == event_layer && (ev0 || ev1);
        if (!hooked) {
            rc = w.add(i);
            continue;
        }
        rc = w.flush();
        if (rc != ABFT_OK) break;
        g_ev_start = ev0;
        g_ev_stop = ev1;
        rc = w.in_place(i);
        g_ev_start = g_ev_stop = nullptr;
    }
    const int rest = w.flush();   // (a call that is refused: the layers before it have run, as ever)
    if (rc == ABFT_OK) rc = rest;
    g_ev_start = ev0;
    g_ev_stop = ev1;
    return rc;
}

int abft_plan_run_chain(abft_plan_t* plan, int first, int count, const void* A, int64_t lda, void* const* C,
                        const int64_t* ldc, uint32_t* fault_flag, void* stream) {
    if (!plan || first < 0 || count <= 0 || first + count > (int)plan->layers.size()) return ABFT_E_PLAN;
    if (!A || !C || !ldc) return ABFT_E_NULL;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    // one launch for the whole chain when every layer qualifies; else layer by layer
    bool one_launch = count <= CHAIN_MAX_LAYERS && plan->chain_flags != nullptr;
    const abft_layer_t& d0 = plan->layers[first].desc;
    bool any_check = false;
    for (int i = 0; i < count && one_launch; ++i) {
        const abft_plan::Layer& L = plan->layers[first + i];
        const abft_layer_t& d = L.desc;
        const void* a_i = i == 0 ? A : C[i - 1];
        const int64_t lda_i = i == 0 ? lda : ldc[i - 1];
        // (layers small enough that a launch of their own would run on 32 x 32 tiles too, and in the same four
        // shares of the k loop: the chain's results are the layers'.  Eight shares in two sets of accumulators
        // per wavefront gave those results in one launch as well, in 46 us for 16 x 4096 -> 1024 -> 4096 -> 1024
        // thread-level, where three launches take 20)
        one_launch = L.chain_beta != nullptr && d.dtype == d0.dtype && d.M == d0.M &&
                     pick_cfg(d.M, d.N, d.K, d.dtype, true, L.mode) == CFG_S32 && !L.report && !L.has_fault &&
                     (L.mode == ABFT_NONE || L.mode == ABFT_GLOBAL || L.mode == ABFT_THREAD) && C[i] != nullptr &&
                     // (else most layers' own launches run on the skinny kernel, and layer by layer is faster: 16 x 512 -> 1024 -> 1024
                     // -> 512 -> 256 -> 1 fp16 thread-level 16.0 us, in one launch 21.5; 1 x 512 -> 256 -> 64 5.8 / 8.5; so, too, where
                     // that kernel leaves a layer of more weights to 32 x 32 tiles: 16 x 2048 -> 8192 -> 2048 18.9 / 77)
                     (d.M > SKINNY_ROWS || L.mode == ABFT_GLOBAL) &&
                     aligned16(a_i) && (lda_i * 2) % 16 == 0 && lda_i >= d.K && ldc[i] >= d.N &&
                     (i == 0 || d.K == plan->layers[first + i - 1].desc.N);
        any_check = any_check || L.mode != ABFT_NONE;
    }
    if (one_launch && any_check && !fault_flag) return ABFT_E_NULL;
    if (!one_launch) {
        // Layer by layer.  A layer under the global scheme takes its activation checksums from the
        // epilogue of the layer before it (Sec. 2.4 step 4) when it reads that layer's output as a
        // plain matrix and both run kernels that can do their part; else it forms them itself.
        int rc = ABFT_OK;
        const float* alpha_in = nullptr;
        for (int i = 0; i < count && rc == ABFT_OK; ++i) {
            float* alpha_out = i + 1 < count ? handover_target(plan, first + i + 1, C[i], ldc[i]) : nullptr;
            const long long ld_alpha = alpha_out ? plan->layers[first + i + 1].desc.K : 0;
            bool emitted = false;
            rc = plan_run_layer(plan, first + i, i == 0 ? A : C[i - 1], i == 0 ? lda : ldc[i - 1], C[i], ldc[i], fault_flag,
                                stream, alpha_out, ld_alpha, &emitted, alpha_in);
            alpha_in = emitted ? alpha_out : nullptr;
        }
        return rc;
    }
    ChainArgs a;
    std::memset(&a, 0, sizeof a);
    a.n_layers = count;
    a.M = d0.M;
    a.flags = plan->chain_flags;
    a.status = plan->chain_flags + CHAIN_FLAG_WORDS;
    a.fault_flag = fault_flag ? fault_flag : plan->chain_flags + CHAIN_FLAG_WORDS + 1;   // (unprotected chain: a word of the plan's own)
    a.spin_limit = plan->chain_spin_limit;
    for (int i = 0; i < count; ++i) {
        const abft_plan::Layer& L = plan->layers[first + i];
        const abft_layer_t& d = L.desc;
        ChainLayer& c = a.layer[i];
        c.A = reinterpret_cast<const char*>(i == 0 ? A : C[i - 1]);
        c.lda = i == 0 ? lda : ldc[i - 1];
        c.B = reinterpret_cast<const char*>(d.B);
        c.ldb = d.ldb;
        c.C = reinterpret_cast<char*>(C[i]);
        c.ldc = ldc[i];
        c.N = d.N;
        c.K = d.K;
        const int nb = (int)cdiv(d.N, 32);
        c.beta_k = reinterpret_cast<const char*>(L.chain_beta) + beta_k_offset(d.K, nb);
        c.beta_p = reinterpret_cast<const char*>(L.chain_beta) + beta_p_offset(d.K, nb);
        c.mode = L.mode;          // ABFT_NONE / GLOBAL / THREAD carry the kernels' own numbers
        c.act = L.act;
        c.depends = i > 0;
        c.tol_coeff = tol_coeff(d.K, d.dtype, L.mode);
        c.tol_l1 = tol_bias_coeff(d.K, d.dtype, L.mode);
    }
    g_chain_launches.fetch_add(1, std::memory_order_relaxed);
    const hipError_t e = d0.dtype == ABFT_F16 ? launch_mlp_chain_f16(a, st) : launch_mlp_chain_bf16(a, st);
    return e == hipSuccess ? ABFT_OK : ABFT_E_HIP;
}

int abft_plan_chain_status(abft_plan_t* plan, uint32_t* status, void* stream) {
    if (!plan || !plan->chain_flags) return ABFT_E_PLAN;
    if (!status) return ABFT_E_NULL;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (hipMemcpyAsync(status, plan->chain_flags + CHAIN_FLAG_WORDS, sizeof(uint32_t), hipMemcpyDeviceToHost, st) != hipSuccess ||
        hipStreamSynchronize(st) != hipSuccess)
        return ABFT_E_HIP;
    return ABFT_OK;
}

int abft_plan_chain_reset(abft_plan_t* plan, int spin_limit, void* stream) {
    if (!plan || !plan->chain_flags) return ABFT_E_PLAN;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (hipMemsetAsync(plan->chain_flags, 0, (size_t)(CHAIN_FLAG_WORDS + 64) * sizeof(unsigned), st) != hipSuccess ||
        hipStreamSynchronize(st) != hipSuccess)
        return ABFT_E_HIP;
    plan->chain_spin_limit = spin_limit >= 0 ? spin_limit : (1 << 20);
    return ABFT_OK;
}

long long abft_handover_launches(void) { return g_handover_launches.load(std::memory_order_relaxed); }
long long abft_chain_launches(void) { return g_chain_launches.load(std::memory_order_relaxed); }
long long abft_shared_launches(void) { return g_shared_launches.load(std::memory_order_relaxed); }

int abft_plan_set_diagnostics(abft_plan_t* plan, int layer, abft_report_t* report, const abft_fault_t* inject) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    abft_plan::Layer& L = plan->layers[layer];
    L.report = report;
    L.has_fault = inject != nullptr;
    if (inject) L.fault = *inject;
    return ABFT_OK;
}

int abft_plan_set_mode(abft_plan_t* plan, int layer, int mode) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    if (mode < ABFT_NONE || mode > ABFT_GLOBAL_WEIGHTED) return ABFT_E_ENUM;
    abft_plan::Layer& L = plan->layers[layer];
    L.mode = mode == ABFT_AUTO ? select_mode(L.desc.M, L.desc.N, L.desc.K, L.desc.dtype) : mode;
    return ABFT_OK;
}

int abft_plan_set_activation(abft_plan_t* plan, int layer, int act) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    if (act != ABFT_ACT_NONE && act != ABFT_ACT_RELU) return ABFT_E_ENUM;
    plan->layers[layer].act = act;
    return ABFT_OK;
}

int abft_plan_activation(const abft_plan_t* plan, int layer) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    return plan->layers[layer].act;
}

int abft_plan_mode(const abft_plan_t* plan, int layer) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    return plan->layers[layer].mode;
}

int abft_plan_times(const abft_plan_t* plan, int layer, double* out3) {
    if (!plan || layer < 0 || layer >= (int)plan->layers.size()) return ABFT_E_PLAN;
    if (!out3) return ABFT_E_NULL;
    for (int i = 0; i < 3; ++i) out3[i] = plan->layers[layer].t_us[i];
    return ABFT_OK;
}

void abft_plan_destroy(abft_plan_t* plan) {
    if (!plan) return;
    for (auto& L : plan->layers) {
        if (L.beta) (void)hipFree(L.beta);
        if (L.workspace) (void)hipFree(L.workspace);
        if (L.lowered_B) (void)hipFree(L.lowered_B);
        if (L.lowered_beta) (void)hipFree(L.lowered_beta);
        if (L.chain_beta) (void)hipFree(L.chain_beta);
        if (L.alpha32) (void)hipFree(L.alpha32);
    }
    if (plan->chain_flags) (void)hipFree(plan->chain_flags);
    delete plan;
}

const char* abft_strerror(int code) {
    switch (code) {
        case ABFT_OK: return "ok";
        case ABFT_E_NULL: return "a required pointer is NULL";
        case ABFT_E_SHAPE: return "bad problem shape";
        case ABFT_E_LD: return "leading dimension smaller than the row length";
        case ABFT_E_ENUM: return "unknown dtype, mode or layout";
        case ABFT_E_WORKSPACE: return "workspace missing, misaligned or too small";
        case ABFT_E_INJECT: return "fault descriptor out of range";
        case ABFT_E_HIP: return "HIP runtime call failed";
        case ABFT_E_PLAN: return "bad plan handle or layer index";
        case ABFT_E_UNSUPPORTED: return "scheme not available for this product";
        case ABFT_E_VALUE: return "a scale, window or page size is out of its range";
    }
    return "unknown error code";
}

int abft_version(void) { return 100; }

}  // extern "C"

namespace {
// MFMAs from registers only: each wavefront keeps the fragments of a 128 x 64 register tile
// (TM + TN fragments of 16 bytes per lane) and multiplies them `iters` times into its TM x TN
// accumulator blocks.  Nothing else runs, so the rate is what the matrix units sustain for these
// operand values under the board's power limit.
template <int DT, int MI>
__global__ __launch_bounds__(512) void mfma_probe_kernel(const i32x4* src, float* sink, int iters) {
    typedef abft::Mma<DT, MI> MMA;
    constexpr int TM = 128 / MI, TN = 64 / MI;
    const long long t = (long long)blockIdx.x * 512 + threadIdx.x;
    i32x4 a[TM], b[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) a[i] = src[t * 16 + i];
#pragma unroll
    for (int j = 0; j < TN; ++j) b[j] = src[t * 16 + TM + j];
    typename MMA::Acc acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < MMA::NACC; ++r) acc[i][j][r] = 0;
    for (int it = 0; it < iters; ++it) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = MMA::run(a[i], b[j], acc[i][j]);
    }
    typename MMA::AccT total = 0;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < MMA::NACC; ++r) total += acc[i][j][r];
    // (no finite sum of these products has this bit pattern's value twice over: never taken)
    if ((float)total == 12345.678f && iters < 0) sink[0] = (float)total;
}

int probe_cus() {
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
    return n;
}
}  // namespace

extern "C" {

size_t abft_mfma_probe_bytes(void) {
    const int cus = probe_cus();
    return (size_t)(cus > 0 ? cus : 256) * 512 * 16 * sizeof(i32x4);
}

int abft_mfma_probe(int shape, int dtype, int iters, const void* operands, float* sink, double* ops, void* stream) {
    if (!valid_dtype(dtype) || (shape != 32 && shape != 16)) return ABFT_E_ENUM;
    if (!operands || !sink || !ops) return ABFT_E_NULL;
    if (iters < 1) return ABFT_E_SHAPE;
    const int cus = probe_cus();
    if (cus <= 0) return ABFT_E_HIP;
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const i32x4* src = reinterpret_cast<const i32x4*>(operands);
    dim3 grid((unsigned)cus), block(512);
    void (*kern)(const i32x4*, float*, int) = nullptr;
    if (dtype == ABFT_F16) kern = shape == 32 ? mfma_probe_kernel<abft::DT_F16, 32> : mfma_probe_kernel<abft::DT_F16, 16>;
    else if (dtype == ABFT_BF16) kern = shape == 32 ? mfma_probe_kernel<abft::DT_BF16, 32> : mfma_probe_kernel<abft::DT_BF16, 16>;
    else kern = shape == 32 ? mfma_probe_kernel<abft::DT_I8, 32> : mfma_probe_kernel<abft::DT_I8, 16>;
    hipLaunchKernelGGL(kern, grid, block, 0, st, src, sink, iters);
    if (hipGetLastError() != hipSuccess) return ABFT_E_HIP;
    // per wavefront and iteration: 8 MFMAs of 32 x 32 x 16 (16384 multiply-adds each) or 32 of
    // 16 x 16 x 32 (8192 each); int8 shapes are twice as deep
    const double macs = (shape == 32 ? 8.0 * 16384.0 : 32.0 * 8192.0) * (dtype == ABFT_I8 ? 2.0 : 1.0);
    *ops = (double)cus * 8.0 * (double)iters * macs * 2.0;
    return ABFT_OK;
}

void abft_set_kernel_events(void* start_event, void* stop_event) {
    g_ev_start = reinterpret_cast<hipEvent_t>(start_event);
    g_ev_stop = reinterpret_cast<hipEvent_t>(stop_event);
}

}  // extern "C"
