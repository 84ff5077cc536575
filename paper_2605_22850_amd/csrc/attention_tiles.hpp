// What the attention kernels over a bfloat16 and over a 4-bit prefix share: the
// order of a launch's row tiles, and the two phases of a wavefront that owns 32
// query rows of a 256-row tile.
#pragma once

#include "mfma_tiles.hpp"

namespace oc {

constexpr int PAGE = 16;          // tokens per pool page (attention requires page_size 16)
constexpr int KB = 64;            // keys per block = 4 pages
constexpr int WAVES = 8;          // two per SIMD: one's softmax overlaps the other's MFMAs
constexpr int QB = 1;             // 32-row query blocks per wavefront
constexpr int WAVE_ROWS = 32 * QB;
constexpr int TILE_ROWS = WAVES * WAVE_ROWS;
constexpr int THREADS = WAVES * 64;
constexpr float RESCALE_SLACK = 8.0f;   // log2 units the running max may lag
constexpr int LOOKAHEAD = 3;              // MFMAs an operand read runs ahead of its use

// A row's P is 2^(s * scale - m), the product unrounded (one fma), and m the rounded
// product of its largest score (log2 units).  All of its P are thus off by one factor
// 2^r, r half a step of m at most, which the row's sum takes out again; but past |m| =
// 2^31 r is more than an exponent holds, and P and sum would all be infinite or 0.
// So each row has a scale of its own, and a row whose largest score is 2^31 or more (m
// past 2^28, r 8) takes 1/4, with which every product is exact.  It need not be the
// right one: two fp32 scores there differ by 2^16 in P or not at all, and with either
// scale the smaller one vanishes.  It is larger than any other (log2(e) / 8 at d = 64),
// so that where such a row meets a part of itself with smaller scores, in another
// wavefront or split, the larger score has the larger m.
constexpr float LARGE_SCORE = 0x1p31f, LARGE_SCALE = 0.25f, LARGE_M = LARGE_SCORE * LARGE_SCALE;
// of a row with running maximum m (-inf, a row without a key, has no P that it matters to)
__device__ __forceinline__ float row_scale(float m, float scale_log2) {
    return __builtin_fabsf(m) >= LARGE_M ? LARGE_SCALE : scale_log2;
}
// the running maximum of a row after scores of at most `top`
__device__ __forceinline__ float raise_row(float m, float scale, float top, float scale_log2) {
    return top * scale > m ? top * (__builtin_fabsf(top) >= LARGE_SCORE ? LARGE_SCALE : scale_log2) : m;
}

// value of the lane 32 positions away (the other half of the wavefront)
__device__ inline float half_swap_max(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float half_swap_sum(float x) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Whether all row tiles of a (KV head, split) group get consecutive slots on
// one XCD (workgroup w runs on XCD w % 8), so that their K/V re-reads hit that
// XCD's L2, or the tiles are dealt out to the XCDs one by one.
//  - A multiple of 8 groups loads the XCDs evenly: by XCD.
//  - 256-row tiles, any other count: dealt.  They re-read little, and XCDs that
//    hold a group less idle (by XCD 0.95 to 1.82 times as long, 1.11 on
//    average, over 87 shapes of 4 to 122 groups).
//  - Tiles of 32 and 64 rows: by XCD where there is a group for every XCD and
//    the busiest XCD's workgroups all run at once on its 32 CUs (0.60 to 1.05
//    times as long as dealt, 0.94 on average, over 123 shapes of 9 to 108
//    groups) or the XCDs are within 1/15 of even (0.48 to 1.12, 0.91 on average,
//    over 36 shapes of 15 to 100 groups).  Otherwise the uneven XCDs cost more
//    than their L2 gives (0.95 to 1.87, 1.28 on average, over 232 shapes), and
//    with fewer groups than XCDs some would idle (1.0 to 6.3).
__host__ __device__ inline bool tiles_by_xcd(int m_tiles, int n_groups, bool small_tiles) {
    if ((n_groups & 7) == 0) return true;
    const int per_xcd = (n_groups + 7) / 8;           // groups of the busiest XCD
    return small_tiles && n_groups > 8 &&
           ((int64_t)per_xcd * m_tiles <= 32 || 2 * (int64_t)n_groups >= 15 * (int64_t)per_xcd);
}

// Workgroup wg of a launch -> its (KV head, split) group and row tile; false
// past the last.  Either way the last row tile comes first: under the causal
// mask later rows see more suffix keys, and dispatching the longest tiles
// first keeps them out of the tail.
__host__ __device__ inline bool tile_of(int wg, int m_tiles, int n_groups, bool small_tiles, int &gamma, int &mt) {
    if (!tiles_by_xcd(m_tiles, n_groups, small_tiles)) {
        gamma = wg % n_groups;
        mt = m_tiles - 1 - wg / n_groups;
        return mt >= 0;
    }
    const int xcd = wg & 7, local = wg >> 3;
    gamma = (local / m_tiles) * 8 + xcd;
    mt = m_tiles - 1 - local % m_tiles;
    return gamma < n_groups;
}

// tile row r of a 32-key MFMA tile reads physical key perm(r): bits 2 and 3 swapped
__device__ inline int key_perm(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// Per-wavefront running state of the online softmax for its 32 query rows.
template <int D>
struct WaveState {
    f32x16 o[D / 32];    // O^T: 32 dims x 32 rows per tile, fp32
    f32x16 s[2];         // scores of the current block, one 32-key half each
    bf16x8 p[2][2];      // P of the last softmaxed block as the PV operand: [half][8-key group]
    float scale, m_use;  // this lane's row: row_scale(), and m, or 0 while that is -inf
    float m, l;          // its running maximum (log2 units) and sum
};

// The first LOOKAHEAD V^T fragments of a PV pass, read ahead of the barrier
// that opens the matrix phase (the V tile of the previous block is already
// readable there), so the phase starts without waiting on LDS.
template <int D>
__device__ __forceinline__ void prefetch_vt(const uint16_t *V, const int (&voff)[D / 32], bf16x8 (&pre)[LOOKAHEAD]) {
#pragma unroll
    for (int n = 0; n < LOOKAHEAD; ++n) pre[n] = load_vt<D>(V, voff, n);
}

// Matrix phase of a wavefront: O^T += V^T P for the previous block (PV:
// 16 MFMAs at d = 128, each V^T fragment from two transposing LDS reads),
// then S^T = K Q^T for the current block (S: 16 MFMAs, K fragments from the
// swizzled tile, the two 32-key halves alternating so that consecutive MFMAs
// are independent).  Written as one flat sequence whose operand reads run
// LOOKAHEAD MFMAs ahead (with PV, the first LOOKAHEAD come preloaded, see
// prefetch_vt); a scheduling fence after every MFMA keeps that order (left
// alone, the compiler hoists every read to the top and runs out of VGPRs).
template <int D, bool PV, bool S>
__device__ __forceinline__ void matrix_phase(WaveState<D> &w, const uint16_t *V, const int (&voff)[D / 32],
                                             const uint16_t *K, const bf16x8 (&qop)[D / 16], int krow, int half,
                                             const bf16x8 (&pre)[LOOKAHEAD]) {
    constexpr int NET = D / 32, NDS = D / 16;
    constexpr int NPV = PV ? 4 * NET : 0;
    constexpr int N = NPV + (S ? 2 * NDS : 0);
    static_assert(!PV || NPV >= LOOKAHEAD, "prefetched fragments must all be V^T fragments");
    auto load = [&](int n) -> bf16x8 {
        if (n < NPV) return load_vt<D>(V, voff, n);
        const int n2 = n - NPV, ds = n2 >> 1, kt = n2 & 1;
        return *reinterpret_cast<const bf16x8 *>(&K[k_lds<D>(kt * 32 + krow, ds * 2 + half)]);
    };
    bf16x8 f[N];
    // the wavefront in its matrix phase issues ahead of its SIMD partner's
    // softmax: the MFMA pipe is the longer of the two (about 3 % per layer)
    __builtin_amdgcn_s_setprio(2);
#pragma unroll
    for (int n = 0; n < LOOKAHEAD && n < N; ++n) f[n] = PV ? pre[n] : load(n);
#pragma unroll
    for (int n = 0; n < N; ++n) {
        if (n + LOOKAHEAD < N) f[n + LOOKAHEAD] = load(n + LOOKAHEAD);
        if (n < NPV) {
            const int et = n % NET, g4 = n / NET;
            w.o[et] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n], w.p[g4 >> 1][g4 & 1], w.o[et], 0, 0, 0);
        } else {
            const int n2 = n - NPV, ds = n2 >> 1, kt = n2 & 1;
            w.s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f[n], qop[ds], ds == 0 ? f32x16{} : w.s[kt], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(1);
}

// Softmax phase of a wavefront for one block: the block maximum (one lane
// swap between the half-waves), the lazy raise of the running maximum (O and
// l rescaled only when the block maximum exceeds it by more than
// 2^RESCALE_SLACK), then P = 2^(s*scale*log2(e) - m) as bf16 and the row sums
// of that rounded P.
template <int D>
__device__ __forceinline__ void softmax_phase(WaveState<D> &w, float scale_log2) {
    float mx[2] = {-__builtin_inff(), -__builtin_inff()};   // two partial maxima
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int i2 = 0; i2 < 16; ++i2) mx[i2 & 1] = fmaxf(mx[i2 & 1], w.s[kt][i2]);
    const float top = half_swap_max(fmaxf(mx[0], mx[1]));
    if (__any(top * w.scale > w.m + RESCALE_SLACK)) {
        const float m_new = raise_row(w.m, w.scale, top, scale_log2);
        w.scale = row_scale(m_new, scale_log2);
        w.m_use = m_new == -__builtin_inff() ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(w.m - (m_new == -__builtin_inff() ? 0.f : m_new));
        w.m = m_new;
        w.l *= alpha;
#pragma unroll
        for (int et = 0; et < D / 32; ++et) w.o[et] *= alpha;
    }
    // row sums of the rounded P (the values the PV product uses), two bf16
    // pairs per dot instruction, two partial sums
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
    float lsum[2] = {0.f, 0.f};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            f32x8 pv;
#pragma unroll
            for (int i2 = 0; i2 < 8; ++i2)
                pv[i2] = __builtin_amdgcn_exp2f(fmaf(w.s[kt][hf * 8 + i2], w.scale, -w.m_use));
            const bf16x8 pp = __builtin_convertvector(pv, bf16x8);
            w.p[kt][hf] = pp;
            lsum[0] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pp, pp, 0, 1), ones, lsum[0], false);
            lsum[1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pp, pp, 2, 3), ones, lsum[1], false);
            lsum[0] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pp, pp, 4, 5), ones, lsum[0], false);
            lsum[1] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(pp, pp, 6, 7), ones, lsum[1], false);
        }
    w.l += lsum[0] + lsum[1];
}

}  // namespace oc
