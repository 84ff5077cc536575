// Attention over a prefix held in 4 bits: the suffix-prefill form (one request's
// new tokens) and the decode form (one new token for each request of a batch).
//
//   out[i][h] = sum_j softmax_j(q[i][h] . k_j / sqrt(d)) v_j
//
// j over the prefix's tokens, dequantised from the pages of the block table, then
// over the new tokens 0..i in bfloat16.
#include <math.h>

#include <algorithm>

#include "kv4.hpp"
#include "mfma_tiles.hpp"

namespace oc {

constexpr int PAGE4 = 16;         // tokens per page
constexpr int UNIT4 = 32;         // keys per unit: two pages
constexpr int NW4 = 8;            // wavefronts of a workgroup
constexpr float SLACK4 = 8.0f;    // log2 units the running maximum may lag

struct Kv4Params {
    const uint16_t *q, *k_new, *v_new;
    unsigned char *pool_k, *pool_v;
    const int32_t *pages, *num_tokens;
    float *o_part;
    float2 *ml_part;
    uint16_t *out;
    int64_t page_bytes, table_stride;
    int code_bytes, Tp, Ts, rows, nq, nkv, grp, m_tiles, n_split, n_groups, units_per_split, max_tokens;
    float scale_log2;
};

// ---------------------------------------------------------------------------
// Row tiles of 16 * NR query rows; the wavefronts of a workgroup split the keys.
//
// A unit is two pages.  Everything is laid out around the 16x16x32 MFMA: lane
// (c, g) = (lane % 16, lane / 16) holds key c of each page, and of that key's row
// the g-th quarter of the dimensions -- at d = 128 one block: 16 bytes of codes and one
// scale byte, so a page's K is one 1 KiB load of a wavefront.  Its dwords, decoded,
// are the K operands of d/32 products (the order of the dimensions in a product is
// free as long as Q has the same), and S^T comes out with query row c and keys 4g..4g+3
// per lane.  The P of two pages is then the second operand of O^T += V^T P as it
// stands, its contraction index 8g + i being key 4g + i%4 of page i/4; V is decoded
// into LDS and read back transposed, four keys of one page per read.
// ---------------------------------------------------------------------------

// 16-byte column of V row r (key in its page), XORed so that a wavefront's
// writes of one column step and its transposing reads each touch every bank once
template <int D>
__device__ __forceinline__ int v4_swz(int r) {
    if constexpr (D == 128) return ((r & 7) << 1) | ((r >> 3) & 1);
    else return (((r >> 1) & 3) << 1) | ((r >> 3) & 1);
}

// codes and scale byte of this lane's piece of one page
template <int D>
struct Piece4 {
    uint32_t c[D / 32], b;
};

template <int D>
__device__ __forceinline__ Piece4<D> load_piece4(const unsigned char *page, uint32_t code_at, uint32_t scale_at) {
    Piece4<D> r;
    if constexpr (D == 128) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(page + code_at);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.c[i] = v[i];
    } else {
        const uint2 v = *reinterpret_cast<const uint2 *>(page + code_at);
        r.c[0] = v.x;
        r.c[1] = v.y;
    }
    r.b = page[scale_at];
    return r;
}

// maximum (and sum) over the four lanes of a query row
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

template <int D, int NR, bool DECODE>
__global__ __launch_bounds__(NW4 * 64) void kv4_ways_kernel(Kv4Params p) {
    constexpr int ROWS = 16 * NR, NDS = D / 32, NT = D / 16;
    constexpr int TILE = PAGE4 * D;                       // V elements of one page
    constexpr int RING = 2 * TILE;                        // elements per wavefront; later 16 rows of O in fp32
    extern __shared__ __align__(1024) uint16_t lds[];     // [NW4][RING], then (m, l) [NW4][ROWS]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;

    const int b = DECODE ? (int)blockIdx.y : 0;
    const int mt = (int)blockIdx.x / p.n_groups, gamma = (int)blockIdx.x - mt * p.n_groups;
    const int h = gamma / p.n_split, split = gamma - h * p.n_split;
    int Tp = p.Tp;
    if (DECODE) {
        Tp = p.num_tokens[b];
        if (Tp < 0) return;                               // an empty place of the batch
        if (Tp > p.max_tokens) Tp = p.max_tokens;
    }
    const int Ts = p.Ts, rows = p.rows, grp = p.grp, nq = p.nq, nkv = p.nkv;
    const int n_pre_pages = (Tp + PAGE4 - 1) / PAGE4, n_pre = (n_pre_pages + 1) / 2;
    const uint16_t *const q_in = p.q + (int64_t)b * nq * D;
    const uint16_t *const k_new = p.k_new + ((int64_t)b * nkv + h) * D, *const v_new = p.v_new + ((int64_t)b * nkv + h) * D;
    const __attribute__((address_space(4))) int32_t *pages_c =
        (const __attribute__((address_space(4))) int32_t *)(p.pages + b * p.table_stride);

    // units of this split: the prefix's, then the suffix's up to the tile's last token
    int row_hi = (mt + 1) * ROWS - 1;
    if (row_hi > rows - 1) row_hi = rows - 1;
    const int n_units = n_pre + row_hi / grp / UNIT4 + 1;
    int per = p.units_per_split;
    if (DECODE) {
        // every request over the same number of splits at most, each of a unit per wavefront at least
        per = (n_units + p.n_split - 1) / p.n_split;
        if (per < NW4) per = NW4;
    }
    const int u0 = split * per;
    int u1 = u0 + per;
    if (u1 > n_units) u1 = n_units;
    if (DECODE && u0 >= n_units) return;
    const int n_used = DECODE ? (n_units + per - 1) / per : p.n_split;

    const uint32_t head_codes = (uint32_t)h * (PAGE4 * D / 2), head_scales = (uint32_t)p.code_bytes + (uint32_t)h * (PAGE4 * D / 32);
    if (DECODE && split == 0 && mt == 0 && wave == NW4 - 1) {
        // the token joins the cache: K by the wavefront's first half, V by its second.
        // No lane of the launch reads this slot.
        const int kv = lane >> 5, i = lane & 31;
        if (i < D / 8) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>((kv ? v_new : k_new) + i * 8);
            uint32_t sb;
            const uint32_t codes = kv4_encode8(x, &sb);
            const int slot = Tp % PAGE4;
            unsigned char *page = (kv ? p.pool_v : p.pool_k) + (int64_t)pages_c[Tp / PAGE4] * p.page_bytes;
            *reinterpret_cast<uint32_t *>(page + head_codes + slot * (D / 2) + i * 4) = codes;
            if ((i & 3) == 0) page[head_scales + slot * (D / 32) + i / 4] = (unsigned char)sb;
        }
    }

    // this lane's quarter of Q's rows: dims g * D/4 + s * 8 .. + 8 for product s
    bf16x8 q[NR][NDS];
    int tok[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = mt * ROWS + r * 16 + c;
        const bool ok = row < rows;
        tok[r] = ok ? row / grp : 0;
        const uint16_t *qr = q_in + ((int64_t)tok[r] * nq + h * grp + (ok ? row % grp : 0)) * D + g * (D / 4);
#pragma unroll
        for (int s = 0; s < NDS; ++s) q[r][s] = ok ? *reinterpret_cast<const bf16x8 *>(qr + s * 8) : bf16x8{};
    }
    const int tok0 = mt * ROWS / grp;

    f32x4 o[NR][NT];
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m[r] = -__builtin_inff();
        l[r] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[r][t] = f32x4{};
    }

    uint16_t *const V = lds + wave * RING;
    const int v_put = c * D, v_sw = v4_swz<D>(c);         // this lane's V row of a page
    const int tr = 4 * g + ((lane >> 2) & 3), tq = lane & 3;
    const int v_get = tr * D + (tq & 1) * 4, v_x = (tq >> 1) ^ v4_swz<D>(tr);

    // softmax of one unit's scores s (two pages), then O^T += V^T P
    auto finish = [&](f32x4 (&s)[NR][2]) {
        bf16x8 pp[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float mx[2] = {-__builtin_inff(), -__builtin_inff()};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mx[0] = fmaxf(mx[0], s[r][0][e]);
                mx[1] = fmaxf(mx[1], s[r][1][e]);
            }
            const float mu = fmaxf(mx[0], mx[1]) * p.scale_log2;
            // the running maximum is raised, and O rescaled, only when a score exceeds it by 2^SLACK4
            if (__any(mu > m[r] + SLACK4)) {
                const float mn = fmaxf(m[r], row_max(mu));
                const float alpha = __builtin_amdgcn_exp2f(m[r] - (mn == -__builtin_inff() ? 0.f : mn));
                m[r] = mn;
                l[r] *= alpha;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[r][t] *= alpha;
            }
            const float m_use = m[r] == -__builtin_inff() ? 0.f : m[r];
            f32x8 e;
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[r][i >> 2][i & 3], p.scale_log2, -m_use));
            // bfloat16 P for the matrix cores; the sum is over the rounded values that the product uses
            const bf16x8 bp = __builtin_convertvector(e, bf16x8);
            pp[r] = bp;
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
            float ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(bp, bp, 0, 1), ones, 0.f, false);
            ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(bp, bp, 2, 3), ones, ls, false);
            ls = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(bp, bp, 4, 5), ones, ls, false);
            l[r] += __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(bp, bp, 6, 7), ones, ls, false);
        }
        // the V rows are written by other lanes of this wavefront; its LDS operations complete in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint16_t *vp = V + v_get + (((2 * t) ^ v_x) << 3);
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)vp);
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(vp + TILE));
            const bf16x8 vt = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int r = 0; r < NR; ++r) o[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pp[r], o[r][t], 0, 0, 0);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    };

    // ---- prefix units ----
    const int first = u0 + wave, end_pre = u1 < n_pre ? u1 : n_pre;
    // A unit's pages and this lane's slots in them, held to the last token's: what
    // lies behind it is never read, and its scores are masked.
    auto fetch = [&](int u, Piece4<D> (&k)[2], Piece4<D> (&v)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int pg = 2 * u + i;
            if (pg > n_pre_pages - 1) pg = n_pre_pages - 1;
            const int left = Tp - 1 - pg * PAGE4;
            const uint32_t slot = (uint32_t)(c < left ? c : left);
            const int64_t at = (int64_t)pages_c[pg] * p.page_bytes;
            const uint32_t code_at = head_codes + slot * (D / 2) + g * (D / 8);
            const uint32_t scale_at = head_scales + slot * (D / 32) + g * D / 128;
            k[i] = load_piece4<D>(p.pool_k + at, code_at, scale_at);
            v[i] = load_piece4<D>(p.pool_v + at, code_at, scale_at);
        }
    };
    Piece4<D> k[2], v[2];
    if (first < end_pre) fetch(first, k, v);
    for (int u = first; u < end_pre; u += NW4) {
        Piece4<D> kc[2], vc[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            kc[i] = k[i];
            vc[i] = v[i];
        }
        if (u + NW4 < end_pre) fetch(u + NW4, k, v);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float sc = kv4_scale(vc[i].b);
#pragma unroll
            for (int s = 0; s < NDS; ++s)
                *reinterpret_cast<bf16x8 *>(V + i * TILE + v_put + (((g * NDS + s) ^ v_sw) << 3)) = kv4_decode8(vc[i].c[s], sc);
        }
        f32x4 s4[NR][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float sc = kv4_scale(kc[i].b);
#pragma unroll
            for (int s = 0; s < NDS; ++s) {
                const bf16x8 kf = kv4_decode8(kc[i].c[s], sc);
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    s4[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[r][s], s == 0 ? f32x4{} : s4[r][i], 0, 0, 0);
            }
        }
        if ((u + 1) * UNIT4 > Tp) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = u * UNIT4 + i * PAGE4 + 4 * g + e < Tp;
#pragma unroll
                    for (int r = 0; r < NR; ++r) s4[r][i][e] = seen ? s4[r][i][e] : -__builtin_inff();
                }
        }
        finish(s4);
    }

    // ---- suffix units ----
    int us = first;
    if (us < n_pre) us += (n_pre - us + NW4 - 1) / NW4 * NW4;
    for (; us < u1; us += NW4) {
        const int t0 = (us - n_pre) * UNIT4;
        const bool hidden = t0 + UNIT4 - 1 > tok0;        // some row of the tile does not see every key
        f32x4 s4[NR][2];
        uint32_t odd = 0;                                 // a value of V is infinite or NaN
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int T = t0 + i * PAGE4 + c;
            if (T > Ts - 1) T = Ts - 1;                   // behind the last token: repeats it, masked
            const int64_t at = (int64_t)T * nkv * D + g * (D / 4);
            bf16x8 kf[NDS];
#pragma unroll
            for (int s = 0; s < NDS; ++s) kf[s] = *reinterpret_cast<const bf16x8 *>(k_new + at + s * 8);
#pragma unroll
            for (int s = 0; s < NDS; ++s) {
                u32x4 x = *reinterpret_cast<const u32x4 *>(v_new + at + s * 8);
                if (hidden) {
                    // a row that does not see a key multiplies its V by 0: only finite values may stand there
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t lo = (x[w] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u;
                        const uint32_t hi = (x[w] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
                        odd |= lo | hi;
                        x[w] &= ~(lo | hi);
                    }
                }
                *reinterpret_cast<u32x4 *>(V + i * TILE + v_put + (((g * NDS + s) ^ v_sw) << 3)) = x;
            }
#pragma unroll
            for (int s = 0; s < NDS; ++s)
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    s4[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[s], q[r][s], s == 0 ? f32x4{} : s4[r][i], 0, 0, 0);
        }
        if (hidden) {
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s4[r][i][e] = t0 + i * PAGE4 + 4 * g + e <= tok[r] ? s4[r][i][e] : -__builtin_inff();
        }
        finish(s4);
        if (__any(odd != 0)) {
            // the values left out above, for the rows that see their keys: a key's
            // weight is positive, so they carry an infinity or NaN into the sum
            for (int t = t0; t < t0 + UNIT4 && t < Ts; ++t) {
#pragma unroll
                for (int x = 0; x < NT; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t w = (uint32_t)v_new[(int64_t)t * nkv * D + x * 16 + 4 * g + e] << 16;
                        if ((w & 0x7F800000u) == 0x7F800000u) {
#pragma unroll
                            for (int r = 0; r < NR; ++r)
                                if (t <= tok[r]) o[r][x][e] += __uint_as_float(w);
                        }
                    }
            }
        }
    }

    // ---- merge the wavefronts, 16 rows at a time ----
    // Row r's 16-byte chunks are stored XOR r, so that neither the writes (one
    // row per lane) nor the reads (one chunk per lane) meet on a bank.
    constexpr int CH = D / 4;
    float2 *const ml = reinterpret_cast<float2 *>(lds + NW4 * RING);
    float *const mine = reinterpret_cast<float *>(V);
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const float lt = row_sum(l[r]);
        if (g == 0) ml[wave * ROWS + r * 16 + c] = float2{m[r], lt};
    }
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        if (r > 0) __syncthreads();
#pragma unroll
        for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4 *>(mine + c * D + (((t * 4 + g) ^ c) & (CH - 1)) * 4) = o[r][t];
        __syncthreads();
        for (int i = tid; i < 16 * CH; i += NW4 * 64) {
            const int rr = i / CH, ch = i % CH;
            const int row = mt * ROWS + r * 16 + rr;
            if (row >= rows) break;
            float2 w[NW4];
            float M = -__builtin_inff();
#pragma unroll
            for (int x = 0; x < NW4; ++x) {
                w[x] = ml[x * ROWS + r * 16 + rr];
                M = fmaxf(M, w[x].x);
            }
            const float Mu = M == -__builtin_inff() ? 0.f : M;
            float L = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < NW4; ++x) {
                const float e = __builtin_amdgcn_exp2f(w[x].x - Mu);
                L += e * w[x].y;
                acc += e * *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(lds) + x * (RING / 2) + rr * D +
                                                           ((ch ^ rr) & (CH - 1)) * 4);
            }
            if (n_used == 1) {
                uint16_t *orow = p.out + ((int64_t)b * nq + (int64_t)(row / grp) * nq + h * grp + row % grp) * D;
                *reinterpret_cast<bf16x4 *>(orow + ch * 4) = __builtin_convertvector(acc * (1.f / L), bf16x4);
            } else {
                const int64_t prow = (((int64_t)b * p.n_split + split) * nkv + h) * rows + row;
                *reinterpret_cast<f32x4 *>(p.o_part + prow * D + ch * 4) = acc;
                if (ch == 0) p.ml_part[prow] = float2{M, L};
            }
        }
    }
}

// Merge the splits of each row: weights 2^(m_s - M), normalised by the matching
// sum of l_s.  d/4 threads per (KV head, row) of request blockIdx.y.
template <int D, bool DECODE>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4Params p) {
    constexpr int TPR = D / 4, RPB = 256 / TPR;
    const int b = DECODE ? (int)blockIdx.y : 0;
    const int64_t gr = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (gr >= (int64_t)p.nkv * p.rows) return;
    int n_split = p.n_split;
    if (DECODE) {
        int Tp = p.num_tokens[b];
        if (Tp < 0) return;
        if (Tp > p.max_tokens) Tp = p.max_tokens;
        const int n_units = ((Tp + PAGE4 - 1) / PAGE4 + 1) / 2 + 1;
        int per = (n_units + p.n_split - 1) / p.n_split;
        if (per < NW4) per = NW4;
        n_split = (n_units + per - 1) / per;
        if (n_split == 1) return;                         // written by the attention itself
    }
    const int h = (int)(gr / p.rows), c4 = threadIdx.x % TPR;
    const int64_t row = gr - (int64_t)h * p.rows, step = (int64_t)p.nkv * p.rows;
    const int64_t prow0 = ((int64_t)b * p.n_split * p.nkv + h) * p.rows + row;
    constexpr int GS = 8;
    float M = -__builtin_inff(), L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n_split; s0 += GS) {
        float2 ml[GS];
        f32x4 o[GS];
#pragma unroll
        for (int i = 0; i < GS; ++i) {
            if (s0 + i < n_split) {
                const int64_t prow = prow0 + (int64_t)(s0 + i) * step;
                ml[i] = p.ml_part[prow];
                o[i] = *reinterpret_cast<const f32x4 *>(p.o_part + prow * D + c4 * 4);
            }
        }
        float Mg = M;
#pragma unroll
        for (int i = 0; i < GS; ++i)
            if (s0 + i < n_split) Mg = fmaxf(Mg, ml[i].x);
        const float Mu = Mg == -__builtin_inff() ? 0.f : Mg;
        const float f = __builtin_amdgcn_exp2f(M - Mu);
        L *= f;
        acc *= f;
#pragma unroll
        for (int i = 0; i < GS; ++i) {
            if (s0 + i < n_split) {
                const float w = __builtin_amdgcn_exp2f(ml[i].x - Mu);
                L += w * ml[i].y;
                acc += w * o[i];
            }
        }
        M = Mg;
    }
    uint16_t *orow = p.out + ((int64_t)b * p.nq + row / p.grp * p.nq + h * p.grp + row % p.grp) * D;
    *reinterpret_cast<bf16x4 *>(orow + c4 * 4) = __builtin_convertvector(acc * (1.f / L), bf16x4);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

static int attention_layout(const oc_layout &l) {
    const int rc = check_kv4_layout(l);
    if (rc) return rc;
    if (l.head_dim != 64 && l.head_dim != 128) return fail(OC_ESHAPE, "4-bit attention supports head_dim 64 or 128");
    if (l.page_size != PAGE4) return fail(OC_ESHAPE, "4-bit attention supports page_size 16");
    return OC_OK;
}

static void size_workspace(Kv4Plan &p, int64_t requests) {
    const int64_t rows = requests * p.n_split * p.nkv * p.rows;
    p.off_ml = p.n_split > 1 ? up256((size_t)rows * p.d * 4) : 0;
    p.total = p.n_split > 1 ? p.off_ml + up256((size_t)rows * 8) : 256;
}

int plan_kv4_attention(const oc_layout &l, int64_t Tp, int64_t Ts, Kv4Plan *pl) {
    const int rc = attention_layout(l);
    if (rc) return rc;
    if (Tp < 0 || Ts < 1) return fail(OC_EINVAL, "attention needs prefix_tokens >= 0 and suffix_tokens >= 1");
    // key positions, query rows and their tokens are 32-bit in the kernels
    if (Tp > (int64_t)1 << 30 || Ts > (int64_t)1 << 30 || Tp + Ts > (int64_t)1 << 30)
        return fail(OC_ERANGE, "prefix + suffix tokens exceed 2^30");
    Kv4Plan p{};
    p.Tp = Tp;
    p.Ts = Ts;
    p.nq = l.num_q_heads;
    p.nkv = l.num_kv_heads;
    p.grp = p.nq / p.nkv;
    p.d = l.head_dim;
    p.rows = Ts * p.grp;
    if (p.rows > (int64_t)1 << 30) return fail(OC_ERANGE, "suffix_tokens * (n_q / n_kv) exceeds 2^30");
    p.row_tile = p.rows <= 16 ? 16 : 32;
    p.m_tiles = (int)((p.rows + p.row_tile - 1) / p.row_tile);
    p.n_units = (int)(((Tp + PAGE4 - 1) / PAGE4 + 1) / 2 + (Ts + UNIT4 - 1) / UNIT4);
    const int64_t tiles = (int64_t)p.nkv * p.m_tiles;
    int64_t ns = std::max<int64_t>(1, std::min<int64_t>(512 / tiles, p.n_units / (2 * NW4)));
    p.units_per_split = (int)((p.n_units + ns - 1) / ns);
    p.n_split = (p.n_units + p.units_per_split - 1) / p.units_per_split;
    if (tiles * p.n_split > OC_MAX_GRID_ITEMS / (NW4 * 64))
        return fail(OC_ERANGE, "attention grid of more than 2^32 work-items");
    if ((int64_t)p.nkv * p.rows * (p.d / 4) > OC_MAX_GRID_ITEMS)
        return fail(OC_ERANGE, "split merge grid exceeds 2^32 work-items");
    size_workspace(p, 1);
    *pl = p;
    return OC_OK;
}

int plan_kv4_decode(const oc_layout &l, int64_t batch, int64_t max_tokens, Kv4Plan *pl) {
    const int rc = attention_layout(l);
    if (rc) return rc;
    if (batch < 1 || max_tokens < 0) return fail(OC_EINVAL, "decode needs batch >= 1 and max_tokens >= 0");
    if (batch > 65535) return fail(OC_ERANGE, "decode takes at most 65535 requests");
    if (max_tokens >= (int64_t)1 << 30) return fail(OC_ERANGE, "max_tokens exceeds 2^30");
    Kv4Plan p{};
    p.batch = (int32_t)batch;
    p.Tp = max_tokens;
    p.Ts = 1;
    p.nq = l.num_q_heads;
    p.nkv = l.num_kv_heads;
    p.grp = p.nq / p.nkv;
    p.d = l.head_dim;
    p.rows = p.grp;
    p.row_tile = p.rows <= 16 ? 16 : 32;
    p.m_tiles = (int)((p.rows + p.row_tile - 1) / p.row_tile);
    p.n_units = (int)(((max_tokens + PAGE4 - 1) / PAGE4 + 1) / 2 + 1);
    const int64_t tiles = batch * p.nkv * p.m_tiles;
    const int64_t per = std::max<int64_t>(2 * NW4, (tiles * p.n_units + 2047) / 2048);
    p.n_split = (int)((p.n_units + per - 1) / per);
    if ((int64_t)p.nkv * p.m_tiles * p.n_split > OC_MAX_GRID_ITEMS / (NW4 * 64))
        return fail(OC_ERANGE, "attention grid of more than 2^32 work-items");
    size_workspace(p, batch);
    *pl = p;
    return OC_OK;
}

template <int D, int NR, bool DECODE>
static hipError_t launch_ways4(const Kv4Plan &pl, const Kv4AttnArgs &a, hipStream_t s) {
    Kv4Params p{};
    p.q = a.q;
    p.k_new = a.k_new;
    p.v_new = a.v_new;
    p.pool_k = a.pool_k;
    p.pool_v = a.pool_v;
    p.pages = a.pages;
    p.num_tokens = a.num_tokens;
    p.o_part = reinterpret_cast<float *>(a.ws);
    p.ml_part = reinterpret_cast<float2 *>(a.ws + pl.off_ml);
    p.out = a.out;
    p.page_bytes = a.page_bytes;
    p.table_stride = a.table_stride;
    p.code_bytes = a.code_bytes;
    p.Tp = (int)pl.Tp;
    p.Ts = (int)pl.Ts;
    p.rows = (int)pl.rows;
    p.nq = pl.nq;
    p.nkv = pl.nkv;
    p.grp = pl.grp;
    p.m_tiles = pl.m_tiles;
    p.n_split = pl.n_split;
    p.n_groups = pl.nkv * pl.n_split;
    p.units_per_split = pl.units_per_split;
    p.max_tokens = a.max_tokens;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
    constexpr int LDS = NW4 * 2 * PAGE4 * D * 2 + NW4 * 16 * NR * 8;
    static_assert(16 * D * 4 == 2 * PAGE4 * D * 2, "the wavefronts' O takes the place of their V");
    const hipError_t e = allow_dynamic_lds<&kv4_ways_kernel<D, NR, DECODE>>(LDS);
    if (e != hipSuccess) return e;
    const unsigned y = DECODE ? (unsigned)pl.batch : 1u;
    hipLaunchKernelGGL((kv4_ways_kernel<D, NR, DECODE>), dim3((unsigned)(p.n_groups * pl.m_tiles), y), dim3(NW4 * 64), LDS, s, p);
    if (p.n_split > 1) {
        constexpr int RPB = 256 / (D / 4);
        const int64_t blocks = ((int64_t)p.nkv * p.rows + RPB - 1) / RPB;
        hipLaunchKernelGGL((kv4_merge_kernel<D, DECODE>), dim3((unsigned)blocks, y), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

hipError_t launch_kv4_attention(const Kv4Plan &p, const Kv4AttnArgs &a, hipStream_t s) {
    if (p.batch) {
        if (p.d == 128) return p.row_tile == 16 ? launch_ways4<128, 1, true>(p, a, s) : launch_ways4<128, 2, true>(p, a, s);
        return p.row_tile == 16 ? launch_ways4<64, 1, true>(p, a, s) : launch_ways4<64, 2, true>(p, a, s);
    }
    if (p.d == 128) return p.row_tile == 16 ? launch_ways4<128, 1, false>(p, a, s) : launch_ways4<128, 2, false>(p, a, s);
    return p.row_tile == 16 ? launch_ways4<64, 1, false>(p, a, s) : launch_ways4<64, 2, false>(p, a, s);
}

}  // namespace oc
