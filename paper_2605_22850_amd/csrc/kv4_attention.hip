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
#include "attention_tiles.hpp"

namespace oc {

constexpr int UNIT4 = 32;         // keys per unit: two pages
constexpr int NW4 = 8;            // wavefronts of a workgroup

struct Kv4Params {
    const uint16_t *q, *k_new, *v_new;
    unsigned char *pool_k, *pool_v;
    const int32_t *pages, *num_tokens;
    float *o_part;
    float2 *ml_part;
    uint16_t *out;
    int64_t page_bytes, table_stride;
    int code_bytes, num_pages, Tp, Ts, rows, nq, nkv, grp, m_tiles, n_split, n_groups, n_units, units_per_split, max_tokens, batch, ranges;
    float scale_log2, per_range;
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
//
// What bounds it, and measured: decode by its codes and scales from memory (eight
// requests of 32K tokens at 64/8/128: 272 MB in 48.5 us, 5.6 TB/s; 30 of 0 to 28560 at
// 32/8/128: 210 MB in 42.6, 4.9 TB/s; matrix units 10 % busy, vector units 30 %).  One new
// token over 32763: 35.7 MB in 9.7 us (10.4 where they are not in the last cache) and a
// merge of 2.8; its 1025 units in 32 splits are 33 each, so that one wavefront of each
// workgroup has a fifth round.  At 128 new tokens over 4096 there is one workgroup to a CU,
// whose eight wavefronts have 16 or 17 units each: 22 us, where the products alone are 7
// at the rate of a large one (matrix units 11 % busy, vector units 33, LDS 28).  Each of a
// head's 32 row tiles reads and decodes all of its keys; by the rule's constants below
// that is 17 us for a workgroup's 132 units, and the chain of 17 dependent rounds (load,
// product, softmax, LDS, product) takes 10.  Sixteen wavefronts to a workgroup, two or three
// units ahead, and the next unit's scores before this one's softmax did not shorten it;
// 64-row tiles with Q in LDS gained at one shape of the 75 below (512 tokens over 1024).
// ---------------------------------------------------------------------------

// XOR on the 16-byte column of V row r (key in its page).  The columns of eight
// rows that a write takes at once differ in their low three bits, and so do the 32-byte
// pairs of the four rows that a transposing read takes at once, so neither meets on
// a bank.  (An XOR by 2 * (r % 8) + r / 8 let every write meet another: 163 LDS cycles a
// unit of one row tile, not 99.)
__device__ __forceinline__ int v4_swz(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }

// Codes and scale byte of this lane's quarter of its key's row, K's or V's.  ONCE (the
// decode form): the codes bypass the caches, since as a rule nothing else reads the page
// in the launch (decode of eight requests of 32K tokens: 58 -> 52.5 us; a lone request's
// 35 MB, which a benchmark finds in the caches again, gains nothing).  Where something
// does, it reads them again: requests that share a prefix, and the further row tiles of
// more than 32 query heads to a KV head.
template <int D>
struct Piece4 {
    uint32_t c[D / 32], b;
};

template <int D, bool ONCE>
__device__ __forceinline__ Piece4<D> load_piece4(const unsigned char *page, uint32_t code_at, uint32_t scale_at) {
    Piece4<D> r;
    if constexpr (D == 128) {
        const u32x4 *from = reinterpret_cast<const u32x4 *>(page + code_at);
        const u32x4 v = ONCE ? __builtin_nontemporal_load(from) : *from;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.c[i] = v[i];
    } else {
        const uint64_t *from = reinterpret_cast<const uint64_t *>(page + code_at);
        const uint64_t v = ONCE ? __builtin_nontemporal_load(from) : *from;
        r.c[0] = (uint32_t)v;
        r.c[1] = (uint32_t)(v >> 32);
    }
    r.b = page[scale_at];
    return r;
}

// max(a, b) in one instruction, NaN left aside; fmaxf() quiets each operand with another
__device__ __forceinline__ float max2(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, __builtin_inff()); }

// maximum (and sum) over the four lanes of a query row
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float row_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// ---- decode: which key range of which request a workgroup has ----
// Sum of x over this lane and the ones before it.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xF, 0xF, false);    // row_shr by 1, 2, 4, 8
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xF, 0xF, false);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xA, 0xF, false);    // row_bcast 15, 31
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xC, 0xF, false);
    return x;
}

// Tokens cached for request b; -1: an empty place, or none.
__device__ __forceinline__ int tokens_of(const Kv4Params &p, int b) {
    if (b >= p.batch) return -1;
    const int t = p.num_tokens[b];
    return t < 0 ? -1 : t > p.max_tokens ? p.max_tokens : t;
}
__device__ __forceinline__ int units_of(int tokens) { return ((tokens + PAGE - 1) / PAGE + 1) / 2; }

// The key ranges of a decode over requests whose lengths only the device knows:
// every request's whole ones of `per` units first, then what is left of each, those of
// more than half a range before the others, so that what starts last is short.  How
// many of each kind there are is one number, ten bits each.  Every wavefront works
// the list out by itself, PER requests to a lane.
__device__ __forceinline__ int kind_of(uint32_t n, int kind) { return (int)(n >> 10 * kind & 1023u); }
__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

template <int PER>
struct RangeList {
    int per;                           // units of a range
    int tokens[PER];                   // this lane's requests
    uint32_t n[PER], upto, all;        // their ranges; those of this lane and the ones before; of all

    // units in all are below 2^24, so a float holds them
    __device__ __forceinline__ RangeList(const Kv4Params &p, int lane) {
        uint32_t sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) tokens[i] = tokens_of(p, lane * PER + i);
#pragma unroll
        for (int i = 0; i < PER; ++i) sum += tokens[i] > 0 ? units_of(tokens[i]) : 0;
        const uint32_t units = lane_of(wave_scan(sum), 63);
        per = ((int)((float)units * p.per_range) + NW4) / NW4 * NW4;     // at least units / ranges
        if (per < p.units_per_split) per = p.units_per_split;
        const float inv = __builtin_amdgcn_rcpf((float)per);
        upto = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int u = tokens[i] > 0 ? units_of(tokens[i]) : 0;
            int whole = (int)((float)u * inv), left = u - whole * per;   // off by one at most
            if (left < 0) --whole, left += per;
            if (left >= per) ++whole, left -= per;
            n[i] = (uint32_t)whole | (left > per / 2 ? 1u << 10 : left || tokens[i] == 0 ? 1u << 20 : 0u);
            upto += n[i];
        }
        upto = wave_scan(upto);
        all = lane_of(upto, 63);
    }
    // Range x of the list: its request, that one's tokens, and which of its ranges; false past the last.
    __device__ __forceinline__ bool find(int x, int &b, int &t, int &split) const {
        int kind = 0;
        while (kind < 3 && x >= kind_of(all, kind)) x -= kind_of(all, kind++);
        if (kind == 3) return false;
        const int at = __ffsll((unsigned long long)__ballot(kind_of(upto, kind) > x)) - 1;
        uint32_t own = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) own += n[i];
        x -= kind_of(lane_of(upto - own, at), kind);
        int in = 0;
#pragma unroll
        for (int i = 0; i + 1 < PER; ++i) {
            const int here = kind_of(lane_of(n[i], at), kind);
            if (in == i && x >= here) x -= here, ++in;
        }
        b = at * PER + in;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (in == i) {
                t = (int)lane_of((uint32_t)tokens[i], at);
                split = kind ? kind_of(lane_of(n[i], at), 0) : x;
            }
        return true;
    }
    // Request b's ranges: how many, its first whole one in the list, and its last one.
    __device__ __forceinline__ int of_request(int b, int &first, int &last) const {
        const int at = b / PER, in = b % PER;
        uint32_t before = upto, mine = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i >= in) before -= n[i];
            if (i == in) mine = n[i];
        }
        before = lane_of(before, at);
        mine = lane_of(mine, at);
        const int whole = kind_of(mine, 0), kind = kind_of(mine, 1) ? 1 : kind_of(mine, 2) ? 2 : 0;
        first = kind_of(before, 0);
        last = kind == 0 ? first + whole - 1
                         : kind_of(all, 0) + (kind == 2 ? kind_of(all, 1) : 0) + kind_of(before, kind);
        return whole + (kind > 0);
    }
};

template <int D, int NR, int PF, bool DECODE>
__global__ __launch_bounds__(NW4 * 64, NR == 1 ? 4 : 2) void kv4_ways_kernel(Kv4Params p) {
    constexpr int ROWS = 16 * NR, NDS = D / 32, NT = D / 16;
    constexpr int TILE = PAGE * D;                       // V elements of one page
    constexpr int RING = 2 * TILE;                        // elements per wavefront; later 16 rows of O in fp32
    extern __shared__ __align__(1024) uint16_t lds[];     // [NW4][RING], then (m, l) [NW4][ROWS]
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c = lane & 15, g = lane >> 4;

    int b = 0, h, mt, split, range, per = p.units_per_split, Tp = p.Tp;
    if (DECODE) {
        // neighbours are of different heads: no XCD gets the long requests
        range = (int)blockIdx.x / p.nkv;
        h = (int)blockIdx.x - range * p.nkv;
        mt = (int)blockIdx.y;
        if (p.ranges) {
            bool some;
            if (p.batch <= 64) {
                const RangeList<1> list(p, lane);
                per = list.per;
                some = list.find(range, b, Tp, split);
            } else {
                const RangeList<2> list(p, lane);
                per = list.per;
                some = list.find(range, b, Tp, split);
            }
            if (!some) return;                            // fewer ranges than workgroups
        } else {
            // first splits, which every request has, come first
            split = range / p.batch;
            b = range - split * p.batch;
            range = b * p.n_split + split;
            Tp = tokens_of(p, b);
            if (Tp < 0) return;                           // an empty place of the batch
        }
    } else {
        mt = (int)blockIdx.x / p.n_groups;
        const int gamma = (int)blockIdx.x - mt * p.n_groups;
        h = gamma / p.n_split;
        split = range = gamma - h * p.n_split;
    }
    const int Ts = p.Ts, rows = p.rows, grp = p.grp, nq = p.nq, nkv = p.nkv;
    const int n_pre_pages = (Tp + PAGE - 1) / PAGE, n_pre = (n_pre_pages + 1) / 2;
    const uint16_t *const q_in = p.q + (int64_t)b * nq * D;
    const uint16_t *const k_new = p.k_new + ((int64_t)b * nkv + h) * D, *const v_new = p.v_new + ((int64_t)b * nkv + h) * D;
    const int32_t *const pages = p.pages + b * p.table_stride;
    const int64_t page_bytes = p.page_bytes;
    const float scale_log2 = p.scale_log2;

    // units of this split: the prefix's, then the suffix's up to the tile's last token
    int row_hi = (mt + 1) * ROWS - 1;
    if (row_hi > rows - 1) row_hi = rows - 1;
    const int n_units = n_pre + row_hi / grp / UNIT4 + 1;
    const int u0 = split * per;
    int u1 = u0 + per, n_used = p.n_split;
    if (DECODE) {
        // the prefix's units are split, and the token's own goes with the last of them
        n_used = n_pre > per ? (n_pre + per - 1) / per : 1;
        if (split >= n_used) return;
        if (split == n_used - 1) u1 = n_units;
    }
    if (u1 > n_units) u1 = n_units;

    const uint32_t head_codes = (uint32_t)h * (PAGE * D / 2), head_scales = (uint32_t)p.code_bytes + (uint32_t)h * (PAGE * D / 32);
    if (DECODE && split == 0 && mt == 0 && wave == NW4 - 1) {
        // the token joins the cache: K by the wavefront's first half, V by its second.
        // No lane of the launch reads this slot.
        const int kv = lane >> 5, i = lane & 31;
        if (i < D / 8) {
            const u32x4 x = *reinterpret_cast<const u32x4 *>((kv ? v_new : k_new) + i * 8);
            uint32_t sb;
            const uint32_t codes = kv4_encode8(x, &sb);
            const int slot = Tp % PAGE;
            const int32_t id = pages[Tp / PAGE];
            if ((uint32_t)id < (uint32_t)p.num_pages) {
                unsigned char *page = (kv ? p.pool_v : p.pool_k) + (int64_t)id * page_bytes;
                *reinterpret_cast<uint32_t *>(page + head_codes + slot * (D / 2) + i * 4) = codes;
                if ((i & 3) == 0) page[head_scales + slot * (D / 32) + i / 4] = (unsigned char)sb;
            }
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
    float m[NR], l[NR], scale[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        scale[r] = scale_log2;
        m[r] = -__builtin_inff();
        l[r] = 0.f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[r][t] = f32x4{};
    }

    uint16_t *const V = lds + wave * RING;
    const int v_put = c * D, v_sw = v4_swz(c);         // this lane's V row of a page
    const int tr = 4 * g + ((lane >> 2) & 3), tq = lane & 3;
    const int v_get = tr * D + (tq & 1) * 4, v_x = (tq >> 1) ^ v4_swz(tr);

    // softmax of one unit's scores s (two pages), then O^T += V^T P
    auto finish = [&](f32x4 (&s)[NR][2]) {
        bf16x8 pp[NR];
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float mx[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) mx[i] = max2(max2(s[r][i][0], s[r][i][1]), max2(s[r][i][2], s[r][i][3]));
            const float top = max2(mx[0], mx[1]);
            // the running maximum is raised, and O rescaled, only when a score exceeds it by 2^RESCALE_SLACK
            if (__any(top * scale[r] > m[r] + RESCALE_SLACK)) {
                const float mn = raise_row(m[r], scale[r], row_max(top), scale_log2);
                scale[r] = row_scale(mn, scale_log2);
                const float alpha = __builtin_amdgcn_exp2f(m[r] - (mn == -__builtin_inff() ? 0.f : mn));
                m[r] = mn;
                l[r] *= alpha;
#pragma unroll
                for (int t = 0; t < NT; ++t) o[r][t] *= alpha;
            }
            const float m_use = m[r] == -__builtin_inff() ? 0.f : m[r];
            f32x8 e;
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[r][i >> 2][i & 3], scale[r], -m_use));
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
    // The addresses of 64 pages at a time, one per lane, K's: a unit's come from there
    // without a wait on memory.
    uint64_t at = 0;
    const int64_t kv_step = p.pool_v - p.pool_k;
    auto load_ids = [&](int u) {
        int pg = 2 * (u + (lane >> 1) * NW4) + (lane & 1);
        if (pg > n_pre_pages - 1) pg = n_pre_pages - 1;
        int32_t id = pages[pg];
        // (the table may hold what a fork or take left that found no page)
        if ((uint32_t)id >= (uint32_t)p.num_pages) id = 0;
        at = reinterpret_cast<uint64_t>(p.pool_k) + (uint64_t)((int64_t)id * page_bytes);
    };
    auto code_at = [&](int slot) { return head_codes + slot * (D / 2) + g * (D / 8); };
    auto scale_at = [&](int slot) { return head_scales + slot * (D / 32) + g * D / 128; };
    const uint32_t my_code = code_at(c), my_scale = scale_at(c);
    Piece4<D> k[PF][2], v[PF][2];
    // the n-th unit of this wavefront, unit u of the prefix
    auto fetch = [&](int n, int u, Piece4<D> (&k)[2], Piece4<D> (&v)[2]) {
        if ((n & 31) == 0) load_ids(u);
        uint32_t ca[2] = {my_code, my_code}, sa[2] = {my_scale, my_scale};
        if ((u + 1) * UNIT4 > Tp) {
            // slots behind the last token repeat it: they are masked, and never read
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                int pg = 2 * u + i;
                if (pg > n_pre_pages - 1) pg = n_pre_pages - 1;
                const int left = Tp - 1 - pg * PAGE, slot = c < left ? c : left;
                ca[i] = code_at(slot);
                sa[i] = scale_at(slot);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int from = (2 * n + i) & 63;
            const unsigned char *const base = reinterpret_cast<const unsigned char *>(
                (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, from) |
                (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(at >> 32), from) << 32);
            k[i] = load_piece4<D, DECODE>(base, ca[i], sa[i]);
            v[i] = load_piece4<D, DECODE>(base + kv_step, ca[i], sa[i]);
        }
    };
    auto unit = [&](int n, int u, Piece4<D> (&k)[2], Piece4<D> (&v)[2]) {
        f32x4 s4[NR][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float sc = kv4_scale(k[i].b);
#pragma unroll
            for (int s = 0; s < NDS; ++s) {
                const bf16x8 kf = kv4_decode8(k[i].c[s], sc);
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    s4[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[r][s], s == 0 ? f32x4{} : s4[r][i], 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float sc = kv4_scale(v[i].b);
#pragma unroll
            for (int s = 0; s < NDS; ++s)
                *reinterpret_cast<bf16x8 *>(V + i * TILE + v_put + (((g * NDS + s) ^ v_sw) << 3)) = kv4_decode8(v[i].c[s], sc);
        }
        // the codes are read: the unit PF further on takes their registers
        if (u + PF * NW4 < end_pre) fetch(n, u + PF * NW4, k, v);
        if ((u + 1) * UNIT4 > Tp) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool seen = u * UNIT4 + i * PAGE + 4 * g + e < Tp;
#pragma unroll
                    for (int r = 0; r < NR; ++r) s4[r][i][e] = seen ? s4[r][i][e] : -__builtin_inff();
                }
        }
        finish(s4);
    };
#pragma unroll
    for (int i = 0; i < PF; ++i)
        if (first + i * NW4 < end_pre) fetch(i, first + i * NW4, k[i], v[i]);
    for (int u = first, n = PF; u < end_pre; u += PF * NW4) {
#pragma unroll
        for (int i = 0; i < PF; ++i, ++n) {
            const int ui = u + i * NW4;
            if (ui >= end_pre) break;
            unit(n, ui, k[i], v[i]);
        }
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
            int T = t0 + i * PAGE + c;
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
                        s4[r][i][e] = t0 + i * PAGE + 4 * g + e <= tok[r] ? s4[r][i][e] : -__builtin_inff();
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
                const int64_t prow = ((int64_t)range * nkv + h) * rows + row;
                *reinterpret_cast<f32x4 *>(p.o_part + prow * D + ch * 4) = acc;
                if (ch == 0) p.ml_part[prow] = float2{M, L};
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Many query rows: 256-row tiles, eight wavefronts of 32 rows each over the same
// 64-key blocks, in the two-phase schedule of the bfloat16 kernel (a wavefront of
// each SIMD in its matrix phase while the other does its softmax).
//
// Only the feed differs.  A wavefront owns one page of each block, waves 0-3 K's
// and waves 4-7 V's: a prefix page's codes come into registers one block ahead (16
// bytes and a scale byte per lane at d = 128), are decoded in a softmax phase, in the
// shadow of the partner's MFMAs, and written to the swizzled bfloat16 tile; a suffix
// page is copied straight to LDS.  Decoding costs 16 conversions per lane and block
// beside some 130 vector operations of the softmax, and the codes a quarter of the
// bytes, so the matrix phases bound this kernel as they do the bfloat16 one.
//
// 512 tokens over 65536 at 32/8/128: 5.52e11 operations in 507 us with its merge, 1.09
// PFLOP/s, where a bfloat16 product of 8192^3 reaches 1.23; matrix units 45 % busy, vector
// units 43 %.  A product with the codes as they are (scaled 4-bit by 8-bit, Q in two
// 8-bit terms) takes as many matrix cycles and a longer start.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(THREADS) void kv4_rows_kernel(Kv4Params p) {
    constexpr int TILE = KB * D, NBUF = 4;
    constexpr int NDW = D / 32;                    // dwords of codes per lane and page
    constexpr int ND = PAGE * D * 2 / 1024;        // 1 KiB copies of a suffix page
    constexpr int KROWS = 512 / D;                 // key rows per copy
    extern __shared__ __align__(1024) uint16_t lds[];   // [NBUF][K tile, V tile], then a flag
    __builtin_amdgcn_s_setprio(1);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const bool is_v = wave >= 4;
    const int my_page = wave & 3;                  // of every block

    const int m_tiles = p.m_tiles, n_split = p.n_split, grp = p.grp, nq = p.nq, nkv = p.nkv;
    const int rows = p.rows, Tp = p.Tp, Ts = p.Ts, n_pre_pages = (Tp + PAGE - 1) / PAGE;
    const float scale_log2 = p.scale_log2;
    const int64_t page_bytes = p.page_bytes;
    const int num_pages = p.num_pages;
    const unsigned char *const pool = is_v ? p.pool_v : p.pool_k;
    const uint16_t *const dense = is_v ? p.v_new : p.k_new;
    const __attribute__((address_space(4))) int32_t *pages_c =
        (const __attribute__((address_space(4))) int32_t *)p.pages;
    int gamma, mt;
    if (!tile_of((int)blockIdx.x, m_tiles, p.n_groups, false, gamma, mt)) return;
    const int g = gamma / n_split, split = gamma - g * n_split;

    const int row = mt * TILE_ROWS + wave * WAVE_ROWS + col;
    const bool row_ok = row < rows;
    const int tok = row_ok ? row / grp : 0;
    bf16x8 qop[D / 16];
    {
        const uint16_t *qr = p.q + ((int64_t)tok * nq + g * grp + (row_ok ? row % grp : 0)) * D + half * 8;
#pragma unroll
        for (int ds = 0; ds < D / 16; ++ds) qop[ds] = row_ok ? *reinterpret_cast<const bf16x8 *>(qr + ds * 16) : bf16x8{};
    }

    const int b0 = split * p.units_per_split;
    int b1 = b0 + p.units_per_split, tok_max;
    {   // causal clip: no row of this tile sees suffix keys past its last token
        int row_hi = (mt + 1) * TILE_ROWS - 1;
        if (row_hi > rows - 1) row_hi = rows - 1;
        tok_max = row_hi / grp;
        const int last = (n_pre_pages + tok_max / PAGE) / 4 + 1;
        if (b1 > last) b1 = last;
        if (b1 > p.n_units) b1 = p.n_units;
    }
    const int nb = b1 > b0 ? b1 - b0 : 0;
    const int tok_tile = mt * TILE_ROWS / grp, tok_min = (mt * TILE_ROWS + wave * WAVE_ROWS) / grp;

    // ---- this wavefront's page of a block ----
    const int key = lane >> 2, piece = lane & 3;   // decoding: this lane's key row and quarter of it
    const uint32_t code_at = (uint32_t)g * (PAGE * D / 2) + piece * (D / 8);
    const uint32_t scale_at = (uint32_t)p.code_bytes + (uint32_t)g * (PAGE * D / 32) + piece * D / 128;
    // V's swizzle moves whole 64-byte units, which all lanes would write in the same
    // order and meet on a bank: a lane starts at a chunk of its own
    const int rot = is_v ? (D == 128 ? key & 3 : (key >> 1) & 1) : 0;
    auto page_of = [&](int j) { return (b0 + j) * 4 + my_page; };
    auto load_pid = [&](int j) -> int {
        int v = page_of(j);
        if (v > n_pre_pages - 1) v = n_pre_pages - 1;
        return v >= 0 ? pages_c[v] : 0;
    };
    struct Raw {
        u32x4 c;
        uint32_t b;
    };
    auto fetch = [&](int j, int pid) -> Raw {
        Raw r{};
        const int v = page_of(j);
        if (v >= n_pre_pages) return r;
        // (the table may hold what a fork or take left that found no page; checked here and
        // not at the load, which is a block ahead and not waited for)
        if ((uint32_t)pid >= (uint32_t)num_pages) pid = 0;
        // slots behind the last token repeat it: they are masked, and never read
        const int left = Tp - 1 - v * PAGE;
        const uint32_t slot = (uint32_t)(key < left ? key : left);
        const unsigned char *base = pool + (int64_t)pid * page_bytes;
        if constexpr (D == 128) {
            r.c = *reinterpret_cast<const u32x4 *>(base + code_at + slot * (D / 2));
        } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(base + code_at + slot * (D / 2));
            r.c = u32x4{x.x, x.y, 0, 0};
        }
        r.b = base[scale_at + slot * (D / 32)];
        return r;
    };
    auto tile_k = [&](int j) -> uint16_t * { return lds + (j % NBUF) * 2 * TILE; };
    auto tile_v = [&](int j) -> uint16_t * { return lds + (j % NBUF) * 2 * TILE + TILE; };
    auto put = [&](int j, const Raw r) {
        uint16_t *const page = (is_v ? tile_v(j) : tile_k(j)) + my_page * PAGE * D;
        const int v = page_of(j);
        if (v < n_pre_pages) {
            const float sc = kv4_scale(r.b);
            u32x4 c = r.c;
            if constexpr (D == 128) {
                c = rot & 1 ? __builtin_shufflevector(c, c, 1, 2, 3, 0) : c;
                c = rot & 2 ? __builtin_shufflevector(c, c, 2, 3, 0, 1) : c;
            } else {
                c = rot ? __builtin_shufflevector(c, c, 1, 0, 2, 3) : c;
            }
            const int rr = my_page * PAGE + key;
            const int swz = is_v ? v_swz<D>(key) : rr & (D / 8 - 1);
#pragma unroll
            for (int i = 0; i < NDW; ++i) {
                const int chunk = piece * NDW + ((i + rot) & (NDW - 1));
                *reinterpret_cast<bf16x8 *>(page + key * D + ((chunk ^ swz) << 3)) = kv4_decode8(c[i], sc);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int r0 = i * KROWS + lane / (D / 8);             // key row within the page
            const int cc = (lane % (D / 8)) ^ (is_v ? v_swz<D>(r0) : r0 & (D / 8 - 1));
            int T = (v - n_pre_pages) * PAGE + r0;
            if (T > Ts - 1) T = Ts - 1;                            // rows past the last one repeat it (masked)
            // below 2^31 bytes: the host limits T_s * n_kv * d * 2
            dma16(dense, ((uint32_t)(T * nkv + g) * D + cc * 8) * 2, page + i * 512);
        }
    };
    int pid = 0;
    Raw raw{};
    // into the buffer of block j - 2, whose last reads have ended (the schedule below)
    auto refill = [&](int j) {
        if (j + 2 < nb) put(j + 2, raw);
        if (j + 3 < nb) {
            raw = fetch(j + 3, pid);
            pid = load_pid(j + 4);
        }
    };
    // This wavefront's copies of block j have landed (its own writes are waited for by
    // the barriers): behind a suffix page come only suffix pages.
    auto await_block = [&](int j) {
        if (page_of(j) < n_pre_pages) return;
        if (j + 1 < nb) wait_vmcnt<ND>();
        else wait_vmcnt<0>();
    };

    WaveState<D> w;
#pragma unroll
    for (int et = 0; et < D / 32; ++et) w.o[et] = f32x16{};
    w.m = -__builtin_inff();
    w.l = 0.f;
    w.scale = scale_log2;
    w.m_use = 0.f;
    const int krow = key_perm(col);
    int voff[D / 32];
#pragma unroll
    for (int et = 0; et < D / 32; ++et) voff[et] = vt_offset<D>(lane, et);

    // Mask of one block, as in the bfloat16 kernel: keys below pe are prefix keys,
    // suffix keys start at ps, and a row sees suffix key k when k - ps <= its token.
    auto mask_block = [&](int b) {
        const int sh = 8 * half;
        const int pe = Tp - b * KB - sh, ps = n_pre_pages * PAGE - b * KB - sh, lim = tok + ps;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int kin = kt * 32 + (i < 8 ? i : 8 + i);
                const uint32_t keep = 0u - (uint32_t)((kin < pe) | ((kin >= ps) & (kin <= lim)));
                w.s[kt][i] = __uint_as_float((__float_as_uint(w.s[kt][i]) & keep) | (0xff800000u & ~keep));
            }
    };
    auto softmax_block = [&](int j) {
        const int b = b0 + j;
        if ((b + 1) * KB > Tp) {
            const int ps = n_pre_pages * PAGE - b * KB, pe = Tp - b * KB;
            const bool partial_prefix = ps > 0 && pe < (ps < KB ? ps : KB);
            const bool unseen_suffix = ps < KB && KB - 1 - ps > tok_min;
            if (partial_prefix || unseen_suffix) mask_block(b);
        }
        softmax_phase<D>(w, scale_log2);
    };
    // Wavefronts 4-7, in phase 2j, each on the V page that it has copied: where some
    // row of the tile does not see a key of the page (its weight there is 0), only
    // finite values may stand; what is taken out is added at the end, row by row.
    uint32_t *const flag = reinterpret_cast<uint32_t *>(lds + NBUF * 2 * TILE);
    auto finite_v = [&](int j) {
        const int v = page_of(j);
        if (j >= nb || v < n_pre_pages || (v - n_pre_pages) * PAGE + PAGE - 1 <= tok_tile) return;
        uint16_t *const page = tile_v(j) + my_page * PAGE * D;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            u32x4 x = *reinterpret_cast<const u32x4 *>(page + i * 512 + lane * 8);
            uint32_t here = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = (x[e] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u;
                const uint32_t hi = (x[e] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
                here |= lo | hi;
                x[e] &= ~(lo | hi);
            }
            if (here) *reinterpret_cast<u32x4 *>(page + i * 512 + lane * 8) = x;
            odd |= here;
        }
        if (odd) *flag = 1;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };

    if (tid == 0) *flag = 0;
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): Q is in registers before the loop
    if (nb > 0) {
        const int p0 = load_pid(0), p1 = load_pid(1), p2 = load_pid(2);
        pid = load_pid(3);
        const Raw r0 = fetch(0, p0), r1 = nb > 1 ? fetch(1, p1) : Raw{};
        if (nb > 2) raw = fetch(2, p2);
        put(0, r0);
        if (nb > 1) put(1, r1);
    }
    // The barriers and buffers are those of the bfloat16 kernel: block j + 2 is put in
    // phase 2j by wavefronts 4-7 and in phase 2j + 1 by wavefronts 0-3, each of them at
    // the start of a softmax phase; the barrier that ends their next matrix phase waits
    // for their LDS writes, before phase 2j + 4, where the tile is first read.
    auto softmax_end = [] { asm volatile("s_barrier" ::: "memory"); };
    if (nb > 0) {
        bf16x8 pre[LOOKAHEAD];
        await_block(0);
        lds_barrier();
        if (!is_v) {
            matrix_phase<D, false, true>(w, nullptr, voff, tile_k(0), qop, krow, half, pre);
            lds_barrier();
            refill(0);
            softmax_block(0);
            for (int j = 1; j < nb; ++j) {
                prefetch_vt<D>(tile_v(j - 1), voff, pre);
                await_block(j);
                softmax_end();
                matrix_phase<D, true, true>(w, tile_v(j - 1), voff, tile_k(j), qop, krow, half, pre);
                lds_barrier();
                refill(j);
                softmax_block(j);
            }
            prefetch_vt<D>(tile_v(nb - 1), voff, pre);
            softmax_end();
            matrix_phase<D, true, false>(w, tile_v(nb - 1), voff, nullptr, qop, krow, half, pre);
            lds_barrier();
        } else {
            refill(0);
            finite_v(0);
            lds_barrier();
            matrix_phase<D, false, true>(w, nullptr, voff, tile_k(0), qop, krow, half, pre);
            for (int j = 1; j < nb; ++j) {
                await_block(j);
                lds_barrier();
                refill(j);
                finite_v(j);
                softmax_block(j - 1);
                prefetch_vt<D>(tile_v(j - 1), voff, pre);
                softmax_end();
                matrix_phase<D, true, true>(w, tile_v(j - 1), voff, tile_k(j), qop, krow, half, pre);
            }
            lds_barrier();
            softmax_block(nb - 1);
            prefetch_vt<D>(tile_v(nb - 1), voff, pre);
            softmax_end();
            matrix_phase<D, true, false>(w, tile_v(nb - 1), voff, nullptr, qop, krow, half, pre);
        }
        if (*flag) {
            // weights are positive, so a row carries the infinities and NaN of the keys it sees
            int t0 = (b0 * 4 - n_pre_pages) * PAGE, t1 = (b1 * 4 - n_pre_pages) * PAGE;
            if (t0 < 0) t0 = 0;
            if (t1 > tok_max + 1) t1 = tok_max + 1;
            for (int t = t0; t < t1; ++t) {
                const uint16_t *vr = p.v_new + ((int64_t)t * nkv + g) * D;
#pragma unroll
                for (int et = 0; et < D / 32; ++et)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t x = (uint32_t)vr[et * 32 + (i >> 2) * 8 + half * 4 + (i & 3)] << 16;
                        if ((x & 0x7F800000u) == 0x7F800000u && t <= tok) w.o[et][i] += __uint_as_float(x);
                    }
            }
        }
    }

    const float l_tot = half_swap_sum(w.l);
    if (!row_ok) return;
    if (n_split == 1) {
        const float inv = 1.f / l_tot;
        uint16_t *orow = p.out + ((int64_t)tok * nq + g * grp + row % grp) * D;
#pragma unroll
        for (int et = 0; et < D / 32; ++et)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) {
                f32x4 o4 = {w.o[et][vq * 4 + 0], w.o[et][vq * 4 + 1], w.o[et][vq * 4 + 2], w.o[et][vq * 4 + 3]};
                *reinterpret_cast<bf16x4 *>(orow + et * 32 + vq * 8 + half * 4) = __builtin_convertvector(o4 * inv, bf16x4);
            }
    } else {
        const int64_t prow = ((int64_t)split * nkv + g) * rows + row;
        float *orow = p.o_part + prow * D;
#pragma unroll
        for (int et = 0; et < D / 32; ++et)
#pragma unroll
            for (int vq = 0; vq < 4; ++vq) {
                f32x4 o4 = {w.o[et][vq * 4 + 0], w.o[et][vq * 4 + 1], w.o[et][vq * 4 + 2], w.o[et][vq * 4 + 3]};
                *reinterpret_cast<f32x4 *>(orow + et * 32 + vq * 8 + half * 4) = o4;
            }
        if (half == 0) p.ml_part[prow] = float2{w.m, l_tot};
    }
}

// Merge the splits of each row: weights 2^(m_s - M), normalised by the matching
// sum of l_s.  d/4 threads of four dimensions for a (KV head, row), and SG such
// groups over the splits of one row: with many splits their partials are all in
// flight at once (61 splits of four rows: 9.4 us with SG = 1, 3.9 with 8).  Bound by
// its bytes where there are many rows: the two splits of 512 tokens of 32 heads, 34 MB,
// in 8.3 us (4.0 TB/s).  Split s is partial first + s, the last one partial `last`.
template <int D, int SG>
__device__ __forceinline__ void merge_rows(const Kv4Params &p, int b, int first, int n_split, int last) {
    constexpr int TPR = D / 4, RPB = 256 / (TPR * SG), GS = 8;
    const int sg = (int)threadIdx.x / TPR % SG, c4 = (int)threadIdx.x % TPR, in = (int)threadIdx.x / (TPR * SG);
    const int64_t gr = (int64_t)blockIdx.x * RPB + in;
    float M = -__builtin_inff(), L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const bool ok = gr < (int64_t)p.nkv * p.rows;
    const int h = ok ? (int)(gr / p.rows) : 0;
    const int64_t row = ok ? gr - (int64_t)h * p.rows : 0;
    if (ok) {
        const int64_t step = (int64_t)p.nkv * p.rows;
        const int64_t prow0 = (int64_t)h * p.rows + row;
        for (int s0 = sg; s0 < n_split; s0 += SG * GS) {
            float2 ml[GS];
            f32x4 o[GS];
#pragma unroll
            for (int i = 0; i < GS; ++i) {
                if (s0 + i * SG < n_split) {
                    const int x = s0 + i * SG;
                    const int64_t prow = prow0 + (int64_t)(x == n_split - 1 ? last : first + x) * step;
                    ml[i] = p.ml_part[prow];
                    o[i] = *reinterpret_cast<const f32x4 *>(p.o_part + prow * D + c4 * 4);
                }
            }
            float Mg = M;
#pragma unroll
            for (int i = 0; i < GS; ++i)
                if (s0 + i * SG < n_split) Mg = fmaxf(Mg, ml[i].x);
            const float Mu = Mg == -__builtin_inff() ? 0.f : Mg;
            const float f = __builtin_amdgcn_exp2f(M - Mu);
            L *= f;
            acc *= f;
#pragma unroll
            for (int i = 0; i < GS; ++i) {
                if (s0 + i * SG < n_split) {
                    const float w = __builtin_amdgcn_exp2f(ml[i].x - Mu);
                    L += w * ml[i].y;
                    acc += w * o[i];
                }
            }
            M = Mg;
        }
    }
    if constexpr (SG > 1) {
        __shared__ float part[RPB][SG][TPR][6];
        float *const mine = part[in][sg][c4];
        mine[0] = M;
        mine[1] = L;
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[2 + i] = acc[i];
        __syncthreads();
        if (sg) return;
        float Mg = M;
        for (int x = 1; x < SG; ++x) Mg = fmaxf(Mg, part[in][x][c4][0]);
        const float Mu = Mg == -__builtin_inff() ? 0.f : Mg;
        const float f = __builtin_amdgcn_exp2f(M - Mu);
        L *= f;
        acc *= f;
        for (int x = 1; x < SG; ++x) {
            const float *const o = part[in][x][c4];
            const float w = __builtin_amdgcn_exp2f(o[0] - Mu);
            L += w * o[1];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += w * o[2 + i];
        }
    }
    if (!ok) return;
    uint16_t *orow = p.out + ((int64_t)b * p.nq + row / p.grp * p.nq + h * p.grp + row % p.grp) * D;
    *reinterpret_cast<bf16x4 *>(orow + c4 * 4) = __builtin_convertvector(acc * (1.f / L), bf16x4);
}

template <int D, int SG>
__global__ __launch_bounds__(256) void kv4_merge_kernel(Kv4Params p) {
    merge_rows<D, SG>(p, 0, 0, p.n_split, p.n_split - 1);
}

// The same for request blockIdx.y of a decode, whose splits only the device knows.
template <int D>
__global__ __launch_bounds__(256) void kv4_decode_merge_kernel(Kv4Params p) {
    const int b = (int)blockIdx.y;
    int n_split, first, last;
    if (p.ranges) {
        const int lane = (int)threadIdx.x & 63;
        n_split = p.batch <= 64 ? RangeList<1>(p, lane).of_request(b, first, last)
                                : RangeList<2>(p, lane).of_request(b, first, last);
    } else {
        const int t = tokens_of(p, b), n = t < 0 ? 0 : units_of(t);
        n_split = (n + p.units_per_split - 1) / p.units_per_split;
        first = b * p.n_split;
        last = first + n_split - 1;
    }
    if (n_split < 2) return;                              // written by the attention itself, or empty
    if (n_split > 8) merge_rows<D, 8>(p, b, first, n_split, last);
    else merge_rows<D, 1>(p, b, first, n_split, last);
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
static size_t up256(size_t x) { return (x + 255) / 256 * 256; }

static int attention_layout(const oc_layout &l) {
    const int rc = check_kv4_layout(l);
    if (rc) return rc;
    if (l.head_dim != 64 && l.head_dim != 128) return fail(OC_ESHAPE, "4-bit attention supports head_dim 64 or 128");
    if (l.page_size != PAGE) return fail(OC_ESHAPE, "4-bit attention supports page_size 16");
    return OC_OK;
}

// workgroups of the 256-row kernel
static int64_t rows_grid(const Kv4Plan &p) {
    const int64_t groups = (int64_t)p.nkv * p.n_split;
    if (groups <= INT32_MAX && tiles_by_xcd(p.m_tiles, (int)groups, false)) return (groups + 7) / 8 * 8 * p.m_tiles;
    return groups * p.m_tiles;
}

static void size_workspace(Kv4Plan &p) {
    const int64_t rows = (int64_t)p.n_split * p.nkv * p.rows;
    p.off_ml = p.n_split > 1 ? up256((size_t)rows * p.d * 4) : 0;
    p.total = p.n_split > 1 ? p.off_ml + up256((size_t)rows * 8) : 256;
}

// Tiles and splits of one request's attention: `ns` key ranges at most.
static Kv4Plan plan_tiles(const oc_layout &l, int64_t Tp, int64_t Ts, int row_tile, int64_t ns) {
    Kv4Plan p{};
    p.Tp = Tp;
    p.Ts = Ts;
    p.nq = l.num_q_heads;
    p.nkv = l.num_kv_heads;
    p.grp = p.nq / p.nkv;
    p.d = l.head_dim;
    p.rows = Ts * p.grp;
    p.row_tile = row_tile;
    p.m_tiles = (int)((p.rows + row_tile - 1) / row_tile);
    const int64_t pre_pages = (Tp + PAGE - 1) / PAGE;
    p.n_units = (int)(row_tile == TILE_ROWS ? (pre_pages + (Ts + PAGE - 1) / PAGE + 3) / 4
                                            : (pre_pages + 1) / 2 + (Ts + UNIT4 - 1) / UNIT4);
    ns = std::max<int64_t>(1, std::min<int64_t>(ns, p.n_units));
    p.units_per_split = (int)((p.n_units + ns - 1) / ns);
    p.n_split = (p.n_units + p.units_per_split - 1) / p.units_per_split;
    size_workspace(p);
    return p;
}

// Estimated time (us) of one request's attention under a plan: the rule that picks
// the row tile and the splits.  Fitted to 75 shapes (n_q/n_kv/d of 32/8/128, 64/8/128,
// 4/1/128, 6/2/128, 32/4/64, 8/8/64, 4/2/64; prefixes of 16 to 65536 tokens, suffixes
// of 1 to 3584) with up to 30 plans each: over them the plan it picks is 2 % slower
// than the best one measured, on average; it loses most (14 to 31 % on five shapes)
// where several hundred new tokens follow a short prefix.
struct Kv4Cost {
    double unit128, unit64;     // one unit of one workgroup, at d = 128 and 64
    double suffix;              // a suffix unit's extra (its rows are not fetched ahead)
    double round;               // the least time of one unit per wavefront (row_tile 256: of a block)
    double start;               // launch, first loads, epilogue
    double wave;                // each further workgroup per CU
};
static const Kv4Cost COST4_16 = {0.132, 0.061, 0.197, 0.588, 4.9, 0.5}, COST4_32 = {0.184, 0.094, 0.191, 0.379, 6.1, 3.3},
                     COST4_256 = {1.76, 1.32, 0., 1.32, 6.0, 0.};

static double plan4_cost(const Kv4Plan &p) {
    const bool large = p.row_tile == TILE_ROWS;
    const Kv4Cost &k = p.row_tile == 16 ? COST4_16 : large ? COST4_256 : COST4_32;
    const double pre = (double)((p.Tp + PAGE - 1) / PAGE), suf = (double)((p.Ts + PAGE - 1) / PAGE);
    // average share of the keys that a row tile sees under the causal mask
    const double seen = p.m_tiles > 1 ? (pre + 0.5 * (suf + 1)) / (pre + suf) : 1.0;
    const double per_cu = (double)p.nkv * p.m_tiles * p.n_split / 256;
    const double crowd = per_cu > 1 ? seen * std::max(1.0, std::min(std::ceil(per_cu), per_cu + 0.55)) : 1.0;
    const double ups = p.units_per_split, suffix_units = std::min(ups, (double)((p.Ts + UNIT4 - 1) / UNIT4));
    double body = ((p.d == 128 ? k.unit128 : k.unit64) * ups + k.suffix * suffix_units) * crowd;
    body = std::max(body, k.round * (large ? ups : std::ceil(ups / NW4)));
    // all inputs and the output once at 5 TB/s
    const double hbm = p.d * (2.0 * p.nq * p.Ts + p.nkv * (1.0625 * p.Tp + 4.0 * p.Ts)) / 5e6;
    double t = k.start + std::sqrt(body * body + hbm * hbm);
    if (per_cu > 1) t += k.wave * (std::ceil(per_cu) - 1);
    // the merge's launch, and its partials written and read
    if (p.n_split > 1) t += 2.1 + 0.585e-6 * p.n_split * p.nkv * (double)p.rows * p.d * 4;
    return t;
}

int plan_kv4_attention(const oc_layout &l, int64_t Tp, int64_t Ts, Kv4Plan *pl) {
    const int rc = attention_layout(l);
    if (rc) return rc;
    if (Tp < 0 || Ts < 1) return fail(OC_EINVAL, "attention needs prefix_tokens >= 0 and suffix_tokens >= 1");
    // key positions, query rows and their tokens are 32-bit in the kernels
    if (Tp > (int64_t)1 << 30 || Ts > (int64_t)1 << 30 || Tp + Ts > (int64_t)1 << 30)
        return fail(OC_ERANGE, "prefix + suffix tokens exceed 2^30");
    // suffix rows are copied to LDS with 32-bit byte offsets from k_new / v_new
    if (Ts * l.num_kv_heads > INT32_MAX / l.head_dim / 2)
        return fail(OC_ERANGE, "suffix K/V of more than 2^31 bytes (suffix_tokens * n_kv * d * 2)");
    if (Ts * (l.num_q_heads / l.num_kv_heads) > (int64_t)1 << 30)
        return fail(OC_ERANGE, "suffix_tokens * (n_q / n_kv) exceeds 2^30");
    Kv4Plan best = plan_tiles(l, Tp, Ts, TILE_ROWS, 1);
    double least = plan4_cost(best);
    for (const int tile : {16, 32, TILE_ROWS})
        for (const int ns : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            const Kv4Plan p = plan_tiles(l, Tp, Ts, tile, ns);
            const int64_t tiles = (int64_t)p.nkv * p.m_tiles;
            if (tile != TILE_ROWS && tiles > 2048) continue;       // long suffixes: 256-row tiles
            if (ns > 1 && (ns > p.n_units || tiles * ns > 1024)) break;
            const double t = plan4_cost(p);
            if (t < least) {
                least = t;
                best = p;
            }
        }
    if (rows_grid(best) > OC_MAX_GRID_ITEMS / THREADS)
        return fail(OC_ERANGE, "attention grid of more than 2^32 work-items");
    if ((int64_t)best.nkv * best.rows * (best.d / 4) * 8 > OC_MAX_GRID_ITEMS)
        return fail(OC_ERANGE, "split merge grid exceeds 2^32 work-items");
    *pl = best;
    return OC_OK;
}

// Decode: the prefix units of each (request, KV head) in ranges that are work for one
// workgroup.  Where lengths that differ can leave CUs idle, the kernels make the list
// of ranges from the lengths (RangeList): one range to a CU if all were whole.  Against
// ranges of one length chosen here for requests of max_tokens: 12 requests of 0 to
// 19248 tokens 41 -> 15.8 us, 50 of up to 32K 52.7 -> 39.3, 53 of up to 32664 with 64
// query heads 64 -> 56; requests of equal length within 4 % either way.  More ranges
// were slower (256 / 512 / 768 of them: 43 / 46 / 44 us for 45 requests, 52 / 55 / 55 for
// eight of 32000 tokens).
//
// Where every CU has a request anyway and none takes more than 160 units (some 30 us), a
// list and a merge only cost (64 requests of up to 3000 tokens 18 us, 21 with them), as
// they do past 128 requests.  Those, and single requests, get ranges of one length: as
// many as would fill the CUs if all were as long as they may be, and of at most 160
// units.  Up to 24 units are one range: a merge costs 2.5 us, as much as two or three
// units per wavefront.
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
    p.n_units = (int)(((max_tokens + PAGE - 1) / PAGE + 1) / 2);
    const int64_t pairs = batch * p.nkv;
    if (p.m_tiles > 65535) return fail(OC_ERANGE, "more than 65535 * 32 query heads to a KV head");
    const int64_t most = OC_MAX_GRID_ITEMS / THREADS / p.nkv;       // ranges a grid can have
    const int64_t fill = 256 / (pairs * p.m_tiles);                // ranges of each pair that fill the CUs
    int64_t n_ranges = batch;
    p.n_split = 1;
    p.units_per_split = std::max(3 * NW4, (p.n_units + NW4 - 1) / NW4 * NW4);
    if (batch > 1 && batch <= 128 && batch * p.n_units < 1 << 24 && p.n_units > (fill ? 3 * NW4 : 160)) {
        p.ranges = (int)std::max<int64_t>(1, 256 / ((int64_t)p.nkv * p.m_tiles));
        p.units_per_split = NW4;                                  // at least
        p.n_split = (p.n_units + NW4 - 1) / NW4;                  // at most, of one request
        n_ranges = std::min(p.ranges + batch, batch * p.n_split);
    } else if (p.n_units > 3 * NW4) {
        const int64_t at_once = std::max<int64_t>(1, fill);
        int64_t ns = (std::max<int64_t>(at_once, (p.n_units + 159) / 160) + at_once - 1) / at_once * at_once;
        ns = std::min(ns, std::max<int64_t>(1, most / batch));
        const int64_t per = (p.n_units + ns - 1) / ns;
        p.units_per_split = (int)((per + NW4 - 1) / NW4 * NW4);
        p.n_split = (p.n_units + p.units_per_split - 1) / p.units_per_split;
        n_ranges = batch * p.n_split;
    }
    if (n_ranges > most) return fail(OC_ERANGE, "attention grid of more than 2^32 work-items");
    p.n_ranges = (int32_t)n_ranges;
    if (pairs * p.rows * (p.d / 4) * 8 > OC_MAX_GRID_ITEMS) return fail(OC_ERANGE, "merge grid exceeds 2^32 work-items");
    const int64_t rows = n_ranges * p.nkv * p.rows;
    p.off_ml = p.n_split > 1 ? up256((size_t)rows * p.d * 4) : 0;
    p.total = p.n_split > 1 ? p.off_ml + up256((size_t)rows * 8) : 256;
    *pl = p;
    return OC_OK;
}

template <int D>
static Kv4Params make_params(const Kv4Plan &pl, const Kv4AttnArgs &a) {
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
    p.num_pages = a.num_pages;
    p.Tp = (int)pl.Tp;
    p.Ts = (int)pl.Ts;
    p.rows = (int)pl.rows;
    p.nq = pl.nq;
    p.nkv = pl.nkv;
    p.grp = pl.grp;
    p.m_tiles = pl.m_tiles;
    p.n_split = pl.n_split;
    p.n_groups = pl.nkv * pl.n_split;
    p.n_units = pl.n_units;
    p.units_per_split = pl.units_per_split;
    p.max_tokens = a.max_tokens;
    p.batch = pl.batch;
    p.ranges = pl.ranges;
    p.per_range = pl.ranges ? 1.f / (float)pl.ranges : 0.f;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)D));
    return p;
}

// `requests`: 0 for one request's suffix
template <int D>
static void launch_merge(const Kv4Params &p, unsigned requests, hipStream_t s) {
    if (p.n_split < 2) return;
    constexpr int RPB = 256 / (D / 4);
    const int64_t n = (int64_t)p.nkv * p.rows * (p.n_split > 8 ? 8 : 1);
    const dim3 grid((unsigned)((n + RPB - 1) / RPB), std::max(1u, requests));
    if (requests) hipLaunchKernelGGL(kv4_decode_merge_kernel<D>, grid, dim3(256), 0, s, p);
    else if (p.n_split > 8) hipLaunchKernelGGL((kv4_merge_kernel<D, 8>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((kv4_merge_kernel<D, 1>), grid, dim3(256), 0, s, p);
}

template <int D>
static hipError_t launch_rows(const Kv4Plan &pl, const Kv4AttnArgs &a, hipStream_t s) {
    constexpr int LDS = 4 * 2 * KB * D * 2 + 16;
    const hipError_t e = allow_dynamic_lds<&kv4_rows_kernel<D>>(LDS);
    if (e != hipSuccess) return e;
    const Kv4Params p = make_params<D>(pl, a);
    hipLaunchKernelGGL(kv4_rows_kernel<D>, dim3((unsigned)rows_grid(pl)), dim3(THREADS), LDS, s, p);
    launch_merge<D>(p, 0, s);
    return hipGetLastError();
}

template <int D, int NR, int PF, bool DECODE>
static hipError_t launch_ways4(const Kv4Plan &pl, const Kv4AttnArgs &a, hipStream_t s) {
    const Kv4Params p = make_params<D>(pl, a);
    constexpr int LDS = NW4 * 2 * PAGE * D * 2 + NW4 * 16 * NR * 8;
    static_assert(16 * D * 4 == 2 * PAGE * D * 2, "the wavefronts' O takes the place of their V");
    static_assert(NW4 * 64 == THREADS, "the grid's limit is shared");
    const hipError_t e = allow_dynamic_lds<&kv4_ways_kernel<D, NR, PF, DECODE>>(LDS);
    if (e != hipSuccess) return e;
    const dim3 grid = DECODE ? dim3((unsigned)(pl.n_ranges * pl.nkv), (unsigned)pl.m_tiles) : dim3((unsigned)(p.n_groups * pl.m_tiles));
    hipLaunchKernelGGL((kv4_ways_kernel<D, NR, PF, DECODE>), grid, dim3(NW4 * 64), LDS, s, p);
    launch_merge<D>(p, DECODE ? (unsigned)pl.batch : 0u, s);
    return hipGetLastError();
}

hipError_t launch_kv4_attention(const Kv4Plan &p, const Kv4AttnArgs &a, hipStream_t s) {
    if (p.row_tile == TILE_ROWS) return p.d == 128 ? launch_rows<128>(p, a, s) : launch_rows<64>(p, a, s);
    if (p.batch) {
        if (p.d == 128) return p.row_tile == 16 ? launch_ways4<128, 1, 1, true>(p, a, s) : launch_ways4<128, 2, 2, true>(p, a, s);
        return p.row_tile == 16 ? launch_ways4<64, 1, 2, true>(p, a, s) : launch_ways4<64, 2, 2, true>(p, a, s);
    }
    if (p.d == 128) return p.row_tile == 16 ? launch_ways4<128, 1, 1, false>(p, a, s) : launch_ways4<128, 2, 2, false>(p, a, s);
    return p.row_tile == 16 ? launch_ways4<64, 1, 2, false>(p, a, s) : launch_ways4<64, 2, 2, false>(p, a, s);
}

}  // namespace oc
