// The 4-bit paged cache: page layout, arguments of its kernels, and the device
// code that turns bfloat16 values into codes and back.
//
// A block is 32 consecutive dimensions of one token's row in one head.  Its
// values are code * 2^(b - 127): a 4-bit code each (sign, two exponent bits, one
// mantissa bit: 0 0.5 1 1.5 2 3 4 6) and one scale byte b for the block.  gfx950
// converts two codes with their scale to two bfloat16 in one instruction, exactly,
// for every b of 0..254, and to NaN for b = 255.
//
// One page of K (or of V) holds, for every KV head and slot, head_dim / 2 bytes
// of codes (two to a byte, the even dimension low), then for every head and slot
// head_dim / 32 scale bytes, padded to a multiple of 16 bytes.
#pragma once

#include "common.hpp"

namespace oc {

inline int64_t kv4_code_bytes(const oc_layout &l) {
    return (int64_t)l.num_kv_heads * l.page_size * (l.head_dim / 2);
}
inline int64_t kv4_page_bytes(const oc_layout &l) {
    return (kv4_code_bytes(l) + (int64_t)l.num_kv_heads * l.page_size * (l.head_dim / 32) + 15) / 16 * 16;
}
// OC_OK, or OC_ESHAPE for a head_dim that is no multiple of 32, OC_ERANGE for
// a page of 2^31 bytes or more
int check_kv4_layout(const oc_layout &l);

// ---- store and read back ----------------------------------------------------
struct Kv4Args {
    const uint16_t *k, *v;        // append: rows [num_tokens][n_kv][d]; ingest: k is the staging
    uint16_t *out;                // gather: the staging
    unsigned char *pool_k, *pool_v;   // the layer's K and V pages
    const int32_t *pages;
    int64_t page_bytes;
    int32_t code_bytes;           // of one page
    int32_t first, end;           // logical positions written or read
    int32_t G, n_kv, d, Ps;
    int32_t num_pages;            // ids outside [0, num_pages) name no page: nothing of them is touched
    int32_t lg_g, lg_d8;          // -1: no power of two (filled by the launcher)
};
hipError_t launch_kv4_ingest(Kv4Args a, hipStream_t s);
hipError_t launch_kv4_append(Kv4Args a, hipStream_t s);
hipError_t launch_kv4_gather(Kv4Args a, hipStream_t s);

// ---- attention ----------------------------------------------------------------
struct Kv4Plan {
    int64_t Tp, Ts;
    int32_t nq, nkv, grp, d;
    int64_t rows;                 // query rows per KV head (decode: of one request)
    int32_t row_tile, m_tiles;
    int32_t n_split, n_units, units_per_split;    // key units of two pages, prefix then suffix
    int32_t batch;                // 0: one request's suffix; else requests with a token each
    int32_t ranges, n_ranges;     // decode: key ranges wanted of all requests (0: n_split of each), and at most
    size_t off_ml, total;         // workspace: partial rows, then their (max, sum) pairs
};
struct Kv4AttnArgs {
    const uint16_t *q, *k_new, *v_new;
    unsigned char *pool_k, *pool_v;   // written by the decode form only
    const int32_t *pages;
    int64_t table_stride;
    const int32_t *num_tokens;    // decode: device lengths
    int32_t max_tokens;
    uint16_t *out;
    unsigned char *ws;
    int64_t page_bytes;
    int32_t code_bytes, num_pages;
};
int plan_kv4_attention(const oc_layout &l, int64_t Tp, int64_t Ts, Kv4Plan *p);
int plan_kv4_decode(const oc_layout &l, int64_t batch, int64_t max_tokens, Kv4Plan *p);
hipError_t launch_kv4_attention(const Kv4Plan &p, const Kv4AttnArgs &a, hipStream_t s);

#ifdef __HIPCC__
typedef __bf16 kv4_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 kv4_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t kv4_u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short kv4_u16x2 __attribute__((ext_vector_type(2)));

// scale byte -> the float whose exponent the conversions take
__device__ inline float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// eight codes of one block -> bfloat16 (exact)
__device__ inline kv4_bf16x8 kv4_decode8(uint32_t codes, float scale) {
    const kv4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    const kv4_bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    const kv4_bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    const kv4_bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return kv4_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A block's scale byte from `top`, the largest magnitude's bfloat16 bits (sign
// cleared; the order of the bits is that of the magnitudes, non-finite ones on
// top): the least power of two of which seven cover it, within 2^-125..2^125.
// With top = 1.m * 2^e that is 2^(e-2) for m <= 0.75, else 2^(e-1): 31 added to
// the bits carries into the exponent just where m (7 bits) exceeds 96.  A
// magnitude of 6 to 7 scales becomes 6, no further off than rounding between 4
// and 6 is; over normal values the 32 are off by 11.2 % in the 2-norm, where a
// scale that covers the maximum by 6 has 11.5 % and one by 8 has 11.5 %.
__device__ inline uint32_t kv4_scale_byte(uint32_t top) {
    if (top >= 0x7F80u) return 255u;
    const int b = (int)((top + 31) >> 7) - 2;
    return (uint32_t)(b < 2 ? 2 : b > 252 ? 252 : b);
}

// Eight values of a block that this lane and the three others of its quad hold:
// their codes and (in all four lanes) the block's scale byte.  All four lanes
// must be active.  Codes round to nearest, ties to the even code, and saturate.
__device__ inline uint32_t kv4_encode8(kv4_u32x4 x, uint32_t *scale_byte) {
    const uint32_t w[4] = {x[0], x[1], x[2], x[3]};     // (a bit cast of x[i] itself takes x[0])
    kv4_u16x2 m = __builtin_bit_cast(kv4_u16x2, w[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(kv4_u16x2, w[i] & 0x7FFF7FFFu));
    uint32_t top = m[0] > m[1] ? m[0] : m[1];
    uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xB1, 0xF, 0xF, true);    // lane ^ 1
    top = top > o ? top : o;
    o = (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4E, 0xF, 0xF, true);             // lane ^ 2
    top = top > o ? top : o;
    const uint32_t b = kv4_scale_byte(top);
    *scale_byte = b;
    const float s = kv4_scale(b);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(kv4_bf16x2, w[0]), s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(kv4_bf16x2, w[1]), s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(kv4_bf16x2, w[2]), s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(kv4_bf16x2, w[3]), s, 3);
    return b == 255u ? 0u : r;
}
#endif

}  // namespace oc
