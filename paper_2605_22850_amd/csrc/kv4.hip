// Store and read-back of the 4-bit paged cache: a layer's payload or a
// request's new rows are quantised into the pages of a block table, and a
// layer's prefix is read back as the bfloat16 values its codes stand for.
//
// Both directions are one pass: 2 bytes a value on the payload's side, 17/32
// of a byte on the pool's.  A wavefront owns one (page, K or V, head): its lanes
// take 16-byte pieces (8 values) of the page's rows in slot order, so a load
// instruction reads whole rows of the payload (d = 128: four rows of 256 bytes) and
// the codes of the page go out as one contiguous stretch.  The four lanes of a quad
// hold one block and find its largest magnitude among themselves.
//
// Bound by memory: a layer of 65536 tokens of 8 heads of 128 is stored in 68 us (340
// MB, 5.0 TB/s) and 66048 of them read back in 50 (342 MB; the codes, just written, are
// partly in the last cache).  A copy of 1 GiB moves 5.1 TB/s.  The least calls (256
// tokens) take 3.2 us, a launch.
#include "kv4.hpp"

namespace oc {

constexpr int kWaves = 4;

// the shift or the division by a positive number
__device__ inline uint32_t div_by(uint32_t x, int lg, uint32_t n) { return lg >= 0 ? x >> lg : x / n; }

// element offset of piece (T, kv, h, c) in a layer payload
__device__ inline int64_t payload_at(const Kv4Args &a, uint32_t T, int kv, int h, int c) {
    const uint32_t j = div_by(T, a.lg_g, (uint32_t)a.G), t = T - j * (uint32_t)a.G;
    return ((((int64_t)j * 2 + kv) * a.G + t) * a.n_kv + h) * a.d + c * 8;
}

// Which page, half and head this wavefront has; false past the last, and where the
// table names no page of the pool (a fork or take that found none leaves -1, which the
// host does not see).
struct Unit {
    int kv, h;
    uint32_t q;              // page of the table
    unsigned char *page;     // its bytes in the pool
};
__device__ inline bool unit_of(const Kv4Args &a, Unit &u) {
    const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const uint32_t i = blockIdx.x * kWaves + wave, per_page = 2u * (uint32_t)a.n_kv;
    const uint32_t n = i / per_page, r = i - n * per_page;
    u.q = (uint32_t)a.first / (uint32_t)a.Ps + n;
    if ((int64_t)u.q * a.Ps >= a.end) return false;
    const int32_t id = a.pages[u.q];
    if ((uint32_t)id >= (uint32_t)a.num_pages) return false;
    u.kv = r >= (uint32_t)a.n_kv;
    u.h = (int)(r - (u.kv ? (uint32_t)a.n_kv : 0u));
    u.page = (u.kv ? a.pool_v : a.pool_k) + (int64_t)id * a.page_bytes;
    return true;
}

template <bool APPEND>
__global__ __launch_bounds__(kWaves * 64) void kv4_store_kernel(Kv4Args a) {
    Unit u;
    if (!unit_of(a, u)) return;
    const int lane = threadIdx.x & 63, d8 = a.d / 8, pieces = a.Ps * d8;
    unsigned char *const codes = u.page + (int64_t)u.h * a.Ps * (a.d / 2);
    unsigned char *const scales = u.page + a.code_bytes + (int64_t)u.h * a.Ps * (a.d / 32);
    // four pieces a lane at a time, so that their loads are in flight together
    for (int p0 = 0; p0 < pieces; p0 += 256) {
        kv4_u32x4 x[4];
        bool ok[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = (uint32_t)(p0 + i * 64 + lane);
            const uint32_t slot = div_by(p, a.lg_d8, (uint32_t)d8), c = p - slot * (uint32_t)d8;
            const uint32_t T = u.q * (uint32_t)a.Ps + slot;
            // a quad's pieces are of one slot: it is wholly in or out
            ok[i] = p < (uint32_t)pieces && T >= (uint32_t)a.first && T < (uint32_t)a.end;
            if (!ok[i]) continue;
            const uint16_t *src;
            if (APPEND) src = (u.kv ? a.v : a.k) + (((int64_t)(T - (uint32_t)a.first) * a.n_kv + u.h) * a.d + c * 8);
            else src = a.k + payload_at(a, T, u.kv, u.h, (int)c);
            x[i] = __builtin_nontemporal_load(reinterpret_cast<const kv4_u32x4 *>(src));
        }
        uint32_t mine = 0;
        bool write = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!ok[i]) continue;
            uint32_t b;
            const uint32_t c8 = kv4_encode8(x[i], &b);
            *reinterpret_cast<uint32_t *>(codes + (int64_t)(p0 + i * 64 + lane) * 4) = c8;
            if ((lane & 3) == i) {
                mine = b;
                write = true;
            }
        }
        // lane i of a quad writes the scale byte of the quad's i-th piece
        if (write) scales[(p0 + (lane & 3) * 64 + (lane & ~3)) / 4] = (unsigned char)mine;
    }
}

__global__ __launch_bounds__(kWaves * 64) void kv4_gather_kernel(Kv4Args a) {
    Unit u;
    if (!unit_of(a, u)) return;
    const int lane = threadIdx.x & 63, d8 = a.d / 8, pieces = a.Ps * d8;
    const unsigned char *const codes = u.page + (int64_t)u.h * a.Ps * (a.d / 2);
    const unsigned char *const scales = u.page + a.code_bytes + (int64_t)u.h * a.Ps * (a.d / 32);
    for (int p0 = 0; p0 < pieces; p0 += 256) {
        uint32_t c8[4], b[4];
        int64_t to[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = (uint32_t)(p0 + i * 64 + lane);
            const uint32_t slot = div_by(p, a.lg_d8, (uint32_t)d8), c = p - slot * (uint32_t)d8;
            const uint32_t T = u.q * (uint32_t)a.Ps + slot;
            to[i] = -1;
            if (p >= (uint32_t)pieces || T >= (uint32_t)a.end) continue;
            c8[i] = *reinterpret_cast<const uint32_t *>(codes + (int64_t)p * 4);
            b[i] = scales[p / 4];
            to[i] = payload_at(a, T, u.kv, u.h, (int)c);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (to[i] < 0) continue;
            const kv4_bf16x8 v = kv4_decode8(c8[i], kv4_scale(b[i]));
            __builtin_nontemporal_store(__builtin_bit_cast(kv4_u32x4, v), reinterpret_cast<kv4_u32x4 *>(a.out + to[i]));
        }
    }
}

static int lg_or_none(int64_t x) {
    if (x <= 0 || (x & (x - 1))) return -1;
    int r = 0;
    while ((INT64_C(1) << r) < x) ++r;
    return r;
}

// wavefronts of the pages from the first position's to the last one's
static dim3 unit_grid(Kv4Args &a) {
    a.lg_g = lg_or_none(a.G);
    a.lg_d8 = lg_or_none(a.d / 8);
    const int64_t pages = (a.end - 1) / a.Ps - a.first / a.Ps + 1;
    return dim3((unsigned)((pages * 2 * a.n_kv + kWaves - 1) / kWaves));
}

hipError_t launch_kv4_ingest(Kv4Args a, hipStream_t s) {
    if (a.end <= a.first) return hipSuccess;
    const dim3 grid = unit_grid(a);
    hipLaunchKernelGGL(kv4_store_kernel<false>, grid, dim3(kWaves * 64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv4_append(Kv4Args a, hipStream_t s) {
    if (a.end <= a.first) return hipSuccess;
    const dim3 grid = unit_grid(a);
    hipLaunchKernelGGL(kv4_store_kernel<true>, grid, dim3(kWaves * 64), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_kv4_gather(Kv4Args a, hipStream_t s) {
    if (a.end <= a.first) return hipSuccess;
    const dim3 grid = unit_grid(a);
    hipLaunchKernelGGL(kv4_gather_kernel, grid, dim3(kWaves * 64), 0, s, a);
    return hipGetLastError();
}

}  // namespace oc
