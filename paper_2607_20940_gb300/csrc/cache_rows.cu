// Appending to the 4-bit cache and reading it back.
//
// A thread takes 16 neighbours of a head (a block: one scale, eight bytes of
// codes) of a token's key and of its value. Bound: HBM; an append reads two bytes
// a value and writes 9/16.
//
// A code is the nearest of the e2m1 values to x / t, t = scale * 2^exponent, ties
// to even. The kernel rounds x * (1 / t) to multiples of 2^-12 first, which gives
// the same code: x has 8 significant bits and a midpoint between two values times
// t has at most 7 (3 and 4), so x is a midpoint exactly or at least 2^-9 of it away;
// the product is within 2^-22 of the quotient, so a midpoint is brought back to
// itself and nothing else reaches one. (Sixteen divisions a block had bound the
// kernel instead of HBM.)
#include <cuda_runtime.h>

#include "cache.h"
#include "internal.h"
#include "kernels.h"
#include "ptx.cuh"

namespace msf {
namespace {

// Two values to e2m1 (nearest, ties to even, saturating): the lower in the low half byte.
__device__ __forceinline__ uint32_t to_e2m1x2(float lo, float hi) {
    uint32_t r;
    asm("{\n.reg .b8 b;\n.reg .b16 h;\ncvt.rn.satfinite.e2m1x2.f32 b, %2, %1;\nmov.b16 h, {b, 0};\ncvt.u32.u16 %0, h;\n}"
        : "=r"(r)
        : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ uint32_t to_e4m3(float x) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(x));
    return r & 0xff;
}
__device__ __forceinline__ float from_e4m3(uint32_t b) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)b));
    float f;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.f32.f16 %0, l;\n}" : "=f"(f) : "r"(r));
    return f;
}
// The two codes of a byte as f16.
__device__ __forceinline__ uint32_t from_e2m1x2(uint32_t byte) {
    uint32_t r;
    asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, a;\n}" : "=r"(r) : "r"(byte));
    return r;
}
__device__ __forceinline__ float f16_lo(uint32_t x) {
    float f;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.f32.f16 %0, l;\n}" : "=f"(f) : "r"(x));
    return f;
}
__device__ __forceinline__ float f16_hi(uint32_t x) { return f16_lo(x >> 16); }

// Where block `blk` of a token's keys (which = 0) or values lies: its codes, and its scale.
__device__ __forceinline__ void block_at(const CacheView& c, int layer, int page, int head, int in_page, int blk, int which,
                                         uint8_t*& codes, uint8_t*& scale) {
    const int group = in_page / kCacheBlock, t = in_page % kCacheBlock;
    uint8_t* rec = c.pool + ((long long)layer * c.pages + page) * c.page_bytes +
                   (long long)(head * (c.P / kCacheBlock) + group) * cache_record_bytes(c.D);
    if (which == 0) {
        codes = rec + t * (c.D / 2) + blk * 8;
        scale = rec + cache_k_scales(c.D) + t * (c.D / kCacheBlock) + blk;
    } else {
        codes = rec + cache_v_codes(c.D) + t * (c.D / 2) + cache_v_code_at(c.D, t, blk * 8);
        scale = rec + cache_v_scales(c.D) + blk * kCacheBlock + cache_v_scale_at(t);
    }
}

// Units: (row of the list, token, head, block); a block of threads takes kSpan
// neighbouring ones of a row of the list.
constexpr int kThreads = 256, kEach = 2, kSpan = kThreads * kEach;

struct UnitGrid {
    FastDiv per_token;  // Hk * D / 16 units
    int nb_log2;        // blocks of a head: 4 or 8
};

__global__ void __launch_bounds__(kThreads) cache_write_kernel(const CacheView c, const CacheRows r, const UnitGrid u,
                                                               const uint16_t* k, const uint16_t* v) {
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    if (__ldcg(c.head + kCacheStatus) & kCacheStop) return;
    for (int i = blockIdx.y; i < r.n; i += gridDim.y) {
        const int s = r.seqs ? r.seqs[i] : i, count = r.at ? r.at[i] : r.tokens;
        if ((unsigned)s >= (unsigned)c.S || count < 0 || count > r.tokens) {
            if (threadIdx.x == 0) atomicOr(c.head + kCacheStatus, kDevIndex);
            continue;
        }
        const long long first = (long long)blockIdx.x * kSpan;
        const int t0 = (int)(first / u.per_token.d), rest = (int)(first - (long long)t0 * u.per_token.d);
        if (t0 >= count) continue;
        const int pos0 = c.lengths[s] - count;
        const int* row = c.table + (size_t)s * c.W;
        uint4 w[kEach][2][2];
        uint8_t *codes[kEach][2], *scale[kEach][2];
        bool live[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int x = rest + e * kThreads + (int)threadIdx.x, dt = u.per_token.div(x);
            const int t = t0 + dt, unit = x - dt * u.per_token.d, h = unit >> u.nb_log2, blk = unit & ((1 << u.nb_log2) - 1);
            const int pos = pos0 + t;
            live[e] = t < count && pos >= 0 && pos < c.W * c.P;
            if (!live[e]) continue;
            const int page = row[pos >> c.log2_p];
            if (!cache_page_ok(c, page) || c.refs[page] > 1) {
                atomicOr(c.head + kCacheStatus, kDevIndex);
                live[e] = false;
                continue;
            }
            const long long at = i * r.st[0] + t * r.st[1] + h * r.st[2] + blk * kCacheBlock;
            w[e][0][0] = *reinterpret_cast<const uint4*>(k + at);
            w[e][0][1] = *reinterpret_cast<const uint4*>(k + at + 8);
            w[e][1][0] = *reinterpret_cast<const uint4*>(v + at);
            w[e][1][1] = *reinterpret_cast<const uint4*>(v + at + 8);
            block_at(c, r.layer, page, h, pos & (c.P - 1), blk, 0, codes[e][0], scale[e][0]);
            block_at(c, r.layer, page, h, pos & (c.P - 1), blk, 1, codes[e][1], scale[e][1]);
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if (!live[e]) continue;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                uint32_t y[8] = {w[e][which][0].x, w[e][which][0].y, w[e][which][0].z, w[e][which][0].w,
                                 w[e][which][1].x, w[e][which][1].y, w[e][which][1].z, w[e][which][1].w};
                uint32_t top = 0;  // largest magnitudes, as bits, of the lower and upper halves
#pragma unroll
                for (int z = 0; z < 8; ++z) top = __vmaxu2(top, y[z] & 0x7fff7fffu);
                top = max(top & 0xffffu, top >> 16);
                if (top >= 0x7f80u) {  // infinities or NaN
                    atomicOr(c.head + kCacheStatus, kDevNonfinite);
                    top = 0;
#pragma unroll
                    for (int z = 0; z < 8; ++z) {
                        uint32_t h[2] = {y[z] & 0xffffu, y[z] >> 16};
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const uint32_t m = h[q] & 0x7fffu;
                            if (m > 0x7f80u) h[q] = 0u;
                            if (m == 0x7f80u) h[q] = (h[q] & 0x8000u) | 0x7f7fu;
                            top = max(top, h[q] & 0x7fffu);
                        }
                        y[z] = h[0] | h[1] << 16;
                    }
                }
                const float unit = which ? c.v_unit : c.k_unit;
                uint32_t sc = to_e4m3(__fdiv_rn(__uint_as_float(top << 16), 6.f * unit));
                if (sc == 0) sc = 1;  // 2^-9
                const float inv = __frcp_rn(from_e4m3(sc) * unit);
                uint32_t code[2] = {0u, 0u};
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    const float lo = __fadd_rn(__fadd_rn(__fmul_rn(__uint_as_float(y[z] << 16), inv), 3072.f), -3072.f);
                    const float hi = __fadd_rn(__fadd_rn(__fmul_rn(__uint_as_float(y[z] & 0xffff0000u), inv), 3072.f), -3072.f);
                    code[z / 4] |= to_e2m1x2(lo, hi) << 8 * (z % 4);
                }
                *reinterpret_cast<uint2*>(codes[e][which]) = make_uint2(code[0], code[1]);
                *scale[e][which] = (uint8_t)sc;
            }
        }
    }
}

__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheView c, const CacheRows r, const UnitGrid u,
                                                              uint16_t* k, uint16_t* v) {
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    for (int i = blockIdx.y; i < r.n; i += gridDim.y) {
        const int s = r.seqs ? r.seqs[i] : i;
        const bool some = (unsigned)s < (unsigned)c.S;
        if (!some && threadIdx.x == 0) atomicOr(c.head + kCacheStatus, kDevIndex);
        const long long first = (long long)blockIdx.x * kSpan;
        const int t0 = (int)(first / u.per_token.d), rest = (int)(first - (long long)t0 * u.per_token.d);
        const int begin = r.at ? r.at[i] : 0, len = some ? min(c.lengths[s], c.W * c.P) : 0;
        const int* row = c.table + (size_t)(some ? s : 0) * c.W;
        uint2 q[kEach][2];
        uint32_t sc[kEach][2];
        long long at[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int x = rest + e * kThreads + (int)threadIdx.x, dt = u.per_token.div(x);
            const int t = t0 + dt, unit = x - dt * u.per_token.d, h = unit >> u.nb_log2, blk = unit & ((1 << u.nb_log2) - 1);
            at[e] = t < r.tokens ? i * r.st[0] + t * r.st[1] + h * r.st[2] + blk * kCacheBlock : -1;
            const long long pos = (long long)begin + t;
            q[e][0] = q[e][1] = make_uint2(0u, 0u);
            sc[e][0] = sc[e][1] = 0u;
            if (at[e] < 0 || pos < 0 || pos >= len) continue;
            const int page = row[(int)pos >> c.log2_p];
            if (!cache_page_ok(c, page)) continue;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                uint8_t *codes, *scale;
                block_at(c, r.layer, page, h, (int)pos & (c.P - 1), blk, which, codes, scale);
                q[e][which] = *reinterpret_cast<const uint2*>(codes);
                sc[e][which] = *scale;
            }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            if (at[e] < 0) continue;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const float step = from_e4m3(sc[e][which]) * (which ? c.v_unit : c.k_unit);
                uint32_t w[8];
#pragma unroll
                for (int z = 0; z < 8; ++z) {
                    const uint32_t h = from_e2m1x2((z < 4 ? q[e][which].x : q[e][which].y) >> 8 * (z % 4));
                    w[z] = ptx::pack_bf16(f16_lo(h) * step, f16_hi(h) * step);
                }
                uint16_t* dst = (which ? v : k) + at[e];
                *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(dst + 8) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        }
    }
}

bool grid_of(const CacheView& c, const CacheRows& r, UnitGrid& u, dim3& grid) {
    u.nb_log2 = c.D == 128 ? 3 : 2;
    u.per_token = FastDiv(c.Hk << u.nb_log2);
    const long long x = ((long long)r.tokens * u.per_token.d + kSpan - 1) / kSpan;
    if (x >= 1ll << 31) return false;
    grid = dim3((unsigned)x, (unsigned)(r.n < 65535 ? r.n : 65535));
    return true;
}

}  // namespace

cudaError_t launch_cache_write(const CacheView& c, const CacheRows& r, const uint16_t* k, const uint16_t* v,
                               cudaStream_t st) {
    UnitGrid u;
    dim3 grid;
    if (!grid_of(c, r, u, grid)) return cudaErrorInvalidValue;
    return launch_pdl(cache_write_kernel, grid, dim3(kThreads), 0, st, c, r, u, k, v);
}

cudaError_t launch_cache_read(const CacheView& c, const CacheRows& r, uint16_t* k, uint16_t* v, cudaStream_t st) {
    UnitGrid u;
    dim3 grid;
    if (!grid_of(c, r, u, grid)) return cudaErrorInvalidValue;
    return launch_pdl(cache_read_kernel, grid, dim3(kThreads), 0, st, c, r, u, k, v);
}

}  // namespace msf
