// Appending to the 4-bit cache and reading it back.
//
// A thread takes 16 neighbours of a head (a block: one scale, eight bytes of
// codes). Bound: HBM; an append reads two bytes a value and writes 9/16.
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

// Place of thread `x`: row i of the list, token t, head h, block blk.
struct Place {
    int i, t, h, blk;
};
__device__ __forceinline__ bool place_of(const CacheView& c, const CacheRows& r, long long x, Place& p) {
    const int nb = c.D / kCacheBlock;
    p.blk = (int)(x % nb);
    x /= nb;
    p.h = (int)(x % c.Hk);
    x /= c.Hk;
    p.t = (int)(x % r.tokens);
    x /= r.tokens;
    p.i = (int)x;
    return x < r.n;
}

__global__ void __launch_bounds__(256) cache_write_kernel(const CacheView c, const CacheRows r, const uint16_t* k,
                                                          const uint16_t* v) {
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    if (__ldcg(c.head + kCacheStatus) & kCacheStop) return;
    Place p;
    if (!place_of(c, r, (long long)blockIdx.x * 256 + threadIdx.x, p)) return;
    const int s = r.seqs ? r.seqs[p.i] : p.i, count = r.at ? r.at[p.i] : r.tokens;
    if ((unsigned)s >= (unsigned)c.S || count < 0 || count > r.tokens) {
        atomicOr(c.head + kCacheStatus, kDevIndex);
        return;
    }
    const int pos = c.lengths[s] - count + p.t;
    if (p.t >= count || pos < 0) return;
    const int page = c.table[(size_t)s * c.W + pos / c.P];
    if (!cache_page_ok(c, page) || c.refs[page] > 1) {
        atomicOr(c.head + kCacheStatus, kDevIndex);
        return;
    }
    const int which = (int)blockIdx.y;
    const uint16_t* src = (which ? v : k) + p.i * r.st[0] + p.t * r.st[1] + p.h * r.st[2] + p.blk * kCacheBlock;
    const float unit = which ? c.v_unit : c.k_unit;
    uint32_t w[8];
    *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(src);
    *reinterpret_cast<uint4*>(w + 4) = *reinterpret_cast<const uint4*>(src + 8);
    float x[16];
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[2 * e] = __uint_as_float(w[e] << 16);
        x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
    float a = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        if (!(fabsf(x[e]) <= 3.38953139e38f)) {  // the largest finite bf16
            odd = true;
            x[e] = x[e] != x[e] ? 0.f : copysignf(3.38953139e38f, x[e]);
        }
        a = fmaxf(a, fabsf(x[e]));
    }
    if (odd) atomicOr(c.head + kCacheStatus, kDevNonfinite);
    uint32_t sc = to_e4m3(__fdiv_rn(a, 6.f * unit));
    if (sc == 0) sc = 1;  // 2^-9
    const float step = from_e4m3(sc) * unit;
    uint32_t code[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        code[e / 4] |= to_e2m1x2(__fdiv_rn(x[2 * e], step), __fdiv_rn(x[2 * e + 1], step)) << 8 * (e % 4);
    uint8_t *codes, *scale;
    block_at(c, r.layer, page, p.h, pos % c.P, p.blk, which, codes, scale);
    *reinterpret_cast<uint2*>(codes) = make_uint2(code[0], code[1]);
    *scale = (uint8_t)sc;
}

__global__ void __launch_bounds__(256) cache_read_kernel(const CacheView c, const CacheRows r, uint16_t* k, uint16_t* v) {
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    Place p;
    if (!place_of(c, r, (long long)blockIdx.x * 256 + threadIdx.x, p)) return;
    const int which = (int)blockIdx.y;
    uint16_t* dst = (which ? v : k) + p.i * r.st[0] + p.t * r.st[1] + p.h * r.st[2] + p.blk * kCacheBlock;
    const int s = r.seqs ? r.seqs[p.i] : p.i;
    uint32_t w[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    if ((unsigned)s < (unsigned)c.S) {
        const long long pos = (long long)(r.at ? r.at[p.i] : 0) + p.t;
        if (pos >= 0 && pos < c.lengths[s]) {
            const int page = c.table[(size_t)s * c.W + (int)pos / c.P];
            if (cache_page_ok(c, page)) {
                uint8_t *codes, *scale;
                block_at(c, r.layer, page, p.h, (int)pos % c.P, p.blk, which, codes, scale);
                const uint2 q = *reinterpret_cast<const uint2*>(codes);
                const float step = from_e4m3(*scale) * (which ? c.v_unit : c.k_unit);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t h = from_e2m1x2((e < 4 ? q.x : q.y) >> 8 * (e % 4));
                    w[e] = ptx::pack_bf16(f16_lo(h) * step, f16_hi(h) * step);
                }
            }
        }
    } else {
        atomicOr(c.head + kCacheStatus, kDevIndex);
    }
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<uint4*>(w);
    *reinterpret_cast<uint4*>(dst + 8) = *reinterpret_cast<uint4*>(w + 4);
}

bool grid_of(const CacheView& c, const CacheRows& r, dim3& grid) {
    const long long x = ((long long)r.n * r.tokens * c.Hk * (c.D / kCacheBlock) + 255) / 256;
    if (x >= 1ll << 31) return false;
    grid = dim3((unsigned)x, 2);
    return true;
}

}  // namespace

cudaError_t launch_cache_write(const CacheView& c, const CacheRows& r, const uint16_t* k, const uint16_t* v,
                               cudaStream_t st) {
    dim3 grid;
    if (!grid_of(c, r, grid)) return cudaErrorInvalidValue;
    return launch_pdl(cache_write_kernel, grid, dim3(256), 0, st, c, r, k, v);
}

cudaError_t launch_cache_read(const CacheView& c, const CacheRows& r, uint16_t* k, uint16_t* v, cudaStream_t st) {
    dim3 grid;
    if (!grid_of(c, r, grid)) return cudaErrorInvalidValue;
    return launch_pdl(cache_read_kernel, grid, dim3(256), 0, st, c, r, k, v);
}

}  // namespace msf
