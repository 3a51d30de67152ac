// Attention over the 4-bit cache on CUDA cores: a block per (sequence, query,
// head), its four warps over the tokens, in fp32 throughout.
#include <cuda_runtime.h>
#include <math.h>

#include "cache.h"
#include "internal.h"
#include "kernels.h"
#include "ptx.cuh"

namespace msf {
namespace {

__device__ __forceinline__ float e4m3_f(uint32_t b) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)b));
    float f;
    asm("{\n.reg .b16 l, h;\nmov.b32 {l, h}, %1;\ncvt.f32.f16 %0, l;\n}" : "=f"(f) : "r"(r));
    return f;
}
__device__ __forceinline__ float2 e2m1_f(uint32_t byte) {
    float2 f;
    asm("{\n.reg .b8 a, b, c, d;\n.reg .b32 r;\n.reg .b16 l, h;\nmov.b32 {a, b, c, d}, %2;\ncvt.rn.f16x2.e2m1x2 r, a;\n"
        "mov.b32 {l, h}, r;\ncvt.f32.f16 %0, l;\ncvt.f32.f16 %1, h;\n}"
        : "=f"(f.x), "=f"(f.y)
        : "r"(byte));
    return f;
}
__device__ __forceinline__ float bf(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Lanes hold neighbouring pairs of the head: D / 64 pairs each, 64 apart.
template <int D>
__global__ void __launch_bounds__(128) cache_attend_kernel(const CacheView c, const CacheAttnArgs a) {
    constexpr int N = D / 64;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int x = (int)blockIdx.x;
    const int h = x % a.heads;
    x /= a.heads;
    const int t = x % a.queries, i = x / a.queries;
    const int s = a.seqs ? a.seqs[i] : i, hk = h / a.group;
    int len = 0;
    if ((unsigned)s < (unsigned)c.S)
        len = min(c.lengths[s], c.W * c.P);
    else if (threadIdx.x == 0)
        atomicOr(c.head + kCacheStatus, kDevIndex);
    if (a.causal) len = max(0, len - a.queries + 1 + t);
    const uint16_t* qp = a.q + i * a.q_st[0] + t * a.q_st[1] + h * a.q_st[2];
    float q[N][2], o[N][2], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(qp + 64 * e + 2 * lane);
        const float f = a.scale * c.k_unit;
        q[e][0] = bf((uint16_t)w) * f;
        q[e][1] = bf((uint16_t)(w >> 16)) * f;
        o[e][0] = o[e][1] = 0.f;
    }
    const int* row = c.table + (size_t)(len ? s : 0) * c.W;
    for (int j = warp; j < len; j += 4) {
        const int page = row[j / c.P];
        if (!cache_page_ok(c, page)) continue;
        const int in = j % c.P, u = in % kCacheBlock;
        const uint8_t* rec = c.pool + ((long long)a.layer * c.pages + page) * c.page_bytes +
                             (long long)(hk * (c.P / kCacheBlock) + in / kCacheBlock) * cache_record_bytes(D);
        float z = 0.f;
        float2 v[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int at = 32 * e + lane, blk = at / 8;
            const float2 k = e2m1_f(rec[u * (D / 2) + at]);
            const float ks = e4m3_f(rec[cache_k_scales(D) + u * (D / 16) + blk]);
            z += (k.x * q[e][0] + k.y * q[e][1]) * ks;
            v[e] = e2m1_f(rec[cache_v_codes(D) + u * (D / 2) + at]);
            const float vs = e4m3_f(rec[cache_v_scales(D) + blk * 16 + u]);
            v[e].x *= vs;
            v[e].y *= vs;
        }
#pragma unroll
        for (int d = 16; d; d /= 2) z += __shfl_xor_sync(0xffffffffu, z, d);
        const float mn = fmaxf(m, z), f = expf(m - mn), p = expf(z - mn);
        m = mn;
        l = l * f + p;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            o[e][0] = o[e][0] * f + p * v[e].x;
            o[e][1] = o[e][1] * f + p * v[e].y;
        }
    }
    __shared__ float so[4][D], sm[4], sl[4];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        so[warp][64 * e + 2 * lane] = o[e][0];
        so[warp][64 * e + 2 * lane + 1] = o[e][1];
    }
    if (lane == 0) {
        sm[warp] = m;
        sl[warp] = l;
    }
    __syncthreads();
    const float M = fmaxf(fmaxf(sm[0], sm[1]), fmaxf(sm[2], sm[3]));
    float w[4], L = 0.f;
    for (int k = 0; k < 4; ++k) {
        w[k] = M == -INFINITY ? 0.f : expf(sm[k] - M);
        L += w[k] * sl[k];
    }
    // this attention's weight in the result, the base's, and the joined log-sum-exp
    float lse = L > 0.f ? M + logf(L) : -INFINITY, own = L > 0.f ? 1.f / L : 0.f, other = 0.f;
    const long long li = i * a.l_st[0] + h * a.l_st[1] + t;
    if (a.base_out) {
        const float b = a.base_lse[li], top = fmaxf(lse, b);
        if (top == -INFINITY) {
            own = 0.f;
        } else {
            const float ea = expf(lse - top), eb = expf(b - top);
            own *= ea / (ea + eb);
            other = eb / (ea + eb);
            lse = top + logf(ea + eb);
        }
    }
    __syncthreads();  // every thread has read base_lse, which may be lse
    if (threadIdx.x == 0 && a.lse) a.lse[li] = lse;
    own *= c.v_unit;
    for (int d = threadIdx.x; d < D; d += 128) {
        float r = (w[0] * so[0][d] + w[1] * so[1][d] + w[2] * so[2][d] + w[3] * so[3][d]) * own;
        const long long at = i * a.o_st[0] + t * a.o_st[1] + h * a.o_st[2] + d;
        if (a.base_out && other != 0.f) r += other * bf(a.base_out[at]);
        a.out[at] = (uint16_t)ptx::pack_bf16(r, 0.f);
    }
}

}  // namespace

cudaError_t launch_cache_attend(const CacheView& c, const CacheAttnArgs& a, cudaStream_t st) {
    const dim3 grid((unsigned)(a.n * a.queries * a.heads));
    return c.D == 128 ? launch_pdl(cache_attend_kernel<128>, grid, dim3(128), 0, st, c, a)
                      : launch_pdl(cache_attend_kernel<64>, grid, dim3(128), 0, st, c, a);
}

}  // namespace msf
