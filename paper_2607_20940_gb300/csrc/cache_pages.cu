// Pages of the 4-bit cache: growing, forking, truncating and compacting.
//
// Each operation is a launch that works on the tables (one CTA, or one cluster
// whose phases are separated by cluster barriers) and, where pages move, a
// second that copies them. The tables' launch checks the whole list before it
// changes anything, so an error leaves the cache as it was. Nothing depends on
// the order of atomics: new pages are ranked by prefix sums (free pages by
// number, requests by their place in the list), references are sums.
//
// Bound: latency for the tables (a few dependent passes over L2), HBM for the
// copies.
#include <cuda_runtime.h>

#include "cache.h"
#include "internal.h"
#include "kernels.h"
#include "ptx.cuh"

namespace msf {
namespace {

constexpr int kThreads = 1024;
constexpr int kCluster = 8;

// Exclusive prefix sum over the block; `total` is the sum. Every thread calls.
__device__ __forceinline__ int block_scan(int x, int* sh, int& total) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int v = x;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, v, d);
        if (lane >= d) v += y;
    }
    if (lane == 31) sh[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int w = sh[lane];
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int y = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += y;
        }
        sh[lane] = w;
    }
    __syncthreads();
    const int before = warp > 0 ? sh[warp - 1] : 0;
    total = sh[31];
    __syncthreads();
    return before + v - x;
}

__device__ __forceinline__ int seq_of(const int* seqs, int i) { return seqs ? seqs[i] : i; }

// Bits of word w that stand for pages.
__device__ __forceinline__ unsigned page_bits(const CacheView& c, int w) {
    const int n = c.pages - 32 * w;
    return n >= 32 ? 0xffffffffu : (1u << n) - 1u;
}

// The lowest `want` free pages into c.free_list. False if there are fewer. One
// block; the list is in place when it returns.
__device__ bool find_free(const CacheView& c, int want, int* sh) {
    const int words = (c.pages + 31) / 32;
    int found = 0;
    for (int w0 = 0; w0 < words && found < want; w0 += kThreads) {
        const int w = w0 + (int)threadIdx.x;
        unsigned f = w < words ? ~__ldcg(c.used + w) & page_bits(c, w) : 0u;
        int total;
        int at = found + block_scan(__popc(f), sh, total);
        while (f && at < want) {
            c.free_list[at++] = 32 * w + __ffs(f) - 1;
            f &= f - 1;
        }
        found += total;
    }
    __syncthreads();
    return found >= want;
}

__device__ __forceinline__ void take_page(const CacheView& c, int page) {
    c.refs[page] = 1;
    atomicOr(c.used + page / 32, 1u << page % 32);
}
__device__ __forceinline__ void drop_page(const CacheView& c, int page) {
    if (!cache_page_ok(c, page)) return;
    if (atomicSub(c.refs + page, 1) == 1) atomicAnd(c.used + page / 32, ~(1u << page % 32));
}

// ------------------------------------------------------------------- growing

__global__ void __launch_bounds__(kThreads) cache_grow_kernel(const CacheView c, const int* seqs, const int* counts,
                                                              int tokens, int n) {
    __shared__ int sh[32];
    __shared__ int n_copies;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const unsigned stop = __ldcg(c.head + kCacheStatus) & kCacheStop;
    if (threadIdx.x == 0) {
        n_copies = 0;
        c.head[kCacheCopies] = 0;
    }
    if (stop) return;
    unsigned bad = 0;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        const int s = seq_of(seqs, i);
        if ((unsigned)s >= (unsigned)c.S)
            bad |= kDevIndex;
        else
            c.claim[s] = i;
    }
    if (__syncthreads_or((int)bad)) {
        if (threadIdx.x == 0) atomicOr(c.head + kCacheStatus, kDevIndex);
        return;
    }
    // Pages that each row needs, and the first of them in the list of free pages.
    long long want = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads) {
        const int i = i0 + (int)threadIdx.x;
        int need = 0, copied = 0;
        if (i < n) {
            const int s = seq_of(seqs, i), count = counts ? counts[i] : tokens, len = c.lengths[s];
            if (c.claim[s] != i || count < 0) bad |= kDevIndex;
            else if (count > c.W * c.P - len) bad |= kDevPages;
            else if (count > 0) {
                if (len % c.P) {
                    const int page = c.table[(size_t)s * c.W + len / c.P];
                    copied = cache_page_ok(c, page) && c.refs[page] > 1;
                }
                need = cache_need(c, len + count) - cache_need(c, len) + copied;
            }
        }
        int total;
        const int before = block_scan(need, sh, total);
        if (want + total > c.pages) bad |= kDevPages;
        else if (i < n) c.row[i] = 2 * ((int)want + before) + copied;
        if (want <= c.pages) want += total;
    }
    // (barriers: the rows' places and the claims are in place)
    int err = __syncthreads_or((int)(bad & kDevIndex)) ? (int)kDevIndex : 0;
    if (__syncthreads_or((int)(bad & kDevPages))) err |= (int)kDevPages;
    if (!err && !find_free(c, (int)want, sh)) err = (int)kDevPages;
    if (err) {
        if (threadIdx.x == 0) atomicOr(c.head + kCacheStatus, (unsigned)err);
        return;
    }
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int i = warp; i < n; i += kThreads / 32) {
        const int s = seq_of(seqs, i), count = counts ? counts[i] : tokens, len = c.lengths[s];
        if (count == 0) continue;
        const int copied = c.row[i] & 1, first = c.row[i] >> 1;
        const int col0 = copied ? len / c.P : cache_need(c, len);
        const int k = cache_need(c, len + count) - col0;
        for (int j = lane; j < k; j += 32) {
            const int page = c.free_list[first + j];
            int* entry = c.table + (size_t)s * c.W + col0 + j;
            if (copied && j == 0) {
                c.copies[atomicAdd(&n_copies, 1)] = make_int2(*entry, page);
                drop_page(c, *entry);
            }
            *entry = page;
            take_page(c, page);
        }
        __syncwarp();
        if (lane == 0) c.lengths[s] = len + count;
    }
    __syncthreads();
    if (threadIdx.x == 0) c.head[kCacheCopies] = (unsigned)n_copies;
}

// ------------------------------------------------------ forking and truncating

// Checks a list on one cluster: rows in [0, n), dst names within the cache and
// once each. Writes c.new_len[i] (of source src[i], or of dst[i] itself) and
// returns true if every CTA may go on.
__device__ bool list_check(const CacheView& c, const int* src, const int* dst, const int* lengths, int keep_all, int n,
                           int t, int T) {
    const unsigned stop = __ldcg(c.head + kCacheStatus) & kCacheStop;
    if (t == 0) c.head[kCacheCopies] = 0;
    if (stop) return false;  // the same for every thread: the word does not change before the first barrier
    for (int i = t; i < n; i += T) {
        const int d = seq_of(dst, i);
        if ((unsigned)d < (unsigned)c.S) c.claim[d] = i;
    }
    ptx::cluster_sync();
    bool bad = false;
    for (int i = t; i < n; i += T) {
        const int d = seq_of(dst, i), s = src ? src[i] : d;
        const int keep = lengths ? lengths[i] : keep_all;
        if ((unsigned)d >= (unsigned)c.S || (unsigned)s >= (unsigned)c.S || keep < 0 || __ldcg(c.claim + d) != i)
            bad = true;
        else
            c.new_len[i] = min(__ldcg(c.lengths + s), keep);
    }
    if (bad) atomicOr(c.head + kCacheBad, 1u);
    ptx::cluster_sync();
    const bool ok = __ldcg(c.head + kCacheBad) == 0;
    ptx::cluster_sync();
    if (!ok && t == 0) {
        c.head[kCacheBad] = 0;
        atomicOr(c.head + kCacheStatus, kDevIndex);
    }
    return ok;
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    cache_fork_kernel(const CacheView c, const int* src, const int* dst, const int* lengths, int n, int copy) {
    __shared__ int sh[32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int t = (int)blockIdx.x * kThreads + (int)threadIdx.x, T = kCluster * kThreads;
    if (!list_check(c, src, dst, lengths, 0x7fffffff, n, t, T)) return;
    if (copy) {
        if (blockIdx.x == 0) {
            long long want = 0;
            for (int i0 = 0; i0 < n; i0 += kThreads) {
                const int i = i0 + (int)threadIdx.x;
                const int need = i < n ? cache_need(c, __ldcg(c.new_len + i)) : 0;
                int total;
                const int before = block_scan(min(need, c.pages + 1), sh, total);
                if (i < n) c.row[i] = (int)want + before;
                want += total;
                if (want > c.pages) break;
            }
            if (want > c.pages || !find_free(c, (int)want, sh)) {
                if (threadIdx.x == 0) {
                    c.head[kCacheBad] = 1;
                    atomicOr(c.head + kCacheStatus, kDevPages);
                }
            } else if (threadIdx.x == 0) {
                c.head[kCacheCopies] = (unsigned)want;
            }
        }
        ptx::cluster_sync();
        const bool ok = __ldcg(c.head + kCacheBad) == 0;
        ptx::cluster_sync();
        if (!ok) {
            if (t == 0) c.head[kCacheBad] = 0;
            return;
        }
    }
    // The new rows, before any table changes.
    const int warp = t / 32, lane = t % 32, warps = T / 32;
    for (int i = warp; i < n; i += warps) {
        const int* from = c.table + (size_t)src[i] * c.W;
        int* to = c.stage + (size_t)i * c.W;
        const int k = min(cache_need(c, __ldcg(c.new_len + i)), c.W), first = copy ? __ldcg(c.row + i) : 0;
        for (int j = lane; j < k; j += 32) {
            int page = __ldcg(from + j);
            if (copy) {
                const int own = __ldcg(c.free_list + first + j);
                c.copies[first + j] = make_int2(page, own);
                take_page(c, own);
                page = own;
            } else if (cache_page_ok(c, page)) {
                atomicAdd(c.refs + page, 1);
            }
            to[j] = page;
        }
    }
    ptx::cluster_sync();
    for (int i = warp; i < n; i += warps) {
        const int d = dst[i], len = __ldcg(c.new_len + i);
        const int* from = c.stage + (size_t)i * c.W;
        int* to = c.table + (size_t)d * c.W;
        const int k = min(cache_need(c, len), c.W), old = min(cache_need(c, __ldcg(c.lengths + d)), c.W);
        for (int j = lane; j < max(k, old); j += 32) {
            if (j < old) drop_page(c, __ldcg(to + j));
            to[j] = j < k ? __ldcg(from + j) : -1;
        }
        __syncwarp();
        if (lane == 0) c.lengths[d] = len;
    }
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kThreads)
    cache_truncate_kernel(const CacheView c, const int* seqs, const int* lengths, int n) {
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int t = (int)blockIdx.x * kThreads + (int)threadIdx.x, T = kCluster * kThreads;
    if (!list_check(c, nullptr, seqs, lengths, 0, n, t, T)) return;
    const int warp = t / 32, lane = t % 32;
    for (int i = warp; i < n; i += T / 32) {
        const int s = seq_of(seqs, i), len = __ldcg(c.new_len + i);
        int* row = c.table + (size_t)s * c.W;
        const int old = min(cache_need(c, __ldcg(c.lengths + s)), c.W);
        for (int j = cache_need(c, len) + lane; j < old; j += 32) {
            drop_page(c, row[j]);
            row[j] = -1;
        }
        __syncwarp();
        if (lane == 0) c.lengths[s] = len;
    }
}

// ---------------------------------------------------------------- compacting

// Which pages move where. With u pages in use: the i-th used page from u on to
// the i-th free one below u, so no page is both read and written.
__global__ void __launch_bounds__(kThreads) cache_compact_kernel(const CacheView c) {
    __shared__ int sh[32];
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const unsigned stop = __ldcg(c.head + kCacheStatus) & kCacheStop;
    if (threadIdx.x == 0) {
        c.head[kCacheCopies] = 0;
        c.head[kCacheLive] = 0x7fffffffu;  // nothing to follow
    }
    if (stop) return;
    const int words = (c.pages + 31) / 32;
    int mine = 0, live;
    for (int w = threadIdx.x; w < words; w += kThreads) mine += __popc(c.used[w] & page_bits(c, w));
    block_scan(mine, sh, live);
    int holes = 0, high = 0;  // found so far
    for (int w0 = 0; w0 < words; w0 += kThreads) {
        const int w = w0 + (int)threadIdx.x;
        const unsigned u = w < words ? c.used[w] & page_bits(c, w) : 0u;
        const int below = min(32, max(0, live - 32 * w));  // bits that stand for pages below u
        const unsigned low = w < words ? (below == 32 ? 0xffffffffu : (1u << below) - 1u) : 0u;
        unsigned f = ~u & low, m = u & ~low;
        int total;
        int at = holes + block_scan(__popc(f), sh, total);
        holes += total;
        for (; f; f &= f - 1) c.copies[at++].y = 32 * w + __ffs(f) - 1;
        at = high + block_scan(__popc(m), sh, total);
        high += total;
        for (; m; m &= m - 1) c.copies[at++].x = 32 * w + __ffs(m) - 1;
    }
    __syncthreads();
    // holes == high: as many pages are missing below u as there are above it
    for (int i = threadIdx.x; i < high; i += kThreads) {
        const int2 p = c.copies[i];
        c.moved[p.x] = p.y;
        c.refs[p.y] = c.refs[p.x];
        c.refs[p.x] = 0;
    }
    for (int w = threadIdx.x; w < words; w += kThreads) {
        const int below = min(32, max(0, live - 32 * w));
        c.used[w] = below == 32 ? 0xffffffffu : (1u << below) - 1u;
    }
    if (threadIdx.x == 0) {
        c.head[kCacheCopies] = (unsigned)high;
        c.head[kCacheLive] = (unsigned)live;
    }
}

// ------------------------------------------------------------------- copying

// The pages of c.copies, all layers, 16 KB at a time; `follow`: and the tables
// of a compaction.
__global__ void __launch_bounds__(256) cache_copy_kernel(const CacheView c, int follow) {
    constexpr int kVec = 4, kSeg = 256 * kVec;
    ptx::grid_dep_wait();
    ptx::grid_dep_launch();
    const int n = (int)__ldcg(c.head + kCacheCopies);
    const long long vecs = c.page_bytes / 16;
    const int segs = (int)((vecs + kSeg - 1) / kSeg);
    const long long items = (long long)n * c.L * segs;
    for (long long it = blockIdx.x; it < items; it += gridDim.x) {
        const int seg = (int)(it % segs);
        const long long pl = it / segs;
        const int layer = (int)(pl % c.L);
        const int2 p = c.copies[pl / c.L];
        if (!cache_page_ok(c, p.x) || !cache_page_ok(c, p.y)) continue;
        const uint4* from = (const uint4*)(c.pool + ((long long)layer * c.pages + p.x) * c.page_bytes);
        uint4* to = (uint4*)(c.pool + ((long long)layer * c.pages + p.y) * c.page_bytes);
        uint4 x[kVec];
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const long long at = (long long)seg * kSeg + k * 256 + threadIdx.x;
            if (at < vecs) x[k] = from[at];
        }
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const long long at = (long long)seg * kSeg + k * 256 + threadIdx.x;
            if (at < vecs) to[at] = x[k];
        }
    }
    if (!follow) return;
    const int live = (int)__ldcg(c.head + kCacheLive);
    if (live == 0x7fffffff) return;
    const int warp = (int)(blockIdx.x * blockDim.x + threadIdx.x) / 32, warps = (int)(gridDim.x * blockDim.x) / 32;
    for (int s = warp; s < c.S; s += warps) {
        int* row = c.table + (size_t)s * c.W;
        const int k = min(cache_need(c, c.lengths[s]), c.W);
        for (int j = threadIdx.x % 32; j < k; j += 32) {
            const int page = row[j];
            if (page >= live && page < c.pages) row[j] = c.moved[page];
        }
    }
}

cudaError_t launch_copies(const CacheView& c, int follow, cudaStream_t st) {
    int sms;
    const cudaError_t e = device_sms(&sms);
    if (e != cudaSuccess) return e;
    return launch_pdl(cache_copy_kernel, dim3(sms * 8), dim3(256), 0, st, c, follow);
}

}  // namespace

cudaError_t launch_cache_grow(const CacheView& c, const int* seqs, const int* counts, int tokens, int n, cudaStream_t st) {
    const cudaError_t e = launch_pdl(cache_grow_kernel, dim3(1), dim3(kThreads), 0, st, c, seqs, counts, tokens, n);
    return e == cudaSuccess ? launch_copies(c, 0, st) : e;
}

cudaError_t launch_cache_fork(const CacheView& c, const int* src, const int* dst, const int* lengths, int n, bool copy,
                              cudaStream_t st) {
    const cudaError_t e = launch_pdl(cache_fork_kernel, dim3(kCluster), dim3(kThreads), 0, st, c, src, dst, lengths, n,
                                     copy ? 1 : 0);
    return e == cudaSuccess && copy ? launch_copies(c, 0, st) : e;
}

cudaError_t launch_cache_truncate(const CacheView& c, const int* seqs, const int* lengths, int n, cudaStream_t st) {
    return launch_pdl(cache_truncate_kernel, dim3(kCluster), dim3(kThreads), 0, st, c, seqs, lengths, n);
}

cudaError_t launch_cache_compact(const CacheView& c, cudaStream_t st) {
    const cudaError_t e = launch_pdl(cache_compact_kernel, dim3(1), dim3(kThreads), 0, st, c);
    return e == cudaSuccess ? launch_copies(c, 1, st) : e;
}

}  // namespace msf
