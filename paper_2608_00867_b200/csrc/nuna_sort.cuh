// Stable counting sort by a cluster of thread blocks.
//
// One pass: the blocks of a cluster take equal, consecutive parts of the items, their warps equal, consecutive parts of
// those.  A warp counts its items by digit (lanes with the same digit find each other with a match), the counts of a block's
// warps are summed bin by bin, every block reads the other blocks' totals out of their shared memory, and an item's place is
//   items of smaller digits + those of its digit in earlier blocks, in earlier warps, earlier in its warp.
// Nothing is decided by the order in which blocks run, there are no atomics, and the only waits are cluster barriers.  One
// cluster of at most 16 blocks sorts all sizes: the rows that are moved by the result take far longer beyond some 10^5 items.
#pragma once
#include "nuna_ops.cuh"

namespace nuna {

constexpr int kSortItems = 8;                            // items of a lane that are fetched together
constexpr unsigned kSortMaxWarps = 32;
constexpr unsigned kSortMaxCluster = 16;                 // beyond 8 blocks a kernel has to ask for it (allow_sort)
constexpr unsigned kNoDigit = 0xFFFFFFFFu;

constexpr unsigned kSortSegments = 8;                    // cuts of a bin's counts by warp

// Dynamic shared memory of a pass over `bins` bins: [warps][bins] counts, [bins] totals, [bins] first places, [bins] items of
// earlier blocks, [segments][bins] sums.
__host__ __device__ constexpr unsigned sort_smem(unsigned warps, unsigned bins) { return (warps + 3u + kSortSegments) * bins * 4u; }

__device__ __forceinline__ unsigned ld_shared_of(const unsigned* local_ptr, unsigned cta)
{
    unsigned remote, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_u32(local_ptr)), "r"(cta));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote) : "memory");
    return v;
}

// Exclusive sum of v over the block's threads, in the order of threads; `total` receives the whole sum.
__device__ __forceinline__ unsigned block_exclusive_sum(unsigned v, unsigned* red, unsigned& total)
{
    const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    unsigned s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned o = __shfl_up_sync(0xFFFFFFFFu, s, d);
        if (lane >= (unsigned)d) s += o;
    }
    __syncthreads();
    if (lane == 31u) red[warp] = s;
    __syncthreads();
    const unsigned w = lane < warps ? red[lane] : 0u;
    unsigned t = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const unsigned o = __shfl_up_sync(0xFFFFFFFFu, t, d);
        if (lane >= (unsigned)d) t += o;
    }
    total = __shfl_sync(0xFFFFFFFFu, t, 31);
    return s - v + __shfl_sync(0xFFFFFFFFu, t - w, warp);
}

// Ids of the caller's, and what blocks of this kernel have written for one another, without waiting for the one before.
__device__ __forceinline__ long long load_id(const long long* p)
{
    long long v;
    asm volatile("ld.global.s64 %0, [%1];" : "=l"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ long long load_id(const int* p) { return (int)ld_src32(reinterpret_cast<const uint32_t*>(p)); }
__device__ __forceinline__ uint2 load_shared_by_cluster(const uint2* p)
{
    uint2 v;
    asm volatile("ld.global.cg.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}

// All threads of the cluster.
__device__ __forceinline__ void sort_sync(unsigned blocks)
{
    if (blocks == 1u) __syncthreads();
    else              cluster_sync();
}

// One pass over items 0 ... n-1 by the grid's first `blocks` blocks, which are a cluster.  load(i): the item (asked twice if a warp has more than 32 * kSortItems of them);
// digit(item): its bin, or kNoDigit to drop it; place(i, item, digit, first, rank): called once for every item, in any
// order; `first` is where its bin begins, `rank` its number within the bin.  `counts` (shared, [bins]), if given, receives what
// all blocks have of each bin.  Returns the number of items that were not dropped.  All threads of the cluster call; shared
// memory may be reused, and what place() wrote to global memory is visible to the whole cluster, when it returns.
template <typename Item, typename Load, typename Digit, typename Place>
__device__ __forceinline__ unsigned sort_pass(unsigned blocks, unsigned n, unsigned bins, unsigned* smem, unsigned* counts, Load load, Digit digit, Place place)
{
    __shared__ unsigned red[32];
    const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const unsigned block = blockIdx.x;
    unsigned *hist = smem, *totals = hist + warps * bins, *first = totals + bins, *ahead = first + bins, *segment = ahead + bins;
    const unsigned parts = blocks * warps;
    const unsigned per_warp = (unsigned)(((unsigned long long)n + parts * 32ull - 1ull) / (parts * 32ull) * 32ull);
    const unsigned long long at = (unsigned long long)(block * warps + warp) * per_warp;
    const unsigned begin = (unsigned)(at < n ? at : n), end = (unsigned)(at + per_warp < n ? at + per_warp : n);
    const bool kept = per_warp <= 32u * kSortItems;
    unsigned* mine = hist + warp * bins;
    Item item[kSortItems];
    unsigned held[kSortItems];                           // an item's number among its warp's items of its digit

    const auto fetch = [&](unsigned base) {
#pragma unroll
        for (int k = 0; k < kSortItems; ++k)
            if (base + k * 32u + lane < end) item[k] = load(base + k * 32u + lane);
    };
    if (kept) fetch(begin);
    for (unsigned b = threadIdx.x; b < warps * bins; b += blockDim.x) hist[b] = 0u;
    __syncthreads();
    for (unsigned base = begin; base < end; base += 32u * kSortItems) {
        if (!kept) fetch(base);
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            if (base + k * 32u >= end) break;
            const unsigned d = base + k * 32u + lane < end ? digit(item[k]) : kNoDigit;
            const unsigned peers = __match_any_sync(0xFFFFFFFFu, d), before = d != kNoDigit ? mine[d] : 0u;
            held[k] = before + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
            if (d != kNoDigit && lane == (unsigned)__ffs(peers) - 1u) mine[d] = before + __popc(peers);
            __syncwarp();
        }
    }
    __syncthreads();
    // What a bin has in earlier warps, and in all: a bin's warps are cut into segments, summed by a thread each.
    unsigned segments = 1;
    while (segments < kSortSegments && segments * 2u <= warps && segments * 2u * bins <= blockDim.x) segments *= 2u;
    const unsigned each = (warps + segments - 1u) / segments;
    for (unsigned t = threadIdx.x; t < segments * bins; t += blockDim.x) {
        const unsigned q = t / bins, b = t - q * bins;
        unsigned sum = 0;
        for (unsigned w = q * each; w < warps && w < (q + 1u) * each; ++w) sum += hist[w * bins + b];
        segment[t] = sum;
    }
    __syncthreads();
    for (unsigned t = threadIdx.x; t < segments * bins; t += blockDim.x) {
        const unsigned q = t / bins, b = t - q * bins;
        unsigned run = 0;
        for (unsigned o = 0; o < q; ++o) run += segment[o * bins + b];
        for (unsigned w = q * each; w < warps && w < (q + 1u) * each; ++w) {
            const unsigned c = hist[w * bins + b];
            hist[w * bins + b] = run;
            run += c;
        }
        if (q == segments - 1u) totals[b] = run;
    }
    sort_sync(blocks);
    unsigned carry = 0;
    for (unsigned b0 = 0; b0 < bins; b0 += blockDim.x) {
        const unsigned b = b0 + threadIdx.x;
        unsigned before = 0, all = 0;
        if (b < bins) {
            if (blocks == 1u) {
                all = totals[b];
            } else {
                unsigned v[kSortMaxCluster];
#pragma unroll
                for (unsigned c = 0; c < kSortMaxCluster; ++c) v[c] = c < blocks ? ld_shared_of(totals + b, c) : 0u;
#pragma unroll
                for (unsigned c = 0; c < kSortMaxCluster; ++c) {
                    before += c < block ? v[c] : 0u;
                    all += v[c];
                }
            }
        }
        unsigned total;
        const unsigned sum = block_exclusive_sum(all, red, total);
        if (b < bins) {
            first[b] = carry + sum;
            ahead[b] = before;
            if (counts) counts[b] = all;
        }
        carry += total;
    }
    __syncthreads();
    if (kept) {
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const unsigned i = begin + k * 32u + lane;
            if (i >= end) break;
            const unsigned d = digit(item[k]);
            if (d == kNoDigit) place(i, item[k], d, 0u, 0u);
            else               place(i, item[k], d, first[d], ahead[d] + mine[d] + held[k]);
        }
    } else {
        for (unsigned base = begin; base < end; base += 32u * kSortItems) {
            fetch(base);
#pragma unroll
            for (int k = 0; k < kSortItems; ++k) {
                if (base + k * 32u >= end) break;
                const unsigned i = base + k * 32u + lane, d = i < end ? digit(item[k]) : kNoDigit;
                const unsigned peers = __match_any_sync(0xFFFFFFFFu, d), before = d != kNoDigit ? mine[d] : 0u;
                __syncwarp();
                if (d != kNoDigit && lane == (unsigned)__ffs(peers) - 1u) mine[d] = before + __popc(peers);
                __syncwarp();
                if (i < end) place(i, item[k], d, d != kNoDigit ? first[d] : 0u, d != kNoDigit ? ahead[d] + before + __popc(peers & ((1u << lane) - 1u)) : 0u);
            }
        }
    }
    sort_sync(blocks);
    return carry;
}

// Blocks of the cluster and warps of a block that sort n items: one block, eight or sixteen, where what the warps save is more
// than the cluster's barriers and the reads of its totals cost (by 128 experts: 1024 pairs 4.7 us in one block, 2048 6.4 | 4.6 in one
// and in eight, 8192 5.8 | 5.6 in eight and in sixteen, 16384 7.9 | 6.0, 65536 18.5 | 12.4).  A warp takes four items a lane
// before there is another one (2 | 4 | 8: 16384 pairs 9.0 | 8.0 | 7.6, 8192 tokens by 32768 rows 21.1 | 21.3 | 26.2 the whole gradient).
constexpr size_t kSortAlone = 1024, kSortWide = 8192;
constexpr size_t kSortEach = 4;
inline Shape sort_shape(size_t n, unsigned bins)
{
    const unsigned cluster = n <= kSortAlone ? 1u : n <= kSortWide ? 8u : kSortMaxCluster;
    const size_t warps = (n / cluster + 32 * kSortEach - 1) / (32 * kSortEach);
    const unsigned per_block = (unsigned)(warps < 4 ? 4 : warps > kSortMaxWarps ? kSortMaxWarps : warps);
    return Shape{cluster, per_block * 32u, sort_smem(per_block, bins), cluster};
}

// Lets a kernel have `bytes` of shared memory in clusters of up to kSortMaxCluster blocks.
template <auto kKernel>
int allow_sort(const Shape& s, int bytes)
{
    if (s.cluster <= 8u && s.smem <= 32 * 1024) return NUNA_OK;
    static std::atomic<bool> done[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return NUNA_ERR_CUDA;
    if (!done[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess ||
            cudaFuncSetAttribute(kKernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
            return NUNA_ERR_CUDA;
        done[dev].store(true, std::memory_order_relaxed);
    }
    return NUNA_OK;
}

}  // namespace nuna
