// Stable counting sort by a cluster of thread blocks.
//
// One pass: the blocks of a cluster take equal, consecutive parts of the items, their warps equal, consecutive parts of
// those.  A warp counts its items by digit (lanes with the same digit find each other with a match), the counts of a block's
// warps are summed bin by bin, every block reads the other blocks' totals out of their shared memory, and an item's place is
//   items of smaller digits + those of its digit in earlier blocks, in earlier warps, earlier in its warp.
// Nothing is decided by the order in which blocks run, there are no atomics, and the only waits are cluster barriers.  One
// cluster of at most 8 blocks sorts all sizes: the rows that are moved by the result take far longer beyond some 10^5 items.
#pragma once
#include "nuna_ops.cuh"

namespace nuna {

constexpr int kSortItems = 8;                            // items of a lane that are fetched together
constexpr unsigned kSortMaxWarps = 32;
constexpr unsigned kSortMaxCluster = 8;
constexpr unsigned kNoDigit = 0xFFFFFFFFu;

// Dynamic shared memory of a pass over `bins` bins: [warps][bins] counts, [bins] totals, [bins] first places.
__host__ __device__ constexpr unsigned sort_smem(unsigned warps, unsigned bins) { return (warps + 2u) * bins * 4u; }

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

// One pass over items 0 ... n-1.  digit(i): the item's bin or kNoDigit (dropped); it is asked twice if a warp has more than
// 32 * kSortItems items.  place(i, digit, first, rank): called once for every item, in any order; `first` is where its bin
// begins, `rank` its number within the bin.  count(bin): with `counts` (shared, [bins]) given, what all blocks have of a bin.
// Returns the number of items that were not dropped.  All threads of the cluster call; shared memory may be reused, and what
// place() wrote to global memory is visible to the whole cluster, when it returns.
template <typename Digit, typename Place>
__device__ __forceinline__ unsigned sort_pass(unsigned n, unsigned bins, unsigned* smem, unsigned* counts, Digit digit, Place place)
{
    __shared__ unsigned red[32];
    const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const unsigned blocks = gridDim.x, block = blockIdx.x;                       // the grid is the cluster
    unsigned *hist = smem, *totals = smem + warps * bins, *first = totals + bins;
    const unsigned parts = blocks * warps;
    const unsigned per_warp = (unsigned)(((unsigned long long)n + parts * 32ull - 1ull) / (parts * 32ull) * 32ull);
    const unsigned long long at = (unsigned long long)(block * warps + warp) * per_warp;
    const unsigned begin = (unsigned)(at < n ? at : n), end = (unsigned)(at + per_warp < n ? at + per_warp : n);
    const bool kept = per_warp <= 32u * kSortItems;
    unsigned* mine = hist + warp * bins;
    unsigned d[kSortItems];

    for (unsigned b = threadIdx.x; b < warps * bins; b += blockDim.x) hist[b] = 0u;
    __syncthreads();
    for (unsigned base = begin; base < end; base += 32u * kSortItems) {
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            const unsigned i = base + k * 32u + lane;
            d[k] = i < end ? digit(i) : kNoDigit;
        }
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            if (base + k * 32u >= end) break;
            const unsigned peers = __match_any_sync(0xFFFFFFFFu, d[k]);
            if (d[k] != kNoDigit && lane == (unsigned)__ffs(peers) - 1u) mine[d[k]] += __popc(peers);
            __syncwarp();
        }
    }
    __syncthreads();
    for (unsigned b = threadIdx.x; b < bins; b += blockDim.x) {
        unsigned run = 0;
        for (unsigned w = 0; w < warps; ++w) {
            const unsigned c = hist[w * bins + b];
            hist[w * bins + b] = run;
            run += c;
        }
        totals[b] = run;
    }
    cluster_sync();
    unsigned carry = 0;
    for (unsigned b0 = 0; b0 < bins; b0 += blockDim.x) {
        const unsigned b = b0 + threadIdx.x;
        unsigned before = 0, all = 0;
        if (b < bins)
            for (unsigned c = 0; c < blocks; ++c) {
                const unsigned v = blocks == 1u ? totals[b] : ld_shared_of(totals + b, c);
                if (c < block) before += v;
                all += v;
            }
        unsigned total;
        const unsigned sum = block_exclusive_sum(all, red, total);
        if (b < bins) {
            first[b] = carry + sum;
            if (counts) counts[b] = all;
            for (unsigned w = 0; w < warps; ++w) hist[w * bins + b] += before;
        }
        carry += total;
    }
    __syncthreads();
    for (unsigned base = begin; base < end; base += 32u * kSortItems) {
        if (!kept) {
#pragma unroll
            for (int k = 0; k < kSortItems; ++k) {
                const unsigned i = base + k * 32u + lane;
                d[k] = i < end ? digit(i) : kNoDigit;
            }
        }
#pragma unroll
        for (int k = 0; k < kSortItems; ++k) {
            if (base + k * 32u >= end) break;
            const unsigned i = base + k * 32u + lane, peers = __match_any_sync(0xFFFFFFFFu, d[k]);
            unsigned rank = 0;
            if (d[k] != kNoDigit) rank = mine[d[k]] + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
            if (d[k] != kNoDigit && lane == (unsigned)__ffs(peers) - 1u) mine[d[k]] += __popc(peers);
            __syncwarp();
            if (i < end) place(i, d[k], d[k] != kNoDigit ? first[d[k]] : 0u, rank);
        }
    }
    cluster_sync();
    return carry;
}

// Blocks of the cluster and warps of a block that sort n items: a warp takes 32 * kSortItems items before there are more of them.
inline Shape sort_shape(size_t n, unsigned bins)
{
    const size_t warps = (n + 32 * kSortItems - 1) / (32 * kSortItems);
    unsigned cluster = 1;
    while (cluster < kSortMaxCluster && cluster * kSortMaxWarps < warps) cluster *= 2;
    unsigned per_block = (unsigned)((warps + cluster - 1) / cluster);
    per_block = per_block < 4u ? 4u : per_block > kSortMaxWarps ? kSortMaxWarps : per_block;
    return Shape{cluster, per_block * 32u, sort_smem(per_block, bins), cluster};
}

}  // namespace nuna
