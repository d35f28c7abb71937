// Device helpers shared by the collectives' kernels and by the operators around them (sm_100a): dependent launch, memory
// access, element types, bulk copies and cluster barriers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "nuna_types.h"

namespace nuna {

// ---- programmatic dependent launch ---------------------------------------------------------------
//
// Every collective kernel opens with pdl_wait() and calls pdl_trigger() when its block has issued
// its main work.  When a kernel is launched with programmatic stream serialization
// (NUNA_LAUNCH_PDL) its blocks may be scheduled while the predecessor in the stream drains:
// griddepcontrol.wait holds them, before their first access to the callers' buffers, until the predecessor grid has
// completed and its memory operations are visible; griddepcontrol.launch_dependents, issued once a
// block is past its main loop, lets the successor's blocks take the freed SM slots so that their
// launch latency overlaps this kernel's tail.  The first warp of a block that issues it does so for the block: in blocks
// wider than their tile an idle warp releases the successor right after the wait, which on cold sources is what its
// prefetch needs (put form, 8 x 512 KiB, tiles of 56: 2.09 us in 256 threads, 2.58 in 64), and full blocks can ask for
// (k_reduce_scatter_ahead).  (Triggering at kernel entry was measured slower -- 8 x 512 KiB one-shot: 3.07 against 2.81 us -- the
// successor's waiting blocks then compete with this kernel's own blocks for slots.)
// Launched normally, both instructions do nothing.
__device__ __forceinline__ void pdl_wait()
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

__device__ __forceinline__ void pdl_trigger()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Asks L2 to fetch `bytes` (a multiple of 16; 16-byte aligned address) of this GPU's memory.  Nothing is
// returned to the thread and nothing is waited for, so it may be issued BEFORE pdl_wait(): L2 is the
// point of coherence, a line the predecessor writes after the fetch is updated in place, and the loads
// after the wait read the current data.  What it buys: the successor's blocks arrive while the
// predecessor's last blocks drain and its writes are flushed; that window covers most of a DRAM round
// trip, so cold sources are L2 hits by the time the wait returns.
__device__ __forceinline__ void prefetch_l2_bulk(const void* g, unsigned bytes)
{
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" :: "l"(g), "r"(bytes) : "memory");
}

// The same for the one line that holds `g`.  Requests of their own for every line are in nobody's way for long: behind a kernel
// that is not the library's, whose end the wait finds already there, a block's loads queue behind what it has just asked for.
__device__ __forceinline__ void prefetch_l2_line(const void* g) { asm volatile("prefetch.global.L2 [%0];" :: "l"(g) : "memory"); }

// Nanoseconds of the device-wide timer (bounds every in-kernel wait; timestamps of the measurement aids).
__device__ __forceinline__ unsigned long long globaltimer_ns()
{
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}

// ---- memory access helpers ----------------------------------------------------------------

// Sources are re-read by other emulated ranks from other SMs: keep them out of L1, let L2 hold them.  Ordinary
// loads, not the non-coherent ones (ld.global.nc, __ldg): those may only read what nobody writes for as long as the
// kernel runs, and a kernel that starts ahead of its predecessor's last stores is already running while its sources
// are written.  griddepcontrol.wait makes those stores visible to ordinary loads.  Same time either way
// (8 ranks x 512 KiB 2.04 us with both, x 64 MiB 156.5; reduce-scatter 8 x 4 MiB 6.37).
__device__ __forceinline__ uint4 ld_src(const uint4* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Data produced earlier in the same kernel by other blocks (two-shot shard): coherent L2 load.
__device__ __forceinline__ uint4 ld_cg(const uint4* p)
{
    uint4 v;
    asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// Destination of a streaming kernel: written once and not read again by this kernel, so it is stored
// with the evict-first policy and does not push the sources out of L2 (measured: two-shot put
// 164.1 -> 160.9 us at 64 MiB per rank, 12.06 -> 11.68 us at 4 MiB; one-shot 234.7 -> 225.8 us).
__device__ __forceinline__ void st_stream(uint4* p, uint4 v)
{
    asm volatile("st.global.cs.v4.u32 [%0], {%1,%2,%3,%4};"
                 :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// Ordinary store: data another block of this kernel reads back (the two-shot shard) and the destinations
// of the placement-aware kernels, which are used when the buffers are meant to stay in L2.
__device__ __forceinline__ void st_dst(uint4* p, uint4 v)
{
    asm volatile("st.global.v4.u32 [%0], {%1,%2,%3,%4};"
                 :: "l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint16_t ld_src16(const uint16_t* p)
{
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}

__device__ __forceinline__ uint32_t ld_src32(const uint32_t* p)
{
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}

// ---- element types ----------------------------------------------------------------------------

// Element types (the values of nuna_dtype_t): 0 = bf16, 1 = f16 (IEEE binary16), 2 = f32.
// Storage is 2 or 4 bytes; a 16-byte vector holds kElems elements; every type is widened exactly
// to binary32, folded in binary32 in rank order, and rounded once to the storage type.
constexpr int kBf16 = 0, kF16 = 1, kF32 = 2;

template <int DT> struct Elem { static constexpr int kElems = 8; static constexpr int kBytes = 2; };
template <> struct Elem<kF32> { static constexpr int kElems = 4; static constexpr int kBytes = 4; };

// bf16 -> binary32 is a 16-bit shift; a 32-bit word holds element 2k in its low half and 2k+1 in
// its high half.  Rank 0's value is widened (shift / mask for bf16, cvt for f16); ranks 1..N-1 are
// folded in with the sm_100 mixed-precision add, d = f32(a) + c rounded once to binary32 (nearest
// even, subnormals kept), so no instruction is spent on widening them.  At large sizes the one-shot is
// limited by instruction issue and L1 throughput (N times the work of a plain sum), which is why the
// instruction count matters.
template <int DT>
__device__ __forceinline__ float add_narrow(float acc, uint16_t h)
{
    float d;
    if (DT == kBf16) asm("add.rn.f32.bf16 %0, %1, %2;" : "=f"(d) : "h"(h), "f"(acc));
    else             asm("add.rn.f32.f16 %0, %1, %2;" : "=f"(d) : "h"(h), "f"(acc));
    return d;
}

template <int DT>
__device__ __forceinline__ void widen_word(float& lo, float& hi, uint32_t w)
{
    if (DT == kBf16) {
        lo = __uint_as_float(w << 16);
        hi = __uint_as_float(w & 0xFFFF0000u);
    } else {
        uint16_t l, h;
        asm("mov.b32 {%0, %1}, %2;" : "=h"(l), "=h"(h) : "r"(w));
        asm("cvt.f32.f16 %0, %1;" : "=f"(lo) : "h"(l));
        asm("cvt.f32.f16 %0, %1;" : "=f"(hi) : "h"(h));
    }
}

// Two binary32 -> one word of two 16-bit elements, round to nearest even, NaN -> 0x7FFF.
template <int DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t d;
    if (DT == kBf16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else             asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// ---- bulk copies ------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, unsigned arrivals)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(smem_u32(bar)), "r"(arrivals) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");   // visible to the bulk-copy engine
}

__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(smem_u32(bar)), "r"(bytes) : "memory");
}

// Bulk copy of `bytes` (a multiple of 16; both addresses 16-byte aligned) from global to this block's shared memory.
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* gsrc, unsigned bytes, uint64_t* bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(smem_u32(smem_dst)), "l"(gsrc), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}

__device__ __forceinline__ bool mbar_try_wait(uint64_t* bar, unsigned parity)
{
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return done != 0;
}

// Bounded wait for phase `parity` of an mbarrier: after timeout_ns the thread latches NUNA_ERR_TIMEOUT in
// *status and gives up (the caller skips its work and returns; nothing traps).
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, unsigned parity, unsigned* status, unsigned long long timeout_ns)
{
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = globaltimer_ns();
    unsigned polls = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++polls & 255u) == 0u && globaltimer_ns() - t0 > timeout_ns) {
            atomicMax(status, 6u);                     // NUNA_ERR_TIMEOUT
            return false;
        }
    }
    return true;
}

// ---- clusters ---------------------------------------------------------------------------------

__device__ __forceinline__ unsigned cluster_ctarank()
{
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace nuna
