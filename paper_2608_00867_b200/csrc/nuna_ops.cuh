// What the operators around the collectives share: argument checks, launches, and rows in 16-byte vectors or single
// elements.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstdio>
#include <cstring>

#include "nuna_device.cuh"
#include "nuna_internal.h"
#include "nuna_spans.h"

namespace nuna {

// ---- host ------------------------------------------------------------------------------------------

// Status of a call's pointers: missing, misaligned, or a written range that overlaps another one.  `twin_a` and `twin_b`
// may be the same matrix (-1: no two may).
inline int check_spans(const Spans& s, int twin_a = -1, int twin_b = -1)
{
    if (s.status != NUNA_OK) return s.status;
    for (int i = 0; i < s.n; ++i) {
        if (s.v[i].required && s.v[i].bytes && !s.v[i].at) return NUNA_ERR_INVALID_ARG;
        if ((uintptr_t)s.v[i].at % s.v[i].align) return NUNA_ERR_ALIGNMENT;
    }
    for (int i = 0; i < s.n; ++i) {
        const Span& a = s.v[i];
        if (!a.written || !a.at || !a.bytes) continue;
        for (int j = 0; j < s.n; ++j) {
            const Span& b = s.v[j];
            if (j == i || !b.at || !b.bytes) continue;
            if (((i == twin_a && j == twin_b) || (i == twin_b && j == twin_a)) && a.at == b.at && a.stride == b.stride) continue;
            if ((uintptr_t)a.at < (uintptr_t)b.at + b.bytes && (uintptr_t)b.at < (uintptr_t)a.at + a.bytes) return NUNA_ERR_ALIAS;
        }
    }
    return NUNA_OK;
}

// Whether every matrix's rows are whole 16-byte vectors at 16-byte addresses.
struct VectorRows {
    bool ok;
    VectorRows& rows(const void* at, size_t elems, size_t stride, size_t size)
    {
        ok = ok && (!at || !(((uintptr_t)at | (stride ? stride : elems) * size | elems * size) & 15u));
        return *this;
    }
};

struct Shape {
    unsigned grid, block, smem, cluster;
};

// Launches an operator's kernel, as a dependent launch if the flags say so (effective_flags has been asked).
template <typename... Args, typename... Act>
int launch_op(void (*kernel)(Args...), const Shape& sh, unsigned flags, void* stream, Act&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sh.grid, 1, 1);
    cfg.blockDim = dim3(sh.block, 1, 1);
    cfg.dynamicSmemBytes = sh.smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (sh.cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = sh.cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (flags & NUNA_LAUNCH_PDL) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, static_cast<Args>(args)...);
    if (e != cudaSuccess) {
        fprintf(stderr, "nuna: kernel launch failed: %s\n", cudaGetErrorString(e));
        return NUNA_ERR_CUDA;
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return NUNA_OK;
}

// Raises the kernel's limit of dynamic shared memory, once per device.
template <auto kKernel>
int allow_smem(int bytes)
{
    static std::atomic<bool> done[kMaxDevices];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return NUNA_ERR_CUDA;
    if (!done[dev].load(std::memory_order_relaxed)) {
        if (cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return NUNA_ERR_CUDA;
        done[dev].store(true, std::memory_order_relaxed);
    }
    return NUNA_OK;
}

// B200's SMs.  Grids and the split of sums are cut for them, so that what a sum's order depends on is the call alone.
constexpr unsigned kSms = 148;

// f(DT) with the element type as a constant.
template <typename F>
int with_dtype(int dtype, F&& f)
{
    switch (dtype) {
        case NUNA_BF16: return f(std::integral_constant<int, kBf16>{});
        case NUNA_F16: return f(std::integral_constant<int, kF16>{});
        default: return f(std::integral_constant<int, kF32>{});
    }
}

// ---- device ----------------------------------------------------------------------------------------

// A pack is what a thread moves at once: a 16-byte vector, or (rows of any length and alignment) one element.
template <int DT, bool kVec> struct Pack {
    static constexpr int kElems = kVec ? Elem<DT>::kElems : 1;
    static constexpr int kWords = kVec ? 4 : 1;
    uint32_t w[kWords];
};

template <int DT, bool kVec>
__device__ __forceinline__ Pack<DT, kVec> load_pack(const void* row, size_t i)
{
    Pack<DT, kVec> p;
    if constexpr (kVec) {
        const uint4 v = ld_src(static_cast<const uint4*>(row) + i);
        p.w[0] = v.x, p.w[1] = v.y, p.w[2] = v.z, p.w[3] = v.w;
    } else if constexpr (DT == kF32) {
        p.w[0] = ld_src32(static_cast<const uint32_t*>(row) + i);
    } else {
        p.w[0] = ld_src16(static_cast<const uint16_t*>(row) + i);
    }
    return p;
}

// kStream: written once and not read again soon (evict-first).
template <int DT, bool kVec, bool kStream = false>
__device__ __forceinline__ void store_pack(void* row, size_t i, const Pack<DT, kVec>& p)
{
    if constexpr (kVec) {
        const uint4 v = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
        if (kStream) st_stream(static_cast<uint4*>(row) + i, v);
        else         st_dst(static_cast<uint4*>(row) + i, v);
    } else if constexpr (DT == kF32) {
        static_cast<uint32_t*>(row)[i] = p.w[0];
    } else {
        static_cast<uint16_t*>(row)[i] = (uint16_t)p.w[0];
    }
}

template <int DT, bool kVec>
__device__ __forceinline__ void unpack(float (&f)[Pack<DT, kVec>::kElems], const Pack<DT, kVec>& p)
{
    if constexpr (DT == kF32) {
#pragma unroll
        for (int i = 0; i < Pack<DT, kVec>::kElems; ++i) f[i] = __uint_as_float(p.w[i]);
    } else if constexpr (kVec) {
#pragma unroll
        for (int i = 0; i < 4; ++i) widen_word<DT>(f[2 * i], f[2 * i + 1], p.w[i]);
    } else {
        float unused;
        widen_word<DT>(f[0], unused, p.w[0]);
    }
}

template <int DT, bool kVec>
__device__ __forceinline__ Pack<DT, kVec> pack(const float (&f)[Pack<DT, kVec>::kElems])
{
    Pack<DT, kVec> p;
    if constexpr (DT == kF32) {
#pragma unroll
        for (int i = 0; i < Pack<DT, kVec>::kElems; ++i) p.w[i] = __float_as_uint(f[i]);
    } else if constexpr (kVec) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p.w[i] = pack2<DT>(f[2 * i], f[2 * i + 1]);
    } else {
        p.w[0] = pack2<DT>(f[0], 0.0f) & 0xFFFFu;
    }
    return p;
}

// N consecutive parameters of type PT from element i * N on, in binary32 (N of 1, 4 or 8; vectors if more than one).
template <int PT, int N>
__device__ __forceinline__ void load_params(float (&f)[N], const void* base, size_t i)
{
    if constexpr (N == 1) {
        unpack<PT, false>(f, load_pack<PT, false>(base, i));
    } else if constexpr (PT == kF32) {
#pragma unroll
        for (int k = 0; k < N / 4; ++k) {
            const uint4 v = *(static_cast<const uint4*>(base) + i * (N / 4) + k);
            f[4 * k] = __uint_as_float(v.x), f[4 * k + 1] = __uint_as_float(v.y);
            f[4 * k + 2] = __uint_as_float(v.z), f[4 * k + 3] = __uint_as_float(v.w);
        }
    } else {
        static_assert(N == 8, "a vector of 16-bit parameters");
        const uint4 v = *(static_cast<const uint4*>(base) + i);
        widen_word<PT>(f[0], f[1], v.x), widen_word<PT>(f[2], f[3], v.y);
        widen_word<PT>(f[4], f[5], v.z), widen_word<PT>(f[6], f[7], v.w);
    }
}

template <typename T>
__device__ __forceinline__ T* row_at(T* base, size_t row, size_t stride_bytes)
{
    return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(base) + row * stride_bytes);
}
__device__ __forceinline__ const void* row_at(const void* base, size_t row, size_t stride_bytes)
{
    return reinterpret_cast<const void*>(reinterpret_cast<uintptr_t>(base) + row * stride_bytes);
}
__device__ __forceinline__ void* row_at(void* base, size_t row, size_t stride_bytes)
{
    return reinterpret_cast<void*>(reinterpret_cast<uintptr_t>(base) + row * stride_bytes);
}

template <int N>
__device__ __forceinline__ void warp_sum(float (&v)[N])
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], d);
}

}  // namespace nuna
