// What the operators around the collectives share: argument checks, launches, and rows in 16-byte vectors or single
// elements.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <cstdio>
#include <cstring>
#include <type_traits>

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

// Whether every matrix's rows are whole 16-byte vectors at 16-byte addresses.  A matrix that is not given has no addresses, but
// its rows' length counts all the same: kernels cut all rows by it (no tokens: a 16-bit dout that need not be there and its
// binary32 dtable, whose rows of 4 elements are a whole vector, are cut in eights).
struct VectorRows {
    bool ok;
    VectorRows& rows(const void* at, size_t elems, size_t stride, size_t size)
    {
        ok = ok && !((elems * size) & 15u) && (!at || !(((uintptr_t)at | (stride ? stride : elems) * size) & 15u));
        return *this;
    }
};

// Kernel arguments, filled up to 32 bytes beyond a multiple of 64: see ParamPad.
template <typename T, size_t kPad = (96 - sizeof(T) % 64) % 64>
struct Padded : T {
    unsigned char unused[kPad];
};
template <typename T>
struct Padded<T, 0> : T {};

struct Shape {
    unsigned grid, block, smem, cluster;
};

// Launches an operator's kernel, as a dependent launch if the flags say so (effective_flags has been asked).
template <typename... Args, typename... Act>
int launch_kernel(void (*kernel)(Args...), const Shape& sh, unsigned flags, void* stream, Act&&... args)
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

template <typename T>
int launch_op(void (*kernel)(Padded<T>), const Shape& sh, unsigned flags, void* stream, const T& args)
{
    static_assert(sizeof(Padded<T>) % 64 == 32, "see ParamPad");
    Padded<T> a = {};
    static_cast<T&>(a) = args;
    return launch_kernel(kernel, sh, flags, stream, a);
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

// What every operator's kernel begins with.  A short grid (`brief`: its blocks do not loop) that leaves SMs free releases its
// successor at once: the slots that the waiting blocks take are not missed, and their launch is out of the way when this grid
// ends (norm of 1 x 8192 3.5 -> 3.15 us; 4096 rows in 148 looping blocks 45.7 -> 46.6, which is why they do not).
__device__ __forceinline__ void pdl_begin(bool brief = true)
{
    if (brief && gridDim.x <= kSms) pdl_trigger();
    pdl_wait();
}

// A pack is what a thread moves at once: a 16-byte vector, or (rows of any length and alignment) one element, or two elements
// that need not be neighbours, each in a word of its own, for arithmetic in pairs.  Where only the first two are meant, a bool
// says which.
constexpr int kElement = 0, kVector = 1, kPair = 2;
template <int DT, int kForm> struct Pack {
    static constexpr int kElems = kForm == kVector ? Elem<DT>::kElems : kForm == kPair ? 2 : 1;
    static constexpr int kWords = kForm == kVector ? 4 : kElems;
    uint32_t w[kWords];
};

template <int DT, int kForm>
__device__ __forceinline__ Pack<DT, kForm> load_pack(const void* row, size_t i)
{
    static_assert(kForm != kPair);
    Pack<DT, kForm> p;
    if constexpr (kForm == kVector) {
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
template <int DT, int kForm, bool kStream = false>
__device__ __forceinline__ void store_pack(void* row, size_t i, const Pack<DT, kForm>& p)
{
    static_assert(kForm != kPair);
    if constexpr (kForm == kVector) {
        const uint4 v = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
        if (kStream) st_stream(static_cast<uint4*>(row) + i, v);
        else         st_dst(static_cast<uint4*>(row) + i, v);
    } else if constexpr (DT == kF32) {
        static_cast<uint32_t*>(row)[i] = p.w[0];
    } else {
        static_cast<uint16_t*>(row)[i] = (uint16_t)p.w[0];
    }
}

// 32 bytes at a 32-byte address in one store: a warp whose lanes hold eight binary32 each writes whole sectors, which two
// 16-byte stores do not (they reach L2 as halves of twice as many).
__device__ __forceinline__ void store8(float* p, const float (&f)[8])
{
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]) : "memory");
}

template <int DT, int kForm>
__device__ __forceinline__ void unpack(float (&f)[Pack<DT, kForm>::kElems], const Pack<DT, kForm>& p)
{
    if constexpr (DT == kF32) {
#pragma unroll
        for (int i = 0; i < Pack<DT, kForm>::kElems; ++i) f[i] = __uint_as_float(p.w[i]);
    } else if constexpr (kForm == kVector) {
#pragma unroll
        for (int i = 0; i < 4; ++i) widen_word<DT>(f[2 * i], f[2 * i + 1], p.w[i]);
    } else {
        float unused;
#pragma unroll
        for (int i = 0; i < Pack<DT, kForm>::kElems; ++i) widen_word<DT>(f[i], unused, p.w[i]);
    }
}

template <int DT, int kForm>
__device__ __forceinline__ Pack<DT, kForm> pack(const float (&f)[Pack<DT, kForm>::kElems])
{
    Pack<DT, kForm> p;
    if constexpr (DT == kF32) {
#pragma unroll
        for (int i = 0; i < Pack<DT, kForm>::kElems; ++i) p.w[i] = __float_as_uint(f[i]);
    } else if constexpr (kForm == kPair) {
        const uint32_t both = pack2<DT>(f[0], f[1]);
        p.w[0] = both & 0xFFFFu, p.w[1] = both >> 16;
    } else if constexpr (kForm == kVector) {
#pragma unroll
        for (int i = 0; i < 4; ++i) p.w[i] = pack2<DT>(f[2 * i], f[2 * i + 1]);
    } else {
        p.w[0] = pack2<DT>(f[0], 0.0f) & 0xFFFFu;
    }
    return p;
}

// N consecutive parameters of type PT (1, 4 or 8; vectors if more than one), kept as they are stored.
template <int PT, int N> struct Params {
    static constexpr int kWords = PT == kF32 ? N : (N + 1) / 2;
    uint32_t w[kWords];
};

// Those from element i * N on; `fill` (a pattern of PT's type) where there are no parameters.
template <int PT, int N>
__device__ __forceinline__ Params<PT, N> load_params(const void* base, size_t i, uint32_t fill)
{
    Params<PT, N> p;
    if (base == nullptr) {
#pragma unroll
        for (int k = 0; k < Params<PT, N>::kWords; ++k) p.w[k] = fill;
    } else if constexpr (N == 1) {
        p.w[0] = load_pack<PT, false>(base, i).w[0];
    } else {
#pragma unroll
        for (int k = 0; k < Params<PT, N>::kWords; k += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint32_t*>(base) + i * Params<PT, N>::kWords + k);
            p.w[k] = v.x, p.w[k + 1] = v.y, p.w[k + 2] = v.z, p.w[k + 3] = v.w;
        }
    }
    return p;
}

// One, as load_params' fill: both halves of a word for the 16-bit types.
template <int PT> constexpr uint32_t kOne = PT == kF32 ? 0x3F800000u : PT == kBf16 ? 0x3F803F80u : 0x3C003C00u;

template <int PT, int N>
__device__ __forceinline__ void unpack_params(float (&f)[N], const Params<PT, N>& p)
{
    if constexpr (PT == kF32) {
#pragma unroll
        for (int k = 0; k < N; ++k) f[k] = __uint_as_float(p.w[k]);
    } else if constexpr (N == 1) {
        float unused;
        widen_word<PT>(f[0], unused, p.w[0]);
    } else {
#pragma unroll
        for (int k = 0; k < N / 2; ++k) widen_word<PT>(f[2 * k], f[2 * k + 1], p.w[k]);
    }
}

// Copies 16 bytes to shared memory without a register; the thread waits for its own copies, group by group.
__device__ __forceinline__ void copy_async(uint32_t to_shared, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to_shared), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until at most kLeft of the thread's latest groups are still on their way.
template <int kLeft>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(kLeft) : "memory"); }

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

// ---- pieces of rows that are not whole vectors ---------------------------------------------------------
//
// Where rows are not whole 16-byte vectors at 16-byte addresses (odd lengths, odd strides), a row that is written is cut at its
// own 16-byte boundaries: piece i is the E elements from E * i - s on, s being how far behind a boundary the row begins.  All
// pieces but the first and the last are then stored as vectors.  A row that is read lies at some other distance from a boundary,
// the same for all of its pieces: a piece is shifted out of the two vectors around it, 2 loads and 4 shifts instead of E loads
// (lookup of 20011 rows of 1037 f16: 26.5 -> 23.6 us).  Those two vectors may reach up to 14 bytes beyond the row, into its
// neighbours or the gaps; what comes from there is not used, and the first and the last row of a matrix, where nothing need be
// there, are read element by element.
template <int DT, bool kWhole> struct Piece {
    uint32_t w[kWhole ? 4 : 8];
};

// Elements from which a row at this address is behind a boundary of E of its elements.
template <int DT, int E>
__device__ __forceinline__ int behind(const void* row) { return (int)(((uintptr_t)row & (E * Elem<DT>::kBytes - 1u)) / Elem<DT>::kBytes); }

// A row that is read in the pieces of a row that begins s elements behind a boundary: piece i is shifted by m bytes out of the
// vectors at at + 16 * i and behind it.
struct Source {
    const char* at;
    unsigned m;
    bool by_element;
};

template <int DT, bool kWhole>
__device__ __forceinline__ Source source_of(const void* base, size_t row, size_t stride, size_t rows, unsigned hidden, int s)
{
    const char* from = static_cast<const char*>(row_at(base, row, stride)) - s * Elem<DT>::kBytes;
    if constexpr (kWhole) return {from, 0u, false};
    if (row == 0 || row + 1 == rows || hidden < (unsigned)Elem<DT>::kElems) return {from, 0u, true};
    const unsigned m = (unsigned)(uintptr_t)from & 15u;
    return {from - m, m, false};
}

// Starts loading piece i, which begins at element e0 = E * i - s; what is outside of the row is not defined.  At least one of
// its elements is inside.
template <int DT, bool kWhole>
__device__ __forceinline__ void fetch_piece(Piece<DT, kWhole>& p, const Source& src, unsigned i, int e0, unsigned hidden)
{
    constexpr int kBytes = Elem<DT>::kBytes, E = Elem<DT>::kElems;
    const char* at = src.at + (size_t)i * 16u;
    if constexpr (kWhole) {
        const uint4 v = ld_src(reinterpret_cast<const uint4*>(at));
        p.w[0] = v.x, p.w[1] = v.y, p.w[2] = v.z, p.w[3] = v.w;
    } else if (src.by_element) {
#pragma unroll
        for (int k = 0; k < 8; ++k) p.w[k] = 0u;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e0 + e >= 0 && e0 + e < (int)hidden) {
                if constexpr (DT == kF32) p.w[e] = ld_src32(reinterpret_cast<const uint32_t*>(at) + e);
                else                      p.w[e / 2] |= (uint32_t)ld_src16(reinterpret_cast<const uint16_t*>(at) + e) << (16 * (e % 2));
            }
    } else {
        // the first vector holds elements e0 - m / kBytes ... + E-1 of the row, the second the E behind them: loaded if one is in the row
        const int left = e0 + E - (int)(src.m / kBytes);
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.gt.s32 p, %9, 0;\n\tsetp.lt.s32 q, %9, %10;\n\tsetp.ne.and.u32 q, %11, 0, q;\n\t"
                     "@p ld.global.v4.u32 {%0,%1,%2,%3}, [%8];\n\t@q ld.global.v4.u32 {%4,%5,%6,%7}, [%8+16];\n\t}"
                     : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[2]), "=r"(p.w[3]), "=r"(p.w[4]), "=r"(p.w[5]), "=r"(p.w[6]), "=r"(p.w[7])
                     : "l"(at), "r"(left), "r"((int)hidden), "r"(src.m));
    }
}

// The elements of a piece that has arrived.
template <int DT, bool kWhole>
__device__ __forceinline__ Pack<DT, true> settle_piece(const Piece<DT, kWhole>& p, const Source& src)
{
    Pack<DT, true> v;
    if constexpr (kWhole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = p.w[i];
    } else {
        // two words, one word, part of a word
        uint32_t t[6], u[5];
#pragma unroll
        for (int i = 0; i < 6; ++i) t[i] = src.m & 8u ? p.w[i + 2] : p.w[i];
#pragma unroll
        for (int i = 0; i < 5; ++i) u[i] = src.m & 4u ? t[i + 1] : t[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = DT == kF32 ? u[i] : __funnelshift_r(u[i], u[i + 1], src.m * 8u);    // modulo 32
    }
    return v;
}

// Whether a piece is wholly inside its row.
template <int E>
__device__ __forceinline__ bool inside(int e0, unsigned hidden) { return e0 >= 0 && (unsigned)e0 + E <= hidden; }

// Whether a piece has an element of its row.
template <int E>
__device__ __forceinline__ bool touches(int e0, unsigned hidden) { return e0 > -E && e0 < (int)hidden; }

// Stores those elements of a piece that are in the row; row + e0 is at a 16-byte boundary.
template <int DT, bool kWhole, bool kStream = false>
__device__ __forceinline__ void store_piece(void* row, unsigned hidden, int e0, const Pack<DT, true>& v)
{
    constexpr int kBytes = Elem<DT>::kBytes, E = Elem<DT>::kElems;
    char* at = static_cast<char*>(row) + (long long)e0 * kBytes;
    if (kWhole || inside<E>(e0, hidden)) {
        store_pack<DT, true, kStream>(at, 0, v);
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e0 + e >= 0 && e0 + e < (int)hidden) {
                if constexpr (DT == kF32) reinterpret_cast<uint32_t*>(at)[e] = v.w[e];
                else                      reinterpret_cast<uint16_t*>(at)[e] = (uint16_t)(v.w[e / 2] >> (16 * (e % 2)));
            }
    }
}

// Pairs of binary32 in one instruction (sm_100's f32x2 forms: each half rounds as the plain instruction does).  The
// element-wise loops of the norm take 40 to 50 % of the issue slots with these, which halve their arithmetic.
struct Two {
    float x, y;
};
__device__ __forceinline__ Two operator+(Two a, Two b)
{
    Two d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two operator*(Two a, Two b)
{
    Two d;
    asm("{\n\t.reg .b64 a, b, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 d, a, b;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ Two mad(Two a, Two b, Two c)
{
    Two d;
    asm("{\n\t.reg .b64 a, b, c, d;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 d, a, b, c;\n\tmov.b64 {%0, %1}, d;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float mad(float a, float b, float c) { return fmaf(a, b, c); }

// What a pack's arithmetic is done in: pairs, or for a single element a float.
template <int DT, int kForm> using Lanes = std::conditional_t<(Pack<DT, kForm>::kElems > 1), Two, float>;
template <typename V> __device__ __forceinline__ V all(float v);
template <> __device__ __forceinline__ Two all<Two>(float v) { return {v, v}; }
template <> __device__ __forceinline__ float all<float>(float v) { return v; }
__device__ __forceinline__ float total(Two v) { return v.x + v.y; }
__device__ __forceinline__ float total(float v) { return v; }
__device__ __forceinline__ float& half(Two& v, int i) { return i % 2 ? v.y : v.x; }
__device__ __forceinline__ float& half(float& v, int) { return v; }

template <int DT, int kForm> constexpr int kLanes = (Pack<DT, kForm>::kElems + 1) / 2;

template <int DT, int kForm>
__device__ __forceinline__ void unpack(Two (&f)[kLanes<DT, kForm>], const Pack<DT, kForm>& p)
{
    float v[Pack<DT, kForm>::kElems];
    unpack<DT, kForm>(v, p);
#pragma unroll
    for (int i = 0; i < kLanes<DT, kForm>; ++i) f[i] = {v[2 * i], v[2 * i + 1]};
}
template <int DT, int kForm>
__device__ __forceinline__ Pack<DT, kForm> pack(const Two (&f)[kLanes<DT, kForm>])
{
    float v[Pack<DT, kForm>::kElems];
#pragma unroll
    for (int i = 0; i < kLanes<DT, kForm>; ++i) v[2 * i] = f[i].x, v[2 * i + 1] = f[i].y;
    return pack<DT, kForm>(v);
}
// f += the pack's elements: one instruction for a 16-bit element, none for widening it.
template <int DT, int kForm>
__device__ __forceinline__ void add_pack(Lanes<DT, kForm> (&f)[kLanes<DT, kForm>], const Pack<DT, kForm>& p)
{
    if constexpr (DT == kF32) {
        Lanes<DT, kForm> r[kLanes<DT, kForm>];
        unpack<DT, kForm>(r, p);
#pragma unroll
        for (int i = 0; i < kLanes<DT, kForm>; ++i) f[i] = f[i] + r[i];
    } else {
#pragma unroll
        for (int i = 0; i < kLanes<DT, kForm>; ++i) {
            half(f[i], 0) = add_narrow<DT>(half(f[i], 0), (uint16_t)p.w[i]);
            if constexpr (kForm == kVector) half(f[i], 1) = add_narrow<DT>(half(f[i], 1), (uint16_t)(p.w[i] >> 16));
            if constexpr (kForm == kPair)   half(f[i], 1) = add_narrow<DT>(half(f[i], 1), (uint16_t)p.w[i + 1]);
        }
    }
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
