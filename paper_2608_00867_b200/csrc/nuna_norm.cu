// Layer norm of the rows that an allreduce has summed, with the residual added, and its gradient.
//
// A row is held by a group of threads, each with up to kPacks 16-byte vectors (or pairs of elements where rows are not
// whole vectors): the sums of a row are a warp's shuffles and one exchange through shared memory, and every operand
// crosses the memory once.  Mean and variance are taken one after the other from the registers, so the variance is a sum
// of squared differences from the mean.  What bounds both directions is the memory: 4 streams of rows, 9 and 16 flops an element.
#include "nuna_ops.cuh"

#include <algorithm>

namespace nuna {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *summed, *y;
    float *mean, *rstd;
    size_t x_stride, residual_stride, summed_stride, y_stride;       // bytes
    unsigned rows, hidden, units, group;                             // vectors or elements in a row, threads of a group
    float eps, count, inverse;                                       // count: hidden; inverse: 1 / hidden
};

struct NormGradArgs {
    const void *dy, *x, *weight, *dsummed;
    const float *mean, *rstd;
    void* dx;
    float* part;                                                     // [gridDim.x][2][part_stride], or null
    size_t dy_stride, x_stride, dsummed_stride, dx_stride;           // bytes
    unsigned rows, hidden, units, group, part_stride;
    float count, inverse;                                            // hidden, 1 / hidden
};

// Sums v over the warps of this thread's group (all threads of the group call; g: the group's number in its block).  Groups
// do not wait for one another.  Two consecutive calls use different halves of `red`, [2][32][N]: the exchange of the second
// separates the uses of the first.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], unsigned warps, unsigned g, float* red)
{
    warp_sum<N>(v);
    if (warps == 1u) return;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, first = g * warps;
    if (lane == 0u)
#pragma unroll
        for (int i = 0; i < N; ++i) red[warp * N + i] = v[i];
    asm volatile("bar.sync %0, %1;" :: "r"(1u + g), "r"(warps * 32u) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < warps ? red[(first + lane) * N + i] : 0.0f;
    warp_sum<N>(v);
}

// sum / count.  The reciprocal's rounding is taken back by the remainder, so that equal elements whose sum is exact have
// themselves as their mean.
__device__ __forceinline__ float quotient(float sum, float count, float inverse)
{
    const float q = sum * inverse;
    const float better = fmaf(fmaf(-q, count, sum), inverse, q);
    return isfinite(q) ? better : q;
}

// The mean of a long sum has been rounded many times over.  Where elements are as fine as the sum itself (binary32 rows; rows of
// any length), and a row lies far from zero for its spread, that error counts in the differences from it: of 8192 equal elements of
// 1e5, 0.98 came out where 0 is right.  Such rows have their differences, which are exact, added too: their mean belongs to
// the mean and off the differences, its square off the variance.  It is at most n * 2^-24 * (|mean| + spread) with n (42 up to 32768
// elements) additions in a row, so rows within 8 spreads of zero, which are left as they are, are off by 2e-5 of a spread at
// most.  (16-bit elements of rows that a block holds: the sums of equal ones are exact, and one step of a few elements is far
// above the mean's error.)  Where the squares overflow the mean alone is settled, if its row is finite.
__device__ __forceinline__ bool far_from_zero(float mean, float variance) { return variance < mean * mean * 0.015625f || isinf(variance); }
__device__ __forceinline__ float settle(float& mean, float& variance, float differences, float count, float inverse)
{
    float shift = quotient(differences, count, inverse);
    if (!isfinite(shift)) shift = 0.0f;
    mean += shift;
    variance = fmaxf(fmaf(-shift, shift, variance), 0.0f);
    return shift;
}

// How rows are cut.  Whole vectors: a thread's are 32 apart, a warp's consecutive.  Otherwise pairs of elements that are 32
// apart, so that loads and stores of a warp are consecutive and sums are taken in pairs at any alignment; a thread's pairs are
// 64 elements apart.  Either way the addresses of a row's packs differ by constants, and a warp whose packs are all in the row
// takes a loop without a question (8000 x 2731 f16 from 67 instructions an element and 69.5 us to 35 and 41.9; gradient 84.4 to
// 59.0).  What rows that are not whole vectors then wait for is latency: 39 to 51 % of the issue slots, 17 to 32 % of the warps.
template <int DT, bool kVec> struct Cut {
    static constexpr int kForm = kVec ? kVector : kPair;
    static constexpr unsigned kStep = kVec ? 32 : 64;                // in units: vectors or elements
    static constexpr unsigned kBytes = kVec ? 16 : Elem<DT>::kBytes; // of a unit
    static __device__ __forceinline__ unsigned first(unsigned lane, unsigned packs) { return lane / 32u * kStep * packs + lane % 32u; }
    static __device__ __forceinline__ void* at(void* row, unsigned first) { return static_cast<char*>(row) + (size_t)first * kBytes; }
    static __device__ __forceinline__ const void* at(const void* row, unsigned first) { return static_cast<const char*>(row) + (size_t)first * kBytes; }
    // Whether the thread, which has `left` units from its first one on, has pack k, and the second element of its pair.
    static __device__ __forceinline__ bool has(unsigned left, int k) { return k * kStep < left; }
    static __device__ __forceinline__ bool second(unsigned left, int k) { return k * kStep + 32u < left; }
};

// Stores pack k of a row from the thread's first unit on.
template <int DT, bool kVec>
__device__ __forceinline__ void put_pack(void* row, unsigned left, int k, const Pack<DT, Cut<DT, kVec>::kForm>& p)
{
    if constexpr (kVec) {
        store_pack<DT, kVector>(row, k * 32, p);
    } else {
        store_pack<DT, kElement>(row, k * 64, {{p.w[0]}});
        if (Cut<DT, kVec>::second(left, k)) store_pack<DT, kElement>(row, k * 64 + 32, {{p.w[1]}});
    }
}

// A pack's parameters, `first` being its first unit.
template <int PT, int E, bool kVec>
__device__ __forceinline__ Params<PT, E> params_of(const void* base, unsigned first, unsigned units, uint32_t fill)
{
    if constexpr (kVec) {
        return load_params<PT, E>(first < units ? base : nullptr, first, fill);
    } else {
        const uint32_t a = load_params<PT, 1>(first < units ? base : nullptr, first, fill).w[0];
        const uint32_t b = load_params<PT, 1>(first + 32u < units ? base : nullptr, first + 32u, fill).w[0];
        if constexpr (PT == kF32) return {{a, b}};
        else                      return {{__byte_perm(a, b, 0x5410u)}};
    }
}

// The rows that a group takes, one after the other, fetched ahead of their use.  Vectors go through shared memory by
// asynchronous copies: a thread fetches, kDepth rows ahead, just the vectors that it will use, so it waits for its own copies
// only, and what is in flight holds no registers.  Pairs are loaded into registers, a row ahead where there are
// enough of them.
template <int DT, int kPacks, bool kVec, int kStreams, int kDepth>
struct RowFetch {
    const void* from[kStreams];
    size_t stride[kStreams];
    bool given[kStreams];
    unsigned rows, first;                                            // the thread's first unit
    uint32_t slots;                                                  // this thread's part of the shared memory: one slot per fetch
    Pack<DT, Cut<DT, kVec>::kForm> next[kVec ? 1 : kStreams][kVec ? 1 : kPacks];     // zeros, where the row has ended

    static constexpr unsigned kSlots = kVec ? kDepth * kStreams * kPacks : 0;       // 16 bytes each, per thread

    __device__ __forceinline__ uint32_t slot(unsigned stage, int s, int k) const { return slots + ((stage * kStreams + s) * kPacks + k) * 512u; }

    // Starts fetching `row` as the stage-th of the ring, the thread having `left` units of it.
    __device__ __forceinline__ void start(unsigned long long row, unsigned stage, unsigned left)
    {
#pragma unroll
        for (int s = 0; s < kStreams; ++s) {
            if (!given[s]) continue;
            const void* at = Cut<DT, kVec>::at(row_at(from[s], (size_t)row, stride[s]), first);
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                if (row < rows && Cut<DT, kVec>::has(left, k)) {
                    if constexpr (kVec) copy_async(slot(stage, s, k), static_cast<const uint4*>(at) + k * 32);
                    else next[s][k].w[0] = load_pack<DT, kElement>(at, k * 64).w[0];
                }
                if constexpr (!kVec)
                    if (row < rows && Cut<DT, kVec>::second(left, k)) next[s][k].w[1] = load_pack<DT, kElement>(at, k * 64 + 32).w[0];
            }
        }
        if constexpr (kVec) copy_commit();
    }
    __device__ __forceinline__ Pack<DT, Cut<DT, kVec>::kForm> take(unsigned stage, int s, int k) const
    {
        if constexpr (kVec) {
            Pack<DT, kVector> p;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(p.w[0]), "=r"(p.w[1]), "=r"(p.w[2]), "=r"(p.w[3]) : "r"(slot(stage, s, k)));
            return p;
        } else {
            return next[s][k];
        }
    }
};

// The parameters of a thread's columns for all of its rows: widened once where there are registers for it, or as they are stored.
template <int PT, int E, int kPacks, bool kWide>
struct KeptParams {
    static constexpr int P = (E + 1) / 2;
    Params<kWide ? kF32 : PT, E> p[kPacks];

    __device__ __forceinline__ void put(int k, const Params<PT, E>& v)
    {
        if constexpr (kWide) {
            float f[E];
            unpack_params<PT, E>(f, v);
#pragma unroll
            for (int e = 0; e < E; ++e) p[k].w[e] = __float_as_uint(f[e]);
        } else {
            p[k] = v;
        }
    }
    template <typename V>
    __device__ __forceinline__ void get(V (&f)[P], int k) const
    {
        float v[E];
        unpack_params<kWide ? kF32 : PT, E>(v, p[k]);
#pragma unroll
        for (int e = 0; e < E; ++e) half(f[e / 2], e) = v[e];
    }
};

// Most threads of a block, and rows that are fetched ahead of the one in work.
__host__ __device__ constexpr int norm_threads(int packs, bool vec) { return (vec && packs > 1) || packs == 8 ? 512 : 1024; }
__host__ __device__ constexpr int norm_depth(int packs, bool vec) { return !vec ? 2 : packs == 4 ? 2 : 3; }

template <int DT, int PT, int kPacks, bool kVec>
__global__ void __launch_bounds__(norm_threads(kPacks, kVec)) k_norm_forward(const Padded<NormArgs> a)
{
    using C = Cut<DT, kVec>;
    constexpr int kForm = C::kForm, E = Pack<DT, kForm>::kElems;
    constexpr int kDepth = norm_depth(kPacks, kVec);
    __shared__ float red[2][32];
    extern __shared__ uint4 ring[];
    const unsigned warps = a.group / 32u, g = threadIdx.x / a.group, lane = threadIdx.x % a.group, groups = blockDim.x / a.group;
    const unsigned first = C::first(lane, kPacks), left = a.units > first ? a.units - first : 0u;
    const unsigned step = gridDim.x * groups;                        // far below 2^31, as is the number of rows
    unsigned row = blockIdx.x * groups + g;
    RowFetch<DT, kPacks, kVec, 2, kDepth> fetch = {{a.x, a.residual}, {a.x_stride, a.residual_stride}, {true, a.residual != nullptr},
                                                   a.rows, first, smem_u32(ring + threadIdx.x / 32u * 32u * RowFetch<DT, kPacks, kVec, 2, kDepth>::kSlots + threadIdx.x % 32u), {}};
    pdl_begin(a.rows <= step);
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch.start(row + d * step, d, left);
    constexpr int P = kLanes<DT, kForm>;
    using V = Lanes<DT, kForm>;
    KeptParams<PT, E, kPacks, (kVec && kPacks <= 2)> w, b;
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
        const unsigned i = first + k * C::kStep;
        w.put(k, params_of<PT, E, kVec>(a.weight, i, a.units, kOne<PT>));
        b.put(k, params_of<PT, E, kVec>(a.bias, i, a.units, 0u));
    }
    unsigned turn = 0, stage = 0;
    const auto work = [&](unsigned left) {
        for (unsigned base = blockIdx.x * groups; base < a.rows; base += step, row += step) {
            const bool live = row < a.rows;
            V f[kPacks][P];
            if constexpr (kVec) {
                fetch.start(row + (kDepth - 1) * step, stage == 0u ? kDepth - 1 : stage - 1u, left);
                copy_wait<kDepth - 1>();
            }
            void* to_sum = C::at(row_at(a.summed, (size_t)row, a.summed_stride), first);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k) {
    #pragma unroll
                for (int e = 0; e < P; ++e) f[k][e] = all<V>(0.0f);
                if (live && C::has(left, k)) {
                    unpack<DT, kForm>(f[k], fetch.take(stage, 0, k));
                    if (a.residual) {
                        add_pack<DT, kForm>(f[k], fetch.take(stage, 1, k));
                        const Pack<DT, kForm> s = pack<DT, kForm>(f[k]);
                        put_pack<DT, kVec>(to_sum, left, k, s);
                        unpack<DT, kForm>(f[k], s);                       // the norm is that of the stored row
                    }
                }
            }
            if constexpr (!kVec) fetch.start(row + step, 0, left);
            V part = all<V>(0.0f);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k)
    #pragma unroll
                for (int e = 0; e < P; ++e) part = part + f[k][e];
            float sum[1] = {total(part)};
            group_sum<1>(sum, warps, g, red[turn]);
            turn ^= 1u;
            float mean = quotient(sum[0], a.count, a.inverse);
            part = all<V>(0.0f);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k)
                if (C::has(left, k))
    #pragma unroll
                    for (int e = 0; e < P; ++e) {
                        f[k][e] = f[k][e] + all<V>(-mean);
                        if (!kVec && !C::second(left, k)) half(f[k][e], 1) = 0.0f;                  // there is none
                        part = mad(f[k][e], f[k][e], part);
                    }
            float sq[1] = {total(part)};
            group_sum<1>(sq, warps, g, red[turn]);
            turn ^= 1u;
            float rstd = rsqrtf(fmaf(sq[0], a.inverse, a.eps)), variance = sq[0] * a.inverse;
            if (DT == kF32 && far_from_zero(mean, variance)) {           // the same for the whole group
                part = all<V>(0.0f);
    #pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (C::has(left, k))
    #pragma unroll
                        for (int e = 0; e < P; ++e) part = part + f[k][e];
                float differences[1] = {total(part)};
                group_sum<1>(differences, warps, g, red[turn]);
                turn ^= 1u;
                const float shift = settle(mean, variance, differences[0], a.count, a.inverse);
                rstd = rsqrtf(variance + a.eps);
    #pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (C::has(left, k))
    #pragma unroll
                        for (int e = 0; e < P; ++e) f[k][e] = f[k][e] + all<V>(-shift);
            }
            if (live && lane == 0u) {
                if (a.mean) a.mean[row] = mean;
                if (a.rstd) a.rstd[row] = rstd;
            }
            void* to = C::at(row_at(a.y, (size_t)row, a.y_stride), first);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                if (live && C::has(left, k)) {
                    V wf[P], bf[P];
                    w.get(wf, k);
                    b.get(bf, k);
    #pragma unroll
                    for (int e = 0; e < P; ++e) f[k][e] = mad(f[k][e] * all<V>(rstd), wf[e], bf[e]);
                    put_pack<DT, kVec>(to, left, k, pack<DT, kForm>(f[k]));
                }
            }
            stage = stage + 1u == kDepth ? 0u : stage + 1u;
        }
    };
    if (first - first % 32u + C::kStep * kPacks <= a.units) work(0xFFFFFFFFu);          // a warp whose packs are all in the row
    else                                                    work(left);
    pdl_trigger();
}

// Rows longer than a block's registers hold: one block per row, which reads the row again for each of the three steps.
template <int DT, int PT, bool kVec>
__global__ void __launch_bounds__(1024) k_norm_forward_long(const Padded<NormArgs> a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    __shared__ float red[3][32];
    pdl_begin(a.rows <= gridDim.x);
    const unsigned warps = blockDim.x / 32u;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void* x = row_at(a.x, row, a.x_stride);
        float sum[1] = {0.0f};
#pragma unroll 4
        for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
            float f[E];
            unpack<DT, kVec>(f, load_pack<DT, kVec>(x, i));
            if (a.residual) {
                float r[E];
                unpack<DT, kVec>(r, load_pack<DT, kVec>(row_at(a.residual, row, a.residual_stride), i));
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = __fadd_rn(f[e], r[e]);
                const Pack<DT, kVec> s = pack<DT, kVec>(f);
                store_pack<DT, kVec>(row_at(a.summed, row, a.summed_stride), i, s);
                unpack<DT, kVec>(f, s);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += f[e];
        }
        const void* s = a.residual ? row_at(a.summed, row, a.summed_stride) : x;         // this thread's own stores
        group_sum<1>(sum, warps, 0u, red[0]);
        float mean = quotient(sum[0], a.count, a.inverse), shift = 0.0f;
        const float from = mean;
        float sq[1] = {0.0f};
#pragma unroll 4
        for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
            float f[E];
            unpack<DT, kVec>(f, load_pack<DT, kVec>(s, i));
#pragma unroll
            for (int e = 0; e < E; ++e) sq[0] = fmaf(f[e] - from, f[e] - from, sq[0]);
        }
        group_sum<1>(sq, warps, 0u, red[1]);
        float rstd = rsqrtf(fmaf(sq[0], a.inverse, a.eps)), variance = sq[0] * a.inverse;
        if (far_from_zero(mean, variance)) {                             // the same for the whole block
            float differences[1] = {0.0f};
#pragma unroll 4
            for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
                float f[E];
                unpack<DT, kVec>(f, load_pack<DT, kVec>(s, i));
#pragma unroll
                for (int e = 0; e < E; ++e) differences[0] += f[e] - from;
            }
            group_sum<1>(differences, warps, 0u, red[2]);
            shift = settle(mean, variance, differences[0], a.count, a.inverse);
            rstd = rsqrtf(variance + a.eps);
        }
        if (threadIdx.x == 0u) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll 4
        for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
            float f[E], w[E], b[E];
            unpack<DT, kVec>(f, load_pack<DT, kVec>(s, i));
            unpack_params<PT, E>(w, load_params<PT, E>(a.weight, i, kOne<PT>));
            unpack_params<PT, E>(b, load_params<PT, E>(a.bias, i, 0u));
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = fmaf((f[e] - from - shift) * rstd, w[e], b[e]);
            store_pack<DT, kVec>(row_at(a.y, row, a.y_stride), i, pack<DT, kVec>(f));
        }
    }
    pdl_trigger();
}

// ---- gradient ------------------------------------------------------------------------------------------
//
// A block's groups take rows in turn and keep their columns' shares of dweight and dbias in registers from row to row;
// at the end the block's groups are added and the block's share goes to the workspace, whose at most 148 rows
// k_norm_params adds up.  Which rows a group takes depends on sizes and types alone, and so do the sums' orders.
// Threads of a block, of which an SM has one, and rows fetched ahead (none: a row's single elements fill the registers).
constexpr int kNormGradThreads = 512;
__host__ __device__ constexpr int norm_grad_depth(int packs, bool vec) { return !vec && packs > 4 ? 1 : packs == 1 ? 4 : 2; }

template <int DT, int PT, int kPacks, bool kVec>
__global__ void __launch_bounds__(kNormGradThreads) k_norm_backward(const Padded<NormGradArgs> a)
{
    using C = Cut<DT, kVec>;
    constexpr int kForm = C::kForm, E = Pack<DT, kForm>::kElems;
    constexpr int kDepth = norm_grad_depth(kPacks, kVec);
    __shared__ float red[2][64];
    extern __shared__ uint4 ring[];                                  // in the end, the groups' shares: [groups - 1][2][kPacks * group * E]
    const unsigned warps = a.group / 32u, g = threadIdx.x / a.group, lane = threadIdx.x % a.group, groups = blockDim.x / a.group;
    const unsigned first = C::first(lane, kPacks), left = a.units > first ? a.units - first : 0u;
    const unsigned long long step = (unsigned long long)gridDim.x * groups;
    unsigned long long row = (unsigned long long)blockIdx.x * groups + g;
    RowFetch<DT, kPacks, kVec, 3, kDepth> fetch = {{a.x, a.dy, a.dsummed}, {a.x_stride, a.dy_stride, a.dsummed_stride}, {true, true, a.dsummed != nullptr},
                                                   a.rows, first, smem_u32(ring + threadIdx.x / 32u * 32u * RowFetch<DT, kPacks, kVec, 3, kDepth>::kSlots + threadIdx.x % 32u), {}};
    pdl_begin(a.rows <= step);
#pragma unroll
    for (int d = 0; d < kDepth - 1; ++d) fetch.start(row + d * step, d, left);
    constexpr int P = kLanes<DT, kForm>;
    using V = Lanes<DT, kForm>;
    V dw[kPacks][P], db[kPacks][P];
    KeptParams<PT, E, kPacks, false> w;
#pragma unroll
    for (int k = 0; k < kPacks; ++k) {
        const unsigned i = first + k * C::kStep;
        w.put(k, params_of<PT, E, kVec>(a.weight, i, a.units, kOne<PT>));
#pragma unroll
        for (int e = 0; e < P; ++e) dw[k][e] = db[k][e] = all<V>(0.0f);
    }
    float next_mean = row < a.rows ? a.mean[row] : 0.0f, next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
    unsigned turn = 0, stage = 0;
    const auto work = [&](unsigned left) {
        for (unsigned long long base = (unsigned long long)blockIdx.x * groups; base < a.rows; base += step, row += step) {
            const bool live = row < a.rows;
            const float mean = next_mean, rstd = next_rstd;
            if (row + step < a.rows) next_mean = a.mean[row + step], next_rstd = a.rstd[row + step];
            constexpr bool kKeep = kPacks * E <= 16 && kDepth > 1;       // registers for a row's xh and g; otherwise they are formed again
            V xh[kKeep ? kPacks : 1][P], gy[kKeep ? kPacks : 1][P], r[kDepth == 2 && !kVec ? kPacks : 1][P];
            const auto normal = [&](V (&x)[P], V (&g)[P], V (&dy)[P], int k) {
                V wf[P];
                unpack<DT, kForm>(x, fetch.take(stage, 0, k));
                unpack<DT, kForm>(dy, fetch.take(stage, 1, k));
                w.get(wf, k);
    #pragma unroll
                for (int e = 0; e < P; ++e) {
                    x[e] = (x[e] + all<V>(-mean)) * all<V>(rstd);
                    g[e] = dy[e] * wf[e];
                }
            };
            if constexpr (kVec) {
                fetch.start(row + (kDepth - 1) * step, stage == 0u ? kDepth - 1 : stage - 1u, left);
                copy_wait<kDepth - 1>();
            } else if constexpr (kDepth == 1) {
                fetch.start(row, 0, left);
            }
            V c0s = all<V>(0.0f), c1s = all<V>(0.0f);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                if (live && C::has(left, k)) {
                    V dy[P];
                    V (&x)[P] = xh[kKeep ? k : 0];
                    V (&g)[P] = gy[kKeep ? k : 0];
                    normal(x, g, dy, k);
                    if constexpr (!kVec && kDepth == 2)
                        if (a.dsummed) unpack<DT, kForm>(r[k], fetch.take(stage, 2, k));
    #pragma unroll
                    for (int e = 0; e < P; ++e) {
                        c0s = c0s + g[e];
                        c1s = mad(g[e], x[e], c1s);
                        dw[k][e] = mad(dy[e], x[e], dw[k][e]);
                        db[k][e] = db[k][e] + dy[e];
                    }
                }
            }
            if constexpr (!kVec && kDepth == 2) fetch.start(row + step, 0, left);
            float c[2] = {total(c0s), total(c1s)};
            group_sum<2>(c, warps, g, red[turn]);
            turn ^= 1u;
            const V c0 = all<V>(-c[0] * a.inverse), c1 = all<V>(-c[1] * a.inverse);
            void* to = C::at(row_at(a.dx, (size_t)row, a.dx_stride), first);
    #pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                if (live && C::has(left, k)) {
                    V (&s)[P] = r[kDepth == 2 && !kVec ? k : 0];
                    V (&x)[P] = xh[kKeep ? k : 0];
                    V (&g)[P] = gy[kKeep ? k : 0];
                    if constexpr (!kKeep) {
                        V dy[P];
                        normal(x, g, dy, k);
                    }
                    if (!a.dsummed) {
    #pragma unroll
                        for (int e = 0; e < P; ++e) s[e] = all<V>(0.0f);
                    } else if constexpr (kVec || kDepth == 1) {
                        unpack<DT, kForm>(s, fetch.take(stage, 2, k));
                    }
    #pragma unroll
                    for (int e = 0; e < P; ++e) s[e] = mad(all<V>(rstd), mad(x[e], c1, g[e] + c0), s[e]);
                    put_pack<DT, kVec>(to, left, k, pack<DT, kForm>(s));
                }
            }
            stage = stage + 1u == kDepth ? 0u : stage + 1u;
        }
    };
    if (first - first % 32u + C::kStep * kPacks <= a.units) work(0xFFFFFFFFu);          // a warp whose packs are all in the row
    else                                                    work(left);
    if (a.part) {
        float* joined = reinterpret_cast<float*>(ring);
        if constexpr (kVec) copy_wait<0>();
        __syncthreads();                                             // every thread is done with its slots
        const unsigned columns = kPacks * a.group * E;
        if (g > 0u) {
            float* to = joined + (size_t)(g - 1u) * 2u * columns;
#pragma unroll
            for (int k = 0; k < kPacks; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    to[(k * E + e) * a.group + lane] = half(dw[k][e / 2], e);
                    to[columns + (k * E + e) * a.group + lane] = half(db[k][e / 2], e);
                }
        }
        __syncthreads();
        if (g == 0u) {
            for (unsigned o = 0; o + 1u < groups; ++o) {
                const float* from = joined + (size_t)o * 2u * columns;
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        half(dw[k][e / 2], e) += from[(k * E + e) * a.group + lane];
                        half(db[k][e / 2], e) += from[columns + (k * E + e) * a.group + lane];
                    }
            }
            float* share = a.part + (size_t)blockIdx.x * 2u * a.part_stride;
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                const unsigned i = first + k * C::kStep;
                if (C::has(left, k)) {
                    if constexpr (kVec) {
#pragma unroll
                        for (int e = 0; e < P; e += 2) {
                            *reinterpret_cast<float4*>(share + (size_t)i * E + 2 * e) = make_float4(dw[k][e].x, dw[k][e].y, dw[k][e + 1].x, dw[k][e + 1].y);
                            *reinterpret_cast<float4*>(share + a.part_stride + (size_t)i * E + 2 * e) =
                                make_float4(db[k][e].x, db[k][e].y, db[k][e + 1].x, db[k][e + 1].y);
                        }
                    } else {
                        share[i] = dw[k][0].x, share[a.part_stride + i] = db[k][0].x;
                        if (C::second(left, k)) share[i + 32u] = dw[k][0].y, share[a.part_stride + i + 32u] = db[k][0].y;
                    }
                }
            }
        }
    }
    pdl_trigger();
}

// Rows longer than a block's registers hold: the sums of kNormBatch of the block's rows first, then their dx column by column,
// with the columns' shares of dweight and dbias in registers from row to row; from batch to batch they are kept in the workspace.
// (One row after the other, with the shares in the workspace, 1000 x 16384 f32 takes 130 us against 80.6, 2000 x 12001 bf16 260 | 207.)
constexpr int kNormBatch = 16;
template <int DT, int PT, bool kVec>
__global__ void __launch_bounds__(1024) k_norm_backward_long(const Padded<NormGradArgs> a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    __shared__ float red[2][64];
    __shared__ float mean[kNormBatch], rstd[kNormBatch], sums[kNormBatch][2];
    pdl_begin(a.rows <= gridDim.x);
    const unsigned warps = blockDim.x / 32u;
    float* share = a.part ? a.part + (size_t)blockIdx.x * 2u * a.part_stride : nullptr;
    const unsigned long long step = gridDim.x;
    for (unsigned long long row0 = blockIdx.x; row0 < a.rows; row0 += step * kNormBatch) {
        const unsigned long long later = (a.rows - 1u - row0) / step + 1u;
        const int rows = later < kNormBatch ? (int)later : kNormBatch;
        for (int j = 0; j < rows; ++j) {
            const size_t row = row0 + j * step;
            const float m = a.mean[row], r = a.rstd[row];
            const void *px = row_at(a.x, row, a.x_stride), *pdy = row_at(a.dy, row, a.dy_stride);
            float c[2] = {0.0f, 0.0f};
#pragma unroll 4
            for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
                float x[E], dy[E], w[E];
                unpack<DT, kVec>(x, load_pack<DT, kVec>(px, i));
                unpack<DT, kVec>(dy, load_pack<DT, kVec>(pdy, i));
                unpack_params<PT, E>(w, load_params<PT, E>(a.weight, i, kOne<PT>));
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float gy = dy[e] * w[e];
                    c[0] += gy;
                    c[1] = fmaf(gy, (x[e] - m) * r, c[1]);
                }
            }
            group_sum<2>(c, warps, 0u, red[j & 1]);
            if (threadIdx.x == 0u) mean[j] = m, rstd[j] = r, sums[j][0] = c[0] * a.inverse, sums[j][1] = c[1] * a.inverse;
        }
        __syncthreads();
        for (unsigned i = threadIdx.x; i < a.units; i += blockDim.x) {
            float w[E], dw[E], db[E];
            unpack_params<PT, E>(w, load_params<PT, E>(a.weight, i, kOne<PT>));
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const size_t at = (size_t)i * E + e;
                const bool more = share && row0 != blockIdx.x;
                dw[e] = more ? share[at] : 0.0f, db[e] = more ? share[a.part_stride + at] : 0.0f;
            }
#pragma unroll 4
            for (int j = 0; j < rows; ++j) {
                const size_t row = row0 + j * step;
                float x[E], dy[E], s[E];
                unpack<DT, kVec>(x, load_pack<DT, kVec>(row_at(a.x, row, a.x_stride), i));
                unpack<DT, kVec>(dy, load_pack<DT, kVec>(row_at(a.dy, row, a.dy_stride), i));
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] = 0.0f;
                if (a.dsummed) unpack<DT, kVec>(s, load_pack<DT, kVec>(row_at(a.dsummed, row, a.dsummed_stride), i));
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xh = (x[e] - mean[j]) * rstd[j];
                    dw[e] = fmaf(dy[e], xh, dw[e]);
                    db[e] += dy[e];
                    s[e] = fmaf(rstd[j], fmaf(-xh, sums[j][1], fmaf(dy[e], w[e], -sums[j][0])), s[e]);
                }
                store_pack<DT, kVec>(row_at(a.dx, row, a.dx_stride), i, pack<DT, kVec>(s));
            }
            if (share)
#pragma unroll
                for (int e = 0; e < E; ++e) share[(size_t)i * E + e] = dw[e], share[a.part_stride + (size_t)i * E + e] = db[e];
        }
        __syncthreads();                                             // the sums are the next batch's
    }
    pdl_trigger();
}

// Adds up the blocks' shares: a block has 32 columns, whose shares its 32 slices of 8 threads take in turn, four columns a
// thread and all loads in flight, and adds the slices in order.
constexpr int kSlices = 32;
template <int PT>
__global__ void __launch_bounds__(8 * kSlices) k_norm_params(const float* part, void* dweight, void* dbias, unsigned shares, unsigned hidden,
                                                             unsigned part_stride, unsigned column_blocks, bool accumulate)
{
    constexpr int kEach = (int)(kNormBlocks + kSlices - 1) / kSlices;
    __shared__ float sum[kSlices][33];
    pdl_begin();
    const unsigned which = blockIdx.x / column_blocks, column = blockIdx.x % column_blocks * 32u, slice = threadIdx.x / 8u, at = threadIdx.x % 8u * 4u;
    void* out = which ? dbias : dweight;
    if (out == nullptr) return;
    float4 v[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const unsigned s = slice + k * kSlices;
        v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (s < shares && column + at < part_stride) v[k] = *reinterpret_cast<const float4*>(part + ((size_t)s * 2u + which) * part_stride + column + at);
    }
#pragma unroll
    for (int k = 1; k < kEach; ++k) v[0].x += v[k].x, v[0].y += v[k].y, v[0].z += v[k].z, v[0].w += v[k].w;
    sum[slice][at] = v[0].x, sum[slice][at + 1u] = v[0].y, sum[slice][at + 2u] = v[0].z, sum[slice][at + 3u] = v[0].w;
    __syncthreads();
    const unsigned mine = column + threadIdx.x;
    if (threadIdx.x < 32u && mine < hidden) {
        float f[1] = {0.0f};
#pragma unroll
        for (int s = 0; s < kSlices; ++s) f[0] += sum[s][threadIdx.x];
        if (accumulate) {
            float old[1];
            unpack<PT, false>(old, load_pack<PT, false>(out, mine));
            f[0] += old[0];
        }
        store_pack<PT, false>(out, mine, pack<PT, false>(f));
    }
    pdl_trigger();
}

// ---- host ------------------------------------------------------------------------------------------------

// Threads for a row of `packs` packs, kPacks each.
static unsigned group_for(size_t packs, int per_thread) { return (unsigned)std::max<size_t>(32, (packs + 32 * per_thread - 1) / (32 * per_thread) * 32); }

template <typename F>
static int with_param(int dtype, int param_dtype, F&& f)
{
    return with_dtype(dtype, [&](auto dt) {
        if (param_dtype == NUNA_F32) return f(dt, std::integral_constant<int, kF32>{});
        return f(dt, dt);
    });
}

template <int N> using Num = std::integral_constant<int, N>;

static int forward(const nuna_layernorm_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype), p = dtype_bytes(n.param_dtype);
    const auto bytes = [&](size_t stride) { return (stride ? stride : n.hidden) * e; };
    const bool vec = VectorRows{true}.rows(n.x, n.hidden, n.x_stride, e).rows(n.residual, n.hidden, n.residual_stride, e)
                         .rows(n.summed, n.hidden, n.summed_stride, e).rows(n.y, n.hidden, n.y_stride, e)
                         .rows(n.weight, n.hidden, 0, p).rows(n.bias, n.hidden, 0, p).ok;
    NormArgs a = {n.x, n.residual, n.weight, n.bias, n.summed, n.y, n.mean, n.rstd, bytes(n.x_stride), bytes(n.residual_stride),
                  bytes(n.summed_stride), bytes(n.y_stride), (unsigned)n.rows, (unsigned)n.hidden,
                  (unsigned)(vec ? n.hidden * e / 16 : n.hidden), 0, n.eps, (float)n.hidden, 1.0f / (float)n.hidden};
    return with_param(n.dtype, n.param_dtype, [&](auto dt, auto pt) {
        constexpr int DT = decltype(dt)::value, PT = decltype(pt)::value;
        // per_block: threads of a block (at least a group); per_sm: threads that an SM shall have
        const auto run = [&](auto per_thread, auto is_vec, unsigned per_block, unsigned per_sm) {
            constexpr int kPacks = decltype(per_thread)::value;
            constexpr bool kVec = decltype(is_vec)::value;
            a.group = group_for(a.units, kVec ? kPacks : 2 * kPacks);
            const unsigned groups = std::min(15u, std::max(1u, per_block / a.group)), threads = groups * a.group, blocks = (a.rows + groups - 1) / groups;
            const unsigned smem = RowFetch<DT, kPacks, kVec, 2, norm_depth(kPacks, kVec)>::kSlots * 16u * threads;
            const int ok = smem > 32 * 1024 ? allow_smem<k_norm_forward<DT, PT, kPacks, kVec>>(227 * 1024 - 1024) : NUNA_OK;
            if (ok != NUNA_OK) return ok;
            const unsigned resident = std::max(1u, std::min(per_sm / threads, 227u * 1024u / (smem + 2048u)));
            return launch_op(k_norm_forward<DT, PT, kPacks, kVec>, Shape{std::min(blocks, kSms * resident), threads, smem, 1}, flags, stream, a);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        // Few rows: 256 threads a row, of which fewer have more to add and more have more sums to exchange (1 x 8192 bf16 with
        // 1024 | 512 | 256 threads 3.15 | 3.01 | 2.84 us, 1 x 2048 with 256 | 128 | 64 1.95 | 2.27 | 2.64).
        // Many: four vectors a thread, so that a warp's part in the sums (40 instructions) is small beside its elements, and two
        // blocks, each of which works while the other one sums (4096 x 8192 bf16 without residual 25.0 us; two vectors a
        // thread in one block 37).  With a residual it is the four streams' traffic that bounds long rows, and fewer rows at a
        // time are ahead: one block with two vectors a thread, where its groups fill it.  Two | four vectors a thread, us for 256
        // MiB, groups that fill the block: bf16 3840 43.1 | 46.6, 4096 42.3 | 46.3, 8192 43.3 | 46.7, f32 4096 43.5 | 46.4, but f32 1920
        // and 2048 48.8 | 46.4; groups that do not: bf16 5120 54.6 | 46.8, 6144 47.6 | 44.6, 7168 46.2 | 46.6, 7680 44.6 | 46.7, f32 3584
        // 42.1 | 46.6; shorter rows: bf16 3584 44.5 | 47.0, 2048 44.9 | 46.1, 1024 55 | 46.4.  So the rule is right for the widths that it takes, but
        // for 1920 to 2048 binary32, and leaves up to a tenth at some that it does not.
        const bool few = a.rows <= 2 * kSms;
        if (vec && (a.units <= 32 || (few && a.units <= 256))) return run(Num<1>{}, Yes{}, 256, 1024);
        if (vec && few && a.units <= 512) return run(Num<2>{}, Yes{}, 256, 1024);
        if (vec && few && a.units <= 2048) return run(Num<4>{}, Yes{}, 256, 512);
        if (vec && a.residual && a.units >= 480 && a.units <= 1024 && 512u % group_for(a.units, 2) == 0u) return run(Num<2>{}, Yes{}, 512, 512);
        if (vec && a.units <= 64) return run(Num<2>{}, Yes{}, 256, 512);
        if (vec && a.units <= 2048) return run(Num<4>{}, Yes{}, 256, 512);
        // Pairs: eight a thread, as far as registers go; f16 four (8000 x 2731 bf16 45.8 us with eight against 56.8, f16 75 | 41.9:
        // the compiler takes half as many instructions again for its eight).
        constexpr int kLong = DT == kF16 ? 4 : 8;
        if (!vec && a.units <= 1024) return run(Num<4>{}, No{}, 256, 1024);
        if (!vec && a.units <= 8192) return run(Num<kLong>{}, No{}, 256, 4096 / kLong);
        return launch_op(vec ? k_norm_forward_long<DT, PT, true> : k_norm_forward_long<DT, PT, false>, Shape{std::min(a.rows, kSms * 2u), 1024, 0, 1}, flags, stream, a);
    });
}

static int backward(const nuna_layernorm_grad_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype), p = dtype_bytes(n.param_dtype);
    const auto bytes = [&](size_t stride) { return (stride ? stride : n.hidden) * e; };
    const bool vec = VectorRows{true}.rows(n.dy, n.hidden, n.dy_stride, e).rows(n.x, n.hidden, n.x_stride, e)
                         .rows(n.dsummed, n.hidden, n.dsummed_stride, e).rows(n.dx, n.hidden, n.dx_stride, e).rows(n.weight, n.hidden, 0, p).ok;
    const bool params = n.dweight || n.dbias;
    const bool accumulate = (flags & NUNA_GRAD_ACCUMULATE) != 0u;
    unsigned shares = 0;
    NormGradArgs a = {n.dy, n.x, n.weight, n.dsummed, n.mean, n.rstd, n.dx, params ? static_cast<float*>(n.workspace) : nullptr,
                      bytes(n.dy_stride), bytes(n.x_stride), bytes(n.dsummed_stride), bytes(n.dx_stride), (unsigned)n.rows, (unsigned)n.hidden,
                      (unsigned)(vec ? n.hidden * e / 16 : n.hidden), 0, (unsigned)((n.hidden + 3) / 4 * 4), (float)n.hidden, 1.0f / (float)n.hidden};
    int st = n.rows == 0 ? NUNA_OK : with_param(n.dtype, n.param_dtype, [&](auto dt, auto pt) {
        constexpr int DT = decltype(dt)::value, PT = decltype(pt)::value;
        const auto run = [&](auto per_thread, auto is_vec) {
            constexpr int kPacks = decltype(per_thread)::value;
            constexpr bool kVec = decltype(is_vec)::value;
            constexpr int E = Pack<DT, Cut<DT, kVec>::kForm>::kElems;
            a.group = group_for(a.units, kVec ? kPacks : 2 * kPacks);
            const unsigned groups = std::min(15u, std::max(1u, (unsigned)kNormGradThreads / a.group));
            shares = (unsigned)norm_blocks((a.rows + groups - 1) / groups);
            const unsigned threads = groups * a.group, shares_smem = params ? (groups - 1) * 2 * kPacks * a.group * E * 4 : 0;
            const unsigned smem = std::max(shares_smem, RowFetch<DT, kPacks, kVec, 3, norm_grad_depth(kPacks, kVec)>::kSlots * 16u * threads);
            if (smem > 32 * 1024) {
                const int ok = allow_smem<k_norm_backward<DT, PT, kPacks, kVec>>(227 * 1024 - 1024);
                if (ok != NUNA_OK) return ok;
            }
            return launch_op(k_norm_backward<DT, PT, kPacks, kVec>, Shape{shares, groups * a.group, smem, 1}, flags, stream, a);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        // Two vectors a thread: with four, xh and g have to be formed twice (4096 x 8192 bf16 73 us against 49.7).
        if (vec && a.units <= 32) return run(Num<1>{}, Yes{});
        if (vec && a.units <= 1024) return run(Num<2>{}, Yes{});
        if (vec && a.units <= 2048) return run(Num<4>{}, Yes{});
        if (!vec && a.units <= 4096) return run(Num<4>{}, No{});
        if (!vec && a.units <= 8192) return run(Num<8>{}, No{});
        shares = (unsigned)norm_blocks(a.rows);
        return launch_op(vec ? k_norm_backward_long<DT, PT, true> : k_norm_backward_long<DT, PT, false>, Shape{shares, 1024, 0, 1}, flags, stream, a);
    });
    if (st != NUNA_OK || !params || (accumulate && n.rows == 0)) return st;
    const unsigned column_blocks = (a.hidden + 31u) / 32u;
    return with_dtype(n.param_dtype, [&](auto pt) {
        return launch_kernel(k_norm_params<decltype(pt)::value>, Shape{2 * column_blocks, 8 * kSlices, 0, 1}, flags, stream, a.part, n.dweight, n.dbias, shares,
                         a.hidden, a.part_stride, column_blocks, accumulate);
    });
}

}  // namespace nuna

using namespace nuna;

extern "C" {

int nuna_layernorm_forward(const nuna_layernorm_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_layernorm_t a = *args;
    if (!is_dtype(a.dtype) || (a.param_dtype != a.dtype && a.param_dtype != NUNA_F32)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    if (!(a.eps >= 0.0f) || (a.residual == nullptr) != (a.summed == nullptr)) return NUNA_ERR_INVALID_ARG;
    const int st = check_spans(spans_of(a), 1, 4);                   // summed may be the residual
    if (st != NUNA_OK || a.rows == 0 || a.hidden == 0) return st;
    return forward(a, effective_flags(flags, stream), stream);
}

int nuna_layernorm_backward(const nuna_layernorm_grad_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~(NUNA_LAUNCH_PDL | NUNA_GRAD_ACCUMULATE))) return NUNA_ERR_INVALID_ARG;
    const nuna_layernorm_grad_t a = *args;
    if (!is_dtype(a.dtype) || (a.param_dtype != a.dtype && a.param_dtype != NUNA_F32)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    const int st = check_spans(spans_of(a), 5, 6);                   // dx may be dsummed
    if (st != NUNA_OK || a.hidden == 0) return st;
    const size_t need = layernorm_workspace_bytes(a.rows, a.hidden);
    if ((a.dweight || a.dbias) && need && (!a.workspace || a.workspace_bytes < need)) return NUNA_ERR_INVALID_ARG;
    if (a.rows == 0 && !a.dweight && !a.dbias) return NUNA_OK;
    return backward(a, effective_flags(flags, stream), stream);
}

size_t nuna_layernorm_workspace(size_t rows, size_t hidden) { return layernorm_workspace_bytes(rows, hidden); }

}  // extern "C"
