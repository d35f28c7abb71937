// Layer norm of the rows that an allreduce has summed, with the residual added, and its gradient.
//
// A row is held by a group of threads, each with up to kPacks 16-byte vectors (or single elements where rows are not
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
    unsigned rows, hidden, packs, group;                             // packs in a row, threads of a group
    float eps, count;                                                // count: hidden
};

struct NormGradArgs {
    const void *dy, *x, *weight, *dsummed;
    const float *mean, *rstd;
    void* dx;
    float* part;                                                     // [gridDim.x][2][part_stride], or null
    size_t dy_stride, x_stride, dsummed_stride, dx_stride;           // bytes
    unsigned rows, hidden, packs, group, part_stride;
    float count;                                                     // hidden
};

// Sums v over the `warps` warps of this thread's group, for every group of the block at once (all threads call).  Two
// consecutive calls use different halves of `red`, [2][32][N]: the exchange of the second separates the uses of the first.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], unsigned warps, float* red)
{
    warp_sum<N>(v);
    if (warps == 1u) return;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, first = warp / warps * warps;
    if (lane == 0u)
#pragma unroll
        for (int i = 0; i < N; ++i) red[warp * N + i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lane < warps ? red[(first + lane) * N + i] : 0.0f;
    warp_sum<N>(v);
}

template <int DT, int PT, int kPacks, bool kVec>
__global__ void __launch_bounds__(1024) k_norm_forward(const NormArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    __shared__ float red[2][32];
    pdl_wait();
    const unsigned warps = a.group / 32u, g = threadIdx.x / a.group, lane = threadIdx.x % a.group, groups = blockDim.x / a.group;
    unsigned turn = 0;
    for (unsigned long long base = (unsigned long long)blockIdx.x * groups; base < a.rows; base += (unsigned long long)gridDim.x * groups) {
        const size_t row = base + g;
        const bool live = row < a.rows;
        float f[kPacks][E];
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = lane + k * a.group;
#pragma unroll
            for (int e = 0; e < E; ++e) f[k][e] = 0.0f;
            if (live && i < a.packs) {
                unpack<DT, kVec>(f[k], load_pack<DT, kVec>(row_at(a.x, row, a.x_stride), i));
                if (a.residual) {
                    float r[E];
                    unpack<DT, kVec>(r, load_pack<DT, kVec>(row_at(a.residual, row, a.residual_stride), i));
#pragma unroll
                    for (int e = 0; e < E; ++e) f[k][e] = __fadd_rn(f[k][e], r[e]);
                    const Pack<DT, kVec> s = pack<DT, kVec>(f[k]);
                    store_pack<DT, kVec>(row_at(a.summed, row, a.summed_stride), i, s);
                    unpack<DT, kVec>(f[k], s);                       // the norm is that of the stored row
                }
            }
        }
        float sum[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[0] += f[k][e];
        group_sum<1>(sum, warps, red[turn]);
        turn ^= 1u;
        const float mean = sum[0] / a.count;
        float sq[1] = {0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
            if (lane + k * a.group < a.packs)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float d = f[k][e] - mean;
                    sq[0] = fmaf(d, d, sq[0]);
                }
        group_sum<1>(sq, warps, red[turn]);
        turn ^= 1u;
        const float rstd = 1.0f / sqrtf(sq[0] / a.count + a.eps);
        if (live && lane == 0u) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = lane + k * a.group;
            if (live && i < a.packs) {
                float w[E], b[E];
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = 1.0f, b[e] = 0.0f;
                if (a.weight) load_params<PT, E>(w, a.weight, i);
                if (a.bias) load_params<PT, E>(b, a.bias, i);
#pragma unroll
                for (int e = 0; e < E; ++e) f[k][e] = fmaf((f[k][e] - mean) * rstd, w[e], b[e]);
                store_pack<DT, kVec>(row_at(a.y, row, a.y_stride), i, pack<DT, kVec>(f[k]));
            }
        }
    }
    pdl_trigger();
}

// Rows longer than a block's registers hold: one block per row, which reads the row again for each of the three steps.
template <int DT, int PT>
__global__ void __launch_bounds__(1024) k_norm_forward_long(const NormArgs a)
{
    __shared__ float red[2][32];
    pdl_wait();
    const unsigned warps = blockDim.x / 32u;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const void* x = row_at(a.x, row, a.x_stride);
        float sum[1] = {0.0f};
        for (unsigned i = threadIdx.x; i < a.hidden; i += blockDim.x) {
            float f[1];
            unpack<DT, false>(f, load_pack<DT, false>(x, i));
            if (a.residual) {
                float r[1];
                unpack<DT, false>(r, load_pack<DT, false>(row_at(a.residual, row, a.residual_stride), i));
                f[0] = __fadd_rn(f[0], r[0]);
                const Pack<DT, false> s = pack<DT, false>(f);
                store_pack<DT, false>(row_at(a.summed, row, a.summed_stride), i, s);
                unpack<DT, false>(f, s);
            }
            sum[0] += f[0];
        }
        const void* s = a.residual ? row_at(a.summed, row, a.summed_stride) : x;         // this thread's own stores
        group_sum<1>(sum, warps, red[0]);
        const float mean = sum[0] / a.count;
        float sq[1] = {0.0f};
        for (unsigned i = threadIdx.x; i < a.hidden; i += blockDim.x) {
            float f[1];
            unpack<DT, false>(f, load_pack<DT, false>(s, i));
            sq[0] = fmaf(f[0] - mean, f[0] - mean, sq[0]);
        }
        group_sum<1>(sq, warps, red[1]);
        const float rstd = 1.0f / sqrtf(sq[0] / a.count + a.eps);
        if (threadIdx.x == 0u) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (unsigned i = threadIdx.x; i < a.hidden; i += blockDim.x) {
            float f[1], w[1] = {1.0f}, b[1] = {0.0f};
            unpack<DT, false>(f, load_pack<DT, false>(s, i));
            if (a.weight) load_params<PT, 1>(w, a.weight, i);
            if (a.bias) load_params<PT, 1>(b, a.bias, i);
            f[0] = fmaf((f[0] - mean) * rstd, w[0], b[0]);
            store_pack<DT, false>(row_at(a.y, row, a.y_stride), i, pack<DT, false>(f));
        }
    }
    pdl_trigger();
}

// ---- gradient ------------------------------------------------------------------------------------------
//
// A block's groups take rows in turn and keep their columns' shares of dweight and dbias in registers from row to row;
// at the end the block's groups are added and the block's share goes to the workspace, whose at most 148 rows
// k_norm_params adds up.  Which rows a group takes depends on sizes and types alone, and so do the sums' orders.
template <int DT, int PT, int kPacks, bool kVec>
__global__ void __launch_bounds__(512, 1) k_norm_backward(const NormGradArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    __shared__ float red[2][64];
    extern __shared__ float joined[];                                // [groups - 1][2][kPacks * group * E], if groups > 1
    pdl_wait();
    const unsigned warps = a.group / 32u, g = threadIdx.x / a.group, lane = threadIdx.x % a.group, groups = blockDim.x / a.group;
    float dw[kPacks][E], db[kPacks][E];
#pragma unroll
    for (int k = 0; k < kPacks; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) dw[k][e] = db[k][e] = 0.0f;
    unsigned turn = 0;
    for (unsigned long long base = (unsigned long long)blockIdx.x * groups; base < a.rows; base += (unsigned long long)gridDim.x * groups) {
        const size_t row = base + g;
        const bool live = row < a.rows;
        const float mean = live ? a.mean[row] : 0.0f, rstd = live ? a.rstd[row] : 0.0f;
        Pack<DT, kVec> px[kPacks], pdy[kPacks];
        float c[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = lane + k * a.group;
            if (live && i < a.packs) {
                px[k] = load_pack<DT, kVec>(row_at(a.x, row, a.x_stride), i);
                pdy[k] = load_pack<DT, kVec>(row_at(a.dy, row, a.dy_stride), i);
            }
        }
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = lane + k * a.group;
            if (live && i < a.packs) {
                float x[E], dy[E], w[E];
                unpack<DT, kVec>(x, px[k]);
                unpack<DT, kVec>(dy, pdy[k]);
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = 1.0f;
                if (a.weight) load_params<PT, E>(w, a.weight, i);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xh = (x[e] - mean) * rstd, gy = dy[e] * w[e];
                    c[0] += gy;
                    c[1] = fmaf(gy, xh, c[1]);
                    dw[k][e] = fmaf(dy[e], xh, dw[k][e]);
                    db[k][e] += dy[e];
                }
            }
        }
        group_sum<2>(c, warps, red[turn]);
        turn ^= 1u;
        const float c0 = c[0] / a.count, c1 = c[1] / a.count;
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = lane + k * a.group;
            if (live && i < a.packs) {
                float x[E], dy[E], w[E], r[E];
                unpack<DT, kVec>(x, px[k]);
                unpack<DT, kVec>(dy, pdy[k]);
#pragma unroll
                for (int e = 0; e < E; ++e) w[e] = 1.0f, r[e] = 0.0f;
                if (a.weight) load_params<PT, E>(w, a.weight, i);
                if (a.dsummed) unpack<DT, kVec>(r, load_pack<DT, kVec>(row_at(a.dsummed, row, a.dsummed_stride), i));
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float xh = (x[e] - mean) * rstd;
                    r[e] = fmaf(rstd, fmaf(dy[e], w[e], -c0) - xh * c1, r[e]);
                }
                store_pack<DT, kVec>(row_at(a.dx, row, a.dx_stride), i, pack<DT, kVec>(r));
            }
        }
    }
    if (a.part) {
        const unsigned half = kPacks * a.group * E;
        if (g > 0u) {
            float* to = joined + (size_t)(g - 1u) * 2u * half;
#pragma unroll
            for (int k = 0; k < kPacks; ++k)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    to[(k * E + e) * a.group + lane] = dw[k][e];
                    to[half + (k * E + e) * a.group + lane] = db[k][e];
                }
        }
        __syncthreads();
        if (g == 0u) {
            for (unsigned o = 0; o + 1u < groups; ++o) {
                const float* from = joined + (size_t)o * 2u * half;
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        dw[k][e] += from[(k * E + e) * a.group + lane];
                        db[k][e] += from[half + (k * E + e) * a.group + lane];
                    }
            }
            float* share = a.part + (size_t)blockIdx.x * 2u * a.part_stride;
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                const unsigned i = lane + k * a.group;
                if (i < a.packs) {
                    if constexpr (E % 4 == 0) {
#pragma unroll
                        for (int e = 0; e < E; e += 4) {
                            *reinterpret_cast<float4*>(share + (size_t)i * E + e) = make_float4(dw[k][e], dw[k][e + 1], dw[k][e + 2], dw[k][e + 3]);
                            *reinterpret_cast<float4*>(share + a.part_stride + (size_t)i * E + e) =
                                make_float4(db[k][e], db[k][e + 1], db[k][e + 2], db[k][e + 3]);
                        }
                    } else {
                        share[i] = dw[k][0];
                        share[a.part_stride + i] = db[k][0];
                    }
                }
            }
        }
    }
    pdl_trigger();
}

// Rows longer than a block's registers hold; the block's shares are kept in the workspace from row to row.
template <int DT, int PT>
__global__ void __launch_bounds__(1024) k_norm_backward_long(const NormGradArgs a)
{
    __shared__ float red[2][64];
    pdl_wait();
    const unsigned warps = blockDim.x / 32u;
    float* share = a.part ? a.part + (size_t)blockIdx.x * 2u * a.part_stride : nullptr;
    unsigned turn = 0;
    bool first = true;
    for (size_t row = blockIdx.x; row < a.rows; row += gridDim.x, first = false) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        const void *px = row_at(a.x, row, a.x_stride), *pdy = row_at(a.dy, row, a.dy_stride);
        float c[2] = {0.0f, 0.0f};
        for (unsigned i = threadIdx.x; i < a.hidden; i += blockDim.x) {
            float x[1], dy[1], w[1] = {1.0f};
            unpack<DT, false>(x, load_pack<DT, false>(px, i));
            unpack<DT, false>(dy, load_pack<DT, false>(pdy, i));
            if (a.weight) load_params<PT, 1>(w, a.weight, i);
            const float xh = (x[0] - mean) * rstd, gy = dy[0] * w[0];
            c[0] += gy;
            c[1] = fmaf(gy, xh, c[1]);
            if (share) {
                share[i] = fmaf(dy[0], xh, first ? 0.0f : share[i]);
                share[a.part_stride + i] = (first ? 0.0f : share[a.part_stride + i]) + dy[0];
            }
        }
        group_sum<2>(c, warps, red[turn]);
        turn ^= 1u;
        const float c0 = c[0] / a.count, c1 = c[1] / a.count;
        for (unsigned i = threadIdx.x; i < a.hidden; i += blockDim.x) {
            float x[1], dy[1], w[1] = {1.0f}, r[1] = {0.0f};
            unpack<DT, false>(x, load_pack<DT, false>(px, i));
            unpack<DT, false>(dy, load_pack<DT, false>(pdy, i));
            if (a.weight) load_params<PT, 1>(w, a.weight, i);
            if (a.dsummed) unpack<DT, false>(r, load_pack<DT, false>(row_at(a.dsummed, row, a.dsummed_stride), i));
            r[0] = fmaf(rstd, fmaf(dy[0], w[0], -c0) - (x[0] - mean) * rstd * c1, r[0]);
            store_pack<DT, false>(row_at(a.dx, row, a.dx_stride), i, pack<DT, false>(r));
        }
    }
    pdl_trigger();
}

// Adds up the blocks' shares: 32 columns a block, whose 16 warps take the shares in turn and are then added in order.
template <int PT>
__global__ void __launch_bounds__(512) k_norm_params(const float* part, void* dweight, void* dbias, unsigned shares, unsigned hidden,
                                                     unsigned part_stride, unsigned column_blocks, bool accumulate)
{
    __shared__ float sum[16][33];
    pdl_wait();
    const unsigned which = blockIdx.x / column_blocks, column = blockIdx.x % column_blocks * 32u + (threadIdx.x & 31u), slice = threadIdx.x >> 5;
    void* out = which ? dbias : dweight;
    float acc = 0.0f;
    if (out && column < hidden) {
#pragma unroll 4
        for (unsigned s = slice; s < shares; s += 16u) acc += part[((size_t)s * 2u + which) * part_stride + column];
    }
    sum[slice][threadIdx.x & 31u] = acc;
    __syncthreads();
    if (slice == 0u && out && column < hidden) {
#pragma unroll
        for (int s = 1; s < 16; ++s) acc += sum[s][threadIdx.x];
        float f[1] = {acc};
        if (accumulate) {
            float old[1];
            unpack<PT, false>(old, load_pack<PT, false>(out, column));
            f[0] += old[0];
        }
        store_pack<PT, false>(out, column, pack<PT, false>(f));
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
                  (unsigned)(vec ? n.hidden * e / 16 : n.hidden), 0, n.eps, (float)n.hidden};
    return with_param(n.dtype, n.param_dtype, [&](auto dt, auto pt) {
        constexpr int DT = decltype(dt)::value, PT = decltype(pt)::value;
        const auto run = [&](auto kernel, int per_thread) {
            a.group = group_for(a.packs, per_thread);
            const unsigned groups = std::max(1u, 256u / a.group);
            return launch_op(kernel, Shape{(a.rows + groups - 1) / groups, groups * a.group, 0, 1}, flags, stream, a);
        };
        if (vec && a.packs <= 128) return run(k_norm_forward<DT, PT, 1, true>, 1);
        if (vec && a.packs <= 4096) return run(k_norm_forward<DT, PT, 4, true>, 4);
        if (!vec && a.packs <= 1024) return run(k_norm_forward<DT, PT, 4, false>, 4);
        if (!vec && a.packs <= 16384) return run(k_norm_forward<DT, PT, 16, false>, 16);
        return launch_op(k_norm_forward_long<DT, PT>, Shape{std::min(a.rows, kSms * 2u), 1024, 0, 1}, flags, stream, a);
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
                      (unsigned)(vec ? n.hidden * e / 16 : n.hidden), 0, (unsigned)((n.hidden + 3) / 4 * 4), (float)n.hidden};
    int st = n.rows == 0 ? NUNA_OK : with_param(n.dtype, n.param_dtype, [&](auto dt, auto pt) {
        constexpr int DT = decltype(dt)::value, PT = decltype(pt)::value;
        const auto run = [&](auto per_thread, auto is_vec) {
            constexpr int kPacks = decltype(per_thread)::value;
            constexpr bool kVec = decltype(is_vec)::value;
            constexpr int E = Pack<DT, kVec>::kElems;
            a.group = group_for(a.packs, kPacks);
            const unsigned groups = std::max(1u, 512u / a.group);
            shares = (unsigned)norm_blocks((a.rows + groups - 1) / groups);
            const unsigned smem = params ? (groups - 1) * 2 * kPacks * a.group * E * 4 : 0;
            if (smem > 32 * 1024) {
                const int ok = allow_smem<k_norm_backward<DT, PT, kPacks, kVec>>(227 * 1024 - 1024);
                if (ok != NUNA_OK) return ok;
            }
            return launch_op(k_norm_backward<DT, PT, kPacks, kVec>, Shape{shares, groups * a.group, smem, 1}, flags, stream, a);
        };
        using Yes = std::true_type;
        using No = std::false_type;
        if (vec && a.packs <= 512) return run(Num<1>{}, Yes{});
        if (vec && a.packs <= 1024) return run(Num<2>{}, Yes{});
        if (vec && a.packs <= 2048) return run(Num<4>{}, Yes{});
        if (!vec && a.packs <= 1024) return run(Num<2>{}, No{});
        if (!vec && a.packs <= 8192) return run(Num<16>{}, No{});
        shares = (unsigned)norm_blocks(a.rows);
        return launch_op(k_norm_backward_long<DT, PT>, Shape{shares, 1024, 0, 1}, flags, stream, a);
    });
    if (st != NUNA_OK || !params || (accumulate && n.rows == 0)) return st;
    const unsigned column_blocks = (a.hidden + 31u) / 32u;
    return with_dtype(n.param_dtype, [&](auto pt) {
        return launch_op(k_norm_params<decltype(pt)::value>, Shape{2 * column_blocks, 512, 0, 1}, flags, stream, a.part, n.dweight, n.dbias, shares,
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
