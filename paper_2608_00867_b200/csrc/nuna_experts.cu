// Tokens sorted by expert, for the alltoall that carries them, and back with the router's weights.
//
// The sort is one pass of the cluster's counting sort (nuna_sort.cuh), the digit being the expert.  The row movers work token
// by token: dispatch reads a token's row once and writes it to all of its experts' rows, combine has the rows of all of a
// token's experts in flight and adds them in registers, and the gradient of the combine reads the token's gradient once for all
// of its rows.  What bounds them is the memory; for a few tokens, the dependent reads of map and row.
#include "nuna_sort.cuh"

#include <algorithm>

namespace nuna {

struct ExpertSortArgs {
    const void* experts;
    int *row_of_pair, *pair_of_row, *offsets, *counts;
    long long first_expert;
    unsigned pairs, num_experts, capacity, rows;
    bool wide;
};

__global__ void __launch_bounds__(1024) k_expert_sort(const ExpertSortArgs a)
{
    extern __shared__ unsigned smem[];
    pdl_wait();
    unsigned* counts = smem;                                         // [num_experts]
    const unsigned threads = gridDim.x * blockDim.x, thread = blockIdx.x * blockDim.x + threadIdx.x;
    const unsigned kept = sort_pass(a.pairs, a.num_experts, smem + a.num_experts, counts,
        [&](unsigned i) {
            const long long e = a.wide ? static_cast<const volatile long long*>(a.experts)[i]
                                       : (long long)static_cast<const volatile int*>(a.experts)[i];
            if (e < a.first_expert || (unsigned long long)e - (unsigned long long)a.first_expert >= a.num_experts) return kNoDigit;
            return (unsigned)(e - a.first_expert);
        },
        [&](unsigned i, unsigned d, unsigned first, unsigned rank) {
            int row = -1;
            if (d != kNoDigit) {
                if (a.capacity == 0u) row = (int)(first + rank);
                else if (rank < a.capacity) row = (int)(d * a.capacity + rank);
            }
            a.row_of_pair[i] = row;
            if (row >= 0) a.pair_of_row[row] = (int)i;
        });
    if (a.capacity == 0u) {
        for (unsigned r = kept + thread; r < a.rows; r += threads) a.pair_of_row[r] = -1;
    } else {
        for (unsigned r = thread; r < a.rows; r += threads)
            if (r % a.capacity >= counts[r / a.capacity]) a.pair_of_row[r] = -1;
    }
    if (blockIdx.x == 0u) {
        unsigned* first = smem + a.num_experts + (blockDim.x / 32u + 1u) * a.num_experts;        // sort_pass's first places
        for (unsigned e = threadIdx.x; e < a.num_experts; e += blockDim.x) {
            a.offsets[e] = (int)(a.capacity ? e * a.capacity : first[e]);
            if (a.counts) a.counts[e] = (int)counts[e];
        }
        if (threadIdx.x == 0u) a.offsets[a.num_experts] = (int)(a.capacity ? a.rows : kept);
    }
    pdl_trigger();
}

// ---- rows -----------------------------------------------------------------------------------------------

struct MoveArgs {
    const void *x, *src;                                             // token rows (read), expert rows (read)
    const int *row_of_pair, *pair_of_row;
    const float* weights;
    void *y, *out;                                                   // token rows (written), expert rows (written)
    float* dweights;
    size_t x_stride, src_stride, y_stride, out_stride;               // bytes
    unsigned long long token_units, row_units;                       // tokens * chunks, rows * chunks (if empty rows are zeroed)
    unsigned topk, rows, packs, chunks, group;                       // packs in a row, chunks of a row, threads of a chunk
};

// Zeroes the chunk of an expert row that no pair has.
template <int DT, int kPacks, bool kVec>
__device__ __forceinline__ void zero_empty_row(const MoveArgs& a, unsigned long long unit, unsigned lane)
{
    const size_t row = unit / a.chunks;
    if (a.pair_of_row[row] >= 0) return;
    const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
    Pack<DT, kVec> zero;
#pragma unroll
    for (int w = 0; w < Pack<DT, kVec>::kWords; ++w) zero.w[w] = 0u;
#pragma unroll
    for (int k = 0; k < kPacks; ++k)
        if (from + k * a.group < a.packs) store_pack<DT, kVec, true>(row_at(a.out, row, a.out_stride), from + k * a.group, zero);
}

template <int DT, int kPacks, bool kVec>
__global__ void __launch_bounds__(256) k_expert_dispatch(const MoveArgs a)
{
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
    if (unit < a.token_units) {
        const size_t token = unit / a.chunks;
        const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
        Pack<DT, kVec> p[kPacks];
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
            if (from + k * a.group < a.packs) p[k] = load_pack<DT, kVec>(row_at(a.x, token, a.x_stride), from + k * a.group);
        for (unsigned j = 0; j < a.topk; ++j) {
            const unsigned row = (unsigned)a.row_of_pair[token * a.topk + j];
            if (row >= a.rows) continue;
            void* out = row_at(a.out, row, a.out_stride);
#pragma unroll
            for (int k = 0; k < kPacks; ++k)
                if (from + k * a.group < a.packs) store_pack<DT, kVec, true>(out, from + k * a.group, p[k]);
        }
    } else if (unit - a.token_units < a.row_units) {
        zero_empty_row<DT, kPacks, kVec>(a, unit - a.token_units, lane);
    }
    pdl_trigger();
}

template <int DT, int kPacks, bool kVec>
__global__ void __launch_bounds__(256) k_expert_combine(const MoveArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    constexpr int kAhead = 4;                                        // expert rows in flight
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
    if (unit < a.token_units) {
        const size_t token = unit / a.chunks;
        const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
        float acc[kPacks][E];
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[k][e] = 0.0f;
        for (unsigned j0 = 0; j0 < a.topk; j0 += kAhead) {
            unsigned row[kAhead];
            Pack<DT, kVec> v[kAhead][kPacks];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) row[j] = j0 + j < a.topk ? (unsigned)a.row_of_pair[token * a.topk + j0 + j] : 0xFFFFFFFFu;
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (row[j] < a.rows)
#pragma unroll
                    for (int k = 0; k < kPacks; ++k)
                        if (from + k * a.group < a.packs) v[j][k] = load_pack<DT, kVec>(row_at(a.src, row[j], a.src_stride), from + k * a.group);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (row[j] < a.rows) {
                    const float w = a.weights ? a.weights[token * a.topk + j0 + j] : 1.0f;
#pragma unroll
                    for (int k = 0; k < kPacks; ++k)
                        if (from + k * a.group < a.packs) {
                            float f[E];
                            unpack<DT, kVec>(f, v[j][k]);
#pragma unroll
                            for (int e = 0; e < E; ++e) acc[k][e] = fmaf(w, f[e], acc[k][e]);
                        }
                }
        }
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
            if (from + k * a.group < a.packs) store_pack<DT, kVec>(row_at(a.y, token, a.y_stride), from + k * a.group, pack<DT, kVec>(acc[k]));
    }
    pdl_trigger();
}

// A token per group of threads, which goes over the row kPacks packs a thread at a time; kBatch pairs' products are summed
// together, and over the group at the end of the row.
template <int DT, int kPacks, bool kVec>
__global__ void __launch_bounds__(256) k_expert_combine_backward(const MoveArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    constexpr int kBatch = 4;
    __shared__ float red[8][kBatch];
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group, warps = a.group / 32u;
    const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
    const unsigned long long first = (unsigned long long)blockIdx.x * groups;
    const size_t token = unit;
    const bool live = unit < a.token_units;
    if (first < a.token_units) {                                     // the whole block: the sums exchange through shared memory
        for (unsigned j0 = 0; j0 < a.topk; j0 += kBatch) {
            unsigned row[kBatch];
            float w[kBatch], dot[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const bool is = live && j0 + j < a.topk;
                row[j] = is ? (unsigned)a.row_of_pair[token * a.topk + j0 + j] : 0xFFFFFFFFu;
                w[j] = is && row[j] < a.rows ? a.weights[token * a.topk + j0 + j] : 0.0f;
                dot[j] = 0.0f;
            }
            for (unsigned base = lane; base < a.packs; base += a.group * kPacks) {
                Pack<DT, kVec> dy[kPacks], v[kBatch][kPacks];
                if (live)
#pragma unroll
                    for (int k = 0; k < kPacks; ++k)
                        if (base + k * a.group < a.packs) dy[k] = load_pack<DT, kVec>(row_at(a.x, token, a.x_stride), base + k * a.group);
                if (a.dweights)
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (row[j] < a.rows)
#pragma unroll
                            for (int k = 0; k < kPacks; ++k)
                                if (base + k * a.group < a.packs)
                                    v[j][k] = load_pack<DT, kVec>(row_at(a.src, row[j], a.src_stride), base + k * a.group);
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (live && base + k * a.group < a.packs) {
                        float g[E];
                        unpack<DT, kVec>(g, dy[k]);
#pragma unroll
                        for (int j = 0; j < kBatch; ++j)
                            if (row[j] < a.rows) {
                                float f[E];
                                if (a.dweights) {
                                    unpack<DT, kVec>(f, v[j][k]);
#pragma unroll
                                    for (int e = 0; e < E; ++e) dot[j] = fmaf(g[e], f[e], dot[j]);
                                }
#pragma unroll
                                for (int e = 0; e < E; ++e) f[e] = w[j] * g[e];
                                store_pack<DT, kVec, true>(row_at(a.out, row[j], a.out_stride), base + k * a.group, pack<DT, kVec>(f));
                            }
                    }
            }
            if (a.dweights) {
                warp_sum<kBatch>(dot);
                if (warps > 1u) {
                    const unsigned warp = threadIdx.x >> 5;
                    __syncthreads();                                 // the last batch's sums have been read
                    if ((threadIdx.x & 31u) == 0u)
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) red[warp][j] = dot[j];
                    __syncthreads();
                    if (lane < kBatch) {
                        float s = 0.0f;
                        for (unsigned o = 0; o < warps; ++o) s += red[warp + o][lane];
                        if (live && j0 + lane < a.topk) a.dweights[token * a.topk + j0 + lane] = s;
                    }
                } else if (live && lane == 0u) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (j0 + j < a.topk) a.dweights[token * a.topk + j0 + j] = dot[j];
                }
            }
        }
    }
    if (!live) {
        // the groups that have no token zero the rows that have no pair, a chunk at a time
        const unsigned long long z = unit - a.token_units;
        if (z < a.row_units) zero_empty_row<DT, kPacks, kVec>(a, z, lane);
    }
    pdl_trigger();
}

// ---- host ------------------------------------------------------------------------------------------------

// Threads (at most 256) and chunks for a row of `packs` packs, kPacks a thread.
static void row_shape(MoveArgs& a, int per_thread)
{
    const unsigned threads = (a.packs + per_thread - 1) / per_thread;
    a.group = std::max(32u, std::min(256u, (threads + 31u) / 32u * 32u));
    a.chunks = std::max(1u, (threads + a.group - 1) / a.group);
}

static size_t stride_bytes(size_t stride, size_t hidden, int dtype) { return (stride ? stride : hidden) * dtype_bytes(dtype); }

// Launches a row mover: `whole` says that a group takes a token's row whole, not a chunk of it.
template <typename Kernel>
static int move_rows(Kernel kernel, MoveArgs& a, size_t tokens, int per_thread, bool whole, unsigned flags, void* stream)
{
    row_shape(a, per_thread);
    a.token_units = (unsigned long long)tokens * (whole ? 1u : a.chunks);
    a.row_units = a.pair_of_row ? (unsigned long long)a.rows * a.chunks : 0u;
    const unsigned groups = 256u / a.group;
    const unsigned long long grid = (a.token_units + a.row_units + groups - 1) / groups;
    if (grid > kMaxExtent) return NUNA_ERR_TOO_LARGE;
    if (grid == 0) return NUNA_OK;
    return launch_op(kernel, Shape{(unsigned)grid, groups * a.group, 0, 1}, flags, stream, a);
}

static int dispatch(const nuna_expert_dispatch_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.x, n.hidden, n.x_stride, e).rows(n.out, n.hidden, n.out_stride, e).ok;
    MoveArgs a = {};
    a.x = n.x, a.row_of_pair = n.row_of_pair, a.pair_of_row = n.pair_of_row, a.out = n.out;
    a.x_stride = stride_bytes(n.x_stride, n.hidden, n.dtype), a.out_stride = stride_bytes(n.out_stride, n.hidden, n.dtype);
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = (unsigned)(vec ? n.hidden * e / 16 : n.hidden);
    const size_t tokens = n.topk ? n.tokens : 0;
    if (vec) {                                                       // bits are copied: a vector is a vector
        return (unsigned long long)tokens * a.packs <= 4ull * kSms * 512ull
                   ? move_rows(k_expert_dispatch<kF32, 1, true>, a, tokens, 1, false, flags, stream)
                   : move_rows(k_expert_dispatch<kF32, 4, true>, a, tokens, 4, false, flags, stream);
    }
    if (n.dtype == NUNA_F32) return move_rows(k_expert_dispatch<kF32, 4, false>, a, tokens, 4, false, flags, stream);
    return move_rows(k_expert_dispatch<kBf16, 4, false>, a, tokens, 4, false, flags, stream);
}

static int combine(const nuna_expert_combine_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.src, n.hidden, n.src_stride, e).rows(n.y, n.hidden, n.y_stride, e).ok;
    MoveArgs a = {};
    a.src = n.src, a.row_of_pair = n.row_of_pair, a.weights = n.weights, a.y = n.y;
    a.src_stride = stride_bytes(n.src_stride, n.hidden, n.dtype), a.y_stride = stride_bytes(n.y_stride, n.hidden, n.dtype);
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = (unsigned)(vec ? n.hidden * e / 16 : n.hidden);
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!vec) return move_rows(k_expert_combine<DT, 4, false>, a, n.tokens, 4, false, flags, stream);
        return (unsigned long long)n.tokens * a.packs <= 2ull * kSms * 512ull
                   ? move_rows(k_expert_combine<DT, 1, true>, a, n.tokens, 1, false, flags, stream)
                   : move_rows(k_expert_combine<DT, 2, true>, a, n.tokens, 2, false, flags, stream);
    });
}

static int combine_backward(const nuna_expert_combine_grad_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.dy, n.hidden, n.dy_stride, e).rows(n.dweights ? n.src : nullptr, n.hidden, n.src_stride, e)
                         .rows(n.dsrc, n.hidden, n.dsrc_stride, e).ok;
    MoveArgs a = {};
    a.x = n.dy, a.src = n.src, a.weights = n.weights, a.row_of_pair = n.row_of_pair, a.pair_of_row = n.pair_of_row;
    a.out = n.dsrc, a.dweights = n.dweights;
    a.x_stride = stride_bytes(n.dy_stride, n.hidden, n.dtype), a.src_stride = stride_bytes(n.src_stride, n.hidden, n.dtype);
    a.out_stride = stride_bytes(n.dsrc_stride, n.hidden, n.dtype);
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = (unsigned)(vec ? n.hidden * e / 16 : n.hidden);
    const size_t tokens = n.topk ? n.tokens : 0;
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!vec) return move_rows(k_expert_combine_backward<DT, 4, false>, a, tokens, 4, true, flags, stream);
        return move_rows(k_expert_combine_backward<DT, 2, true>, a, tokens, 2, true, flags, stream);
    });
}

}  // namespace nuna

using namespace nuna;

extern "C" {

int nuna_expert_sort(const nuna_expert_sort_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_expert_sort_t a = *args;
    if ((a.id_bytes != 4 && a.id_bytes != 8) || a.num_experts < 1 || a.first_expert < 0) return NUNA_ERR_INVALID_ARG;
    if (a.num_experts > NUNA_MAX_EXPERTS) return NUNA_ERR_TOO_LARGE;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK) return st;
    const size_t pairs = a.tokens * a.topk, rows = a.capacity ? a.num_experts * a.capacity : pairs;
    const ExpertSortArgs k = {a.experts, a.row_of_pair, a.pair_of_row, a.offsets, a.counts, a.first_expert, (unsigned)pairs,
                              (unsigned)a.num_experts, (unsigned)a.capacity, (unsigned)rows, a.id_bytes == 8};
    Shape s = sort_shape(pairs, k.num_experts);
    s.smem += k.num_experts * 4u;
    if (s.smem > 32 * 1024) {
        const int ok = allow_smem<k_expert_sort>(sort_smem(kSortMaxWarps, NUNA_MAX_EXPERTS) + NUNA_MAX_EXPERTS * 4);
        if (ok != NUNA_OK) return ok;
    }
    return launch_op(k_expert_sort, s, effective_flags(flags, stream), stream, k);
}

int nuna_expert_dispatch(const nuna_expert_dispatch_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_expert_dispatch_t a = *args;
    if (!is_dtype(a.dtype)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK || a.hidden == 0 || a.rows == 0) return st;
    return dispatch(a, effective_flags(flags, stream), stream);
}

int nuna_expert_combine(const nuna_expert_combine_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_expert_combine_t a = *args;
    if (!is_dtype(a.dtype)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK || a.hidden == 0 || a.tokens == 0) return st;
    return combine(a, effective_flags(flags, stream), stream);
}

int nuna_expert_combine_backward(const nuna_expert_combine_grad_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_expert_combine_grad_t a = *args;
    if (!is_dtype(a.dtype)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK) return st;
    return combine_backward(a, effective_flags(flags, stream), stream);
}

}  // extern "C"
