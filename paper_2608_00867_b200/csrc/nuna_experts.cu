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
};

template <typename Id>
__global__ void __launch_bounds__(1024) k_expert_sort(const Padded<ExpertSortArgs> a)
{
    extern __shared__ unsigned smem[];
    pdl_begin();
    unsigned* counts = smem;                                         // [num_experts]
    const unsigned threads = gridDim.x * blockDim.x, thread = blockIdx.x * blockDim.x + threadIdx.x;
    const Id* ids = static_cast<const Id*>(a.experts);
    const unsigned kept = sort_pass<long long>(gridDim.x, a.pairs, a.num_experts, smem + a.num_experts, counts,
        [&](unsigned i) { return load_id(ids + i); },
        [&](long long e) {
            const unsigned long long from = (unsigned long long)e - (unsigned long long)a.first_expert;
            return e >= a.first_expert && from < a.num_experts ? (unsigned)from : kNoDigit;
        },
        [&](unsigned i, long long, unsigned d, unsigned first, unsigned rank) {
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
    unsigned units, zero_blocks;                                     // tokens * chunks; blocks that zero rows that no pair has
    unsigned tokens, topk, rows, hidden, packs, chunks, group;       // pieces in a row at most, chunks of a row, threads of a chunk
};

constexpr unsigned kZeroRows = 32;                                   // rows that a block looks at

// Zeroes those of the block's kZeroRows expert rows that no pair has.  These blocks come first: one that has to write all of
// its rows would otherwise be what the kernel ends with.
template <int DT, bool kWhole>
__device__ __forceinline__ void zero_empty_rows(const MoveArgs& a)
{
    constexpr int E = Elem<DT>::kElems;
    const unsigned first = blockIdx.x * kZeroRows, lane = threadIdx.x & 31u;
    const unsigned empty = __ballot_sync(0xFFFFFFFFu, first + lane < a.rows && a.pair_of_row[first + lane] < 0);        // every warp for itself
    const Pack<DT, true> zero = {};
    for (unsigned left = empty; left; left &= left - 1u) {
        char* row = static_cast<char*>(row_at(a.out, (size_t)first + __ffs(left) - 1u, a.out_stride));
        const unsigned s = kWhole ? 0u : (unsigned)behind<DT, E>(row);
        if constexpr (!kWhole) {                                     // what is in front of the first boundary and behind the last
            const unsigned head = s ? E - s : 0u, tail = (a.hidden + s) / E * E - s, i = threadIdx.x;
            if (a.hidden < 2u * E) {
                if (i < a.hidden) store_pack<DT, false>(row, i, {0u});
                continue;
            }
            if (i < head) store_pack<DT, false>(row, i, {0u});
            if (tail + i < a.hidden) store_pack<DT, false>(row, tail + i, {0u});
        }
        const unsigned from = s ? 1u : 0u, to = (a.hidden + s) / E;
        row -= s * Elem<DT>::kBytes;
#pragma unroll 4
        for (unsigned i = from + threadIdx.x; i < to; i += blockDim.x) store_pack<DT, true, true>(row, i, zero);
    }
}

// Every token's row to its pairs' rows.  Whole vectors are read once; rows that are cut otherwise are cut as each of the rows
// that are written, and read again for each (from L1).
template <int DT, int kPacks, bool kWhole>
__global__ void __launch_bounds__(256) k_expert_dispatch(const Padded<MoveArgs> a)
{
    constexpr int E = Elem<DT>::kElems;
    // Rows of the map that are fetched together; pieces, also the rows that are written together (1 | 2 | 4: 8192 x 2050 f32, 2 of 16:
    // 45 | 50 | 74 us, 4096 x 2051 bf16, 8 of 64: 38.8 | 37.6 | 43.8).
    constexpr int kAhead = kWhole ? 8 : DT == kF32 ? 1 : 2;
    pdl_begin();
    if (blockIdx.x < a.zero_blocks) {
        zero_empty_rows<DT, kWhole>(a);
    } else {
        const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
        const unsigned unit = (blockIdx.x - a.zero_blocks) * groups + threadIdx.x / a.group;
        if (unit < a.units) {
            const size_t token = unit / a.chunks;
            const unsigned from = unit % a.chunks * a.group * kPacks + lane;
            const int* map = a.row_of_pair + token * a.topk;
            Piece<DT, kWhole> p[kWhole ? 1 : kAhead][kPacks];
            Source source[kWhole ? 1 : kAhead];
            if constexpr (kWhole) {
                source[0] = source_of<DT, kWhole>(a.x, token, a.x_stride, a.tokens, a.hidden, 0);
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (from + k * a.group < a.packs) fetch_piece<DT, kWhole>(p[0][k], source[0], from + k * a.group, 0, a.hidden);
            }
            for (unsigned j0 = 0; j0 < a.topk; j0 += kAhead) {
                unsigned row[kAhead];
                int s[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j) row[j] = j0 + j < a.topk ? (unsigned)map[j0 + j] : 0xFFFFFFFFu;
#pragma unroll
                for (int j = 0; j < kAhead; ++j) {
                    s[j] = 0;
                    if constexpr (!kWhole) {
                        if (row[j] < a.rows) {
                            s[j] = behind<DT, E>(row_at(a.out, row[j], a.out_stride));
                            source[j] = source_of<DT, kWhole>(a.x, token, a.x_stride, a.tokens, a.hidden, s[j]);
#pragma unroll
                            for (int k = 0; k < kPacks; ++k) {
                                const int e0 = (int)((from + k * a.group) * E) - s[j];
                                if (touches<E>(e0, a.hidden)) fetch_piece<DT, kWhole>(p[j][k], source[j], from + k * a.group, e0, a.hidden);
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (row[j] < a.rows)
#pragma unroll
                        for (int k = 0; k < kPacks; ++k) {
                            const int e0 = (int)((from + k * a.group) * E) - s[j];
                            if (touches<E>(e0, a.hidden))
                                store_piece<DT, kWhole, true>(row_at(a.out, row[j], a.out_stride), a.hidden, e0,
                                                              settle_piece<DT, kWhole>(p[kWhole ? 0 : j][k], source[kWhole ? 0 : j]));
                        }
            }
        }
    }
    pdl_trigger();
}

template <int DT, int kPacks, bool kWhole>
__global__ void __launch_bounds__(256) k_expert_combine(const Padded<MoveArgs> a)
{
    constexpr int E = Elem<DT>::kElems;
    // Expert rows in flight.  Pieces hold twice the registers of vectors: blocks are worth more than rows ahead in each (one and four:
    // 8192 x 2050 f32, 2 of 16: 56 and 116 us, 4096 x 2051 bf16, 8 of 64: 46 | 59), but for few tokens, which have the SMs to themselves.
    constexpr int kAhead = kWhole ? (kPacks == 1 ? 8 : 4) : kPacks == 1 ? 4 : 1;
    pdl_begin();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned unit = blockIdx.x * groups + threadIdx.x / a.group;
    if (unit < a.units) {
        const size_t token = unit / a.chunks;
        const unsigned from = unit % a.chunks * a.group * kPacks + lane;
        const int* map = a.row_of_pair + token * a.topk;
        const float* weights = a.weights ? a.weights + token * a.topk : nullptr;
        void* y = row_at(a.y, token, a.y_stride);
        const int s = kWhole ? 0 : behind<DT, E>(y);
        Two acc[kPacks][E / 2];
#pragma unroll
        for (int k = 0; k < kPacks; ++k)
#pragma unroll
            for (int e = 0; e < E / 2; ++e) acc[k][e] = all<Two>(0.0f);
        for (unsigned j0 = 0; j0 < a.topk; j0 += kAhead) {
            unsigned row[kAhead];
            float w[kAhead];
            Piece<DT, kWhole> v[kAhead][kPacks];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                row[j] = j0 + j < a.topk ? (unsigned)map[j0 + j] : 0xFFFFFFFFu;
                w[j] = weights && j0 + j < a.topk ? weights[j0 + j] : 1.0f;
            }
            Source source[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (row[j] < a.rows) {
                    source[j] = source_of<DT, kWhole>(a.src, row[j], a.src_stride, a.rows, a.hidden, s);
#pragma unroll
                    for (int k = 0; k < kPacks; ++k) {
                        const int e0 = (int)((from + k * a.group) * E) - s;
                        if (touches<E>(e0, a.hidden)) fetch_piece<DT, kWhole>(v[j][k], source[j], from + k * a.group, e0, a.hidden);
                    }
                }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (row[j] < a.rows)
#pragma unroll
                    for (int k = 0; k < kPacks; ++k) {
                        Two f[E / 2];
                        unpack<DT, true>(f, settle_piece<DT, kWhole>(v[j][k], source[j]));
#pragma unroll
                        for (int e = 0; e < E / 2; ++e) acc[k][e] = mad(all<Two>(w[j]), f[e], acc[k][e]);
                    }
        }
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const int e0 = (int)((from + k * a.group) * E) - s;
            if (touches<E>(e0, a.hidden)) store_piece<DT, kWhole>(y, a.hidden, e0, pack<DT, true>(acc[k]));
        }
    }
    pdl_trigger();
}

// A token per group of threads, which goes over the row kPacks pieces a thread at a time; kBatch pairs' products are summed
// together, and over the group at the end of the row.  Pieces of rows that are not whole vectors hold three times the registers:
// one pair at a time and five blocks on an SM, instead of two pairs in two or three (4096 x 2051 bf16, 8 of 64: 103 against 138 us,
// 2048 x 2050 f32, 2 of 16: 25 | 39); where all tokens find a place at once with two pairs, two (100 x 2050, 4 of 16: 7.4 against 9.3,
// 450 x 2051 12.1 | 10.2, 1000 x 333 10.7 | 13.4).
template <int DT, int kPacks, bool kWhole, int kBatch>
__global__ void __launch_bounds__(256, kBatch > 1 ? 2 : DT == kF32 ? 4 : 5) k_expert_combine_backward(const Padded<MoveArgs> a)
{
    constexpr int E = Elem<DT>::kElems;
    __shared__ float red[2][8][kBatch];
    pdl_begin();
    if (blockIdx.x < a.zero_blocks) {
        zero_empty_rows<DT, kWhole>(a);
    } else {
        const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group, warps = a.group / 32u;
        const unsigned unit = (blockIdx.x - a.zero_blocks) * groups + threadIdx.x / a.group;
        const size_t token = unit;
        const bool live = unit < a.units;
        unsigned turn = 0;
        for (unsigned j0 = 0; j0 < a.topk; j0 += kBatch, turn ^= 1u) {
            unsigned row[kBatch];
            float w[kBatch];
            int s[kBatch];
            Two dot[kBatch];
            Source src[kBatch], x[kWhole ? 1 : kBatch];              // whole vectors of dy serve all rows; otherwise each row has them cut as itself
            if constexpr (kWhole) x[0] = source_of<DT, kWhole>(a.x, token, a.x_stride, a.tokens, a.hidden, 0);
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const bool is = live && j0 + j < a.topk;
                row[j] = is ? (unsigned)a.row_of_pair[token * a.topk + j0 + j] : 0xFFFFFFFFu;
                w[j] = is ? a.weights[token * a.topk + j0 + j] : 0.0f;
                dot[j] = all<Two>(0.0f);
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                s[j] = kWhole || row[j] >= a.rows ? 0 : behind<DT, E>(row_at(a.out, row[j], a.out_stride));
                src[j] = source_of<DT, kWhole>(a.src, row[j], a.src_stride, a.rows, a.hidden, s[j]);
                if constexpr (!kWhole) x[j] = source_of<DT, kWhole>(a.x, token, a.x_stride, a.tokens, a.hidden, s[j]);
            }
            for (unsigned base = lane; base < a.packs; base += a.group * kPacks) {
                Piece<DT, kWhole> dy[kWhole ? 1 : kBatch][kPacks], v[kBatch][kPacks];
                if constexpr (kWhole) {
                    if (live) {
#pragma unroll
                        for (int k = 0; k < kPacks; ++k)
                            if (base + k * a.group < a.packs) fetch_piece<DT, kWhole>(dy[0][k], x[0], base + k * a.group, 0, a.hidden);
                    }
                }
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (row[j] < a.rows)
#pragma unroll
                        for (int k = 0; k < kPacks; ++k) {
                            const int e0 = (int)((base + k * a.group) * E) - s[j];
                            if (touches<E>(e0, a.hidden)) {
                                if constexpr (!kWhole) fetch_piece<DT, kWhole>(dy[j][k], x[j], base + k * a.group, e0, a.hidden);
                                if (a.dweights) fetch_piece<DT, kWhole>(v[j][k], src[j], base + k * a.group, e0, a.hidden);
                            }
                        }
#pragma unroll
                for (int j = 0; j < kBatch; ++j)
                    if (row[j] < a.rows)
#pragma unroll
                        for (int k = 0; k < kPacks; ++k) {
                            const int e0 = (int)((base + k * a.group) * E) - s[j];
                            if (touches<E>(e0, a.hidden)) {
                                Two g[E / 2], f[E / 2];
                                unpack<DT, true>(g, settle_piece<DT, kWhole>(dy[kWhole ? 0 : j][k], x[kWhole ? 0 : j]));
                                if (a.dweights) {
                                    unpack<DT, true>(f, settle_piece<DT, kWhole>(v[j][k], src[j]));
                                    if (!kWhole && !inside<E>(e0, a.hidden)) {
#pragma unroll
                                        for (int e = 0; e < E; ++e)
                                            if (e0 + e < 0 || e0 + e >= (int)a.hidden) half(f[e / 2], e) = half(g[e / 2], e) = 0.0f;
                                    }
#pragma unroll
                                    for (int e = 0; e < E / 2; ++e) dot[j] = mad(g[e], f[e], dot[j]);
                                }
#pragma unroll
                                for (int e = 0; e < E / 2; ++e) f[e] = all<Two>(w[j]) * g[e];
                                store_piece<DT, kWhole, true>(row_at(a.out, row[j], a.out_stride), a.hidden, e0, pack<DT, true>(f));
                            }
                        }
            }
            if (a.dweights) {
                float sum[kBatch];
#pragma unroll
                for (int j = 0; j < kBatch; ++j) sum[j] = total(dot[j]);
                warp_sum<kBatch>(sum);
                if (warps > 1u) {
                    const unsigned warp = threadIdx.x >> 5;
                    if ((threadIdx.x & 31u) == 0u)
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) red[turn][warp][j] = sum[j];
                    __syncthreads();                                 // the next batch has the other half of `red`
                    if (lane < kBatch) {
                        float s = 0.0f;
                        for (unsigned o = 0; o < warps; ++o) s += red[turn][warp + o][lane];
                        if (live && j0 + lane < a.topk) a.dweights[token * a.topk + j0 + lane] = s;
                    }
                } else if (live && lane == 0u) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j)
                        if (j0 + j < a.topk) a.dweights[token * a.topk + j0 + j] = sum[j];
                }
            }
        }
    }
    pdl_trigger();
}

// ---- host ------------------------------------------------------------------------------------------------

static size_t stride_bytes(size_t stride, size_t hidden, int dtype) { return (stride ? stride : hidden) * dtype_bytes(dtype); }

// Pieces of 16 bytes that a row may be cut into.
static unsigned pieces(size_t hidden, size_t size, bool whole) { return (unsigned)(whole ? hidden * size / 16 : (hidden + 2 * (16 / size) - 2) / (16 / size)); }

// Threads of a group, at most `most`, for a row in steps of about the same length.
static unsigned group_of(unsigned packs, int per_thread, unsigned most)
{
    const unsigned threads = (packs + per_thread - 1) / per_thread, steps = std::max(1u, (threads + most - 1) / most);
    return std::max(32u, ((threads + steps - 1) / steps + 31u) / 32u * 32u);
}

// Launches a row mover with kPacks pieces a thread in groups of at most `most` threads, which take chunks of a row, or (`whole`)
// a row in several steps.
template <typename Kernel>
static int move_rows(Kernel kernel, MoveArgs& a, size_t tokens, int per_thread, unsigned most, bool whole, unsigned flags, void* stream)
{
    const unsigned threads = (a.packs + per_thread - 1) / per_thread, steps = std::max(1u, (threads + most - 1) / most);
    a.group = group_of(a.packs, per_thread, most);
    a.chunks = whole ? 1u : steps;
    const unsigned groups = std::max(1u, 256u / a.group);
    const unsigned long long units = (unsigned long long)tokens * a.chunks;
    if (units > 0xFFFFFF00ull) return NUNA_ERR_TOO_LARGE;            // 32 bits count the units
    a.units = (unsigned)units;
    a.zero_blocks = a.pair_of_row ? (unsigned)((a.rows + kZeroRows - 1ull) / kZeroRows) : 0u;
    const unsigned long long grid = a.zero_blocks + (units + groups - 1) / groups;
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
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = pieces(n.hidden, e, vec), a.hidden = (unsigned)n.hidden, a.tokens = (unsigned)n.tokens;
    const size_t tokens = n.topk ? n.tokens : 0;
    if (vec) {                                                       // bits are copied: a vector is a vector
        a.hidden = (unsigned)(n.hidden * e / 4);
        return (unsigned long long)tokens * a.packs <= 4ull * kSms * 512ull
                   ? move_rows(k_expert_dispatch<kF32, 1, true>, a, tokens, 1, 256, false, flags, stream)
                   : move_rows(k_expert_dispatch<kF32, 4, true>, a, tokens, 4, 256, false, flags, stream);
    }
    if (n.dtype == NUNA_F32) return move_rows(k_expert_dispatch<kF32, 1, false>, a, tokens, 1, 256, false, flags, stream);
    return move_rows(k_expert_dispatch<kBf16, 1, false>, a, tokens, 1, 256, false, flags, stream);
}

static int combine(const nuna_expert_combine_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.src, n.hidden, n.src_stride, e).rows(n.y, n.hidden, n.y_stride, e).ok;
    MoveArgs a = {};
    a.src = n.src, a.row_of_pair = n.row_of_pair, a.weights = n.weights, a.y = n.y;
    a.src_stride = stride_bytes(n.src_stride, n.hidden, n.dtype), a.y_stride = stride_bytes(n.y_stride, n.hidden, n.dtype);
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = pieces(n.hidden, e, vec), a.hidden = (unsigned)n.hidden, a.tokens = (unsigned)n.tokens;
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const bool few = (unsigned long long)n.tokens * a.packs <= 2ull * kSms * 512ull;       // too few for two pieces a thread
        if (!vec) return few ? move_rows(k_expert_combine<DT, 1, false>, a, n.tokens, 1, 256, false, flags, stream)
                             : move_rows(k_expert_combine<DT, 2, false>, a, n.tokens, 2, 256, false, flags, stream);
        return few ? move_rows(k_expert_combine<DT, 1, true>, a, n.tokens, 1, 256, false, flags, stream)
                   : move_rows(k_expert_combine<DT, 2, true>, a, n.tokens, 2, 256, false, flags, stream);
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
    a.topk = (unsigned)n.topk, a.rows = (unsigned)n.rows, a.packs = pieces(n.hidden, e, vec), a.hidden = (unsigned)n.hidden, a.tokens = (unsigned)n.tokens;
    const size_t tokens = n.topk ? n.tokens : 0;
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const bool few = tokens <= kSms * (512u / group_of(a.packs, 1, 256));                 // all at once with two pairs
        if (!vec) return few ? move_rows(k_expert_combine_backward<DT, 1, false, 2>, a, tokens, 1, 256, true, flags, stream)
                             : move_rows(k_expert_combine_backward<DT, 1, false, 1>, a, tokens, 1, 256, true, flags, stream);
        return move_rows(k_expert_combine_backward<DT, 2, true, 4>, a, tokens, 2, 128, true, flags, stream);
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
                              (unsigned)a.num_experts, (unsigned)a.capacity, (unsigned)rows};
    Shape s = sort_shape(pairs, k.num_experts);
    s.smem += k.num_experts * 4u;
    constexpr int kMost = sort_smem(kSortMaxWarps, NUNA_MAX_EXPERTS) + NUNA_MAX_EXPERTS * 4;
    const bool wide = a.id_bytes == 8;
    const int ok = wide ? allow_sort<k_expert_sort<long long>>(s, kMost) : allow_sort<k_expert_sort<int>>(s, kMost);
    if (ok != NUNA_OK) return ok;
    return launch_op(wide ? k_expert_sort<long long> : k_expert_sort<int>, s, effective_flags(flags, stream), stream, k);
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
