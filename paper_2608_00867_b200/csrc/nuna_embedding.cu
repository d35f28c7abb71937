// Embedding lookup over a slice of the vocabulary, and its gradient by sorted tokens.
//
// Both are rows moved by an index: what bounds them is the memory, and for a few tokens the two dependent reads, id and row.
// The gradient sorts the tokens by id (k_embedding_sort), so that the tokens of a table row are a run of consecutive positions,
// in the tokens' order; then every table row is written once, by the threads that have added its run in registers.  Runs of
// more than kRunPart tokens are cut at the positions that are multiples of kRunPart, their parts added by blocks of their own
// and joined in order, so that one frequent id does not keep one block busy.
#include "nuna_sort.cuh"

#include <algorithm>

namespace nuna {

struct LookupArgs {
    const void *ids, *table;
    void* out;
    size_t table_stride, out_stride;                                 // bytes
    long long vocab_start;
    unsigned long long units;                                        // tokens * chunks
    unsigned vocab_rows, packs, chunks, group;                       // packs in a row, chunks of a row, threads of a chunk
    float scale;
    bool wide;                                                       // ids are int64
};

// The row of the slice that id i names, or -1.
__device__ __forceinline__ long long slice_row(const void* ids, bool wide, size_t i, long long start, unsigned rows)
{
    const long long id = wide ? static_cast<const volatile long long*>(ids)[i] : (long long)static_cast<const volatile int*>(ids)[i];
    // without overflow: id - start is formed only where it is small
    if (id < start || (unsigned long long)id - (unsigned long long)start >= rows) return -1;
    return id - start;
}

// One chunk of one token's row per group of threads, kPacks packs a thread, all of them in flight at once.
template <int DT, int kPacks, bool kVec>
__global__ void __launch_bounds__(256) k_embedding_lookup(const LookupArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
    if (unit < a.units) {
        const size_t token = unit / a.chunks;
        const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
        const long long row = slice_row(a.ids, a.wide, token, a.vocab_start, a.vocab_rows);
        Pack<DT, kVec> p[kPacks];
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = from + k * a.group;
#pragma unroll
            for (int w = 0; w < Pack<DT, kVec>::kWords; ++w) p[k].w[w] = 0u;
            if (row >= 0 && i < a.packs) p[k] = load_pack<DT, kVec>(row_at(a.table, (size_t)row, a.table_stride), i);
        }
#pragma unroll
        for (int k = 0; k < kPacks; ++k) {
            const unsigned i = from + k * a.group;
            if (i < a.packs) {
                if (row >= 0) {
                    float f[E];
                    unpack<DT, kVec>(f, p[k]);
#pragma unroll
                    for (int e = 0; e < E; ++e) f[e] *= a.scale;
                    p[k] = pack<DT, kVec>(f);
                }
                store_pack<DT, kVec>(row_at(a.out, token, a.out_stride), i, p[k]);
            }
        }
    }
    pdl_trigger();
}

// ---- gradient ------------------------------------------------------------------------------------------

struct SortArgs {
    const void* ids;
    unsigned *token[2], *id[2], *begin, *end, *count;
    long long vocab_start;
    unsigned tokens, vocab_rows, passes, bits;                       // bits of a digit
    bool wide, clear;                                                // clear: rows without a token get end = 0
};

// token[passes & 1 ^ 1] / id[...]: the tokens with a row in the slice, by row and then by token; begin / end: each row's run.
__global__ void __launch_bounds__(1024) k_embedding_sort(const SortArgs a)
{
    extern __shared__ unsigned smem[];
    pdl_wait();
    const unsigned bins = 1u << a.bits, threads = gridDim.x * blockDim.x, thread = blockIdx.x * blockDim.x + threadIdx.x;
    if (a.clear)
        for (unsigned long long v = thread; v < a.vocab_rows; v += threads) a.end[v] = 0u;
    unsigned n = a.tokens;
    for (unsigned pass = 0; pass < a.passes; ++pass) {
        const unsigned shift = pass * a.bits;
        unsigned *token = a.token[pass & 1u], *id = a.id[pass & 1u];
        const volatile unsigned *from_token = a.token[(pass & 1u) ^ 1u], *from_id = a.id[(pass & 1u) ^ 1u];
        if (pass == 0u) {
            n = sort_pass(n, bins, smem, nullptr,
                [&](unsigned i) {
                    const long long row = slice_row(a.ids, a.wide, i, a.vocab_start, a.vocab_rows);
                    return row < 0 ? kNoDigit : (unsigned)row & (bins - 1u);
                },
                [&](unsigned i, unsigned d, unsigned first, unsigned rank) {
                    if (d == kNoDigit) return;
                    token[first + rank] = i;
                    id[first + rank] = (unsigned)slice_row(a.ids, a.wide, i, a.vocab_start, a.vocab_rows);
                });
        } else {
            sort_pass(n, bins, smem, nullptr,
                [&](unsigned i) { return (from_id[i] >> shift) & (bins - 1u); },
                [&](unsigned i, unsigned, unsigned first, unsigned rank) {
                    token[first + rank] = from_token[i];
                    id[first + rank] = from_id[i];
                });
        }
    }
    const volatile unsigned* id = a.id[(a.passes & 1u) ^ 1u];
    for (unsigned long long p = thread; p < n; p += threads) {
        const unsigned v = id[p];
        if (p == 0 || id[p - 1] != v) a.begin[v] = (unsigned)p;
        if (p + 1 == n || id[p + 1] != v) a.end[v] = (unsigned)p + 1u;
    }
    if (thread == 0u) *a.count = n;
    pdl_trigger();
}

struct TableArgs {
    const void* dout;
    void* dtable;
    const unsigned *token, *id, *begin, *end, *count;
    float* part;                                                     // [parts][2][part_stride]
    size_t dout_stride, dtable_stride;                               // bytes
    unsigned long long row_units;                                    // table rows (positions, if accumulating) * chunks
    unsigned parts, part_blocks;                                     // cuts of the positions, blocks that add them
    unsigned hidden, packs, chunks, group, part_stride;
    float scale;
    bool accumulate;
};

// acc += the packs i + k * group of the rows of dout that positions p ... end-1 name, in their order.
template <int DT, int kPacks, bool kVec>
__device__ __forceinline__ void add_run(float (&acc)[kPacks][Pack<DT, kVec>::kElems], const TableArgs& a, unsigned p, unsigned end, unsigned from)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    constexpr int kAhead = kPacks >= 4 ? 2 : 4;                      // rows in flight
    for (; p < end; p += kAhead) {
        Pack<DT, kVec> v[kAhead][kPacks];
#pragma unroll
        for (int r = 0; r < kAhead; ++r)
            if (p + r < end) {
                const void* row = row_at(a.dout, a.token[p + r], a.dout_stride);
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (from + k * a.group < a.packs) v[r][k] = load_pack<DT, kVec>(row, from + k * a.group);
            }
#pragma unroll
        for (int r = 0; r < kAhead; ++r)
            if (p + r < end)
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (from + k * a.group < a.packs) {
                        float f[E];
                        unpack<DT, kVec>(f, v[r][k]);
#pragma unroll
                        for (int e = 0; e < E; ++e) acc[k][e] += f[e];
                    }
    }
}

// E values of dtable's type GT from element i * E of a row on: rne(scale * sum), or added to what is there.
template <int GT, int E>
__device__ __forceinline__ void put_gradient(void* row, unsigned i, const float (&sum)[E], float scale, bool accumulate)
{
    constexpr bool kVec = E > 1;
    constexpr int G = Pack<GT, kVec>::kElems, kParts = E / G;
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
        float f[G];
#pragma unroll
        for (int e = 0; e < G; ++e) f[e] = sum[q * G + e] * scale;
        if (accumulate) {
            float old[G];
            unpack<GT, kVec>(old, load_pack<GT, kVec>(row, (size_t)i * kParts + q));
#pragma unroll
            for (int e = 0; e < G; ++e) f[e] = __fadd_rn(old[e], f[e]);
        }
        store_pack<GT, kVec, true>(row, (size_t)i * kParts + q, pack<GT, kVec>(f));
    }
}

// Blocks below part_blocks add the parts of cut runs; the others take one chunk of a table row per group of threads.
template <int DT, int GT, int kPacks, bool kVec>
__global__ void __launch_bounds__(256) k_embedding_rows(const TableArgs a)
{
    constexpr int E = Pack<DT, kVec>::kElems;
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    float acc[kPacks][E];
#pragma unroll
    for (int k = 0; k < kPacks; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[k][e] = 0.0f;
    if (blockIdx.x < a.part_blocks) {
        const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
        const unsigned part = (unsigned)(unit / a.chunks / 2u), n = *a.count;
        const bool last = unit / a.chunks % 2u != 0u;                // the run of the part's last position, or of its first
        const unsigned long long lo = (unsigned long long)part * kRunPart;
        if (part < a.parts && lo < n) {
            const unsigned hi = (unsigned)(lo + kRunPart < n ? lo + kRunPart : n);
            const unsigned v = a.id[last ? hi - 1u : lo], b = a.begin[v], e = a.end[v];
            if (e - b > kRunPart && !(last && b <= lo)) {
                const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
                add_run<DT, kPacks, kVec>(acc, a, b > lo ? b : (unsigned)lo, e < hi ? e : hi, from);
                float* to = a.part + ((size_t)part * 2u + last) * a.part_stride;
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (from + k * a.group < a.packs)
#pragma unroll
                        for (int x = 0; x < E; ++x) to[(size_t)(from + k * a.group) * E + x] = acc[k][x];
            }
        }
    } else {
        const unsigned long long unit = (unsigned long long)(blockIdx.x - a.part_blocks) * groups + threadIdx.x / a.group;
        if (unit < a.row_units) {
            unsigned v = (unsigned)(unit / a.chunks), b, e;
            bool mine = true;
            if (a.accumulate) {                                      // v is a position: the first of a run stands for its row
                const unsigned p = v;
                mine = p < *a.count && (v = a.id[p], a.begin[v] == p);
                b = p, e = mine ? a.end[v] : 0u;
            } else {
                e = a.end ? a.end[v] : 0u;                           // no tokens at all: nothing was sorted
                b = e ? a.begin[v] : 0u;
            }
            if (mine && e - b <= kRunPart) {
                const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
                add_run<DT, kPacks, kVec>(acc, a, b, e, from);
                void* row = row_at(a.dtable, v, a.dtable_stride);
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
                    if (from + k * a.group < a.packs) put_gradient<GT, E>(row, from + k * a.group, acc[k], a.scale, a.accumulate);
            }
        }
    }
    pdl_trigger();
}

// Joins the parts of each cut run: the part in which it begins does it, one chunk per group of threads.
template <int GT, int E, int kPacks>
__global__ void __launch_bounds__(256) k_embedding_join(const TableArgs a)
{
    pdl_wait();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned long long unit = (unsigned long long)blockIdx.x * groups + threadIdx.x / a.group;
    const unsigned part = (unsigned)(unit / a.chunks), n = *a.count;
    const unsigned long long lo = (unsigned long long)part * kRunPart;
    if (part < a.parts && lo < n) {
        const unsigned hi = (unsigned)(lo + kRunPart < n ? lo + kRunPart : n);
        const unsigned v = a.id[hi - 1u], b = a.begin[v], e = a.end[v];
        if (b >= lo && e - b > kRunPart) {
            const unsigned from = (unsigned)(unit % a.chunks) * a.group * kPacks + lane;
            const unsigned ends = (unsigned)((e - 1u) / kRunPart);
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                const unsigned i = from + k * a.group;
                if (i < a.packs) {
                    float acc[E];
#pragma unroll
                    for (int x = 0; x < E; ++x) acc[x] = 0.0f;
#pragma unroll 4
                    for (unsigned q = part; q <= ends; ++q) {
                        const float* share = a.part + ((size_t)q * 2u + (q == part && b > lo)) * a.part_stride + (size_t)i * E;
                        if constexpr (E % 4 == 0) {
#pragma unroll
                            for (int x = 0; x < E; x += 4) {
                                const float4 s = *reinterpret_cast<const float4*>(share + x);
                                acc[x] += s.x, acc[x + 1] += s.y, acc[x + 2] += s.z, acc[x + 3] += s.w;
                            }
                        } else {
                            acc[0] += share[0];
                        }
                    }
                    put_gradient<GT, E>(row_at(a.dtable, v, a.dtable_stride), i, acc, a.scale, a.accumulate);
                }
            }
        }
    }
    pdl_trigger();
}

// ---- host ------------------------------------------------------------------------------------------------

struct RowShape {
    unsigned group, chunks;
};

// Threads and chunks for a row of `packs` packs, kPacks a thread: chunks of at most 256 threads.
static RowShape row_shape(size_t packs, int per_thread)
{
    const size_t threads = (packs + per_thread - 1) / per_thread, group = std::min<size_t>(256, (threads + 31) / 32 * 32);
    return {(unsigned)group, (unsigned)((threads + group - 1) / group)};
}

static int lookup(const nuna_embedding_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.table, n.hidden, n.table_stride, e).rows(n.out, n.hidden, n.out_stride, e).ok;
    LookupArgs a = {};
    a.ids = n.ids, a.table = n.table, a.out = n.out;
    a.table_stride = (n.table_stride ? n.table_stride : n.hidden) * e;
    a.out_stride = (n.out_stride ? n.out_stride : n.hidden) * e;
    a.vocab_start = n.vocab_start, a.vocab_rows = (unsigned)n.vocab_rows;
    a.packs = (unsigned)(vec ? n.hidden * e / 16 : n.hidden);
    a.scale = n.scale, a.wide = n.id_bytes == 8;
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto run = [&](auto kernel, int per_thread) {
            const RowShape s = row_shape(a.packs, per_thread);
            a.group = s.group, a.chunks = s.chunks;
            a.units = (unsigned long long)n.tokens * s.chunks;
            const unsigned groups = 256u / s.group;
            const unsigned long long grid = (a.units + groups - 1) / groups;
            if (grid > kMaxExtent) return (int)NUNA_ERR_TOO_LARGE;
            return launch_op(kernel, Shape{(unsigned)grid, groups * s.group, 0, 1}, flags, stream, a);
        };
        const bool few = (unsigned long long)n.tokens * a.packs <= 4ull * kSms * 512ull;     // too few for every SM to hold four a thread
        if (vec) return few ? run(k_embedding_lookup<DT, 1, true>, 1) : run(k_embedding_lookup<DT, 4, true>, 4);
        return few ? run(k_embedding_lookup<DT, 1, false>, 1) : run(k_embedding_lookup<DT, 8, false>, 8);
    });
}

static int table_gradient(const nuna_embedding_grad_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype), ge = dtype_bytes(n.grad_dtype);
    const bool accumulate = (flags & NUNA_GRAD_ACCUMULATE) != 0u;
    if (n.vocab_rows == 0 || (accumulate && n.tokens == 0)) return NUNA_OK;
    const EmbeddingWorkspace w = embedding_workspace(n.tokens, n.hidden, n.vocab_rows);
    const auto words = [&](size_t at) { return reinterpret_cast<unsigned*>(static_cast<char*>(n.workspace) + at); };
    SortArgs s = {};
    s.ids = n.ids, s.vocab_start = n.vocab_start, s.tokens = (unsigned)n.tokens, s.vocab_rows = (unsigned)n.vocab_rows;
    s.wide = n.id_bytes == 8, s.clear = !accumulate;
    for (int i = 0; i < 2; ++i) s.token[i] = words(w.token[i]), s.id[i] = words(w.id[i]);
    s.begin = words(w.begin), s.end = words(w.end), s.count = words(w.count);
    unsigned bits = 1;
    while (bits < 32u && (n.vocab_rows - 1) >> bits) ++bits;
    s.passes = (bits + 9u) / 10u;                                    // digits of at most 10 bits: 1024 bins a warp fit a block's shared memory
    s.bits = (bits + s.passes - 1u) / s.passes;
    if (n.tokens) {
        const Shape sort = sort_shape(n.tokens, 1u << s.bits);
        int st = sort.smem > 32 * 1024 ? allow_smem<k_embedding_sort>(sort_smem(kSortMaxWarps, 1024)) : NUNA_OK;
        if (st != NUNA_OK || (st = launch_op(k_embedding_sort, sort, flags, stream, s)) != NUNA_OK) return st;
    }

    const bool vec = VectorRows{true}.rows(n.dout, n.hidden, n.dout_stride, e).rows(n.dtable, n.hidden, n.dtable_stride, ge).ok;
    TableArgs a = {};
    a.dout = n.dout, a.dtable = n.dtable;
    a.token = s.token[(s.passes & 1u) ^ 1u], a.id = s.id[(s.passes & 1u) ^ 1u], a.begin = s.begin, a.end = n.tokens ? s.end : nullptr, a.count = s.count;
    a.part = reinterpret_cast<float*>(words(w.part));
    a.dout_stride = (n.dout_stride ? n.dout_stride : n.hidden) * e;
    a.dtable_stride = (n.dtable_stride ? n.dtable_stride : n.hidden) * ge;
    a.hidden = (unsigned)n.hidden, a.packs = (unsigned)(vec ? n.hidden * e / 16 : n.hidden), a.part_stride = (unsigned)((n.hidden + 3) / 4 * 4);
    a.scale = n.scale, a.accumulate = accumulate;
    a.parts = n.tokens > kRunPart ? (unsigned)((n.tokens + kRunPart - 1) / kRunPart) : 0u;
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto run = [&](auto rows, auto join, int per_thread) {
            const RowShape sh = row_shape(a.packs, per_thread);
            a.group = sh.group, a.chunks = sh.chunks;
            const unsigned groups = 256u / sh.group;
            const auto blocks = [&](unsigned long long units) { return (units + groups - 1) / groups; };
            a.row_units = (unsigned long long)(accumulate ? n.tokens : n.vocab_rows) * sh.chunks;
            const unsigned long long part_blocks = blocks(2ull * a.parts * sh.chunks), grid = part_blocks + blocks(a.row_units);
            if (grid > kMaxExtent) return (int)NUNA_ERR_TOO_LARGE;
            a.part_blocks = (unsigned)part_blocks;
            const int ok = launch_op(rows, Shape{(unsigned)grid, groups * sh.group, 0, 1}, flags, stream, a);
            if (ok != NUNA_OK || a.parts == 0u) return ok;
            return launch_op(join, Shape{(unsigned)blocks((unsigned long long)a.parts * sh.chunks), groups * sh.group, 0, 1}, flags, stream, a);
        };
        const auto typed = [&](auto gt) {
            constexpr int GT = decltype(gt)::value;
            if (vec) return run(k_embedding_rows<DT, GT, 2, true>, k_embedding_join<GT, Elem<DT>::kElems, 2>, 2);
            return run(k_embedding_rows<DT, GT, 4, false>, k_embedding_join<GT, 1, 4>, 4);
        };
        return n.grad_dtype == NUNA_F32 ? typed(std::integral_constant<int, kF32>{}) : typed(dt);
    });
}

}  // namespace nuna

using namespace nuna;

extern "C" {

int nuna_embedding_forward(const nuna_embedding_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~NUNA_LAUNCH_PDL)) return NUNA_ERR_INVALID_ARG;
    const nuna_embedding_t a = *args;
    if (!is_dtype(a.dtype)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    if ((a.id_bytes != 4 && a.id_bytes != 8) || a.vocab_start < 0) return NUNA_ERR_INVALID_ARG;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK || a.tokens == 0 || a.hidden == 0) return st;
    return lookup(a, effective_flags(flags, stream), stream);
}

int nuna_embedding_backward(const nuna_embedding_grad_t* args, unsigned flags, void* stream)
{
    if (!args || (flags & ~(NUNA_LAUNCH_PDL | NUNA_GRAD_ACCUMULATE))) return NUNA_ERR_INVALID_ARG;
    const nuna_embedding_grad_t a = *args;
    if (!is_dtype(a.dtype) || (a.grad_dtype != a.dtype && a.grad_dtype != NUNA_F32)) return NUNA_ERR_UNSUPPORTED_DTYPE;
    if ((a.id_bytes != 4 && a.id_bytes != 8) || a.vocab_start < 0) return NUNA_ERR_INVALID_ARG;
    const int st = check_spans(spans_of(a));
    if (st != NUNA_OK || a.hidden == 0) return st;
    if (a.tokens && a.workspace_bytes < embedding_workspace(a.tokens, a.hidden, a.vocab_rows).bytes) return NUNA_ERR_INVALID_ARG;
    return table_gradient(a, effective_flags(flags, stream), stream);
}

size_t nuna_embedding_workspace(size_t tokens, size_t hidden, size_t vocab_rows) { return embedding_workspace(tokens, hidden, vocab_rows).bytes; }

}  // extern "C"
