// Embedding lookup over a slice of the vocabulary, and its gradient by sorted tokens.
//
// Both are rows moved by an index: what bounds them is the memory, and for a few tokens the two dependent reads, id and row.
// The gradient sorts the tokens by id (k_embedding_sort: a few by comparing all of them, more digit by digit), so that the tokens of a table row are a run of consecutive positions,
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
    unsigned tokens, units;                                          // units: (tokens / kTokens) * chunks
    unsigned vocab_rows, hidden, chunks, group;                      // chunks of a row, threads of a chunk
    float scale;
};

// One chunk of kTokens tokens' rows per group of threads, kPacks pieces a thread and token: the tokens' ids are fetched together,
// and then all of their pieces.
template <typename Id, int DT, int kTokens, int kPacks, bool kWhole>
__global__ void __launch_bounds__(256) k_embedding_lookup(const Padded<LookupArgs> a)
{
    constexpr int E = Elem<DT>::kElems;
    pdl_begin();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    const unsigned unit = blockIdx.x * groups + threadIdx.x / a.group;
    if (unit < a.units) {
        const unsigned first = unit / a.chunks * kTokens, from = unit % a.chunks * a.group * kPacks + lane;
        long long id[kTokens];
        Piece<DT, kWhole> p[kTokens][kPacks];
        Source source[kTokens];
        int s[kTokens];                                              // by how much the output row is behind a boundary
#pragma unroll
        for (int t = 0; t < kTokens; ++t) id[t] = first + t < a.tokens ? load_id(static_cast<const Id*>(a.ids) + first + t) : -1;
        unsigned found = 0;
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            const unsigned long long row = (unsigned long long)id[t] - (unsigned long long)a.vocab_start;
            s[t] = kWhole ? 0 : behind<DT, E>(row_at(a.out, (size_t)first + t, a.out_stride));
            if (id[t] >= a.vocab_start && row < a.vocab_rows) {
                found |= 1u << t;
                source[t] = source_of<DT, kWhole>(a.table, row, a.table_stride, a.vocab_rows, a.hidden, s[t]);
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    const unsigned i = from + k * a.group;
                    const int e0 = (int)(i * E) - s[t];
                    if (touches<E>(e0, a.hidden)) fetch_piece<DT, kWhole>(p[t][k], source[t], i, e0, a.hidden);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < kTokens; ++t) {
            if (first + t >= a.tokens) break;
            void* out = row_at(a.out, (size_t)first + t, a.out_stride);
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                const int e0 = (int)((from + k * a.group) * E) - s[t];
                if (touches<E>(e0, a.hidden)) {
                    Pack<DT, true> v = {};                           // zeros, which are not scaled: the scale may be infinite
                    if (found >> t & 1u) {
                        v = settle_piece<DT, kWhole>(p[t][k], source[t]);
                        if (a.scale != 1.0f) {
                            Two f[E / 2];
                            unpack<DT, true>(f, v);
#pragma unroll
                            for (int e = 0; e < E / 2; ++e) f[e] = f[e] * all<Two>(a.scale);
                            v = pack<DT, true>(f);
                        }
                    }
                    store_piece<DT, kWhole>(out, a.hidden, e0, v);
                }
            }
        }
    }
    pdl_trigger();
}

// ---- gradient ------------------------------------------------------------------------------------------

struct SortArgs {
    const void* ids;
    uint2* items[2];                                                 // token and row of the slice
    unsigned *begin, *end, *count, *cut;
    long long vocab_start;
    unsigned tokens, vocab_rows, passes, bits;                       // bits of a digit
    unsigned sorters;                                                // blocks that sort; the others zero the table
    unsigned per, slices;                                            // by rank: a block's tokens, threads that count for one; 0: by digits
    bool clear;                                                      // rows without a token get end = 0
    uint4* zero;
    unsigned long long zero_vectors;
    uint16_t *head, *tail;                                           // what the table has in front of those vectors and behind them
    unsigned head_halves, tail_halves;
};

// The place of each of a few tokens is the number of tokens that belong before it: a block has all tokens' rows in its shared
// memory, and `slices` threads compare a share of them each with the row of one of its `per` tokens.  Returns how many tokens
// have a row; keys, [tokens + 3] and [tokens] behind, holds their rows and, if one block sorts, those in order.
template <typename RowAt>
__device__ __forceinline__ unsigned rank_tokens(const SortArgs& a, unsigned* keys, uint2* to, RowAt row_at_token)
{
    const unsigned vectors = (a.tokens + 3u) / 4u;
    unsigned *sorted = keys + vectors * 4u, *part = sorted + a.tokens, n = 0;
    for (unsigned base = 0; base < vectors * 4u; base += blockDim.x) {
        const unsigned j = base + threadIdx.x, key = j < a.tokens ? row_at_token(j) : kNoDigit;
        if (j < vectors * 4u) keys[j] = key;
        n += __syncthreads_count(key != kNoDigit);
    }
    const unsigned slice = threadIdx.x / a.per, mine = threadIdx.x - slice * a.per, i = blockIdx.x * a.per + mine;
    const unsigned key = i < a.tokens ? keys[i] : kNoDigit;
    if (slice < a.slices) {
        const unsigned each = (vectors + a.slices - 1u) / a.slices, from = slice * each, to_vector = from + each < vectors ? from + each : vectors;
        const unsigned own = (i - threadIdx.x % 32u) / 4u;           // the first of the eight vectors that hold this warp's tokens
        const uint4* all = reinterpret_cast<const uint4*>(keys);
        unsigned count = 0, j = from;
#pragma unroll 4
        for (; j < to_vector && j < own; ++j) {                      // earlier tokens come first among equals
            const uint4 k = all[j];
            count += (unsigned)(k.x <= key) + (unsigned)(k.y <= key) + (unsigned)(k.z <= key) + (unsigned)(k.w <= key);
        }
        for (; j < to_vector && j < own + 8u; ++j) {
            const uint4 k = all[j];
            const unsigned t = j * 4u;
            count += (unsigned)(k.x < key || (k.x == key && t < i)) + (unsigned)(k.y < key || (k.y == key && t + 1u < i)) +
                     (unsigned)(k.z < key || (k.z == key && t + 2u < i)) + (unsigned)(k.w < key || (k.w == key && t + 3u < i));
        }
#pragma unroll 4
        for (; j < to_vector; ++j) {
            const uint4 k = all[j];
            count += (unsigned)(k.x < key) + (unsigned)(k.y < key) + (unsigned)(k.z < key) + (unsigned)(k.w < key);
        }
        part[threadIdx.x] = count;
    }
    __syncthreads();
    if (slice == 0u && key != kNoDigit) {
        unsigned rank = 0;
        for (unsigned s = 0; s < a.slices; ++s) rank += part[s * a.per + mine];
        to[rank] = make_uint2(i, key);
        sorted[rank] = key;
    }
    sort_sync(a.sorters);
    return n;
}

// items[passes & 1 ^ 1]: the tokens with a row in the slice, by row and then by token; begin / end: each row's run; count: how
// many tokens that is, and how many runs are cut; cut: where those begin, in no order (each of them is joined by itself).
template <typename Id>
__global__ void __launch_bounds__(1024) k_embedding_sort(const Padded<SortArgs> a)
{
    extern __shared__ unsigned smem[];
    pdl_begin(a.sorters == gridDim.x);
    if (blockIdx.x >= a.sorters) {
        // a stretch of its own for every block
        const unsigned blocks = gridDim.x - a.sorters;
        const unsigned long long each = (a.zero_vectors + blocks - 1u) / blocks, from = (blockIdx.x - a.sorters) * each;
        const unsigned long long to = from + each < a.zero_vectors ? from + each : a.zero_vectors;
#pragma unroll 4
        for (unsigned long long i = from + threadIdx.x; i < to; i += blockDim.x) st_stream(a.zero + i, make_uint4(0u, 0u, 0u, 0u));
        return;
    }
    const unsigned bins = 1u << a.bits, threads = a.sorters * blockDim.x, thread = blockIdx.x * blockDim.x + threadIdx.x;
    const Id* ids = static_cast<const Id*>(a.ids);
    if (thread == 0u) a.count[1] = 0u;                               // like `end`, before the first pass
    if (thread < a.head_halves) a.head[thread] = 0;
    if (thread < a.tail_halves) a.tail[thread] = 0;
    if (a.clear)                                                     // whose barriers order it
        // 16 bytes a store; the rest of the last vector is the workspace's padding
        for (unsigned long long v = thread; v * 4u < a.vocab_rows; v += threads) reinterpret_cast<uint4*>(a.end)[v] = make_uint4(0u, 0u, 0u, 0u);
    const auto row_of = [&](long long id) {
        const unsigned long long from = (unsigned long long)id - (unsigned long long)a.vocab_start;
        return id >= a.vocab_start && from < a.vocab_rows ? (unsigned)from : kNoDigit;
    };
    uint2 *to = a.items[0], *from = a.items[1];
    unsigned n;
    if (a.per) {
        n = rank_tokens(a, smem, to, [&](unsigned i) { return row_of(load_id(ids + i)); });
    } else {
        n = sort_pass<long long>(a.sorters, a.tokens, bins, smem, nullptr,
            [&](unsigned i) { return load_id(ids + i); },
            [&](long long id) {
                const unsigned row = row_of(id);
                return row == kNoDigit ? kNoDigit : row & (bins - 1u);
            },
            [&](unsigned i, long long id, unsigned d, unsigned first, unsigned rank) {
                if (d != kNoDigit) to[first + rank] = make_uint2(i, row_of(id));
            });
        for (unsigned pass = 1; pass < a.passes; ++pass) {
            uint2* last = to;
            to = from, from = last;
            sort_pass<uint2>(a.sorters, n, bins, smem, nullptr, [&](unsigned i) { return load_shared_by_cluster(from + i); },
                [&](uint2 item) { return (item.y >> (pass * a.bits)) & (bins - 1u); },
                [&](unsigned, uint2 item, unsigned, unsigned first, unsigned rank) { to[first + rank] = item; });
        }
    }
    const auto row_in_order = [&](size_t p) { return a.per && a.sorters == 1u ? smem[(a.tokens + 3u) / 4u * 4u + p] : load_shared_by_cluster(to + p).y; };
    for (unsigned long long p = thread; p < n; p += threads) {
        const unsigned v = row_in_order(p), left = p > 0 ? row_in_order(p - 1) : kNoDigit, right = p + 1 < n ? row_in_order(p + 1) : kNoDigit;
        if (left != v) a.begin[v] = (unsigned)p;
        if (right != v) a.end[v] = (unsigned)p + 1u;
        if (left != v && p + kRunPart < n && row_in_order(p + kRunPart) == v) a.cut[atomicAdd(a.count + 1, 1u)] = (unsigned)p;
    }
    if (thread == 0u) a.count[0] = n;
    pdl_trigger();
}

struct TableArgs {
    const void* dout;
    void* dtable;
    const uint2* items;                                              // (token, row) by row
    const unsigned *begin, *end, *count, *cut;
    float* part;                                                     // [parts][2][part_stride]
    size_t dout_stride, dtable_stride;                               // bytes
    unsigned rows, row_units, each;                                  // table rows (positions, if by_position); (rows / each) * chunks
    unsigned parts, part_blocks;                                     // cuts of the positions, blocks that add them
    unsigned tokens, hidden, chunks, group, part_stride;
    float scale;
    bool accumulate, by_position;                                    // by_position: rows without a token are left alone, or zero already
    bool whole_sectors;                                              // rows of dtable are at 32-byte addresses
};

// acc += pieces from + k * group, which begin at E times that minus s, of the rows of dout that positions p ... end-1 name, in
// their order.  A warp fetches 32 positions' tokens at once, and then kAhead rows.  All lanes of a warp have the same run.
template <int DT, int kPacks, bool kWhole>
__device__ __forceinline__ void add_run(Two (&acc)[kPacks][Elem<DT>::kElems / 2], const TableArgs& a, unsigned p, unsigned end, unsigned from, int s)
{
    constexpr int E = Elem<DT>::kElems;
    constexpr int kAhead = 4;
    for (; p < end; p += 32u) {
        const unsigned lane = threadIdx.x & 31u, n = end - p < 32u ? end - p : 32u;
        const unsigned token = lane < n ? a.items[p + lane].x : 0u;
        for (unsigned r0 = 0; r0 < n; r0 += kAhead) {
            Piece<DT, kWhole> v[kAhead][kPacks];
            Source source[kAhead];
#pragma unroll
            for (int r = 0; r < kAhead; ++r) {
                source[r] = source_of<DT, kWhole>(a.dout, __shfl_sync(0xFFFFFFFFu, token, r0 + r), a.dout_stride, a.tokens, a.hidden, s);
                if (r0 + r < n)
#pragma unroll
                    for (int k = 0; k < kPacks; ++k) {
                        const int e0 = (int)((from + k * a.group) * E) - s;
                        if (touches<E>(e0, a.hidden)) fetch_piece<DT, kWhole>(v[r][k], source[r], from + k * a.group, e0, a.hidden);
                    }
            }
#pragma unroll
            for (int r = 0; r < kAhead; ++r)
                if (r0 + r < n)
#pragma unroll
                    for (int k = 0; k < kPacks; ++k) add_pack<DT, true>(acc[k], settle_piece<DT, kWhole>(v[r][k], source[r]));
        }
    }
}

// E values of dtable's type GT from element e0 of a row on: rne(scale * sum), or added to what is there.
template <int GT, int E, bool kWhole>
__device__ __forceinline__ void put_gradient(const TableArgs& a, void* row, int e0, const Two (&acc)[E / 2])
{
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = e % 2 ? acc[e / 2].y : acc[e / 2].x;
    if (!kWhole && !inside<E>(e0, a.hidden)) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e0 + e >= 0 && e0 + e < (int)a.hidden) {
                float f[1] = {sum[e] * a.scale};
                if (a.accumulate) {
                    float old[1];
                    unpack<GT, false>(old, load_pack<GT, false>(row, (size_t)(e0 + e)));
                    f[0] = __fadd_rn(old[0], f[0]);
                }
                store_pack<GT, false>(row, (size_t)(e0 + e), pack<GT, false>(f));
            }
        return;
    }
    constexpr int G = Elem<GT>::kElems, kParts = E / G;
    void* at = static_cast<char*>(row) + (long long)e0 * Elem<GT>::kBytes;
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
        float old[G];
        if (a.accumulate) unpack<GT, true>(old, load_pack<GT, true>(at, q));
#pragma unroll
        for (int e = 0; e < G; ++e) {
            sum[q * G + e] *= a.scale;
            if (a.accumulate) sum[q * G + e] = __fadd_rn(old[e], sum[q * G + e]);
        }
    }
    bool done = false;
    if constexpr (GT == kF32 && E == 8) {
        done = !kWhole || a.whole_sectors;
        if (done) store8(static_cast<float*>(at), sum);          // pieces of eight are cut at 32-byte boundaries
    }
    if (!done) {
#pragma unroll
        for (int q = 0; q < kParts; ++q) {
            float f[G];
#pragma unroll
            for (int e = 0; e < G; ++e) f[e] = sum[q * G + e];
            store_pack<GT, true, true>(at, q, pack<GT, true>(f));
        }
    }
}

// Blocks below part_blocks add the parts of cut runs; the others take one chunk of `each` table rows per group of threads,
// whose runs are fetched together: most rows of a large vocabulary have none, and are only written.
template <int DT, int GT, int kPacks, bool kWhole>
__global__ void __launch_bounds__(256, 3) k_embedding_rows(const Padded<TableArgs> a)
{
    constexpr int E = Elem<DT>::kElems;
    pdl_begin();
    const unsigned groups = blockDim.x / a.group, lane = threadIdx.x % a.group;
    Two acc[kPacks][E / 2];
    if (blockIdx.x < a.part_blocks) {
        const unsigned unit = blockIdx.x * groups + threadIdx.x / a.group;
        const unsigned part = unit / a.chunks, n = a.count[0], from = unit % a.chunks * a.group * kPacks + lane;
        const unsigned long long lo = (unsigned long long)part * kRunPart;
        if (part < a.parts && lo < n) {
            const unsigned hi = (unsigned)(lo + kRunPart < n ? lo + kRunPart : n);
            const unsigned row[2] = {a.items[lo].y, a.items[hi - 1u].y};
            for (int last = 0; last < 2; ++last) {                   // the run of the part's first position, and of its last if another
                const unsigned v = row[last], b = a.begin[v], e = a.end[v];
                if (e - b <= kRunPart || (last && b <= lo)) continue;
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
#pragma unroll
                    for (int x = 0; x < E / 2; ++x) acc[k][x] = all<Two>(0.0f);
                add_run<DT, kPacks, kWhole>(acc, a, b > lo ? b : (unsigned)lo, e < hi ? e : hi, from, 0);
                float* to = a.part + ((size_t)part * 2u + last) * a.part_stride;
#pragma unroll
                for (int k = 0; k < kPacks; ++k)                     // a whole piece at the row's end too: part_stride is a multiple of eight
                    if ((from + k * a.group) * E < a.hidden) {
                        float f[E];
#pragma unroll
                        for (int x = 0; x < E; ++x) f[x] = x % 2 ? acc[k][x / 2].y : acc[k][x / 2].x;
                        if constexpr (E == 8) store8(to + (size_t)(from + k * a.group) * 8u, f);
                        else                  *reinterpret_cast<float4*>(to + (size_t)(from + k * a.group) * 4u) = make_float4(f[0], f[1], f[2], f[3]);
                    }
            }
        }
    } else {
        const unsigned unit = (blockIdx.x - a.part_blocks) * groups + threadIdx.x / a.group;
        if (unit < a.row_units) {
            const unsigned first = unit / a.chunks * a.each, from = unit % a.chunks * a.group * kPacks + lane, me = threadIdx.x & 31u;
            unsigned v = first + me, b = 0, e = 0;                   // of the row that this lane looks at
            bool mine = me < a.each && v < a.rows;
            if (mine && a.by_position) {                             // a position: the first of a run stands for its row
                const unsigned p = v;
                mine = p < a.count[0];
                if (mine) v = a.items[p].y, b = a.begin[v], e = a.end[v];
                mine = mine && b == p;
            } else if (mine && a.end) {                              // no tokens at all: nothing was sorted
                e = a.end[v];
                if (e) b = a.begin[v];
            }
            const unsigned only = mine && e - b == 1u ? a.items[b].x : 0u;       // the token of a run of one, as most are
            const unsigned empty = __ballot_sync(0xFFFFFFFFu, mine && e == b), single = __ballot_sync(0xFFFFFFFFu, mine && e - b == 1u),
                           todo = __ballot_sync(0xFFFFFFFFu, mine && e - b > 1u && e - b <= kRunPart);
            // Rows without a token: one after the other, they are only stores, of consecutive vectors by consecutive lanes.
            constexpr int G = Elem<GT>::kElems, kParts = E / G;
            const Pack<GT, true> zero = {};
            const unsigned zero_from = (from - lane) * kParts + lane;
            for (unsigned left = empty; left; left &= left - 1u) {
                void* row = row_at(a.dtable, (size_t)first + __ffs(left) - 1, a.dtable_stride);
                const int s = kWhole ? 0 : behind<GT, E>(row);
#pragma unroll
                for (int k = 0; k < kPacks * kParts; ++k) {
                    const int e0 = (int)((zero_from + k * a.group) * G) - s;
                    if (touches<G>(e0, a.hidden)) store_piece<GT, kWhole, true>(row, a.hidden, e0, zero);
                }
            }
            // Rows with one token: several at a time.
            constexpr int kRows = 4;
            for (unsigned left = single; left;) {
                Piece<DT, kWhole> p[kRows][kPacks];
                Source source[kRows];
                void* row[kRows];
                int s[kRows], n = 0;
#pragma unroll
                for (int q = 0; q < kRows; ++q) {
                    const int r = left ? __ffs(left) - 1 : 0;
                    const unsigned row_v = __shfl_sync(0xFFFFFFFFu, v, r), token = __shfl_sync(0xFFFFFFFFu, only, r);
                    if (left) {
                        left &= left - 1u;
                        ++n;
                        row[q] = row_at(a.dtable, row_v, a.dtable_stride);
                        s[q] = kWhole ? 0 : behind<GT, E>(row[q]);
                        source[q] = source_of<DT, kWhole>(a.dout, token, a.dout_stride, a.tokens, a.hidden, s[q]);
#pragma unroll
                        for (int k = 0; k < kPacks; ++k) {
                            const int e0 = (int)((from + k * a.group) * E) - s[q];
                            if (touches<E>(e0, a.hidden)) fetch_piece<DT, kWhole>(p[q][k], source[q], from + k * a.group, e0, a.hidden);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < kRows; ++q)
                    if (q < n)
#pragma unroll
                        for (int k = 0; k < kPacks; ++k) {
                            const int e0 = (int)((from + k * a.group) * E) - s[q];
                            Two f[E / 2];
                            unpack<DT, true>(f, settle_piece<DT, kWhole>(p[q][k], source[q]));
                            if (touches<E>(e0, a.hidden)) put_gradient<GT, E, kWhole>(a, row[q], e0, f);
                        }
            }
            for (unsigned left = todo; left; left &= left - 1u) {
                const int r = __ffs(left) - 1;
                const unsigned row_v = __shfl_sync(0xFFFFFFFFu, v, r), row_b = __shfl_sync(0xFFFFFFFFu, b, r), row_e = __shfl_sync(0xFFFFFFFFu, e, r);
                void* row = row_at(a.dtable, row_v, a.dtable_stride);
                const int s = kWhole ? 0 : behind<GT, E>(row);
#pragma unroll
                for (int k = 0; k < kPacks; ++k)
#pragma unroll
                    for (int x = 0; x < E / 2; ++x) acc[k][x] = all<Two>(0.0f);
                add_run<DT, kPacks, kWhole>(acc, a, row_b, row_e, from, s);
#pragma unroll
                for (int k = 0; k < kPacks; ++k) {
                    const int e0 = (int)((from + k * a.group) * E) - s;
                    if (touches<E>(e0, a.hidden)) put_gradient<GT, E, kWhole>(a, row, e0, acc[k]);
                }
            }
        }
    }
    pdl_trigger();
}

// Joins the parts of the cut runs, 128 columns of one run at a time: eight warps take its parts in turn, and are added in order.
constexpr unsigned kJoinColumns = 128;
template <int GT>
__global__ void __launch_bounds__(256) k_embedding_join(const Padded<TableArgs> a)
{
    __shared__ float4 sum[8][32];
    pdl_begin();
    const unsigned slice = threadIdx.x >> 5, lane = threadIdx.x & 31u, chunks = (a.hidden + kJoinColumns - 1u) / kJoinColumns;
    const unsigned long long todo = (unsigned long long)a.count[1] * chunks;
    for (unsigned long long t = blockIdx.x; t < todo; t += gridDim.x) {
        const unsigned b = a.cut[t / chunks], column = (unsigned)(t % chunks) * kJoinColumns, v = a.items[b].y, e = a.end[v];
        const unsigned first = b / (unsigned)kRunPart, last = (e - 1u) / (unsigned)kRunPart;
        float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (column + lane * 4u < a.part_stride) {
#pragma unroll 4
            for (unsigned q = first + slice; q <= last; q += 8u) {
                const float4 f = *reinterpret_cast<const float4*>(a.part + ((size_t)q * 2u + (q == first && b % (unsigned)kRunPart != 0u)) * a.part_stride + column + lane * 4u);
                s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
            }
        }
        sum[slice][lane] = s;
        __syncthreads();
        if (threadIdx.x < kJoinColumns && column + threadIdx.x < a.hidden) {
            float f[1] = {0.0f}, old[1];
#pragma unroll
            for (int o = 0; o < 8; ++o) f[0] += reinterpret_cast<const float*>(sum[o])[threadIdx.x];
            f[0] *= a.scale;
            void* row = row_at(a.dtable, v, a.dtable_stride);
            if (a.accumulate) {
                unpack<GT, false>(old, load_pack<GT, false>(row, column + threadIdx.x));
                f[0] = __fadd_rn(old[0], f[0]);
            }
            store_pack<GT, false>(row, column + threadIdx.x, pack<GT, false>(f));
        }
        __syncthreads();
    }
    pdl_trigger();
}

// ---- host ------------------------------------------------------------------------------------------------

struct RowShape {
    unsigned group, chunks;
};

// Pieces of E elements that a row of `hidden` may be cut into.
static size_t pieces(size_t hidden, int elems, bool whole) { return whole ? hidden / elems : (hidden + 2 * elems - 2) / elems; }

// Threads (at most 256) and chunks, of about the same length, for a row of `packs` pieces, per_thread of them a thread.
static RowShape row_shape(size_t packs, int per_thread)
{
    const size_t threads = (packs + per_thread - 1) / per_thread, chunks = (threads + 255) / 256;
    return {(unsigned)(((threads + chunks - 1) / chunks + 31) / 32 * 32), (unsigned)chunks};
}

constexpr unsigned long long kMaxUnits = 0xFFFFFF00ull;              // 32 bits count the units of a launch

static int lookup(const nuna_embedding_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype);
    const bool vec = VectorRows{true}.rows(n.table, n.hidden, n.table_stride, e).rows(n.out, n.hidden, n.out_stride, e).ok;
    LookupArgs a = {};
    a.ids = n.ids, a.table = n.table, a.out = n.out;
    a.table_stride = (n.table_stride ? n.table_stride : n.hidden) * e;
    a.out_stride = (n.out_stride ? n.out_stride : n.hidden) * e;
    a.vocab_start = n.vocab_start, a.vocab_rows = (unsigned)n.vocab_rows, a.tokens = (unsigned)n.tokens;
    a.hidden = (unsigned)n.hidden, a.scale = n.scale;
    const size_t packs = pieces(n.hidden, 16 / (int)e, vec);
    const auto typed = [&](auto id, auto dt) {
        using Id = decltype(id);
        constexpr int DT = decltype(dt)::value;
        const auto run = [&](auto kernel, int tokens, int per_thread) {
            const RowShape s = row_shape(packs, per_thread);
            a.group = s.group, a.chunks = s.chunks;
            const unsigned long long units = (n.tokens + tokens - 1) / tokens * s.chunks;
            if (units > kMaxUnits) return (int)NUNA_ERR_TOO_LARGE;
            a.units = (unsigned)units;
            const unsigned groups = 256u / s.group;
            return launch_op(kernel, Shape{(unsigned)((units + groups - 1) / groups), groups * s.group, 0, 1}, flags, stream, a);
        };
        const bool few = (unsigned long long)n.tokens * packs <= 4ull * kSms * 512ull;     // too few for every SM to hold more than one a thread
        if (vec) return few ? run(k_embedding_lookup<Id, DT, 1, 1, true>, 1, 1) : run(k_embedding_lookup<Id, DT, 4, 2, true>, 4, 2);
        // (two tokens and two pieces, against four and one: 16384 x 4001 bf16 43.8 | 50.2 us, 20011 x 1037 f32 30.7 | 37.6)
        return few ? run(k_embedding_lookup<Id, DT, 1, 1, false>, 1, 1) : run(k_embedding_lookup<Id, DT, 2, 2, false>, 2, 2);
    };
    return with_dtype(n.dtype, [&](auto dt) { return n.id_bytes == 8 ? typed((long long)0, dt) : typed(0, dt); });
}

// Tokens that are placed by rank, in one block and at all.  Comparisons grow with the square, but there is one pass and one wait
// instead of a dozen a digit (the whole gradient, to 32768 rows: 32 tokens 9.6 -> 5.3 us, 128 10.9 -> 6.9, 400 16.3 -> 9.4, 1024 16.6 ->
// 13.4; 2048 18.8 by digits against 21.6; in one block and in eight 64 tokens 6.1 both, 128 6.9 | 7.2, 256 8.6 | 8.0).
constexpr size_t kRankAlone = 128, kRankTokens = 1024;

constexpr size_t kZeroBytes = 384 << 10;                             // that a block zeroes, about: 7.2 TB/s; with 113 KB and 3.6 MB 7.0 and 6.5

static int table_gradient(const nuna_embedding_grad_t& n, unsigned flags, void* stream)
{
    const size_t e = dtype_bytes(n.dtype), ge = dtype_bytes(n.grad_dtype);
    const bool accumulate = (flags & NUNA_GRAD_ACCUMULATE) != 0u;
    if (n.vocab_rows == 0 || (accumulate && n.tokens == 0)) return NUNA_OK;
    const EmbeddingWorkspace w = embedding_workspace(n.tokens, n.hidden, n.vocab_rows);
    const auto words = [&](size_t at) { return reinterpret_cast<unsigned*>(static_cast<char*>(n.workspace) + at); };
    SortArgs s = {};
    s.ids = n.ids, s.vocab_start = n.vocab_start, s.tokens = (unsigned)n.tokens, s.vocab_rows = (unsigned)n.vocab_rows;
    // Few tokens beside the table's rows: one block sorts, the others zero the table meanwhile, and only rows with a token are
    // visited (8192 tokens, a quarter of them in the slice of 32768 x 4096 f32: 94.7 us against 103; 1000 tokens, 50000 x 1024: 40 | 50;
    // 128 tokens, 4096 x 4096: 15 | 19).  With more tokens too much is written twice (8192 tokens to 32768 rows 116 | 114), or the
    // sort outlasts the stores (3 ns a token in one block).
    const bool vec = VectorRows{true}.rows(n.dout, n.hidden, n.dout_stride, e).rows(n.dtable, n.hidden, n.dtable_stride, ge).ok;
    const bool whole = n.dtable_stride == 0 || n.dtable_stride == n.hidden;
    const bool zero_first = !accumulate && whole && n.tokens && n.tokens * 4 <= n.vocab_rows && n.tokens <= 16384 &&
                            n.vocab_rows * n.hidden * ge >= n.tokens * (24 << 10);
    s.clear = !accumulate && !zero_first;
    for (int i = 0; i < 2; ++i) s.items[i] = reinterpret_cast<uint2*>(words(w.items[i]));
    s.begin = words(w.begin), s.end = words(w.end), s.count = words(w.count), s.cut = words(w.cut);
    unsigned bits = 1;
    while (bits < 32u && (n.vocab_rows - 1) >> bits) ++bits;
    s.passes = (bits + 9u) / 10u;                                    // digits of at most 10 bits: 1024 bins a warp fit a block's shared memory
    s.bits = (bits + s.passes - 1u) / s.passes;
    if (n.tokens) {
        Shape sort = sort_shape(n.tokens, 1u << s.bits);
        if (n.tokens <= (zero_first ? kRankTokens / 2 : kRankTokens)) {
            s.passes = 1;
            sort.grid = sort.cluster = n.tokens <= kRankAlone || zero_first ? 1 : 8;
            s.per = (unsigned)((n.tokens + sort.grid - 1) / sort.grid + 31) / 32 * 32;
            s.slices = std::max(1u, std::min(1024u / s.per, (unsigned)n.tokens / 16u));
            sort.block = std::max(s.per * s.slices, zero_first ? 1024u : 128u);
            sort.smem = (unsigned)(n.tokens * 2 + 3 + sort.block) * 4;
        }
        s.sorters = sort.grid;
        if (zero_first) {
            const uintptr_t begin = (uintptr_t)n.dtable, end = begin + n.vocab_rows * n.hidden * ge, from = std::min(end, (begin + 15) / 16 * 16);
            s.zero = reinterpret_cast<uint4*>(from), s.zero_vectors = (end - from) / 16;
            s.head = static_cast<uint16_t*>(n.dtable), s.head_halves = (unsigned)(from - begin) / 2;
            s.tail = reinterpret_cast<uint16_t*>(from + s.zero_vectors * 16), s.tail_halves = (unsigned)(end - from) % 16 / 2;
            s.sorters = 1;                                           // the sort is hidden: a cluster would only leave SMs without a block
            const size_t wave = (kSms - 1) * kZeroBytes;             // one of these blocks is resident on an SM
            const unsigned blocks = (kSms - 1) * (unsigned)std::max<size_t>(1, (n.vocab_rows * n.hidden * ge + wave / 2) / wave);
            sort = Shape{1 + blocks, kSortMaxWarps * 32u, s.per ? sort.smem : sort_smem(kSortMaxWarps, 1u << s.bits), 1};
        }
        constexpr int kMost = sort_smem(kSortMaxWarps, 1024);
        const bool wide = n.id_bytes == 8;
        int st = wide ? allow_sort<k_embedding_sort<long long>>(sort, kMost) : allow_sort<k_embedding_sort<int>>(sort, kMost);
        if (st != NUNA_OK) return st;
        if ((st = launch_op(wide ? k_embedding_sort<long long> : k_embedding_sort<int>, sort, flags, stream, s)) != NUNA_OK) return st;
    }

    TableArgs a = {};
    a.dout = n.dout, a.dtable = n.dtable;
    a.items = s.items[(s.passes & 1u) ^ 1u], a.begin = s.begin, a.end = n.tokens ? s.end : nullptr, a.count = s.count, a.cut = s.cut;
    a.part = reinterpret_cast<float*>(words(w.part));
    a.dout_stride = (n.dout_stride ? n.dout_stride : n.hidden) * e;
    a.dtable_stride = (n.dtable_stride ? n.dtable_stride : n.hidden) * ge;
    a.part_stride = (unsigned)part_stride(n.hidden), a.hidden = (unsigned)n.hidden, a.tokens = (unsigned)n.tokens;
    a.scale = n.scale, a.accumulate = accumulate, a.whole_sectors = !(((uintptr_t)n.dtable | a.dtable_stride) & 31u);
    a.parts = n.tokens > kRunPart ? (unsigned)((n.tokens + kRunPart - 1) / kRunPart) : 0u;
    a.by_position = accumulate || zero_first;
    a.rows = (unsigned)(a.by_position ? n.tokens : n.vocab_rows);
    return with_dtype(n.dtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const auto run = [&](auto rows, auto join, int per_thread) {
            const RowShape sh = row_shape(pieces(n.hidden, Elem<DT>::kElems, vec), per_thread);
            a.group = sh.group, a.chunks = sh.chunks;
            const unsigned groups = 256u / sh.group;
            const auto blocks = [&](unsigned long long units) { return (units + groups - 1) / groups; };
            // as many rows at once as leave each SM 32 warps' work
            a.each = 1;
            while (a.each < 8u && (unsigned long long)a.rows / (2u * a.each) * sh.chunks * (sh.group / 32u) >= 32ull * kSms) a.each *= 2u;
            const unsigned long long row_units = ((unsigned long long)a.rows + a.each - 1) / a.each * sh.chunks, part_units = (unsigned long long)a.parts * sh.chunks;
            if (row_units > kMaxUnits || part_units > kMaxUnits) return (int)NUNA_ERR_TOO_LARGE;
            a.row_units = (unsigned)row_units;
            a.part_blocks = (unsigned)blocks(part_units);
            const unsigned long long grid = a.part_blocks + blocks(row_units);
            if (grid > kMaxExtent) return (int)NUNA_ERR_TOO_LARGE;
            const int ok = launch_op(rows, Shape{(unsigned)grid, groups * sh.group, 0, 1}, flags, stream, a);
            if (ok != NUNA_OK || a.parts == 0u) return ok;
            const size_t most = (size_t)a.parts * ((n.hidden + kJoinColumns - 1) / kJoinColumns);   // there are no more cut runs than parts
            return launch_op(join, Shape{(unsigned)std::min<size_t>(most, 4 * kSms), 256, 0, 1}, flags, stream, a);
        };
        const auto typed = [&](auto gt) {
            constexpr int GT = decltype(gt)::value;
            if (vec) return run(k_embedding_rows<DT, GT, 2, true>, k_embedding_join<GT>, 2);
            return run(k_embedding_rows<DT, GT, 1, false>, k_embedding_join<GT>, 1);
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
