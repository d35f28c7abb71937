// The memory that an operator's call names: one entry for every pointer of its argument structure, in the structure's
// order.  The library refuses calls whose ranges overlap by it, and the Python binding calls whose tensors are too small.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/nuna.h"

namespace nuna {

constexpr size_t kMaxExtent = (size_t)0x7FFFFFFF;        // rows, tokens, table rows
constexpr size_t kMaxHidden = (size_t)1 << 30;           // elements in a row: a 32-bit index may step beyond its end
constexpr size_t kMaxMatrixBytes = (size_t)1 << 46;
constexpr int kMaxSpans = 10;

struct Span {
    const void* at = nullptr;
    size_t bytes = 0;                // from the first byte to the last
    size_t stride = 0;               // bytes between rows
    unsigned align = 1;
    bool written = false;
    bool required = false;
};

struct Spans {
    Span v[kMaxSpans];
    int n = 0;
    int status = NUNA_OK;

    // rows of `elems` elements of `size` bytes, `stride` elements apart (0: elems)
    void matrix(const void* at, size_t rows, size_t elems, size_t stride, size_t size, bool written, bool required = true)
    {
        if (elems > kMaxHidden) fail(NUNA_ERR_TOO_LARGE);
        extent(at, rows, elems, stride, size, written, required);
    }
    void array(const void* at, size_t elems, size_t size, bool written, bool required = true) { extent(at, 1, elems, 0, size, written, required); }
    // `bytes` (a multiple of 32) that kernels write 32 bytes at a time
    void workspace(const void* at, size_t bytes, bool required) { array(at, bytes / 32, 32, true, required); }
    void extent(const void* at, size_t rows, size_t elems, size_t stride, size_t size, bool written, bool required)
    {
        Span& s = v[n++];
        s.at = at;
        s.align = (unsigned)size;
        s.written = written;
        s.required = required;
        if (stride == 0) stride = elems;
        if (rows > kMaxExtent || elems > kMaxExtent || stride > kMaxMatrixBytes) {
            fail(NUNA_ERR_TOO_LARGE);
            return;
        }
        if (stride < elems) fail(NUNA_ERR_INVALID_ARG);
        if (rows == 0 || elems == 0) return;
        const unsigned __int128 bytes = ((unsigned __int128)(rows - 1) * stride + elems) * size;
        if (bytes > kMaxMatrixBytes) {
            fail(NUNA_ERR_TOO_LARGE);
            return;
        }
        s.stride = stride * size;
        s.bytes = (size_t)bytes;
    }
    void fail(int st)
    {
        if (status == NUNA_OK) status = st;
    }
};

// ---- workspaces --------------------------------------------------------------------------------------
//
// Layer norm: the row blocks' shares of dweight and dbias, [blocks][2][hidden] in binary32.
constexpr size_t kNormBlocks = 148;                      // at most one block per SM sums over rows
inline size_t norm_blocks(size_t rows) { return rows < kNormBlocks ? rows : kNormBlocks; }
inline size_t layernorm_workspace_bytes(size_t rows, size_t hidden)
{
    if (rows > kMaxExtent || hidden > kMaxExtent) return 0;
    return norm_blocks(rows) * 2 * ((hidden + 3) / 4 * 4) * sizeof(float);
}

// Embedding: the tokens with their rows, in the order of the rows (two buffers, between which the sort's passes alternate),
// where each row's run of tokens begins and ends, how many tokens have a row and how many runs are cut, which those are, and
// their shares: two rows for every kRunPart positions.
constexpr size_t kRunPart = 32;
inline size_t part_stride(size_t hidden) { return (hidden + 7) / 8 * 8; }
struct EmbeddingWorkspace {
    size_t items[2], begin, end, count, cut, part, bytes;
};
inline EmbeddingWorkspace embedding_workspace(size_t tokens, size_t hidden, size_t vocab_rows)
{
    EmbeddingWorkspace w = {};
    if (tokens > kMaxExtent || hidden > kMaxExtent || vocab_rows > kMaxExtent) return w;
    const auto take = [&](size_t n) {
        const size_t at = w.bytes;
        w.bytes += (n * 4 + 255) / 256 * 256;
        return at;
    };
    w.items[0] = take(2 * tokens), w.items[1] = take(2 * tokens);
    w.begin = take(vocab_rows), w.end = take(vocab_rows), w.count = take(2);
    w.cut = take(tokens > kRunPart ? tokens / kRunPart : 0);
    w.part = take(tokens > kRunPart ? (tokens + kRunPart - 1) / kRunPart * 2 * part_stride(hidden) : 0);
    return w;
}

inline size_t dtype_bytes(int dtype) { return dtype == NUNA_F32 ? 4 : 2; }
inline bool is_dtype(int dtype) { return dtype == NUNA_BF16 || dtype == NUNA_F16 || dtype == NUNA_F32; }
inline size_t id_size(int id_bytes) { return id_bytes == 4 ? 4 : 8; }
// pairs of (token, choice), or something too large
inline size_t pair_count(size_t tokens, size_t topk)
{
    const unsigned __int128 n = (unsigned __int128)tokens * topk;
    return n > kMaxExtent ? kMaxExtent + 1 : (size_t)n;
}

inline Spans spans_of(const nuna_layernorm_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype), p = dtype_bytes(a.param_dtype);
    s.matrix(a.x, a.rows, a.hidden, a.x_stride, e, false);
    s.matrix(a.residual, a.rows, a.hidden, a.residual_stride, e, false, false);
    s.array(a.weight, a.hidden, p, false, false);
    s.array(a.bias, a.hidden, p, false, false);
    s.matrix(a.summed, a.rows, a.hidden, a.summed_stride, e, true, false);
    s.matrix(a.y, a.rows, a.hidden, a.y_stride, e, true);
    s.array(a.mean, a.rows, 4, true, false);
    s.array(a.rstd, a.rows, 4, true, false);
    return s;
}

inline Spans spans_of(const nuna_layernorm_grad_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype), p = dtype_bytes(a.param_dtype);
    s.matrix(a.dy, a.rows, a.hidden, a.dy_stride, e, false);
    s.matrix(a.x, a.rows, a.hidden, a.x_stride, e, false);
    s.array(a.mean, a.rows, 4, false);
    s.array(a.rstd, a.rows, 4, false);
    s.array(a.weight, a.hidden, p, false, false);
    s.matrix(a.dsummed, a.rows, a.hidden, a.dsummed_stride, e, false, false);
    s.matrix(a.dx, a.rows, a.hidden, a.dx_stride, e, true);
    s.array(a.dweight, a.hidden, p, true, false);
    s.array(a.dbias, a.hidden, p, true, false);
    s.array(a.workspace, (a.dweight || a.dbias) ? layernorm_workspace_bytes(a.rows, a.hidden) / 16 : 0, 16, true, false);
    return s;
}

inline Spans spans_of(const nuna_embedding_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype);
    s.array(a.ids, a.tokens, id_size(a.id_bytes), false);
    s.matrix(a.table, a.vocab_rows, a.hidden, a.table_stride, e, false, a.vocab_rows != 0);
    s.matrix(a.out, a.tokens, a.hidden, a.out_stride, e, true);
    return s;
}

inline Spans spans_of(const nuna_embedding_grad_t& a)
{
    Spans s;
    s.array(a.ids, a.tokens, id_size(a.id_bytes), false, a.tokens != 0);
    s.matrix(a.dout, a.tokens, a.hidden, a.dout_stride, dtype_bytes(a.dtype), false, a.tokens != 0);
    s.matrix(a.dtable, a.vocab_rows, a.hidden, a.dtable_stride, dtype_bytes(a.grad_dtype), true);
    s.workspace(a.workspace, embedding_workspace(a.tokens, a.hidden, a.vocab_rows).bytes, a.tokens != 0);
    return s;
}

inline Spans spans_of(const nuna_expert_sort_t& a)
{
    Spans s;
    const size_t pairs = pair_count(a.tokens, a.topk), rows = a.capacity ? pair_count(a.num_experts, a.capacity) : pairs;
    s.array(a.experts, pairs, id_size(a.id_bytes), false, pairs != 0);
    s.array(a.row_of_pair, pairs, 4, true, pairs != 0);
    s.array(a.pair_of_row, rows, 4, true, rows != 0);
    s.array(a.offsets, a.num_experts + 1, 4, true);
    s.array(a.counts, a.num_experts, 4, true, false);
    return s;
}

inline Spans spans_of(const nuna_expert_dispatch_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype), pairs = pair_count(a.tokens, a.topk);
    s.matrix(a.x, a.tokens, a.hidden, a.x_stride, e, false, pairs != 0);
    s.array(a.row_of_pair, pairs, 4, false, pairs != 0);
    s.array(a.pair_of_row, a.rows, 4, false, false);
    s.matrix(a.out, a.rows, a.hidden, a.out_stride, e, true, a.rows != 0);
    return s;
}

inline Spans spans_of(const nuna_expert_combine_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype), pairs = pair_count(a.tokens, a.topk);
    s.matrix(a.src, a.rows, a.hidden, a.src_stride, e, false, a.rows != 0);
    s.array(a.row_of_pair, pairs, 4, false, pairs != 0);
    s.array(a.weights, pairs, 4, false, false);
    s.matrix(a.y, a.tokens, a.hidden, a.y_stride, e, true);
    return s;
}

inline Spans spans_of(const nuna_expert_combine_grad_t& a)
{
    Spans s;
    const size_t e = dtype_bytes(a.dtype), pairs = pair_count(a.tokens, a.topk);
    s.matrix(a.dy, a.tokens, a.hidden, a.dy_stride, e, false, pairs != 0);
    s.matrix(a.src, a.rows, a.hidden, a.src_stride, e, false, a.rows != 0 && a.dweights);
    s.array(a.weights, pairs, 4, false, pairs != 0);
    s.array(a.row_of_pair, pairs, 4, false, pairs != 0);
    s.array(a.pair_of_row, a.rows, 4, false, false);
    s.matrix(a.dsrc, a.rows, a.hidden, a.dsrc_stride, e, true, a.rows != 0);
    s.array(a.dweights, pairs, 4, true, false);
    return s;
}

}  // namespace nuna
