"""Tokens sorted by expert and back, and the gradients.  The sort is compared entry by entry with a stable sort on the host; with
small integers and weights that are powers of two the sums are exact, so rows are compared bit for bit."""
import numpy as np
import pytest
import torch

from operator_cases import DTYPES, GUARD, Rows, U, generator, guarded, half_step, integers, normal, smallest, within
from paper_2608_00867_b200 import binding as nb

pytestmark = pytest.mark.gpu

# (tokens, choices, experts of the slice, its first, all experts, capacity)
SORTS = [(1, 1, 1, 0, 1, 0), (1, 1, 1, 0, 1, 3), (5, 2, 3, 0, 3, 0), (5, 2, 3, 1, 7, 2), (32, 8, 64, 0, 64, 0), (33, 3, 17, 4, 60, 0),
         (300, 1, 8, 0, 8, 0), (257, 4, 256, 0, 256, 5), (1000, 8, 128, 0, 128, 0), (2047, 3, 24, 12, 48, 117), (4096, 8, 64, 0, 64, 512),
         (4097, 8, 1024, 0, 1024, 0), (8192, 8, 128, 0, 128, 0), (20001, 7, 31, 3, 40, 0), (40000, 8, 1000, 0, 1000, 300), (0, 4, 8, 0, 8, 0),
         (0, 4, 8, 0, 8, 4), (7, 0, 8, 0, 8, 0), (100, 2, 5, 50, 60, 0), (3, 2, 4, 0, 4, 100000)]
IDS = {"i32": torch.int32, "i64": torch.int64}


def sort_reference(ids, experts, first, capacity):
    """One expert after the other, in plain numpy."""
    pairs = ids.size
    rows = experts * capacity if capacity else pairs
    row, pair = np.full(pairs, -1, np.int32), np.full(rows, -1, np.int32)
    offsets, counts, at = np.zeros(experts + 1, np.int32), np.zeros(experts, np.int32), 0
    order = np.argsort(ids, kind="stable")
    bounds = np.searchsorted(ids[order], np.arange(first, first + experts + 1))
    for e in range(experts):
        mine = order[bounds[e]:bounds[e + 1]]
        counts[e], offsets[e] = mine.size, at
        mine = mine[:capacity] if capacity else mine
        row[mine] = at + np.arange(mine.size)
        pair[at:at + mine.size] = mine
        at += capacity if capacity else mine.size
    offsets[experts] = at
    return row, pair, offsets, counts


def make_experts(gen, tokens, topk, total, kind, skew=False):
    if skew:
        ids = (torch.rand(tokens, topk, generator=gen, device="cuda") ** 6 * total).long()
    else:
        ids = torch.randint(0, total, (tokens, topk), generator=gen, device="cuda")
    if tokens * topk > 8:
        flat = ids.view(-1)
        flat[3], flat[5], flat[8] = -1, torch.iinfo(IDS[kind]).max, torch.iinfo(IDS[kind]).min
    return ids.to(IDS[kind])


def plan_of(ids, tokens, topk, experts, first, capacity, counts=True, flags=0):
    pairs, rows = tokens * topk, experts * capacity if capacity else tokens * topk
    outs = [guarded(n, torch.int32, 77) for n in (pairs, rows, experts + 1, experts)]
    nb.nuna_expert_sort(ids, outs[0][0], outs[1][0], outs[2][0], tokens, topk, experts, counts=outs[3][0] if counts else None,
                        first_expert=first, capacity=capacity, id_bytes=ids.element_size(), flags=flags)
    torch.cuda.synchronize()
    for (got, whole), n in zip(outs, (pairs, rows, experts + 1, experts)):
        assert bool((whole[n:] == 77).all()), "written beyond the end"
    if not counts:
        assert bool((outs[3][0] == 77).all())
    return [got for got, _ in outs]


@pytest.mark.parametrize("kind", sorted(IDS))
@pytest.mark.parametrize("shape", SORTS)
def test_sort(shape, kind):
    tokens, topk, experts, first, total, capacity = shape
    for skew in (False, True):
        ids = make_experts(generator(*shape), tokens, topk, total, kind, skew)
        got = plan_of(ids, tokens, topk, experts, first, capacity)
        want = sort_reference(ids.cpu().numpy().reshape(-1).astype(np.int64), experts, first, capacity)
        for g, w, name in zip(got, want, ("row_of_pair", "pair_of_row", "offsets", "counts")):
            assert np.array_equal(g.cpu().numpy(), w), (shape, kind, skew, name)
        again = plan_of(ids, tokens, topk, experts, first, capacity, counts=False)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], again[:3]))


@pytest.mark.parametrize("pairs", [255, 256, 257, 8191, 8192, 8193, 16385, 32769, 65535, 65536, 65537, 131073, 500000])
def test_sort_at_the_sizes_where_its_shape_changes(pairs):
    ids = torch.randint(0, 61, (pairs, 1), generator=generator(pairs), device="cuda")
    row, pair, offsets, counts = plan_of(ids, pairs, 1, 61, 0, 0)
    order = torch.argsort(ids.view(-1), stable=True)
    assert torch.equal(pair.long(), order)
    assert torch.equal(row.long()[order], torch.arange(pairs, device="cuda"))
    assert torch.equal(counts.long(), torch.bincount(ids.view(-1), minlength=61)) and int(offsets[-1]) == pairs


def test_sort_of_one_expert_and_of_nobody():
    for fill, kept in ((3, 5000), (-1, 0), (8, 0)):
        ids = torch.full((1250, 4), fill, device="cuda")
        row, pair, offsets, counts = plan_of(ids, 1250, 4, 8, 0, 0)
        assert int((row >= 0).sum()) == kept and int(offsets[-1]) == kept and int(counts.sum()) == kept
        assert torch.equal(pair[:kept], torch.arange(kept, device="cuda", dtype=torch.int32)) and bool((pair[kept:] == -1).all())
        row, pair, offsets, counts = plan_of(ids, 1250, 4, 8, 0, 100)
        assert int((row >= 0).sum()) == min(kept, 100) and int((pair >= 0).sum()) == min(kept, 100) and int(counts.sum()) == kept


# (tokens, choices, hidden, experts, all experts, capacity)
MOVES = [(1, 1, 1, 1, 1, 0), (1, 8, 64, 8, 8, 0), (5, 2, 8, 3, 5, 0), (32, 8, 4096, 64, 64, 0), (33, 3, 31, 7, 20, 0), (40, 9, 1037, 6, 6, 0),
         (17, 5, 1032, 4, 4, 30), (100, 2, 520, 10, 20, 3), (64, 4, 8192, 16, 16, 0), (9, 3, 16392, 4, 4, 8), (700, 6, 264, 30, 60, 50),
         (3, 17, 100, 40, 40, 0), (3000, 2, 48, 8, 8, 0), (4, 3, 65537, 4, 4, 0),
         (500, 4, 2051, 16, 16, 0), (700, 3, 2051, 9, 16, 0), (1300, 3, 333, 8, 8, 0), (470, 3, 1031, 12, 30, 40)]


def setup(shape, pads, shift, dtype):
    tokens, topk, hidden, experts, total, capacity = shape
    gen = generator(*shape)
    ids = make_experts(gen, tokens, topk, total, "i64")
    row, pair, _, _ = plan_of(ids, tokens, topk, experts, 0, capacity)
    return gen, row, pair, pair.numel(), DTYPES[dtype]


def pair_rows(rows_buffer, row, topk):
    """[tokens][choices][hidden] in 64 bits, zeros for dropped pairs."""
    at = row.long().view(-1, topk)
    taken = rows_buffer.double()[at.clamp(min=0)] if rows_buffer.shape[0] else torch.zeros(*at.shape, rows_buffer.shape[1], device="cuda").double()
    return torch.where((at >= 0)[..., None], taken, torch.zeros_like(taken))


LAYOUTS = [(0, 0), (8, 0), (8, 8), (5, 0), (0, 1), (3, 7)]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("shape", MOVES)
def test_dispatch(shape, dtype):
    tokens, topk, hidden, experts, total, capacity = shape
    for pad, shift in LAYOUTS:
        gen, row, pair, rows, (tdt, code) = setup(shape, pad, shift, dtype)
        x = Rows(tokens, hidden, tdt, pad, shift, normal(gen, tokens, hidden))
        for zero in (False, True):
            out = Rows(rows, hidden, tdt, 2 * pad, shift)
            nb.nuna_expert_dispatch(x.flat, row, out.flat, tokens, topk, rows, hidden, pair_of_row=pair if zero else None, dtype=code,
                                    x_stride=x.stride, out_stride=out.stride)
            torch.cuda.synchronize()
            full = pair >= 0
            assert torch.equal(out.v[full], x.v[pair[full].long() // topk]), (shape, dtype, pad, shift)
            assert bool((out.v[~full] == (0.0 if zero else GUARD)).all()), (shape, dtype, pad, shift, zero)
            assert out.untouched() and x.untouched()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("shape", MOVES)
def test_combine(shape, dtype):
    tokens, topk, hidden, experts, total, capacity = shape
    for pad, shift in LAYOUTS:
        gen, row, pair, rows, (tdt, code) = setup(shape, pad, shift, dtype)
        for exact in (True, False):
            src = Rows(rows, hidden, tdt, pad, shift, integers(gen, -8, 8, rows, hidden) if exact else normal(gen, rows, hidden))
            weights = 2.0 ** integers(gen, -3, 0, tokens, topk) if exact else torch.rand(tokens, topk, generator=gen, device="cuda")
            src.v[pair < 0] = float("nan")                             # rows that no pair has are not looked at
            weights.view(-1)[row < 0] = float("nan")                   # nor the weights of dropped pairs
            for w in (weights, None):
                y = Rows(tokens, hidden, tdt, 2 * pad, shift)
                nb.nuna_expert_combine(src.flat, row, y.flat, tokens, topk, rows, hidden, weights=w, dtype=code, src_stride=src.stride,
                                       y_stride=y.stride)
                torch.cuda.synchronize()
                parts = pair_rows(src.v, row, topk)
                if w is not None:
                    parts = parts * torch.where(row.view(-1, topk) >= 0, w, torch.zeros_like(w)).double()[..., None]
                want, what = parts.sum(1), (shape, dtype, pad, shift, w is not None)
                if exact:
                    assert torch.equal(y.v.double(), want.to(tdt).double()), what
                else:
                    bound = (topk + 1) * U * parts.abs().sum(1)        # a rounding for each of the sum's terms
                    within(y.v, want, bound + half_step(tdt) * (want.abs() + bound) + smallest(tdt), what)
                nobody = (row.view(-1, topk) < 0).all(-1)
                assert bool((y.v[nobody] == 0).all()) and y.untouched()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("shape", MOVES)
def test_combine_backward(shape, dtype):
    tokens, topk, hidden, experts, total, capacity = shape
    for pad, shift in LAYOUTS:
        gen, row, pair, rows, (tdt, code) = setup(shape, pad, shift, dtype)
        for exact in (True, False):
            make = (lambda *s: integers(gen, -8, 8, *s)) if exact else (lambda *s: normal(gen, *s))
            src, dy = Rows(rows, hidden, tdt, pad, shift, make(rows, hidden)), Rows(tokens, hidden, tdt, pad, shift, make(tokens, hidden))
            weights = 2.0 ** integers(gen, -3, 0, tokens, topk) if exact else torch.rand(tokens, topk, generator=gen, device="cuda")
            src.v[pair < 0] = float("nan")
            weights.view(-1)[row < 0] = float("nan")
            for zero, dots in ((False, True), (True, True), (True, False)):
                dsrc = Rows(rows, hidden, tdt, 2 * pad, shift)
                dw, dw_all = guarded(tokens * topk, torch.float32)
                nb.nuna_expert_combine_backward(dy.flat, src.flat if dots else None, weights, row, dsrc.flat, dw if dots else None, tokens, topk,
                                                rows, hidden, pair_of_row=pair if zero else None, dtype=code, dy_stride=dy.stride,
                                                src_stride=src.stride, dsrc_stride=dsrc.stride)
                torch.cuda.synchronize()
                what = (shape, dtype, pad, shift, exact, zero, dots)
                full = pair >= 0
                of = pair[full].long()
                want = dy.v[of // topk].double() * weights.view(-1)[of].double()[:, None]
                if exact:
                    assert torch.equal(dsrc.v[full].double(), want.to(tdt).double()), what
                else:
                    within(dsrc.v[full], want, (half_step(tdt) + 2 * U) * want.abs() + smallest(tdt), what)
                assert bool((dsrc.v[~full] == (0.0 if zero else GUARD)).all()) and dsrc.untouched(), what
                if dots:
                    terms = pair_rows(src.v, row, topk) * dy.v.double()[:, None]
                    total64 = terms.sum(-1).reshape(-1)
                    # integers up to 64, at most 65537 of them: exact in binary32 (the sum stays below 2^23); otherwise every addition
                    # rounds, of which a thread makes hidden / 32 in a row at most and the group ten more
                    bound = torch.zeros_like(total64) if exact else (hidden / 32 + 16) * U * terms.abs().sum(-1).reshape(-1)
                    within(dw, total64, bound, what)
                    assert bool((dw[row < 0] == 0).all()), what
                assert bool((dw_all[tokens * topk if dots else 0:] == GUARD).all()), what


def test_maps_that_name_no_row_are_dropped():
    """Entries beyond the rows that the call has are dropped pairs, so a map and a buffer that do not belong together stay harmless."""
    tokens, topk, hidden, rows = 6, 2, 64, 5
    row = torch.tensor([0, 5, 4, -1, 2 ** 31 - 1, 1, -2 ** 31, 2, 3, 100, 7, 6], dtype=torch.int32, device="cuda")
    kept = ((row >= 0) & (row < rows)).view(tokens, topk)
    x, src = normal(generator(1), tokens, hidden), integers(generator(2), -8, 8, rows, hidden)
    out = Rows(rows, hidden, torch.float32)
    nb.nuna_expert_dispatch(x, row, out.flat, tokens, topk, rows, hidden, dtype=nb.NUNA_F32)
    assert out.untouched() and all(torch.equal(out.v[row[p]], x[p // topk]) for p in range(12) if kept.view(-1)[p])
    y = torch.empty(tokens, hidden, device="cuda")
    nb.nuna_expert_combine(src, row, y, tokens, topk, rows, hidden, dtype=nb.NUNA_F32)
    want = torch.where(kept[..., None], src[row.view(tokens, topk).long().clamp(0, rows - 1)], torch.zeros((), device="cuda")).sum(1)
    assert torch.equal(y, want)
    dsrc, dw = Rows(rows, hidden, torch.float32), torch.empty(tokens * topk, device="cuda")
    nb.nuna_expert_combine_backward(x, src, torch.ones(12, device="cuda"), row, dsrc.flat, dw, tokens, topk, rows, hidden, dtype=nb.NUNA_F32)
    assert dsrc.untouched() and bool((dw.view(tokens, topk)[~kept] == 0).all())
    assert all(torch.equal(dsrc.v[row[p]], x[p // topk]) for p in range(12) if kept.view(-1)[p])


def test_gradients_against_differences():
    """combine(dispatch(x), weights) with an expert's factor on every row: its slopes in x and in the weights."""
    gen = generator(3)
    tokens, topk, hidden, experts = 4, 2, 24, 3
    ids = torch.randint(0, experts, (tokens, topk), generator=gen, device="cuda")
    row, pair, offsets, _ = plan_of(ids, tokens, topk, experts, 0, 0)
    rows = tokens * topk
    factor = torch.tensor([0.5, -1.5, 2.0], device="cuda")[ids.view(-1)[pair.long()]][:, None]
    x, w, up = normal(gen, tokens, hidden), torch.rand(tokens, topk, generator=gen, device="cuda"), normal(gen, tokens, hidden)
    f32 = dict(dtype=nb.NUNA_F32)
    out, dsrc, dx, dw = torch.empty(rows, hidden, device="cuda"), torch.empty(rows, hidden, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    nb.nuna_expert_dispatch(x, row, out, tokens, topk, rows, hidden, **f32)
    src = out * factor
    nb.nuna_expert_combine_backward(up, src, w, row, dsrc, dw, tokens, topk, rows, hidden, **f32)
    dout = dsrc * factor
    nb.nuna_expert_combine(dout, row, dx, tokens, topk, rows, hidden, **f32)

    def loss(x, w):
        parts = (x[pair.long() // topk] * factor.double())[row.long()].view(tokens, topk, hidden)
        return ((parts * w[..., None]).sum(1) * up.double()).sum()

    h = 1e-4
    for name, got in (("x", dx), ("w", dw)):
        args = {"x": x.double(), "w": w.double()}
        for i in range(got.numel()):
            step = torch.zeros(got.numel(), dtype=torch.float64, device="cuda")
            step[i] = h
            step = step.view(got.shape)
            slope = (loss(**{**args, name: args[name] + step}) - loss(**{**args, name: args[name] - step})) / (2 * h)
            # the loss is bilinear, so the difference is exact but for 64-bit rounding; the kernels round some 50 terms of size 2
            assert abs(float(slope) - float(got.view(-1)[i])) < 1e-4, (name, i)


def test_captured_and_replayed():
    tokens, topk, hidden, experts = 96, 4, 1024, 16
    gen = generator(8)
    ids = torch.randint(0, experts, (tokens, topk), generator=gen, device="cuda")
    x = integers(gen, -4, 4, tokens, hidden).bfloat16()
    weights = torch.full((tokens, topk), 0.25, device="cuda")
    for flags in (0, nb.NUNA_LAUNCH_PDL):
        row, pair = torch.zeros(tokens * topk, dtype=torch.int32, device="cuda"), torch.zeros(tokens * topk, dtype=torch.int32, device="cuda")
        offsets = torch.zeros(experts + 1, dtype=torch.int32, device="cuda")
        out, y = torch.zeros(tokens * topk, hidden, dtype=torch.bfloat16, device="cuda"), torch.zeros_like(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            nb.nuna_expert_sort(ids, row, pair, offsets, tokens, topk, experts, flags=flags)
            nb.nuna_expert_dispatch(x, row, out, tokens, topk, tokens * topk, hidden, flags=flags)
            nb.nuna_expert_combine(out, row, y, tokens, topk, tokens * topk, hidden, weights=weights, flags=flags)
        for _ in range(3):
            ids.random_(0, experts, generator=gen)                     # other routes, the same graph
            y.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, x)
            assert torch.equal(pair.long(), torch.argsort(ids.view(-1), stable=True))


def test_tensors_that_are_too_short_are_refused():
    ids = torch.zeros(4, 2, dtype=torch.int64, device="cuda")
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    call = lambda *a, **k: nb.nuna_expert_sort(*a, check=False, **k)
    assert call(ids, i32(8), i32(8), i32(4), 4, 2, 3) == nb.NUNA_OK
    for bad in ((ids.int(), i32(8), i32(8), i32(4)), (ids, i32(7), i32(8), i32(4)), (ids, i32(8), i32(7), i32(4)), (ids, i32(8), i32(8), i32(3))):
        assert call(*bad, 4, 2, 3) == nb.NUNA_ERR_INVALID_ARG
    assert call(ids, i32(8), i32(8), i32(4), 4, 2, 3, capacity=3) == nb.NUNA_ERR_INVALID_ARG         # nine rows
    assert call(ids, i32(8), i32(9), i32(4), 4, 2, 3, capacity=3) == nb.NUNA_OK
    x, out = torch.zeros(4, 8, device="cuda"), torch.zeros(8, 8, device="cuda")
    assert nb.nuna_expert_dispatch(x[1:], i32(8), out, 4, 2, 8, 8, dtype=nb.NUNA_F32, check=False) == nb.NUNA_ERR_INVALID_ARG
    assert nb.nuna_expert_combine(out, i32(8), x, 4, 2, 8, 8, weights=torch.zeros(7, device="cuda"), dtype=nb.NUNA_F32,
                                  check=False) == nb.NUNA_ERR_INVALID_ARG
    torch.cuda.synchronize()
