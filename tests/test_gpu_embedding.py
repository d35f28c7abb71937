"""Embedding lookup over a slice of the vocabulary and its gradient.  Small integers and scales that are powers of two make every
sum exact, so most results are compared bit for bit; random values against 64 bits."""
import pytest
import torch

from operator_cases import DTYPES, GUARD, Rows, U, generator, half_step, integers, normal, smallest, within
from paper_2608_00867_b200 import binding as nb

pytestmark = pytest.mark.gpu

# (tokens, hidden, rows of the slice, its start, the vocabulary)
SHAPES = [(1, 1, 1, 0, 1), (1, 8, 5, 0, 5), (3, 7, 4, 2, 9), (64, 64, 16, 0, 16), (65, 64, 16, 0, 16), (63, 33, 1, 0, 1), (129, 40, 1, 0, 2),
          (1000, 256, 37, 100, 200), (257, 1024, 1000, 0, 1000), (500, 1037, 300, 17, 400), (2500, 520, 3, 0, 3), (300, 8192, 50, 0, 64),
          (8193, 72, 1025, 0, 1025), (20000, 24, 131072, 0, 131072), (70000, 16, 2049, 5, 3000), (37, 16392, 9, 0, 9), (4, 65537, 3, 0, 4),
          (150000, 8, 40000, 0, 40000), (300, 520, 5000, 100, 6000), (5000, 4096, 30000, 0, 60000), (16390, 40, 70000, 0, 70000),
          (100, 1001, 4000, 5, 5000), (128, 24, 77, 3, 90), (513, 1001, 16000, 0, 16000), (512, 72, 300, 0, 300), (1024, 33, 5000, 9, 5100),
          (1025, 40, 2000, 0, 2000)]
IDS = {"i32": torch.int32, "i64": torch.int64}


def make_ids(gen, tokens, vocab, kind, outside=True):
    """Half of the tokens share a few ids; some are negative or beyond every vocabulary."""
    few = torch.randint(0, min(vocab, 3), (tokens,), generator=gen, device="cuda")
    many = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
    ids = torch.where(torch.rand(tokens, generator=gen, device="cuda") < 0.5, few, many)
    if outside and tokens > 8:
        ids[3], ids[5], ids[7] = -1, torch.iinfo(IDS[kind]).max, torch.iinfo(IDS[kind]).min
    return ids.to(IDS[kind])


def run_forward(tokens, hidden, rows, start, vocab, dtype, kind, scale=0.5, pad=0, shift=0):
    tdt, code = DTYPES[dtype]
    gen = generator(tokens, hidden, rows, pad)
    ids = make_ids(gen, tokens, vocab, kind)
    table = Rows(rows, hidden, tdt, pad, shift, normal(gen, rows, hidden))
    out = Rows(tokens, hidden, tdt, 2 * pad, shift)
    nb.nuna_embedding_forward(ids, table.flat, out.flat, tokens, hidden, rows, vocab_start=start, scale=scale, dtype=code,
                              id_bytes=ids.element_size(), table_stride=table.stride, out_stride=out.stride)
    torch.cuda.synchronize()
    at = ids.long() - start
    mine = (ids.long() >= start) & (at < rows) & (at >= 0)
    want = torch.zeros(tokens, hidden, dtype=torch.float64, device="cuda")
    want[mine] = table.v[at[mine]].double() * torch.tensor(scale).double().item()
    what = (tokens, hidden, rows, dtype, kind, scale, pad, shift)
    # one rounding of the product to binary32, one to the type
    within(out.v, want, (half_step(tdt) + 2 * U) * want.abs() + smallest(tdt), what)
    if scale in (1.0, 0.5):
        assert torch.equal(out.v.double(), want.to(tdt).double()), what
    assert bool((out.v[~mine] == 0).all()) and out.untouched() and table.untouched(), what


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype):
    for kind in IDS:
        run_forward(*shape, dtype, kind)
    run_forward(*shape, dtype, "i64", scale=1.0)
    run_forward(*shape, dtype, "i64", scale=22.627417)
    for pad, shift in ((8, 0), (8, 8), (5, 0), (0, 1), (3, 7)):
        run_forward(*shape, dtype, "i32", pad=pad, shift=shift)


def run_backward(tokens, hidden, rows, start, vocab, dtype, grad, kind, scale=0.5, pad=0, shift=0, accumulate=False, exact=True, same=None):
    tdt, code = DTYPES[dtype]
    gdt, gcode = DTYPES[grad]
    gen = generator(tokens, hidden, rows, pad, accumulate, exact)
    ids = make_ids(gen, tokens, vocab, kind) if same is None else torch.full((tokens,), same, dtype=IDS[kind], device="cuda")
    # integers up to 4 in size: sums of 70000 of them stay below 2^24, so binary32 holds them exactly in any order
    values = integers(gen, -4, 4, tokens, hidden) if exact else normal(gen, tokens, hidden)
    dout = Rows(tokens, hidden, tdt, pad, shift, values)
    old = integers(gen, -8, 8, rows, hidden) if accumulate else None
    dtable = Rows(rows, hidden, gdt, 2 * pad, shift, old)
    need = nb.nuna_embedding_workspace(tokens, hidden, rows)
    ws = torch.full((need + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    nb.nuna_embedding_backward(ids, dout.flat, dtable.flat, tokens, hidden, rows, workspace=ws[:need], vocab_start=start, scale=scale,
                               dtype=code, grad_dtype=gcode, id_bytes=ids.element_size(), dout_stride=dout.stride,
                               dtable_stride=dtable.stride, flags=nb.NUNA_GRAD_ACCUMULATE if accumulate else 0)
    torch.cuda.synchronize()
    at = ids.long() - start
    mine = (ids.long() >= start) & (at < rows) & (at >= 0)
    want = torch.zeros(rows, hidden, dtype=torch.float64, device="cuda").index_add_(0, at[mine], dout.v[mine].double()) * scale
    what = (tokens, hidden, rows, dtype, grad, kind, pad, shift, accumulate)
    if exact:
        total = want + old.double() if accumulate else want
        assert torch.equal(dtable.v.double(), total.to(gdt).double()), what
    else:
        # at most 32 additions in a part and as many as there are parts, of values whose absolute sum is `size`
        size = torch.zeros_like(want).index_add_(0, at[mine], dout.v[mine].double().abs()) * scale
        bound = (32 + tokens // 32 + 4) * U * size
        within(dtable.v, want, bound + half_step(gdt) * (want.abs() + bound) + smallest(gdt), what)
    if accumulate:
        present = torch.zeros(rows, dtype=torch.bool, device="cuda").index_fill_(0, at[mine], True)
        assert torch.equal(dtable.v[~present], old.to(gdt)[~present]), what
    assert dtable.untouched() and dout.untouched() and bool((ws[need:] == 0x7F).all()), what
    return dtable.v


@pytest.mark.parametrize("dtype,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, dtype, grad):
    for kind in IDS:
        run_backward(*shape, dtype, grad, kind)
        run_backward(*shape, dtype, grad, kind, accumulate=True)
    run_backward(*shape, dtype, grad, "i64", exact=False)
    for pad, shift in ((8, 0), (8, 8), (5, 0), (0, 1), (3, 7)):
        run_backward(*shape, dtype, grad, "i32", pad=pad, shift=shift)
        run_backward(*shape, dtype, grad, "i32", pad=pad, shift=shift, accumulate=True)


@pytest.mark.parametrize("tokens", [1, 2, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 191, 1000, 4096])
def test_all_tokens_are_one_id(tokens):
    for same in (0, 6):
        run_backward(tokens, 48, 7, 0, 7, "bf16", "f32", "i64", same=same)
        run_backward(tokens, 48, 7, 0, 7, "bf16", "f32", "i64", same=same, accumulate=True)
        run_backward(tokens, 31, 7, 0, 7, "f16", "f16", "i32", same=same)
    run_backward(tokens, 48, 7, 0, 7, "bf16", "f32", "i64", same=-1)          # nobody's: every row is written with zeros
    run_backward(tokens, 48, 7, 0, 7, "bf16", "f32", "i64", same=7, accumulate=True)


@pytest.mark.parametrize("lengths", [[64, 64, 64], [65, 63, 64], [1, 64, 65, 1], [63, 65, 128], [200, 1, 1, 1, 70, 64, 129], [32, 65, 31, 65],
                                     [32, 32, 33], [33, 31, 32, 33, 1, 30], [1, 33, 33, 33], [5, 32, 33, 26, 33], [500, 31, 33, 900]])
def test_runs_that_end_inside_and_between_the_parts(lengths):
    """Runs of given lengths, in the order of their ids: cut and whole ones, at and around the places where runs are cut."""
    ids = torch.cat([torch.full((n,), i) for i, n in enumerate(lengths)]).cuda()
    order = torch.randperm(ids.numel(), generator=generator(1, len(lengths)), device="cuda")
    ids = ids[order]
    dout = integers(generator(2), -8, 8, ids.numel(), 40).bfloat16()
    got = torch.full((len(lengths), 40), GUARD, device="cuda")
    ws = torch.empty(nb.nuna_embedding_workspace(ids.numel(), 40, len(lengths)), dtype=torch.uint8, device="cuda")
    nb.nuna_embedding_backward(ids, dout, got, ids.numel(), 40, len(lengths), workspace=ws, grad_dtype=nb.NUNA_F32)
    assert torch.equal(got, torch.zeros_like(got).index_add_(0, ids, dout.float()))


def test_the_same_call_gives_the_same_bits():
    for shape in ((5000, 520, 40, 0, 40), (3000, 129, 700, 0, 700)):
        first = run_backward(*shape, "bf16", "f32", "i64", exact=False)
        for _ in range(3):
            assert torch.equal(first, run_backward(*shape, "bf16", "f32", "i64", exact=False))


@pytest.mark.parametrize("first,second,want", [([1, 0, -1], [0, 1, -1], [0.0, 0.0]), ([1, -1, 0], [0, 1, -1], [1.0, 0.0])])
def test_the_sum_is_in_the_tokens_order(first, second, want):
    """Sums of 2^24 (1), 1 (0) and -2^24 (-1), in which 2^24 + 1 rounds to 2^24 (a tie, to even): a one is lost unless it comes last."""
    values = [(1.0, 2.0 ** 24, -2.0 ** 24)[i] for i in first + second]
    dout = torch.tensor(values, device="cuda")[:, None].contiguous()
    ids = torch.tensor([4, 4, 4, 2, 2, 2], device="cuda")
    got = torch.empty(5, 1, device="cuda")
    ws = torch.empty(nb.nuna_embedding_workspace(6, 1, 5), dtype=torch.uint8, device="cuda")
    nb.nuna_embedding_backward(ids, dout, got, 6, 1, 5, workspace=ws, dtype=nb.NUNA_F32, grad_dtype=nb.NUNA_F32)
    assert got[:, 0].tolist() == [0, 0, want[1], 0, want[0]]


def test_not_finite_values_stay_in_their_rows():
    ids = torch.tensor([0, 1, 2, 3, -1, 9], device="cuda")
    table = torch.tensor([[1.0], [float("inf")], [float("nan")], [2.0]], device="cuda")
    out = torch.empty(6, 1, device="cuda")
    nb.nuna_embedding_forward(ids, table, out, 6, 1, 4, dtype=nb.NUNA_F32, scale=2.0)
    assert out[:2, 0].tolist() == [2.0, float("inf")] and bool(torch.isnan(out[2])) and out[3:, 0].tolist() == [4.0, 0.0, 0.0]
    dout = torch.tensor([[1.0], [float("inf")], [1.0], [1.0], [float("nan")], [float("nan")]], device="cuda")
    grad = torch.empty(4, 1, device="cuda")
    ws = torch.empty(nb.nuna_embedding_workspace(6, 1, 4), dtype=torch.uint8, device="cuda")
    nb.nuna_embedding_backward(ids, dout, grad, 6, 1, 4, workspace=ws, dtype=nb.NUNA_F32, grad_dtype=nb.NUNA_F32)
    assert grad[:, 0].tolist() == [1.0, float("inf"), 1.0, 1.0]               # what no row of the slice has is not read


def test_zeros_of_no_row_are_not_scaled():
    table = torch.ones(2, 24, device="cuda")
    for scale, want in ((float("inf"), float("inf")), (0.0, 0.0), (float("nan"), float("nan"))):
        out = torch.full((3, 24), GUARD, device="cuda")
        nb.nuna_embedding_forward(torch.tensor([1, 2, -5], device="cuda"), table, out, 3, 24, 2, scale=scale, dtype=nb.NUNA_F32)
        assert bool((out[1:] == 0).all()) and torch.equal(out[0], torch.full_like(out[0], want)) or want != want and bool(torch.isnan(out[0]).all())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("hidden", [1, 24, 37, 1032])
@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan"), 0.0, 3.0])
def test_rows_of_no_token_are_zeros_at_any_scale(scale, hidden, dtype):
    tdt, code = DTYPES[dtype]
    for tokens in (3, 3000):
        ids = torch.tensor([1, 2, -5], device="cuda").repeat(tokens // 3)
        out = torch.full((tokens, hidden), GUARD, dtype=tdt, device="cuda")
        nb.nuna_embedding_forward(ids, torch.ones(2, hidden, dtype=tdt, device="cuda"), out, tokens, hidden, 2, scale=scale, dtype=code)
        assert bool((out[ids != 1] == 0).all())
        if scale != scale:
            assert bool(torch.isnan(out[ids == 1]).all())
        else:
            assert bool((out[ids == 1] == scale).all())


def test_the_first_call_of_a_process_may_be_captured():
    code = """
import torch
from paper_2608_00867_b200 import binding as nb
f32 = dict(dtype=nb.NUNA_F32)
i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
tokens, hidden, rows = 20000, 256, 300
ids = torch.arange(tokens, device="cuda") % rows
table, out, grad = torch.randn(rows, hidden, device="cuda"), torch.zeros(tokens, hidden, device="cuda"), torch.zeros(rows, hidden, device="cuda")
y, mean, rstd, dx, dw = torch.zeros_like(out), torch.zeros(tokens, device="cuda"), torch.zeros(tokens, device="cuda"), torch.zeros_like(out), torch.zeros(hidden, device="cuda")
row, pair, offsets, moved, back = i32(tokens), i32(tokens), i32(301), torch.zeros_like(out), torch.zeros_like(out)
ws = torch.empty(nb.nuna_embedding_workspace(tokens, hidden, rows), dtype=torch.uint8, device="cuda")
wn = torch.empty(nb.nuna_layernorm_workspace(tokens, hidden), dtype=torch.uint8, device="cuda")
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g):
    nb.nuna_embedding_forward(ids, table, out, tokens, hidden, rows, **f32)
    nb.nuna_layernorm_forward(out, y, tokens, hidden, mean=mean, rstd=rstd, param_dtype=nb.NUNA_F32, **f32)
    nb.nuna_layernorm_backward(y, out, mean, rstd, dx, tokens, hidden, dweight=dw, workspace=wn, param_dtype=nb.NUNA_F32, **f32)
    nb.nuna_expert_sort(ids, row, pair, offsets, tokens, 1, 300)
    nb.nuna_expert_dispatch(y, row, moved, tokens, 1, tokens, hidden, **f32)
    nb.nuna_expert_combine(moved, row, back, tokens, 1, tokens, hidden, **f32)
    nb.nuna_embedding_backward(ids, torch.ones_like(out), grad, tokens, hidden, rows, workspace=ws, grad_dtype=nb.NUNA_F32, **f32)
g.replay()
torch.cuda.synchronize()
assert torch.equal(out, table[ids]) and torch.equal(back, y) and float(y.abs().max()) > 0
assert torch.equal(grad.sum(1), torch.bincount(ids, minlength=rows) * float(hidden))
assert torch.equal(pair.long(), torch.argsort(ids, stable=True))
"""
    import os
    import subprocess
    import sys
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True,
                          text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_empty_calls_that_write():
    """No tokens: the dense gradient is zeros, gaps between its rows stay."""
    for pad in (0, 3, 8):
        for grad in ("bf16", "f32"):
            dtable = Rows(9, 24, DTYPES[grad][0], pad)
            nb.nuna_embedding_backward(None, None, dtable.flat, 0, 24, 9, grad_dtype=DTYPES[grad][1], dtable_stride=dtable.stride)
            torch.cuda.synchronize()
            assert bool((dtable.v == 0).all()) and dtable.untouched()
    none = torch.empty(0, 24, device="cuda")
    out = torch.full((5, 24), GUARD, device="cuda")
    nb.nuna_embedding_forward(torch.arange(5, device="cuda"), none, out, 5, 24, 0, dtype=nb.NUNA_F32)        # a slice without rows
    assert bool((out == 0).all())
    nb.nuna_embedding_backward(torch.arange(5, device="cuda"), out, none, 5, 24, 0, dtype=nb.NUNA_F32, grad_dtype=nb.NUNA_F32,
                               workspace=torch.empty(nb.nuna_embedding_workspace(5, 24, 0), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype,grad", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("hidden", [1, 4, 12, 20, 516, 1028, 1540, 2052, 4100, 8196])
def test_empty_calls_write_every_column(hidden, dtype, grad):
    """No tokens and no dout: all of the gradient is zeros, where its rows are whole vectors and dout's would not be, too."""
    for pad in (0, 4):
        for tokens_of in (None, torch.empty(0, hidden, dtype=DTYPES[dtype][0], device="cuda")):
            dtable = Rows(9, hidden, DTYPES[grad][0], pad)
            nb.nuna_embedding_backward(None, tokens_of, dtable.flat, 0, hidden, 9, dtype=DTYPES[dtype][1], grad_dtype=DTYPES[grad][1],
                                       dtable_stride=dtable.stride)
            torch.cuda.synchronize()
            assert bool((dtable.v == 0).all()) and dtable.untouched()


def test_rows_beyond_32_bits():
    """A table of more than 2^32 elements: the last row is reached, and its gradient written, at the right place."""
    hidden, rows = 4096, (1 << 20) + 3
    table = torch.zeros(rows, hidden, dtype=torch.bfloat16, device="cuda")
    table[-1] = 3.0
    table[rows - (1 << 20) - 1] = 5.0                                  # where a row number that wrapped would end up
    out = torch.empty(2, hidden, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([rows - 1, 0], device="cuda")
    nb.nuna_embedding_forward(ids, table, out, 2, hidden, rows)
    assert bool((out[0] == 3.0).all()) and bool((out[1] == 0.0).all())
    ws = torch.empty(nb.nuna_embedding_workspace(2, hidden, rows), dtype=torch.uint8, device="cuda")
    nb.nuna_embedding_backward(ids, out, table, 2, hidden, rows, workspace=ws)
    assert bool((table[-1] == 3.0).all()) and float(table[:-1].abs().max()) == 0.0


def test_captured_twice_with_a_workspace_each():
    gen = generator(4)
    tokens, hidden, rows = 700, 256, 90
    ids = torch.randint(0, rows, (tokens,), generator=gen, device="cuda")
    dout = integers(gen, -4, 4, tokens, hidden).bfloat16()
    want = torch.zeros(rows, hidden, device="cuda").index_add_(0, ids, dout.float())
    out = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")
    for flags in (0, nb.NUNA_LAUNCH_PDL):
        graphs, grads = [], []
        for _ in range(2):
            grad = torch.zeros(rows, hidden, device="cuda")
            ws = torch.empty(nb.nuna_embedding_workspace(tokens, hidden, rows), dtype=torch.uint8, device="cuda")
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                nb.nuna_embedding_backward(ids, dout, grad, tokens, hidden, rows, workspace=ws, grad_dtype=nb.NUNA_F32, flags=flags)
                nb.nuna_embedding_forward(ids, grad, grad.new_empty(tokens, hidden), tokens, hidden, rows, dtype=nb.NUNA_F32, flags=flags)
            graphs.append(g), grads.append((grad, ws))
        streams = [torch.cuda.Stream() for _ in graphs]
        torch.cuda.synchronize()
        for _ in range(3):
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, want) for g, _ in grads)
    del out


def test_tensors_that_are_too_short_are_refused():
    ids, table, out = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    call = lambda *a, **k: nb.nuna_embedding_forward(*a, dtype=nb.NUNA_F32, check=False, **k)
    assert call(ids, table, out, 4, 8, 5) == nb.NUNA_OK
    assert call(ids[:3], table, out, 4, 8, 5) == nb.NUNA_OK                     # the storage goes on
    assert call(ids[:3].clone(), table, out, 4, 8, 5) == nb.NUNA_ERR_INVALID_ARG
    assert call(ids.int(), table, out, 4, 8, 5) == nb.NUNA_ERR_INVALID_ARG      # int32 ids passed as int64
    assert call(ids, table, out, 4, 8, 6) == nb.NUNA_ERR_INVALID_ARG
    assert call(ids, table[1:], out, 4, 8, 5) == nb.NUNA_ERR_INVALID_ARG
    assert call(ids, table.bfloat16(), out, 4, 8, 5) == nb.NUNA_ERR_INVALID_ARG
    assert call(ids, table, out, 4, 8, 5, out_stride=9) == nb.NUNA_ERR_INVALID_ARG
    torch.cuda.synchronize()
