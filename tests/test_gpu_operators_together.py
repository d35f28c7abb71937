"""A layer's path through the operators and the collectives, as eight emulated ranks of a tensor-parallel program run it: vocabulary
slices looked up and added by an allreduce, residual and norm, tokens to their experts by alltoall and back, and the way back with the
gradients, against the same path in 64 bits."""
import pytest
import torch

from operator_cases import DTYPES, U, generator, half_step, integers, normal, within
from paper_2608_00867_b200 import binding as nb

pytestmark = pytest.mark.gpu

RANKS, TOKENS, HIDDEN, VOCAB, EXPERTS, TOPK, CAPACITY = 8, 24, 512, 80, 16, 2, 6
F32 = dict(dtype=nb.NUNA_F32)


def zeros(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("flags", [0, nb.NUNA_LAUNCH_PDL])
@pytest.mark.parametrize("graph", [False, True])
def test_lookup_allreduce_norm_and_back(flags, graph):
    """Each rank holds an eighth of the vocabulary."""
    gen = generator(1)
    per = VOCAB // RANKS
    ids = torch.randint(0, VOCAB, (TOKENS,), generator=gen, device="cuda")
    table, residual, up = normal(gen, VOCAB, HIDDEN), normal(gen, TOKENS, HIDDEN), normal(gen, TOKENS, HIDDEN)
    w, b = 1 + 0.1 * normal(gen, HIDDEN), normal(gen, HIDDEN)
    slices = [table[r * per:(r + 1) * per].contiguous() for r in range(RANKS)]
    part, whole = [zeros(TOKENS, HIDDEN) for _ in range(RANKS)], [zeros(TOKENS, HIDDEN) for _ in range(RANKS)]
    summed, y, mean, rstd, dx = zeros(TOKENS, HIDDEN), zeros(TOKENS, HIDDEN), zeros(TOKENS), zeros(TOKENS), zeros(TOKENS, HIDDEN)
    dw, db, grads = zeros(HIDDEN), zeros(HIDDEN), [zeros(per, HIDDEN) for _ in range(RANKS)]
    ws = zeros(nb.nuna_layernorm_workspace(TOKENS, HIDDEN), dtype=torch.uint8)
    ews = [zeros(nb.nuna_embedding_workspace(TOKENS, HIDDEN, per), dtype=torch.uint8) for _ in range(RANKS)]

    def step():
        for r in range(RANKS):
            nb.nuna_embedding_forward(ids, slices[r], part[r], TOKENS, HIDDEN, per, vocab_start=r * per, scale=2.0, flags=flags, **F32)
        nb.nuna_allreduce(part, whole, TOKENS * HIDDEN, flags=flags | nb.NUNA_PLACE_AUTO, **F32)
        nb.nuna_layernorm_forward(whole[3], y, TOKENS, HIDDEN, weight=w, bias=b, residual=residual, summed=summed, mean=mean, rstd=rstd,
                                  param_dtype=nb.NUNA_F32, flags=flags, **F32)
        nb.nuna_layernorm_backward(up, summed, mean, rstd, dx, TOKENS, HIDDEN, weight=w, dsummed=y, dweight=dw, dbias=db, workspace=ws,
                                   param_dtype=nb.NUNA_F32, flags=flags, **F32)
        for r in range(RANKS):
            nb.nuna_embedding_backward(ids, dx, grads[r], TOKENS, HIDDEN, per, workspace=ews[r], vocab_start=r * per, scale=2.0,
                                       grad_dtype=nb.NUNA_F32, flags=flags, **F32)

    if graph:
        nb.nuna_init(4 * TOKENS * HIDDEN)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        g.replay()
        g.replay()
    else:
        step()
        step()
    torch.cuda.synchronize()
    for r in range(RANKS):
        assert torch.equal(whole[r], table[ids] * 2.0)                 # one rank's row and seven zeros
    s = (whole[3] + residual).double()
    assert torch.equal(summed.double(), s)
    x = s.clone().requires_grad_()
    w64, b64 = w.double().requires_grad_(), b.double().requires_grad_()
    xh = (x - x.mean(-1, keepdim=True)) * (x.var(-1, unbiased=False, keepdim=True) + 1e-5).rsqrt()
    out = xh * w64 + b64
    # 42 additions in a row at most (32 and 10 levels) of values near 1, a handful of roundings, doubled; xh and the weights are below 8
    within(y, out.detach(), torch.full_like(out.detach(), 2 * 64 * 8 * U), "y")
    (out * up.double()).sum().backward()
    want = x.grad + y.double()
    within(dx, want, torch.full_like(want, 2 * 64 * 32 * U), "dx")
    within(dw, w64.grad, torch.full_like(dw.double(), 2 * 64 * TOKENS * 16 * U), "dweight")
    within(db, b64.grad, torch.full_like(db.double(), 2 * TOKENS * TOKENS * 4 * U), "dbias")
    want = torch.zeros(VOCAB, HIDDEN, dtype=torch.float64, device="cuda").index_add_(0, ids, dx.double()) * 2.0
    within(torch.cat(grads), want, TOKENS * U * 2 * torch.zeros_like(want).index_add_(0, ids, dx.double().abs()), "dtable")
    assert nb.nuna_device_status() == nb.NUNA_OK


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_to_experts_on_other_ranks_and_back(dtype):
    """Every rank sorts its own tokens into equal blocks, an alltoall carries them to the experts' ranks and back.  Integers and
    weights of one half: exact throughout, dropped pairs included."""
    tdt, code = {"bf16": (torch.bfloat16, nb.NUNA_BF16), "f32": (torch.float32, nb.NUNA_F32)}[dtype]
    rows, per = EXPERTS * CAPACITY, EXPERTS // RANKS
    block = per * CAPACITY * HIDDEN
    gens = [generator(2, r) for r in range(RANKS)]
    ids = [torch.stack([torch.randperm(EXPERTS, generator=g, device="cuda")[:TOPK] for _ in range(TOKENS)]) for g in gens]
    x = [integers(g, -3, 3, TOKENS, HIDDEN).to(tdt) for g in gens]
    up = [integers(g, -1, 1, TOKENS, HIDDEN).to(tdt) for g in gens]
    weights = [torch.full((TOKENS, TOPK), 0.5, device="cuda") for _ in gens]
    ints = lambda n: [zeros(n, dtype=torch.int32) for _ in gens]
    row, pair, offsets, counts = ints(TOKENS * TOPK), ints(rows), ints(EXPERTS + 1), ints(EXPERTS)
    many = lambda: [torch.full((rows, HIDDEN), float("nan"), dtype=tdt, device="cuda") for _ in gens]
    send, arrived, back, y = many(), many(), many(), [zeros(TOKENS, HIDDEN, dtype=tdt) for _ in gens]
    factor = torch.arange(1, EXPERTS + 1, device="cuda") % 4 + 1       # expert e multiplies by e % 4 + 1
    for r in range(RANKS):
        nb.nuna_expert_sort(ids[r], row[r], pair[r], offsets[r], TOKENS, TOPK, EXPERTS, counts=counts[r], capacity=CAPACITY)
        nb.nuna_expert_dispatch(x[r], row[r], send[r], TOKENS, TOPK, rows, HIDDEN, pair_of_row=pair[r], dtype=code)
    nb.nuna_alltoall(send, arrived, block, dtype=code)
    own = lambda r: factor[r * per:(r + 1) * per].repeat_interleave(CAPACITY).repeat(RANKS)[:, None]
    made = [(arrived[r] * own(r)).to(tdt) for r in range(RANKS)]
    nb.nuna_alltoall(made, back, block, dtype=code)
    dsrc, dweights, dmade, dout, dx = many(), [zeros(TOKENS, TOPK) for _ in gens], many(), many(), [zeros(TOKENS, HIDDEN, dtype=tdt) for _ in gens]
    for r in range(RANKS):
        nb.nuna_expert_combine(back[r], row[r], y[r], TOKENS, TOPK, rows, HIDDEN, weights=weights[r], dtype=code)
        nb.nuna_expert_combine_backward(up[r], back[r], weights[r], row[r], dsrc[r], dweights[r], TOKENS, TOPK, rows, HIDDEN,
                                        pair_of_row=pair[r], dtype=code)
    nb.nuna_alltoall(dsrc, dmade, block, dtype=code)
    darrived = [(dmade[r] * own(r)).to(tdt) for r in range(RANKS)]
    nb.nuna_alltoall(darrived, dout, block, dtype=code)
    for r in range(RANKS):
        nb.nuna_expert_combine(dout[r], row[r], dx[r], TOKENS, TOPK, rows, HIDDEN, dtype=code)
    torch.cuda.synchronize()
    dropped = 0
    for r in range(RANKS):
        kept = torch.zeros(TOKENS, TOPK, dtype=torch.float64, device="cuda")
        seen = [0] * EXPERTS
        for t, choices in enumerate(ids[r].tolist()):
            for j, e in enumerate(choices):
                kept[t, j] = float(seen[e] < CAPACITY)
                seen[e] += 1
        assert counts[r].tolist() == seen
        dropped += int((kept == 0).sum())
        f = factor.double()[ids[r]] * kept
        assert torch.equal(y[r].double(), (f.sum(1) * 0.5)[:, None] * x[r].double())
        assert torch.equal(dx[r].double(), (f.sum(1) * 0.5)[:, None] * up[r].double())
        assert torch.equal(dweights[r].double(), f * (x[r].double() * up[r].double()).sum(1)[:, None])
        for e in range(EXPERTS):                                       # empty rows were sent as zeros
            n = min(seen[e], CAPACITY)
            assert bool((send[r][e * CAPACITY + n:(e + 1) * CAPACITY] == 0).all())
    assert dropped > 0
    assert half_step(tdt) > 0 and nb.nuna_device_status() == nb.NUNA_OK


@pytest.mark.parametrize("pad,shift", [(3, 0), (1, 1), (11, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_gaps_that_hold_nan_change_nothing(dtype, pad, shift):
    """Rows of an odd length with NaN between and around them give, bit for bit, what rows without gaps give.  Integers and halves, so
    that sums are exact whatever the rows' addresses."""
    tdt, code = DTYPES[dtype]
    tokens, hidden, rows, topk, experts = 61, 37, 23, 3, 8
    pairs = tokens * topk
    gen = generator(5, pad)
    ids = torch.randint(-2, rows + 2, (tokens,), generator=gen, device="cuda")
    choices = torch.randint(0, experts + 1, (tokens, topk), generator=gen, device="cuda")
    weights = integers(gen, 1, 4, tokens, topk) * 0.5
    values = {n: integers(gen, -3, 3, r, hidden) for n, r in dict(table=rows, x=tokens, residual=tokens, dy=tokens, src=pairs).items()}
    row, pair, offsets = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (pairs, pairs, experts + 1))
    nb.nuna_expert_sort(choices, row, pair, offsets, tokens, topk, experts)

    def run(pad, shift):
        stride = hidden + pad

        def rows_of(values, count=None):
            n = count or values.shape[0]
            whole = torch.full((shift + n * stride + 64,), float("nan"), dtype=tdt, device="cuda")
            v = torch.as_strided(whole, (n, hidden), (stride, 1), shift)
            if count is None:
                v.copy_(values)
            return whole[shift:], v

        at = {n: rows_of(v)[0] for n, v in values.items()}
        out = {n: rows_of(None, c) for n, c in dict(looked=tokens, dtable=rows, summed=tokens, y=tokens, dx=tokens, moved=pairs, back=tokens,
                                                    dsrc=pairs).items()}
        to = {n: o[0] for n, o in out.items()}
        mean, rstd, dw, db, dweights = zeros(tokens), zeros(tokens), zeros(hidden), zeros(hidden), zeros(tokens, topk)
        ws = zeros(max(nb.nuna_embedding_workspace(tokens, hidden, rows), nb.nuna_layernorm_workspace(tokens, hidden)), dtype=torch.uint8)
        strides = lambda *names: {f"{n}_stride": stride for n in names}
        nb.nuna_embedding_forward(ids, at["table"], to["looked"], tokens, hidden, rows, dtype=code, **strides("table", "out"))
        nb.nuna_embedding_backward(ids, at["dy"], to["dtable"], tokens, hidden, rows, workspace=ws, dtype=code, grad_dtype=code,
                                   **strides("dout", "dtable"))
        nb.nuna_layernorm_forward(at["x"], to["y"], tokens, hidden, residual=at["residual"], summed=to["summed"], mean=mean, rstd=rstd,
                                  dtype=code, param_dtype=nb.NUNA_F32, **strides("x", "residual", "summed", "y"))
        nb.nuna_layernorm_backward(at["dy"], to["summed"], mean, rstd, to["dx"], tokens, hidden, dsummed=at["x"], dweight=dw, dbias=db,
                                   workspace=ws, dtype=code, param_dtype=nb.NUNA_F32, **strides("dy", "x", "dsummed", "dx"))
        nb.nuna_expert_dispatch(at["x"], row, to["moved"], tokens, topk, pairs, hidden, pair_of_row=pair, dtype=code, **strides("x", "out"))
        nb.nuna_expert_combine(at["src"], row, to["back"], tokens, topk, pairs, hidden, weights=weights, dtype=code, **strides("src", "y"))
        nb.nuna_expert_combine_backward(at["dy"], at["src"], weights, row, to["dsrc"], dweights, tokens, topk, pairs, hidden,
                                        pair_of_row=pair, dtype=code, **strides("dy", "src", "dsrc"))
        torch.cuda.synchronize()
        return {**{n: o[1].clone() for n, o in out.items()}, "mean": mean, "rstd": rstd, "dw": dw, "db": db, "dweights": dweights}

    want, got = run(0, 0), run(pad, shift)
    for n in want:
        assert not bool(torch.isnan(want[n]).any()) and torch.equal(want[n], got[n]), (n, dtype, pad, shift)


@pytest.mark.parametrize("flags", [0, nb.NUNA_LAUNCH_PDL])
@pytest.mark.parametrize("n,vectors", [(2, 40), (4, 148 * 32 + 1), (8, 148 * 96 + 7), (8, 148 * 8 - 1), (3, (7 << 20) // 16)])
def test_two_shots_with_short_operators_between_them(n, vectors, flags):
    """Short grids release their successor ahead of their own wait, so a two-shot, which may draw its tickets ahead of its wait, can
    start while the two-shot before the operator still runs.  A lookup writes what the first two-shot sums, a combine copies each one's
    result before the next one overwrites it; eager and replayed, in the tagged form and beyond it.  Small integers: exact."""
    hidden, tokens = 64, 4
    count, head = 8 * vectors + 8, tokens * hidden
    gen = generator(n, vectors)
    ids = torch.tensor([3, 9, 0, 1], device="cuda")
    src = [[integers(gen, -2, 2, count).bfloat16() for _ in range(n)] for _ in range(2)]
    tables = [integers(gen, -2, 2, 4, hidden).bfloat16() for _ in range(2)]
    dst = [torch.zeros(count, dtype=torch.bfloat16, device="cuda") for _ in range(n)]
    seen = [torch.zeros(tokens, hidden, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    row = torch.arange(tokens, dtype=torch.int32, device="cuda")
    want = []
    for i in range(2):
        looked = torch.where((ids < 4)[:, None], tables[i][ids.clamp(max=3)].float() * 2, torch.zeros(1, device="cuda"))
        src[i][0][:head] = looked.reshape(-1).bfloat16()
        want.append(torch.stack([s.float() for s in src[i]]).sum(0).bfloat16())
    nb.nuna_init(2 * count)

    def look(i):
        nb.nuna_embedding_forward(ids, tables[i], src[i][0], tokens, hidden, 4, scale=2.0, flags=flags)

    def reduce(i):
        nb.nuna_allreduce_twoshot(src[i], dst, count, flags=flags)
        nb.nuna_expert_combine(dst[n - 1], row, seen[i], tokens, 1, tokens, hidden, flags=flags)

    def steps():
        for _ in range(4):
            look(0), reduce(0), reduce(1), look(1)

    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        steps()
    for run in (steps, g.replay):
        src[0][0][:head] = src[1][0][:head] = 5.0                      # written by the lookups, for the second of them in a pass before
        for d in dst + seen:
            d.fill_(7.0)
        run(), run(), run()
        torch.cuda.synchronize()
        assert all(torch.equal(d, want[1]) for d in dst)
        assert all(torch.equal(s.reshape(-1), w[:head]) for s, w in zip(seen, want))
    assert nb.nuna_device_status() == nb.NUNA_OK
