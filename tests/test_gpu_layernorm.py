"""Layer norm and its gradient against the formulas in 64 bits."""
import pytest
import torch

from operator_cases import DTYPES, GUARD, Rows, U, generator, guarded, half_step, normal, smallest, within
from paper_2608_00867_b200 import binding as nb

pytestmark = pytest.mark.gpu

# (rows, hidden): a warp, part of a warp, several groups a block, whole blocks, both sides of every change of kernel, long rows
SHAPES = [(1, 1), (3, 2), (5, 8), (2, 31), (7, 33), (300, 64), (17, 257), (1, 1024), (9, 1032), (33, 2048), (5, 2731), (4, 4096), (151, 4104),
          (300, 8192), (2, 8200), (3, 12288), (2, 16384), (3, 16392), (2, 16391), (2, 32768), (2, 40000), (1, 65537), (0, 64), (2000, 128)]
PARAMS = [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32"), ("f32", "f32")]
EPS = 1e-5


def serial(hidden):
    """Additions that follow one another in a sum over a row: at most 32 values a thread while a row fits the block's registers,
    hidden / 1024 beyond, then 10 levels across the block."""
    return max(32, hidden // 1024 + 1) + 10


def forward_reference(x, residual, weight, bias, dtype, eps=EPS):
    s = x.double()
    if residual is not None:
        s = (x.float() + residual.float()).to(dtype).double()          # one rounding to binary32 (exact or not), one to the type
    mean = s.mean(-1, keepdim=True)
    var = ((s - mean) ** 2).mean(-1, keepdim=True)
    rstd = (var + eps) ** -0.5
    xh = (s - mean) * rstd
    y = xh
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return s, mean, rstd, xh, y


def forward_bounds(s, mean, rstd, xh, y, weight, dtype):
    """The mean is off by at most n*U*mean|s| (n additions in a row), which moves xh by that times rstd; the sum of squares by n*U
    relative plus the square of the mean's error, so rstd by about half of that; centring, scaling, weight and bias round once each.
    Doubled, then the rounding of y."""
    n = serial(s.shape[-1])
    dmean = 2 * n * U * s.abs().mean(-1, keepdim=True)
    rel = 2 * (n + 6) * U + dmean * dmean * rstd * rstd
    w = 1.0 if weight is None else weight.double().abs()
    dy = w * (dmean * rstd + xh.abs() * rel) + 4 * U * (y.abs() + w * xh.abs())
    tiny = smallest(dtype)
    return dmean, rel * rstd, dy + half_step(dtype) * (y.abs() + dy) + tiny


def run_forward(rows, hidden, dtype, param, residual=False, affine=True, pad=0, shift=0, stats=True, in_place=False, offset=0.0, **kw):
    tdt, code = DTYPES[dtype]
    pdt, pcode = DTYPES[param]
    gen = generator(rows, hidden, pad, residual)
    x = Rows(rows, hidden, tdt, pad, shift, normal(gen, rows, hidden) * 2 + offset)
    r = Rows(rows, hidden, tdt, pad + 8 if pad else 0, shift, normal(gen, rows, hidden)) if residual else None
    summed = (r if in_place else Rows(rows, hidden, tdt, 0, shift)) if residual else None
    y = Rows(rows, hidden, tdt, 2 * pad, shift)
    w, b = ((1 + 0.3 * normal(gen, hidden)).to(pdt), normal(gen, hidden).to(pdt)) if affine else (None, None)
    (mean, mean_all), (rstd, rstd_all) = guarded(rows, torch.float32), guarded(rows, torch.float32)
    want = forward_reference(x.v, r.v if r else None, w, b, tdt)
    residual_before = r.v.clone() if r else None
    nb.nuna_layernorm_forward(x.flat, y.flat, rows, hidden, weight=w, bias=b, residual=r.flat if r else None,
                              summed=summed.flat if r else None, mean=mean if stats else None, rstd=rstd if stats else None, eps=EPS,
                              dtype=code, param_dtype=pcode, x_stride=x.stride, residual_stride=r.stride if r else 0,
                              summed_stride=summed.stride if r else 0, y_stride=y.stride, **kw)
    torch.cuda.synchronize()
    what = (rows, hidden, dtype, param, residual, pad, shift)
    s, m, rs, xh, yy = want
    if rows:
        dmean, drstd, dy = forward_bounds(s, m, rs, xh, yy, w, tdt)
        within(y.v, yy, dy, (what, "y"))
        if stats:
            within(mean, m[:, 0], dmean[:, 0], (what, "mean"))
            within(rstd, rs[:, 0], drstd[:, 0], (what, "rstd"))
    if r:
        assert torch.equal(summed.v.double(), s), (what, "summed")
        if not in_place:
            assert torch.equal(r.v, residual_before)
    for t in [x, y] + ([r, summed] if r else []):
        assert t.untouched(), (what, "written beyond the rows")
    for t in (mean_all, rstd_all):
        assert bool((t[rows if stats else 0:] == GUARD).all()), (what, "written beyond the statistics")
    return y.v


@pytest.mark.parametrize("dtype,param", PARAMS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_forward(rows, hidden, dtype, param):
    run_forward(rows, hidden, dtype, param)
    run_forward(rows, hidden, dtype, param, residual=True)


@pytest.mark.parametrize("dtype,param", PARAMS)
@pytest.mark.parametrize("rows,hidden", [(5, 64), (19, 2048), (7, 1027), (3, 8192), (2, 16400), (2, 33000)])
def test_forward_with_gaps_odd_alignment_and_without_options(rows, hidden, dtype, param):
    for pad, shift in ((8, 0), (8, 8), (5, 0), (0, 1), (3, 7)):
        run_forward(rows, hidden, dtype, param, residual=True, pad=pad, shift=shift)
    run_forward(rows, hidden, dtype, param, residual=True, in_place=True)
    run_forward(rows, hidden, dtype, param, residual=True, in_place=True, pad=5)
    run_forward(rows, hidden, dtype, param, affine=False, stats=False)
    run_forward(rows, hidden, dtype, param, residual=True, stats=False)


@pytest.mark.parametrize("hidden", [64, 1000, 1001, 8192, 33000])
def test_forward_far_from_zero(hidden):
    """The variance is a sum of squared differences: a mean 1000 times the spread costs it nothing."""
    run_forward(6, hidden, "f32", "f32", offset=2000.0)
    run_forward(6, hidden, "bf16", "f32", offset=16.0)


@pytest.mark.parametrize("hidden", [64, 1001, 8192, 40000])
def test_rows_that_are_constant_or_not_finite(hidden):
    x = torch.randn(6, hidden, device="cuda")
    x[1] = 3.0                                                        # no spread: y = bias
    x[2, hidden // 2] = float("inf")
    x[3, 0] = float("nan")
    x[4, hidden - 1] = -torch.finfo(torch.float32).max                # the square overflows: rstd = 0
    y = torch.empty_like(x)
    mean, rstd = torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    bias = torch.randn(hidden, device="cuda")
    nb.nuna_layernorm_forward(x, y, 6, hidden, bias=bias, mean=mean, rstd=rstd, eps=1e-5, dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    assert torch.equal(y[1], bias) and float(mean[1]) == 3.0
    for r in (2, 3):
        assert bool(torch.isnan(y[r]).all())
    assert float(rstd[4]) == 0.0 and bool(torch.isfinite(y[4]).all())
    clean = torch.empty_like(y)
    nb.nuna_layernorm_forward(x[[0, 5]].contiguous(), clean, 2, hidden, bias=bias, dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    assert torch.equal(clean[:2], y[[0, 5]])                          # the others are none the worse for their neighbours


@pytest.mark.parametrize("hidden", [31, 64, 1000, 1001, 2731, 5120, 8192, 8193, 12288, 16392, 40000, 65537])
def test_constant_rows_whose_sum_is_not_exact(hidden):
    """Equal elements have themselves as their mean and no spread, whatever rounding did to their sum: every difference from a mean
    that is off by a few steps is exact, equal, and a small multiple of such a step, so their sum is exact too."""
    values = torch.tensor([12345.678, 1e5 / 3, -99999.37, 1e-3, 16777215.0, 1e30 / 7, -0.1], device="cuda")
    rows = values.numel()
    x = values[:, None].expand(rows, hidden).contiguous()
    bias = normal(generator(hidden), hidden)
    y, summed, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    f32 = dict(bias=bias, mean=mean, rstd=rstd, eps=EPS, dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    nb.nuna_layernorm_forward(x, y, rows, hidden, **f32)
    assert torch.equal(y, bias.expand_as(y)) and torch.equal(mean, values)
    nb.nuna_layernorm_forward(x, y, rows, hidden, residual=torch.zeros_like(x), summed=summed, **f32)
    assert torch.equal(y, bias.expand_as(y)) and torch.equal(mean, values) and torch.equal(summed, x)


@pytest.mark.parametrize("offset,spread", [(1e5, 0.05), (-3e4, 1e-2), (1e6, 4.0), (7777.7, 1e-3)])
@pytest.mark.parametrize("hidden", [64, 1001, 2731, 5120, 8192, 12288, 16391, 40000])
def test_rows_a_few_steps_of_their_mean_wide(hidden, offset, spread):
    """Rows whose spread is that of a few steps of binary32 at their mean, against 64 bits."""
    rows = 5
    x = normal(generator(hidden), rows, hidden) * spread + offset
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    nb.nuna_layernorm_forward(x, y, rows, hidden, mean=mean, rstd=rstd, eps=EPS, dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    s, m, rs, xh, want = forward_reference(x, None, None, None, torch.float32)
    n = serial(hidden)
    # The first mean is off by d0 <= n*U*mean|s|; the differences from it are exact.  Their sum is off by n*U of their absolute values,
    # and so is the settled mean, beside its own rounding.  The mean square m2 of the differences is var + d0^2, off by n + 6
    # roundings; d0^2 comes off it again, with 2*d0 times the settled mean's error.  Doubled, as elsewhere.
    d0 = n * U * s.abs().mean(-1, keepdim=True)
    dm = 2 * n * U * ((s - m).abs().mean(-1, keepdim=True) + d0)
    m2 = ((s - m) ** 2).mean(-1, keepdim=True) + d0 ** 2
    rel = (2 * (n + 6) * U * m2 + 2 * d0 * dm + dm ** 2) * rs ** 2 + 4 * U
    within(mean, m[:, 0], (dm + U * m.abs())[:, 0], (hidden, offset, "mean"))
    within(rstd, rs[:, 0], (rel * rs)[:, 0], (hidden, offset, "rstd"))
    within(y, want, dm * rs + xh.abs() * (rel + 4 * U) + 2 * U * want.abs(), (hidden, offset, "y"))


def backward_reference(dy, x, mean, rstd, weight, dsummed):
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    g = dy.double() if weight is None else dy.double() * weight.double()
    c0, c1 = g.mean(-1, keepdim=True), (g * xh).mean(-1, keepdim=True)
    dx = rstd.double()[:, None] * (g - c0 - xh * c1)
    if dsummed is not None:
        dx = dx + dsummed.double()
    return xh, g, c0, c1, dx


def run_backward(rows, hidden, dtype, param, affine=True, dsummed=False, pad=0, shift=0, in_place=False, accumulate=False,
                 want_weight=True, want_bias=True, stream=None):
    tdt, code = DTYPES[dtype]
    pdt, pcode = DTYPES[param]
    gen = generator(rows, hidden, pad, dsummed, accumulate)
    x = Rows(rows, hidden, tdt, pad, shift, normal(gen, rows, hidden) * 2 + 0.5)
    dy = Rows(rows, hidden, tdt, 2 * pad, shift, normal(gen, rows, hidden))
    ds = Rows(rows, hidden, tdt, pad, shift, normal(gen, rows, hidden)) if dsummed else None
    dx = ds if in_place else Rows(rows, hidden, tdt, 3 * pad, shift)
    w = (1 + 0.3 * normal(gen, hidden)).to(pdt) if affine else None
    mean = x.v.double().mean(-1).float()
    rstd = (x.v.double().var(-1, unbiased=False) + EPS).rsqrt().float()
    (dw, dw_all), (db, db_all) = guarded(hidden, pdt), guarded(hidden, pdt)
    old = None
    if accumulate:
        old = (normal(gen, hidden).to(pdt), normal(gen, hidden).to(pdt))
        dw.copy_(old[0]), db.copy_(old[1])
    xh, g, c0, c1, dx64 = backward_reference(dy.v, x.v, mean, rstd, w, ds.v if ds else None)
    ds_before = ds.v.double() if ds else 0.0
    need = nb.nuna_layernorm_workspace(rows, hidden)
    ws = torch.full((need + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    nb.nuna_layernorm_backward(dy.flat, x.flat, mean, rstd, dx.flat, rows, hidden, weight=w, dsummed=ds.flat if ds else None,
                               dweight=dw if want_weight else None, dbias=db if want_bias else None, workspace=ws[:need], dtype=code,
                               param_dtype=pcode, dy_stride=dy.stride, x_stride=x.stride, dsummed_stride=ds.stride if ds else 0,
                               dx_stride=dx.stride, flags=nb.NUNA_GRAD_ACCUMULATE if accumulate else 0)
    torch.cuda.synchronize()
    what = (rows, hidden, dtype, param, dsummed, pad, shift, accumulate)
    # xh rounds twice (4U of it), the two sums over the row n*U of their absolute values, the rest once each; doubled
    if rows:
        n, r = serial(hidden), rstd.double().abs()[:, None]
        e0, e1 = 2 * (n + 2) * U * g.abs().mean(-1, keepdim=True), 2 * (n + 6) * U * (g * xh).abs().mean(-1, keepdim=True)
        d = r * (e0 + xh.abs() * e1 + 12 * U * (g.abs() + c0.abs() + (xh * c1).abs())) + 2 * U * (dx64.abs() + torch.as_tensor(ds_before).abs())
        within(dx.v, dx64, d + half_step(tdt) * (dx64.abs() + d) + smallest(tdt), (what, "dx"))
    # sums over the rows: at most rows / 148 + 1 rows one after the other in a group, up to 16 groups, then 148 blocks in 16 slices
    n = rows // 148 + 1 + 16 + 10 + 16 + 6
    for got, whole, term, o, asked, name in ((dw, dw_all, dy.v.double() * xh, 0, want_weight, "dweight"),
                                             (db, db_all, dy.v.double(), 1, want_bias, "dbias")):
        if not asked:
            assert bool((whole == GUARD).all()) or accumulate
            continue
        total = term.sum(0)
        b = 2 * n * U * term.abs().sum(0) + 2 * U * total.abs()
        if accumulate:
            total = total + old[o].double()
            b = b + 2 * U * total.abs()
        within(got, total, b + half_step(pdt) * (total.abs() + b) + smallest(pdt), (what, name))
        assert bool((whole[hidden:] == GUARD).all()), (what, name)
    for t in [x, dy, dx] + ([ds] if ds else []):
        assert t.untouched(), (what, "written beyond the rows")
    assert bool((ws[need:] == 0x7F).all()), (what, "written beyond the workspace")
    return dx.v, dw, db


@pytest.mark.parametrize("dtype,param", PARAMS)
@pytest.mark.parametrize("rows,hidden", SHAPES)
def test_backward(rows, hidden, dtype, param):
    run_backward(rows, hidden, dtype, param)
    run_backward(rows, hidden, dtype, param, dsummed=True)


@pytest.mark.parametrize("dtype,param", PARAMS)
@pytest.mark.parametrize("rows,hidden", [(5, 64), (601, 2048), (149, 1027), (30, 8192), (2, 16400), (2, 33000), (0, 40)])
def test_backward_with_gaps_odd_alignment_and_without_options(rows, hidden, dtype, param):
    for pad, shift in ((8, 0), (8, 8), (5, 0), (0, 1), (3, 7)):
        run_backward(rows, hidden, dtype, param, dsummed=True, pad=pad, shift=shift)
    run_backward(rows, hidden, dtype, param, dsummed=True, in_place=True)
    run_backward(rows, hidden, dtype, param, dsummed=True, in_place=True, pad=5)
    run_backward(rows, hidden, dtype, param, affine=False, want_weight=False, want_bias=False)
    run_backward(rows, hidden, dtype, param, want_weight=False)
    run_backward(rows, hidden, dtype, param, want_bias=False)
    run_backward(rows, hidden, dtype, param, accumulate=True)
    run_backward(rows, hidden, dtype, param, accumulate=True, want_bias=False)


@pytest.mark.parametrize("dtype,param", PARAMS)
@pytest.mark.parametrize("hidden", [63, 65, 255, 257, 511, 512, 513, 1023, 1024, 1025, 1537, 4095, 4096, 4097, 6001, 8191, 8192, 8193])
def test_rows_that_end_at_and_around_a_warps_columns(hidden, dtype, param):
    for rows in (1, 17):
        for residual in (False, True):
            run_forward(rows, hidden, dtype, param, residual=residual, pad=5)
            run_backward(rows, hidden, dtype, param, dsummed=residual, pad=5)
    run_forward(400, hidden, dtype, param, residual=True, pad=3, shift=1)                 # more rows than there are SMs: fetched ahead
    run_backward(400, hidden, dtype, param, dsummed=True, pad=3, shift=1)


@pytest.mark.parametrize("dtype,param,hidden", [("bf16", "f32", 8193), ("f16", "f16", 16392), ("f32", "f32", 8200)])
@pytest.mark.parametrize("rows", [148, 149, 148 * 16, 148 * 16 + 1, 148 * 33 + 5])
def test_long_rows_in_several_batches(rows, hidden, dtype, param):
    run_backward(rows, hidden, dtype, param, dsummed=True)
    run_backward(rows, hidden, dtype, param, accumulate=True, pad=3)


@pytest.mark.parametrize("rows,hidden", [(1500, 96), (700, 1001), (333, 8192)])
def test_the_same_call_gives_the_same_bits(rows, hidden):
    first = run_backward(rows, hidden, "bf16", "f32", dsummed=True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run_backward(rows, hidden, "bf16", "f32", dsummed=True)))


def test_gradient_against_differences():
    """The formula's gradient is that of the forward pass: central differences of a weighted sum of y, in 64 bits, of the kernel's
    own inputs."""
    gen = generator(5)
    rows, hidden = 3, 40
    x, w, b, up = normal(gen, rows, hidden), normal(gen, hidden), normal(gen, hidden), normal(gen, rows, hidden)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dw, db = (torch.empty(n, device="cuda") for n in (rows, rows, hidden, hidden))
    f32 = dict(dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    nb.nuna_layernorm_forward(x, y, rows, hidden, weight=w, bias=b, mean=mean, rstd=rstd, **f32)
    ws = torch.empty(nb.nuna_layernorm_workspace(rows, hidden), dtype=torch.uint8, device="cuda")
    nb.nuna_layernorm_backward(up, x, mean, rstd, dx, rows, hidden, weight=w, dweight=dw, dbias=db, workspace=ws, **f32)

    def loss(x, w, b):
        return (forward_reference(x, None, w, b, torch.float64)[4] * up.double()).sum()

    h = 1e-5
    for name, got in (("x", dx), ("w", dw), ("b", db)):
        args = {"x": x.double(), "w": w.double(), "b": b.double()}
        for i in range(0, got.numel(), 7):
            step = torch.zeros(got.numel(), dtype=torch.float64, device="cuda")
            step[i] = h
            step = step.view(got.shape)
            slope = (loss(**{**args, name: args[name] + step}) - loss(**{**args, name: args[name] - step})) / (2 * h)
            # binary32 kernel: 1e-5 of the gradient's scale (about 40 terms of size 1); differences: h^2 times third derivatives, 1e-8
            assert abs(float(slope) - float(got.reshape(-1)[i])) < 1e-4, (name, i)


def test_captured_and_replayed_and_on_another_stream():
    rows, hidden = 64, 8192
    gen = generator(9)
    x, r, up = (normal(gen, rows, hidden).bfloat16() for _ in range(3))
    w, b = normal(gen, hidden), normal(gen, hidden)
    make = lambda: dict(summed=torch.zeros_like(x), y=torch.zeros_like(x), mean=torch.zeros(rows, device="cuda"),
                        rstd=torch.zeros(rows, device="cuda"), dx=torch.zeros_like(x), dw=torch.zeros(hidden, device="cuda"),
                        db=torch.zeros(hidden, device="cuda"),
                        ws=torch.empty(nb.nuna_layernorm_workspace(rows, hidden), dtype=torch.uint8, device="cuda"))

    def step(t, flags):
        nb.nuna_layernorm_forward(x, t["y"], rows, hidden, weight=w, bias=b, residual=r, summed=t["summed"], mean=t["mean"], rstd=t["rstd"],
                                  param_dtype=nb.NUNA_F32, flags=flags)
        nb.nuna_layernorm_backward(up, t["summed"], t["mean"], t["rstd"], t["dx"], rows, hidden, weight=w, dsummed=t["y"], dweight=t["dw"],
                                   dbias=t["db"], workspace=t["ws"], param_dtype=nb.NUNA_F32, flags=flags)

    want = make()
    step(want, 0)
    torch.cuda.synchronize()
    for flags in (0, nb.NUNA_LAUNCH_PDL):
        got = make()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(got, flags)
            step(got, flags)
        for t in got.values():
            t.zero_()
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(want[k], got[k]) for k in want if k != "ws"), flags
    stream = torch.cuda.Stream()
    got = make()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(5):
            step(got, 0)
    stream.synchronize()
    assert all(torch.equal(want[k], got[k]) for k in want if k != "ws")


def test_tensors_that_are_too_short_are_refused():
    x, y = torch.zeros(4 * 64 - 1, device="cuda"), torch.zeros(4 * 64, device="cuda")
    before = nb.nuna_launch_count()
    with pytest.raises(nb.NunaError, match="shorter than the call's sizes"):
        nb.nuna_layernorm_forward(x, y, 4, 64, dtype=nb.NUNA_F32)
    assert nb.nuna_layernorm_forward(y, y[1:], 4, 64, dtype=nb.NUNA_F32, check=False) == nb.NUNA_ERR_INVALID_ARG
    assert nb.nuna_layernorm_forward(y, x.new_zeros(256), 4, 64, x_stride=65, dtype=nb.NUNA_F32, check=False) == nb.NUNA_ERR_INVALID_ARG
    ws = torch.zeros(nb.nuna_layernorm_workspace(4, 64) - 1, dtype=torch.uint8, device="cuda")
    stats = torch.zeros(4, device="cuda")
    assert nb.nuna_layernorm_backward(y, y, stats, stats, x.new_zeros(256), 4, 64, dweight=x.new_zeros(64), workspace=ws, dtype=nb.NUNA_F32,
                                      param_dtype=nb.NUNA_F32, check=False) == nb.NUNA_ERR_INVALID_ARG
    assert nb.nuna_launch_count() == before
