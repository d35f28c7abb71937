"""Refusals and empty calls of the operators around the collectives: everything that is decided before any CUDA call."""
import ctypes
import inspect
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2608_00867_b200 import binding as nb
from paper_2608_00867_b200 import build as nbuild

A = 1 << 24                                  # fake aligned addresses, 1 MiB apart; refused calls never dereference them
BUF = [A + (i << 20) for i in range(12)]
BF16, F16, F32 = nb.NUNA_BF16, nb.NUNA_F16, nb.NUNA_F32
HUGE = 1 << 31

# name: the arguments of a valid call on BUF
NORM = dict(x=BUF[0], y=BUF[1], rows=4, hidden=64, weight=BUF[2], bias=BUF[3], residual=BUF[4], summed=BUF[5], mean=BUF[6], rstd=BUF[7])
NORM_GRAD = dict(dy=BUF[0], x=BUF[1], mean=BUF[2], rstd=BUF[3], dx=BUF[4], rows=4, hidden=64, weight=BUF[5], dsummed=BUF[6],
                 dweight=BUF[7], dbias=BUF[8], workspace=BUF[9], workspace_bytes=1 << 20)
LOOKUP = dict(ids=BUF[0], table=BUF[1], out=BUF[2], tokens=4, hidden=64, vocab_rows=16)
LOOKUP_GRAD = dict(ids=BUF[0], dout=BUF[1], dtable=BUF[2], tokens=4, hidden=64, vocab_rows=16, workspace=BUF[3], workspace_bytes=1 << 20)
SORT = dict(experts=BUF[0], row_of_pair=BUF[1], pair_of_row=BUF[2], offsets=BUF[3], tokens=4, topk=2, num_experts=8, counts=BUF[4])
DISPATCH = dict(x=BUF[0], row_of_pair=BUF[1], out=BUF[2], tokens=4, topk=2, rows=8, hidden=64, pair_of_row=BUF[3])
COMBINE = dict(src=BUF[0], row_of_pair=BUF[1], y=BUF[2], tokens=4, topk=2, rows=8, hidden=64, weights=BUF[3])
COMBINE_GRAD = dict(dy=BUF[0], src=BUF[1], weights=BUF[2], row_of_pair=BUF[3], dsrc=BUF[4], dweights=BUF[5], tokens=4, topk=2, rows=8,
                    hidden=64, pair_of_row=BUF[6])
OPS = {"nuna_layernorm_forward": NORM, "nuna_layernorm_backward": NORM_GRAD, "nuna_embedding_forward": LOOKUP,
       "nuna_embedding_backward": LOOKUP_GRAD, "nuna_expert_sort": SORT, "nuna_expert_dispatch": DISPATCH,
       "nuna_expert_combine": COMBINE, "nuna_expert_combine_backward": COMBINE_GRAD}
WRITTEN = {"nuna_layernorm_forward": ["y", "summed", "mean", "rstd"], "nuna_layernorm_backward": ["dx", "dweight", "dbias", "workspace"],
           "nuna_embedding_forward": ["out"], "nuna_embedding_backward": ["dtable", "workspace"],
           "nuna_expert_sort": ["row_of_pair", "pair_of_row", "offsets", "counts"], "nuna_expert_dispatch": ["out"],
           "nuna_expert_combine": ["y"], "nuna_expert_combine_backward": ["dsrc", "dweights"]}
OPTIONAL = {"weight", "bias", "residual", "summed", "mean", "rstd", "dsummed", "dweight", "dbias", "workspace", "counts", "pair_of_row",
            "weights", "dweights"}
REQUIRED = {"nuna_layernorm_backward": {"mean", "rstd"}, "nuna_embedding_backward": {"workspace"}, "nuna_expert_sort": {"pair_of_row"},
            "nuna_expert_combine_backward": {"weights"}}


@pytest.fixture(scope="module", autouse=True)
def built_library():
    nbuild.build()


def status(name, **kw):
    return getattr(nb, name)(**{**OPS[name], **kw}, stream=0, check=False)


def buffers(name):
    return [k for k, v in OPS[name].items() if v in BUF]


@pytest.mark.parametrize("name", sorted(OPS))
def test_missing_misaligned_and_overlapping_buffers(name):
    for k in buffers(name):
        assert status(name, **{k: OPS[name][k] + 1}) == nb.NUNA_ERR_ALIGNMENT, k
        optional = k in OPTIONAL - REQUIRED.get(name, set())
        if not optional:
            assert status(name, **{k: 0}) == nb.NUNA_ERR_INVALID_ARG, k
            assert status(name, **{k: None}) == nb.NUNA_ERR_INVALID_ARG, k
    for w in WRITTEN[name]:
        for k in buffers(name):
            if k == w or {k, w} in ({"residual", "summed"}, {"dsummed", "dx"}):
                continue
            assert status(name, **{w: OPS[name][k]}) == nb.NUNA_ERR_ALIAS, (w, k)


@pytest.mark.parametrize("name", sorted(OPS))
def test_types_flags_and_sizes(name):
    if name != "nuna_expert_sort":
        assert status(name, dtype=3) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
        assert status(name, dtype=-1) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
        assert status(name, hidden=HUGE) == nb.NUNA_ERR_TOO_LARGE
        assert status(name, hidden=(1 << 30) + 1) == nb.NUNA_ERR_TOO_LARGE
    allowed = nb.NUNA_LAUNCH_PDL | (nb.NUNA_GRAD_ACCUMULATE if name in ("nuna_layernorm_backward", "nuna_embedding_backward") else 0)
    for bit in range(32):
        if not (1 << bit) & allowed:
            assert status(name, flags=1 << bit) == nb.NUNA_ERR_INVALID_ARG, bit
    rows = "rows" if "layernorm" in name else "tokens"
    assert status(name, **{rows: HUGE}) == nb.NUNA_ERR_TOO_LARGE
    for k in OPS[name]:
        stride = f"{k}_stride"
        if stride in inspect.signature(getattr(nb, name)).parameters and OPS[name][k] in BUF:
            assert status(name, **{stride: 63}) == nb.NUNA_ERR_INVALID_ARG, stride
            assert status(name, **{stride: 1 << 47}) == nb.NUNA_ERR_TOO_LARGE, stride
            assert status(name, **{stride: 1 << 45}) == nb.NUNA_ERR_TOO_LARGE, stride      # 4 rows: beyond 2^46 bytes
    L = nb.lib()
    assert getattr(L, name)(None, 0, None) == nb.NUNA_ERR_INVALID_ARG


def test_what_only_one_operator_refuses():
    assert status("nuna_layernorm_forward", param_dtype=F16) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
    assert status("nuna_layernorm_forward", dtype=F32, param_dtype=BF16) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
    assert status("nuna_layernorm_backward", param_dtype=F16) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
    for eps in (-1e-6, float("nan")):
        assert status("nuna_layernorm_forward", eps=eps) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_layernorm_forward", residual=None) == nb.NUNA_ERR_INVALID_ARG      # a sum without a residual
    assert status("nuna_layernorm_forward", summed=None) == nb.NUNA_ERR_INVALID_ARG        # a residual without a place for the sum
    # the sum may be the residual itself, but not with other rows
    assert status("nuna_layernorm_forward", summed=BUF[4], summed_stride=72) == nb.NUNA_ERR_ALIAS
    assert status("nuna_layernorm_forward", summed=BUF[4] + 16) == nb.NUNA_ERR_ALIAS
    assert status("nuna_layernorm_backward", dx=BUF[6], dx_stride=72) == nb.NUNA_ERR_ALIAS
    need = nb.nuna_layernorm_workspace(4, 64)
    assert need == 4 * 2 * 64 * 4
    assert status("nuna_layernorm_backward", workspace_bytes=need - 1) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_layernorm_backward", workspace=None) == nb.NUNA_ERR_INVALID_ARG
    need = nb.nuna_embedding_workspace(4, 64, 16)
    assert status("nuna_embedding_backward", workspace=OPS["nuna_embedding_backward"]["workspace"] + 16) == nb.NUNA_ERR_ALIGNMENT    # 32 bytes a store
    assert status("nuna_embedding_backward", workspace_bytes=need - 1) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_embedding_backward", workspace=None) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_embedding_backward", grad_dtype=F16) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
    for name in ("nuna_embedding_forward", "nuna_embedding_backward", "nuna_expert_sort"):
        for size in (0, 1, 2, 16):
            assert status(name, id_bytes=size) == nb.NUNA_ERR_INVALID_ARG
    for name in ("nuna_embedding_forward", "nuna_embedding_backward"):
        assert status(name, vocab_start=-1) == nb.NUNA_ERR_INVALID_ARG
        assert status(name, vocab_rows=HUGE) == nb.NUNA_ERR_TOO_LARGE
    assert status("nuna_expert_sort", num_experts=0) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_expert_sort", num_experts=nb.NUNA_MAX_EXPERTS + 1) == nb.NUNA_ERR_TOO_LARGE
    assert status("nuna_expert_sort", first_expert=-1) == nb.NUNA_ERR_INVALID_ARG
    assert status("nuna_expert_sort", capacity=HUGE // 8) == nb.NUNA_ERR_TOO_LARGE         # 2^31 rows
    for name in ("nuna_expert_sort", "nuna_expert_dispatch", "nuna_expert_combine", "nuna_expert_combine_backward"):
        assert status(name, tokens=1 << 20, topk=1 << 11) == nb.NUNA_ERR_TOO_LARGE         # 2^31 pairs
        assert status(name, tokens=1 << 40, topk=1 << 40) == nb.NUNA_ERR_TOO_LARGE         # more than 2^64
    for name in ("nuna_expert_dispatch", "nuna_expert_combine", "nuna_expert_combine_backward"):
        assert status(name, rows=HUGE) == nb.NUNA_ERR_TOO_LARGE


def test_empty_calls_launch_nothing():
    before = nb.nuna_launch_count()
    assert status("nuna_layernorm_forward", rows=0) == nb.NUNA_OK
    assert status("nuna_layernorm_forward", hidden=0) == nb.NUNA_OK
    assert status("nuna_layernorm_backward", hidden=0) == nb.NUNA_OK
    assert status("nuna_layernorm_backward", rows=0, dweight=None, dbias=None) == nb.NUNA_OK
    assert status("nuna_layernorm_backward", rows=0, flags=nb.NUNA_GRAD_ACCUMULATE) == nb.NUNA_OK
    assert status("nuna_embedding_forward", tokens=0) == nb.NUNA_OK
    assert status("nuna_embedding_forward", hidden=0) == nb.NUNA_OK
    assert status("nuna_embedding_backward", hidden=0) == nb.NUNA_OK
    assert status("nuna_embedding_backward", vocab_rows=0, dtable=None) == nb.NUNA_OK
    assert status("nuna_embedding_backward", tokens=0, flags=nb.NUNA_GRAD_ACCUMULATE) == nb.NUNA_OK
    assert status("nuna_expert_dispatch", rows=0) == nb.NUNA_OK
    assert status("nuna_expert_dispatch", tokens=0, pair_of_row=None) == nb.NUNA_OK
    assert status("nuna_expert_combine", tokens=0) == nb.NUNA_OK
    assert status("nuna_expert_combine", hidden=0) == nb.NUNA_OK
    assert status("nuna_expert_combine_backward", tokens=0, pair_of_row=None) == nb.NUNA_OK
    assert nb.nuna_launch_count() == before


@pytest.mark.parametrize("hidden", [1, 4, 12, 516, 8196])
def test_a_gradient_of_no_tokens_reaches_its_launch(hidden):
    """Absent rows of a 16-bit dout beside a binary32 table whose own rows are whole vectors.  In a process that sees no GPU, where
    the launch is refused and the addresses are never used."""
    code = f"""
from paper_2608_00867_b200 import binding as nb
for dtype in (nb.NUNA_BF16, nb.NUNA_F16):
    st = nb.nuna_embedding_backward(None, None, {BUF[2]}, 0, {hidden}, 9, dtype=dtype, grad_dtype=nb.NUNA_F32, stream=0, check=False)
    assert st == nb.NUNA_ERR_CUDA, st
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True,
                          text=True, timeout=300, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert done.returncode == 0, (done.returncode, done.stderr[-2000:])


def test_workspaces_of_impossible_sizes():
    assert nb.nuna_layernorm_workspace(HUGE, 64) == 0 and nb.nuna_layernorm_workspace(4, HUGE) == 0
    assert nb.nuna_layernorm_workspace(0, 64) == 0
    assert nb.nuna_embedding_workspace(HUGE, 64, 16) == 0 and nb.nuna_embedding_workspace(4, 64, HUGE) == 0
    # the parts of cut runs: none up to 32 tokens, two rows of binary32 for every 32 tokens beyond
    assert nb.nuna_embedding_workspace(33, 64, 16) - nb.nuna_embedding_workspace(32, 64, 16) >= 4 * 64 * 4
    big = nb.nuna_embedding_workspace(HUGE - 1, HUGE - 1, HUGE - 1)
    assert big > 1 << 56                                             # not wrapped


@pytest.mark.parametrize("name", sorted(OPS))
def test_tensors_that_cannot_be_meant(name):
    """A tensor of the host's memory is refused whatever its size: its address means nothing to a kernel."""
    for k in buffers(name):
        kw = {k: torch.zeros(1 << 16, dtype=torch.int64)}
        assert status(name, **kw) == nb.NUNA_ERR_INVALID_ARG
        with pytest.raises(nb.NunaError, match=f"{name}: a tensor that is not on the current device") as e:
            getattr(nb, name)(**{**OPS[name], **kw}, stream=0)
        assert e.value.status == nb.NUNA_ERR_INVALID_ARG


@pytest.mark.parametrize("name", sorted(OPS))
def test_arguments_by_name_and_position(name):
    stand_in = nb._STAND_INS[name]
    status(name, flags=1)                                            # loads the native module
    native = getattr(nb, name)
    assert native is not stand_in
    a, b = inspect.signature(stand_in).parameters, inspect.signature(native).parameters
    assert list(a) == list(b) and list(a)[-3:] == ["flags", "stream", "check"]
    for k in a:
        if k != "workspace_bytes":
            assert a[k].default == b[k].default, k
    order = [k for k in a if a[k].default is inspect.Parameter.empty]
    assert order == list(OPS[name])[:len(order)]
    args = [OPS[name][k] for k in order]
    rest = {k: v for k, v in OPS[name].items() if k not in order}
    for f in (stand_in, native):
        assert f(*args, **rest, flags=1, stream=0, check=False) == nb.NUNA_ERR_INVALID_ARG
        assert f(check=False, stream=0, flags=np.int64(1), **dict(reversed(OPS[name].items()))) == nb.NUNA_ERR_INVALID_ARG
        with pytest.raises(nb.NunaError, match=name):
            f(*args, **rest, flags=1, stream=0)
        for bad_args, bad_kw in ((args[:-1], {}), (args, {order[0]: args[0]}), (args, {"nosuch": 1}), (args * 5, {})):
            with pytest.raises(TypeError):
                f(*bad_args, **bad_kw, stream=0)
        with pytest.raises(TypeError):
            f(*args[:-1], "8", **rest, stream=0)


@pytest.mark.parametrize("name", ["nuna_layernorm_backward", "nuna_embedding_backward"])
def test_no_size_of_a_workspace_is_none(name):
    """The default that the documented signature has may be passed, before and after the native module took over."""
    stand_in = nb._STAND_INS[name]
    status(name, flags=1)
    native = getattr(nb, name)
    for f in (stand_in, native):
        assert inspect.signature(f).parameters["workspace_bytes"].default is None
        for kw, want in ((dict(hidden=0), nb.NUNA_OK), (dict(), nb.NUNA_ERR_INVALID_ARG)):       # an address has no size of its own
            assert f(**{**OPS[name], **kw, "workspace_bytes": None}, stream=0, check=False) == want
        with pytest.raises(TypeError):
            f(**{**OPS[name], "hidden": None}, stream=0)


def test_structures_match_the_header():
    """The library's own view of a call made through ctypes: field order and sizes of one of the structures."""
    class Sort(ctypes.Structure):
        _fields_ = [(n, ctypes.c_size_t) for n in ("tokens", "topk", "num_experts", "capacity")] + \
                   [(n, ctypes.c_void_p) for n in ("experts", "row_of_pair", "pair_of_row", "offsets", "counts")] + \
                   [("first_expert", ctypes.c_longlong), ("id_bytes", ctypes.c_int)]
    a = Sort(4, 2, 8, 0, *BUF[:5], 0, 8)
    L = nb.lib()
    a.row_of_pair = BUF[0]
    assert L.nuna_expert_sort(ctypes.byref(a), 0, None) == nb.NUNA_ERR_ALIAS
    a.row_of_pair, a.id_bytes = BUF[1], 3
    assert L.nuna_expert_sort(ctypes.byref(a), 0, None) == nb.NUNA_ERR_INVALID_ARG
