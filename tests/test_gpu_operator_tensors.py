"""What a tensor says of itself is held against the operators' calls: its element type, and where its elements are.  Every refusal is
the host's, before any launch; the tensors are as long as the calls reach all the same."""
import pytest
import torch

from paper_2608_00867_b200 import binding as nb

pytestmark = pytest.mark.gpu

T, H, V, E, K = 6, 16, 10, 4, 2                # tokens, hidden, table rows, experts, choices
TYPES = {torch.bfloat16: nb.NUNA_BF16, torch.float16: nb.NUNA_F16, torch.float32: nb.NUNA_F32}
WRONG = {torch.bfloat16: [torch.float16, torch.float32, torch.int16, torch.int32], torch.float16: [torch.bfloat16, torch.float32, torch.float64],
         torch.float32: [torch.float64, torch.int32, torch.int64], torch.int32: [torch.int64, torch.float32], torch.int64: [torch.int32, torch.float64]}


def made(shape, dtype):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def ops(rows=torch.bfloat16, param=torch.float32, ids=torch.int64):
    """name: (tensors by argument, with their shapes; the other arguments)."""
    f32, i32 = torch.float32, torch.int32
    d, p = TYPES[rows], TYPES[param]
    norm = dict(rows=T, hidden=H, dtype=d, param_dtype=p)
    pairs = T * K
    work = made((1 << 16,), torch.uint8)
    m = lambda *s, t=rows: made(s, t)
    return {
        "nuna_layernorm_forward": (dict(x=m(T, H), y=m(T, H), weight=m(H, t=param), bias=m(H, t=param), residual=m(T, H), summed=m(T, H),
                                        mean=m(T, t=f32), rstd=m(T, t=f32)), norm),
        "nuna_layernorm_backward": (dict(dy=m(T, H), x=m(T, H), mean=m(T, t=f32), rstd=m(T, t=f32), dx=m(T, H), weight=m(H, t=param), dsummed=m(T, H),
                                         dweight=m(H, t=param), dbias=m(H, t=param)), dict(norm, workspace=work)),
        "nuna_embedding_forward": (dict(ids=m(T, t=ids), table=m(V, H), out=m(T, H)),
                                   dict(tokens=T, hidden=H, vocab_rows=V, dtype=d, id_bytes=ids.itemsize)),
        "nuna_embedding_backward": (dict(ids=m(T, t=ids), dout=m(T, H), dtable=m(V, H, t=param)),
                                    dict(tokens=T, hidden=H, vocab_rows=V, dtype=d, grad_dtype=p, id_bytes=ids.itemsize, workspace=work)),
        "nuna_expert_sort": (dict(experts=m(T, K, t=ids), row_of_pair=m(pairs, t=i32), pair_of_row=m(pairs, t=i32), offsets=m(E + 1, t=i32),
                                  counts=m(E, t=i32)), dict(tokens=T, topk=K, num_experts=E, id_bytes=ids.itemsize)),
        "nuna_expert_dispatch": (dict(x=m(T, H), row_of_pair=m(pairs, t=i32), out=m(pairs, H), pair_of_row=m(pairs, t=i32)),
                                 dict(tokens=T, topk=K, rows=pairs, hidden=H, dtype=d)),
        "nuna_expert_combine": (dict(src=m(pairs, H), row_of_pair=m(pairs, t=i32), y=m(T, H), weights=m(T, K, t=f32)),
                                dict(tokens=T, topk=K, rows=pairs, hidden=H, dtype=d)),
        "nuna_expert_combine_backward": (dict(dy=m(T, H), src=m(pairs, H), weights=m(T, K, t=f32), row_of_pair=m(pairs, t=i32), dsrc=m(pairs, H),
                                              dweights=m(T, K, t=f32), pair_of_row=m(pairs, t=i32)),
                                         dict(tokens=T, topk=K, rows=pairs, hidden=H, dtype=d)),
    }


def call(name, tensors, rest, **kw):
    before = nb.nuna_launch_count()
    st = getattr(nb, name)(**{**rest, **tensors, **kw}, check=False)
    assert (nb.nuna_launch_count() > before) == (st == nb.NUNA_OK)
    return st


@pytest.mark.parametrize("rows,param,ids", [(torch.bfloat16, torch.float32, torch.int64), (torch.float16, torch.float16, torch.int32),
                                            (torch.float32, torch.float32, torch.int64)])
def test_other_types_are_refused(rows, param, ids):
    for name, (tensors, rest) in ops(rows, param, ids).items():
        assert call(name, tensors, rest) == nb.NUNA_OK, name
        for k, t in tensors.items():
            for wrong in WRONG[t.dtype]:
                other = made((4 * t.numel(),), wrong)                   # longer than the call reaches whatever its type
                assert call(name, {**tensors, k: other}, rest) == nb.NUNA_ERR_INVALID_ARG, (name, k, wrong)
                with pytest.raises(nb.NunaError, match=f"{name}: {k} is a tensor of another type"):
                    getattr(nb, name)(**{**rest, **tensors, k: other})
            for raw in (torch.uint8, torch.uint16, torch.uint32):       # memory, of any type
                assert call(name, {**tensors, k: made((8 * t.numel(),), raw)}, rest) == nb.NUNA_OK, (name, k, raw)
            assert call(name, {**tensors, k: t.data_ptr()}, rest) == nb.NUNA_OK, (name, k)
    torch.cuda.synchronize()


def test_types_that_the_library_refuses_stay_its_own():
    for name, (tensors, rest) in ops().items():
        if "dtype" in rest:
            assert call(name, tensors, rest, dtype=3) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
        for k in ("param_dtype", "grad_dtype"):
            if k in rest:
                assert call(name, tensors, rest, **{k: nb.NUNA_F16}) == nb.NUNA_ERR_UNSUPPORTED_DTYPE
        if "id_bytes" in rest:
            assert call(name, tensors, rest, id_bytes=2) == nb.NUNA_ERR_INVALID_ARG
    tensors, rest = ops(torch.float32, torch.float32)["nuna_layernorm_forward"]
    assert call("nuna_layernorm_forward", tensors, {**rest, "param_dtype": nb.NUNA_BF16}) == nb.NUNA_ERR_UNSUPPORTED_DTYPE


def test_elements_elsewhere_are_refused():
    """Transposed rows, every second element, slices of wider rows whose stride the call does not say, rows that are not evenly spaced."""
    for name, (tensors, rest) in ops().items():
        for k, t in tensors.items():
            bad = [made(tuple(reversed(t.shape)), t.dtype).t()] if t.dim() == 2 else []
            bad.append(made((4 * t.numel(),), t.dtype)[::2])
            bad.append(made((t.shape[0], 2 * (t.shape[1] if t.dim() == 2 else 1) + 1), t.dtype)[:, :t.shape[1] if t.dim() == 2 else 1])
            bad.append(made((3, 4, t.numel()), t.dtype)[:, 1:])
            bad.append(made((1, 1), t.dtype).expand(4, t.numel()))
            for other in bad:
                assert not other.is_contiguous()
                kw = {**tensors, k: other}
                assert call(name, kw, rest) == nb.NUNA_ERR_INVALID_ARG, (name, k, other.shape, other.stride())
                if other.untyped_storage().nbytes() >= 4 * t.numel() * t.element_size():
                    with pytest.raises(nb.NunaError, match=f"{name}: {k} is a tensor whose elements are not where"):
                        getattr(nb, name)(**{**rest, **kw})
    torch.cuda.synchronize()


def test_rows_at_the_distance_that_the_call_says():
    stride = H + 8
    for name, (tensors, rest) in ops().items():
        for k, t in tensors.items():
            if t.dim() != 2 or t.shape[1] != H:
                continue
            wide = made((2 * t.shape[0], stride), t.dtype)
            for view, said in ((wide[:t.shape[0], :H], stride), (wide[::2, :H], 2 * stride), (wide[:, 8:], stride), (wide[:, 8:], 2 * stride),
                               (wide.view(2, t.shape[0], stride)[:, :, :H], stride), (wide, stride), (wide, 0), (wide.view(-1), stride)):
                assert call(name, {**tensors, k: view}, rest, **{f"{k}_stride": said}) == nb.NUNA_OK, (name, k, view.shape, said)
            for view, said in ((wide[:, :H], 0), (wide[:, :H], stride + 8), (wide[::2, :H], stride)):
                assert call(name, {**tensors, k: view}, rest, **{f"{k}_stride": said}) == nb.NUNA_ERR_INVALID_ARG, (name, k, view.shape, said)
    column = made((T, 5), torch.float32)
    y = made((T,), torch.float32)
    one = dict(rows=T, hidden=1, dtype=nb.NUNA_F32, param_dtype=nb.NUNA_F32)
    for view in (column[:, 2], column[:, 2:3]):                         # rows of one element
        assert call("nuna_layernorm_forward", dict(x=view, y=y), one, x_stride=5) == nb.NUNA_OK
        assert call("nuna_layernorm_forward", dict(x=view, y=y), one) == nb.NUNA_ERR_INVALID_ARG
    torch.cuda.synchronize()


def test_one_row_needs_no_distance():
    wide, y = made((T, H + 8), torch.bfloat16), made((1, H), torch.bfloat16)
    one = dict(rows=1, hidden=H, param_dtype=nb.NUNA_F32)
    assert call("nuna_layernorm_forward", dict(x=wide[:, :H], y=y), one) == nb.NUNA_OK
    assert call("nuna_layernorm_forward", dict(x=wide[:, :H], y=y), one, x_stride=H + 1) == nb.NUNA_OK
    assert call("nuna_layernorm_forward", dict(x=wide[:, :2 * H:2], y=y), one) == nb.NUNA_ERR_INVALID_ARG
    assert call("nuna_layernorm_forward", dict(x=wide.t(), y=y), one) == nb.NUNA_ERR_INVALID_ARG
    assert call("nuna_layernorm_forward", dict(x=wide[:, :H], y=made((2, H), torch.bfloat16)), dict(one, rows=2)) == nb.NUNA_ERR_INVALID_ARG
    torch.cuda.synchronize()
