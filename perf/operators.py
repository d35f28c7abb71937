"""What stands around the collectives of a tensor-parallel program, as cases that can be timed and compared.

Three families, each with its gradient: the layer norm (with the residual added) that follows every allreduce, the
embedding lookup whose vocabulary slices an allreduce adds up, and the tokens sorted by expert that an alltoall carries,
and their way back with the router's weights.  ``run`` makes the calls a user makes (``own``) or computes the same in
elementary torch operations; ``exact`` is the definition in 64 bits.

Sizes: hidden 8192 and the token counts 1 ... 4096 are those of this repository's decode and prefill workloads; the
others (vocabularies, expert counts, odd sizes) are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"bf16": 0, "f16": 1, "f32": 2}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
HIDDEN = 8192


def listed():
    return [
        # decode, one token: the norm after the allreduce, residual added; its latency is all that matters
        dict(name="norm_t1", op="norm", rows=1, hidden=HIDDEN, dtype="bf16", param="bf16", residual=True, pad=0),
        # prefill or a training forward pass: 4096 tokens, statistics kept
        dict(name="norm_t4096", op="norm", rows=4096, hidden=HIDDEN, dtype="bf16", param="bf16", residual=True, pad=0),
        # training: the same rows' gradient, with the residual stream's gradient added and binary32 parameters
        dict(name="norm_grad_t4096", op="norm_grad", rows=4096, hidden=HIDDEN, dtype="bf16", param="f32", residual=True, pad=0),
        # an odd hidden size in rows that are a slice of wider ones
        dict(name="norm_grad_ragged_f16", op="norm_grad", rows=1003, hidden=2731, dtype="f16", param="f16", residual=False, pad=5),
        # decode, batch of 32: one rank's slice of a vocabulary of 131072 (the other ids give zero rows)
        dict(name="embedding_t32", op="embedding", tokens=32, hidden=HIDDEN, vocab=131072, start=0, rows=16384, dtype="bf16",
             scale=1.0, ids="i64"),
        # prefill with a whole, scaled table
        dict(name="embedding_t16384", op="embedding", tokens=16384, hidden=4096, vocab=32768, start=0, rows=32768, dtype="bf16",
             scale=64.0, ids="i64"),
        # training: the dense binary32 gradient of a vocabulary slice from 8192 tokens
        dict(name="embedding_grad_t8192", op="embedding_grad", tokens=8192, hidden=4096, vocab=131072, start=0, rows=32768,
             dtype="bf16", grad="f32", scale=1.0, ids="i64"),
        # many tokens over few, odd rows: long runs of the same id
        dict(name="embedding_grad_ragged", op="embedding_grad", tokens=20011, hidden=1037, vocab=5003, start=17, rows=4801,
             dtype="f16", grad="f16", scale=32.0, ids="i32"),
        # decode, batch of 32: sort, dispatch, and the experts' outputs back with their weights
        dict(name="experts_t32", op="experts", tokens=32, topk=8, hidden=4096, total=64, first=0, local=64, capacity=0,
             dtype="bf16", ids="i64"),
        # prefill: 8192 tokens to 8 of 128 experts
        dict(name="experts_t8192", op="experts", tokens=8192, topk=8, hidden=4096, total=128, first=0, local=128, capacity=0,
             dtype="bf16", ids="i64"),
        # training: the gradients of both ways, 4096 tokens to 4 of 64 experts
        dict(name="experts_grad_t4096", op="experts_grad", tokens=4096, topk=4, hidden=HIDDEN, total=64, first=0, local=64,
             capacity=0, dtype="bf16", ids="i64"),
        # expert parallel with a capacity per expert (equal blocks for the alltoall), odd sizes, binary32
        dict(name="experts_grad_capacity_f32", op="experts_grad", tokens=2047, topk=3, hidden=1030, total=48, first=12,
             local=24, capacity=117, dtype="f32", ids="i32"),
    ]


def draw(rng):
    def between(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def width(lo, hi):
        h = between(lo, hi)
        return max(8, h // 8 * 8) if rng.random() < 0.7 else h | 1

    op = rng.choice(["norm", "norm_grad", "embedding", "embedding_grad", "experts", "experts_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    ids = rng.choice(["i64", "i32"])
    if op in ("norm", "norm_grad"):
        hidden = width(64, 16384)
        rows = between(1, max(2, min(65536, 4096 * HIDDEN // hidden)))
        return dict(op=op, rows=rows, hidden=hidden, dtype=dtype, param=rng.choice([dtype, "f32"]),
                    residual=rng.random() < 0.5, pad=rng.choice([0, 0, 8, 5]))
    hidden = width(64, 8192)
    if op in ("embedding", "embedding_grad"):
        tokens = between(1, max(2, min(65536, 16384 * 4096 // hidden)))
        rows = between(16, max(32, min(131072, 32768 * 4096 // hidden)))
        vocab = rows * rng.choice([1, 1, 2, 8])
        case = dict(op=op, tokens=tokens, hidden=hidden, vocab=vocab, start=rng.randrange(vocab - rows + 1), rows=rows,
                    dtype=dtype, scale=rng.choice([1.0, round(math.sqrt(hidden), 3)]), ids=ids)
        if op == "embedding_grad":
            case["grad"] = rng.choice([dtype, "f32"])
        return case
    topk = rng.choice([1, 2, 3, 4, 6, 8])
    total = rng.choice([8, 16, 31, 60, 64, 128, 256])
    local = total if rng.random() < 0.6 else max(1, total // rng.choice([2, 4, 8]))
    tokens = between(1, max(2, min(32768, 8192 * 8 * 4096 // (topk * hidden * (2 if op == "experts_grad" else 1) * SIZES[dtype] // 2))))
    capacity = 0 if rng.random() < 0.6 else max(1, int(tokens * topk / total * rng.choice([0.8, 1.0, 1.25])))
    return dict(op=op, tokens=tokens, topk=topk, hidden=hidden, total=total, first=rng.randrange(total - local + 1), local=local,
                capacity=capacity, dtype=dtype, ids=ids)


# ---- inputs ------------------------------------------------------------------------------------------------------

def _rows(gen, n, hidden, dtype, pad=0):
    """n rows of unit normal values, each `pad` elements short of the next."""
    full = torch.randn(n, hidden + pad, generator=gen, device="cuda", dtype=torch.float32).to(DTYPES[dtype])
    return full[:, :hidden]


def _ids(case, gen):
    """Token ids with the skew of text (frequency ~ 1 / rank), the ranks scattered over the vocabulary."""
    v = case["vocab"]
    share = np.cumsum(1.0 / (np.arange(v) + 2.7))                 # on the host: the same sums in every run
    drawn = torch.rand(case["tokens"], generator=gen, device="cuda", dtype=torch.float64) * float(share[-1])
    ranks = torch.searchsorted(torch.from_numpy(share).cuda(), drawn).clamp_(max=v - 1)
    at = torch.randperm(v, generator=gen, device="cuda")
    return at[ranks].to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _row_count(case):
    return case["local"] * case["capacity"] if case["capacity"] else case["tokens"] * case["topk"]


def _plan(case, experts):
    """The plan of a sort by expert: a stable sort of the (token, choice) pairs."""
    n, e, cap, rows = case["tokens"] * case["topk"], case["local"], case["capacity"], _row_count(case)
    key = experts.reshape(-1).long() - case["first"]
    mine = (key >= 0) & (key < e)
    key = torch.where(mine, key, torch.full_like(key, e))
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(e + 1, dtype=torch.int64, device="cuda").scatter_add_(0, key, torch.ones_like(key))
    starts = torch.cumsum(counts, 0) - counts
    place = torch.empty_like(key)
    place[order] = torch.arange(n, device="cuda") - starts[key[order]]
    if cap:
        offsets = torch.arange(e + 1, device="cuda") * cap
        mine = mine & (place < cap)
    else:
        offsets = starts
    row = torch.where(mine, offsets[key] + place, torch.full_like(key, -1))
    pair = torch.full((rows + 1,), -1, dtype=torch.int64, device="cuda")
    pair[torch.where(mine, row, torch.full_like(row, rows))] = torch.arange(n, device="cuda")
    return row.int(), pair[:rows].int(), offsets.int(), counts[:e].int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 11)
    s = {"case": case}
    op, dtype, hidden = case["op"], case["dtype"], case["hidden"]
    empty = lambda *shape, dt=dtype: torch.zeros(*shape, dtype=DTYPES[dt], device="cuda")
    if op in ("norm", "norm_grad"):
        n, param = case["rows"], DTYPES[case["param"]]
        s["x"] = _rows(gen, n, hidden, dtype, case["pad"])
        s["weight"] = (1.0 + 0.1 * torch.randn(hidden, generator=gen, device="cuda")).to(param)
        s["bias"] = (0.1 * torch.randn(hidden, generator=gen, device="cuda")).to(param)
        other = _rows(gen, n, hidden, dtype, case["pad"]) if case["residual"] else None
        if op == "norm":
            s["residual"] = other
            s["summed"] = empty(n, hidden) if case["residual"] else None
            s["y"] = empty(n, hidden)
            s["mean"], s["rstd"] = empty(n, dt="f32"), empty(n, dt="f32")
        else:
            s["dsummed"] = other
            s["dy"] = _rows(gen, n, hidden, dtype, case["pad"])
            x = s["x"].double()
            s["mean"] = x.mean(-1).float()
            s["rstd"] = (x.var(-1, unbiased=False) + EPS).rsqrt().float()
            s["dx"] = empty(n, hidden)
            s["dweight"], s["dbias"] = torch.zeros_like(s["weight"]), torch.zeros_like(s["bias"])
    elif op in ("embedding", "embedding_grad"):
        s["ids"] = _ids(case, gen)
        if op == "embedding":
            s["table"] = _rows(gen, case["rows"], hidden, dtype)
            s["out"] = empty(case["tokens"], hidden)
        else:
            s["dout"] = _rows(gen, case["tokens"], hidden, dtype)
            s["dtable"] = empty(case["rows"], hidden, dt=case["grad"])
    else:
        n, k, rows = case["tokens"], case["topk"], _row_count(case)
        logits = torch.randn(n, case["total"], generator=gen, device="cuda")
        logits += 0.7 * torch.randn(case["total"], generator=gen, device="cuda")           # some experts are asked more often
        top = torch.topk(logits, k, dim=-1)
        s["experts"] = top.indices.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        s["weights"] = torch.softmax(top.values, -1)
        s["src"] = _rows(gen, rows, hidden, dtype)                                         # what the experts made of their rows
        if op == "experts":
            s["x"] = _rows(gen, n, hidden, dtype)
            s["out"], s["y"] = empty(rows, hidden), empty(n, hidden)
            integers = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda")
            s["row_of_pair"], s["pair_of_row"] = integers(n * k), integers(rows)
            s["offsets"], s["counts"] = integers(case["local"] + 1), integers(case["local"])
        else:
            s["row_of_pair"], s["pair_of_row"], _, _ = _plan(case, s["experts"])           # kept from the forward pass
            s["dy"] = _rows(gen, n, hidden, dtype)
            s["dout"] = _rows(gen, rows, hidden, dtype)                                    # gradient of the experts' inputs
            s["dsrc"], s["dx"] = empty(rows, hidden), empty(n, hidden)
            s["dweights"] = torch.zeros_like(s["weights"])
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _plain_norm(s):
    x, dt = s["x"].float(), s["x"].dtype
    summed = None
    if s["residual"] is not None:
        summed = (x + s["residual"].float()).to(dt)
        x = summed.float()
    mean = x.mean(-1, keepdim=True)
    centred = x - mean
    rstd = 1.0 / torch.sqrt((centred * centred).mean(-1, keepdim=True) + EPS)
    y = (centred * rstd * s["weight"].float() + s["bias"].float()).to(dt)
    return {"summed": summed, "y": y, "mean": mean[:, 0], "rstd": rstd[:, 0]}


def _plain_norm_grad(s):
    dy = s["dy"].float()
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)) * s["rstd"][:, None]
    if s["dsummed"] is not None:
        dx = dx + s["dsummed"].float()
    param = s["weight"].dtype
    return {"dx": dx.to(s["x"].dtype), "dweight": (dy * xhat).sum(0).to(param), "dbias": dy.sum(0).to(param)}


def _slice(case, ids):
    """Each id's row of the slice, and whether it has one."""
    at = ids.long() - case["start"]
    return at, (at >= 0) & (at < case["rows"])


def _plain_embedding(s):
    at, mine = _slice(s["case"], s["ids"])
    rows = s["table"][torch.where(mine, at, torch.zeros_like(at))].float() * s["case"]["scale"]
    return torch.where(mine[:, None], rows, torch.zeros_like(rows)).to(s["table"].dtype)


def _plain_embedding_grad(s):
    case = s["case"]
    at, mine = _slice(case, s["ids"])
    total = torch.zeros(case["rows"] + 1, case["hidden"], device="cuda")
    total.index_add_(0, torch.where(mine, at, torch.full_like(at, case["rows"])), s["dout"].float())
    return (total[:-1] * case["scale"]).to(DTYPES[case["grad"]])


def _plain_gather(src, row):
    """The rows of src that the pairs have, in 32 bits, [tokens][choices][hidden]; zeros for a pair without one."""
    at = row.long()
    rows = src[at.clamp(min=0)].float()
    return torch.where((at >= 0)[..., None], rows, torch.zeros_like(rows))


def _plain_experts(s):
    case = s["case"]
    k = case["topk"]
    row, pair, offsets, counts = _plan(case, s["experts"])
    taken = s["x"][pair.long().clamp(min=0) // k]
    out = torch.where((pair >= 0)[:, None], taken, torch.zeros_like(taken))
    rows = _plain_gather(s["src"], row.view(-1, k))
    y = (rows * s["weights"][..., None]).sum(1).to(s["src"].dtype)
    return {"row_of_pair": row, "pair_of_row": pair, "offsets": offsets, "counts": counts, "out": out, "y": y}


def _plain_experts_grad(s):
    k, dt = s["case"]["topk"], s["src"].dtype
    row, pair = s["row_of_pair"].view(-1, k), s["pair_of_row"].long()
    dweights = (_plain_gather(s["src"], row) * s["dy"].float()[:, None]).sum(-1)
    of = pair.clamp(min=0)
    dsrc = s["weights"].reshape(-1)[of][:, None] * s["dy"][of // k].float()
    dsrc = torch.where((pair >= 0)[:, None], dsrc, torch.zeros_like(dsrc)).to(dt)
    dx = _plain_gather(s["dout"], row).sum(1).to(dt)
    return {"dsrc": dsrc, "dweights": dweights, "dx": dx}


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "embedding": _plain_embedding,
          "embedding_grad": _plain_embedding_grad, "experts": _plain_experts, "experts_grad": _plain_experts_grad}


# ---- the library's calls -------------------------------------------------------------------------------------------

def _workspace(s, nbytes):
    """The caller's workspace, made by the first call and kept as a program keeps it."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_norm(nb, s, case):
    nb.nuna_layernorm_forward(s["x"], s["y"], case["rows"], case["hidden"], weight=s["weight"], bias=s["bias"],
                              residual=s["residual"], summed=s["summed"], mean=s["mean"], rstd=s["rstd"], eps=EPS,
                              dtype=CODES[case["dtype"]], param_dtype=CODES[case["param"]],
                              x_stride=case["hidden"] + case["pad"], residual_stride=case["hidden"] + case["pad"])
    return {"summed": s["summed"], "y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}


def _own_norm_grad(nb, s, case):
    stride = case["hidden"] + case["pad"]
    ws = _workspace(s, nb.nuna_layernorm_workspace(case["rows"], case["hidden"]))
    nb.nuna_layernorm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["dx"], case["rows"], case["hidden"], weight=s["weight"],
                               dsummed=s["dsummed"], dweight=s["dweight"], dbias=s["dbias"], workspace=ws,
                               dtype=CODES[case["dtype"]], param_dtype=CODES[case["param"]],
                               dy_stride=stride, x_stride=stride, dsummed_stride=stride)
    return {"dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}


def _own_embedding(nb, s, case):
    nb.nuna_embedding_forward(s["ids"], s["table"], s["out"], case["tokens"], case["hidden"], case["rows"],
                              vocab_start=case["start"], scale=case["scale"], dtype=CODES[case["dtype"]],
                              id_bytes=s["ids"].element_size())
    return s["out"]


def _own_embedding_grad(nb, s, case):
    ws = _workspace(s, nb.nuna_embedding_workspace(case["tokens"], case["hidden"], case["rows"]))
    nb.nuna_embedding_backward(s["ids"], s["dout"], s["dtable"], case["tokens"], case["hidden"], case["rows"],
                               vocab_start=case["start"], scale=case["scale"], workspace=ws, dtype=CODES[case["dtype"]],
                               grad_dtype=CODES[case["grad"]], id_bytes=s["ids"].element_size())
    return s["dtable"]


def _empty_rows(s, case):
    """The rows' map where rows may have no pair (a capacity, other ranks' experts): those are zeros then."""
    return s["pair_of_row"] if case["capacity"] or case["local"] < case["total"] else None


def _own_experts(nb, s, case):
    n, k, rows, hidden, code = case["tokens"], case["topk"], _row_count(case), case["hidden"], CODES[case["dtype"]]
    nb.nuna_expert_sort(s["experts"], s["row_of_pair"], s["pair_of_row"], s["offsets"], n, k, case["local"], counts=s["counts"],
                        first_expert=case["first"], capacity=case["capacity"], id_bytes=s["experts"].element_size())
    nb.nuna_expert_dispatch(s["x"], s["row_of_pair"], s["out"], n, k, rows, hidden,
                            pair_of_row=_empty_rows(s, case), dtype=code)
    nb.nuna_expert_combine(s["src"], s["row_of_pair"], s["y"], n, k, rows, hidden, weights=s["weights"], dtype=code)
    return {name: s[name] for name in ("row_of_pair", "pair_of_row", "offsets", "counts", "out", "y")}


def _own_experts_grad(nb, s, case):
    n, k, rows, hidden, code = case["tokens"], case["topk"], _row_count(case), case["hidden"], CODES[case["dtype"]]
    nb.nuna_expert_combine_backward(s["dy"], s["src"], s["weights"], s["row_of_pair"], s["dsrc"], s["dweights"], n, k, rows, hidden,
                                    pair_of_row=_empty_rows(s, case), dtype=code)
    nb.nuna_expert_combine(s["dout"], s["row_of_pair"], s["dx"], n, k, rows, hidden, dtype=code)
    return {"dsrc": s["dsrc"], "dweights": s["dweights"], "dx": s["dx"]}


_OWN = {"norm": _own_norm, "norm_grad": _own_norm_grad, "embedding": _own_embedding,
        "embedding_grad": _own_embedding_grad, "experts": _own_experts, "experts_grad": _own_experts_grad}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2608_00867_b200 import binding as nb
        return _OWN[op](nb, state, state["case"])
    return _PLAIN[op](state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------

def _touched(case):
    """Expected ids inside the slice, and expected distinct rows among them, under _ids' frequencies (the slice's share of
    them is that of its size: the ranks are scattered)."""
    v, n, share = case["vocab"], case["tokens"], case["rows"] / case["vocab"]
    p = 1.0 / (np.arange(v) + 2.7)
    p /= p.sum()
    distinct = float(-np.expm1(n * np.log1p(-p)).sum())
    return n * share, distinct * share


def work(case):
    op, h, size = case["op"], case["hidden"], SIZES[case["dtype"]]
    if op in ("norm", "norm_grad"):
        n, psize = case["rows"], SIZES[case["param"]]
        if op == "norm":
            return {"bytes": n * h * size * (4 if case["residual"] else 2) + 2 * h * psize + 8 * n, "flops": 9 * n * h}
        return {"bytes": n * h * size * (4 if case["residual"] else 3) + 3 * h * psize + 8 * n, "flops": 16 * n * h}
    isize = 4 if case["ids"] == "i32" else 8
    if op == "embedding":
        _, distinct = _touched(case)
        return {"bytes": case["tokens"] * (isize + h * size) + distinct * h * size, "flops": case["tokens"] * h}
    if op == "embedding_grad":
        mine, _ = _touched(case)
        return {"bytes": case["tokens"] * isize + mine * h * size + case["rows"] * h * SIZES[case["grad"]], "flops": mine * h}
    n, pairs = case["tokens"], case["tokens"] * case["topk"]
    kept = pairs * case["local"] / case["total"]
    if case["capacity"]:
        kept = min(kept, case["local"] * case["capacity"])
    filled = _row_count(case) if case["capacity"] else kept
    if op == "experts":
        return {"bytes": pairs * (isize + 4 + 4) + _row_count(case) * 4 + (2 * n + filled + kept) * h * size, "flops": 2 * kept * h}
    return {"bytes": pairs * (4 + 4 + 4) + (2 * n + 2 * kept + filled) * h * size, "flops": 4 * kept * h}


# ---- the definition in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f = lambda name: None if s.get(name) is None else s[name].to(torch.float64)
    op, h = case["op"], case["hidden"]
    if op == "norm":
        x, stored = f("x"), None
        if case["residual"]:
            stored = x + f("residual")
            x = stored.to(DTYPES[case["dtype"]]).to(torch.float64)            # the norm is that of the rows as they are kept
        mean = x.sum(1) / h
        variance = (x - mean.unsqueeze(1)).square().sum(1) / h
        rstd = (variance + EPS).pow(-0.5)
        y = torch.addcmul(f("bias"), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), f("weight"))
        return {"summed": stored, "y": y, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        dy, r = f("dy"), f("rstd").unsqueeze(1)
        normal = (f("x") - f("mean").unsqueeze(1)) * r
        g = dy * f("weight")
        dx = r * (g - g.sum(1, keepdim=True) / h - normal * ((g * normal).sum(1, keepdim=True) / h))
        if case["residual"]:
            dx += f("dsummed")
        return {"dx": dx, "dweight": torch.einsum("th,th->h", dy, normal), "dbias": dy.sum(0)}
    if op in ("embedding", "embedding_grad"):
        ids = s["ids"].cpu().numpy().astype(np.int64) - case["start"]
        inside = np.nonzero((ids >= 0) & (ids < case["rows"]))[0]
        tokens, rows = torch.from_numpy(inside).cuda(), torch.from_numpy(ids[inside]).cuda()
        if op == "embedding":
            out = torch.zeros(case["tokens"], h, dtype=torch.float64, device="cuda")
            out[tokens] = f("table")[rows] * case["scale"]
            return out
        out = torch.zeros(case["rows"], h, dtype=torch.float64, device="cuda")
        out.index_add_(0, rows, f("dout")[tokens] * case["scale"])
        return out
    # the sort, one expert after the other
    ids, k, rows = s["experts"].cpu().numpy().reshape(-1).astype(np.int64), case["topk"], _row_count(case)
    row, pair = np.full(ids.size, -1, np.int32), np.full(rows, -1, np.int32)
    offsets, counts = np.zeros(case["local"] + 1, np.int32), np.zeros(case["local"], np.int32)
    at = 0
    for e in range(case["local"]):
        pairs = np.nonzero(ids == case["first"] + e)[0]
        counts[e], offsets[e] = pairs.size, at
        pairs = pairs[:case["capacity"]] if case["capacity"] else pairs
        row[pairs] = at + np.arange(pairs.size)
        pair[at:at + pairs.size] = pairs
        at += case["capacity"] if case["capacity"] else pairs.size
    offsets[-1] = at
    there, to = torch.from_numpy(np.nonzero(row >= 0)[0]).cuda(), torch.from_numpy(row[row >= 0].astype(np.int64)).cuda()
    weights = f("weights").reshape(-1)

    def back(name, weighted):
        total = torch.zeros(case["tokens"], h, dtype=torch.float64, device="cuda")
        taken = f(name)[to]
        return total.index_add_(0, there // k, taken * weights[there].unsqueeze(1) if weighted else taken)

    if op == "experts":
        out = torch.zeros(rows, h, dtype=torch.float64, device="cuda")
        out[to] = f("x")[there // k]
        return {"row_of_pair": row, "pair_of_row": pair, "offsets": offsets, "counts": counts, "out": out, "y": back("src", True)}
    dy = f("dy")[there // k]
    dsrc = torch.zeros(rows, h, dtype=torch.float64, device="cuda")
    dsrc[to] = dy * weights[there].unsqueeze(1)
    dweights = torch.zeros(weights.numel(), dtype=torch.float64, device="cuda")
    dweights[there] = torch.einsum("ph,ph->p", dy, f("src")[to])
    return {"dsrc": dsrc, "dweights": dweights.view(-1, k), "dx": back("dout", False)}
