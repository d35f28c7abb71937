"""What the GPU tests of the operators share: rows with gaps and guards around them, and comparisons."""
import torch

from paper_2608_00867_b200 import binding as nb

DTYPES = {"bf16": (torch.bfloat16, nb.NUNA_BF16), "f16": (torch.float16, nb.NUNA_F16), "f32": (torch.float32, nb.NUNA_F32)}
GUARD = 13.0                                   # exact in every type
U = 2.0 ** -24                                 # half a step of binary32


def half_step(dtype):
    """Relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """The step between the type's smallest values."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


class Rows:
    """rows x hidden elements, `pad` elements between rows and `shift` before them, in a buffer that is guarded throughout."""

    def __init__(self, rows, hidden, dtype, pad=0, shift=0, values=None):
        self.rows, self.hidden, self.stride = rows, hidden, hidden + pad
        self.whole = torch.full((shift + rows * self.stride + 64,), GUARD, dtype=dtype, device="cuda")
        self.flat = self.whole[shift:]
        self.v = torch.as_strided(self.whole, (rows, hidden), (self.stride, 1), shift)
        if values is not None:
            self.v.copy_(values)

    def untouched(self):
        """Whether everything around the rows is as it was."""
        left = self.whole.clone()
        torch.as_strided(left, (self.rows, self.hidden), (self.stride, 1), self.whole.numel() - self.flat.numel()).fill_(GUARD)
        return bool((left == GUARD).all())


def guarded(n, dtype, fill=GUARD):
    """A vector of n elements with a guard behind it: (what a call gets, the whole)."""
    whole = torch.full((n + 16,), fill, dtype=dtype, device="cuda")
    return whole[:n], whole


def generator(*seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(hash(seed) & 0x7FFFFFFF)
    return gen


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def integers(gen, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=gen, device="cuda").float()


def within(got, want, bound, what):
    """|got - want| <= bound, element by element, in 64 bits; NaN where NaN is wanted."""
    got = got.double()
    assert got.shape == want.shape, what
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), (what, "NaN")
    excess = torch.where(nan | (got == want), torch.zeros_like(want), (got - want).abs() - bound)
    worst = float(excess.max()) if excess.numel() else 0.0
    assert worst <= 0.0, (what, worst, int((excess > 0).sum()), "of", excess.numel())
