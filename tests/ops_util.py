"""What the tests of the operators share: inputs from a seed, matrices at awkward places, half steps of the types."""
import torch

U = 2.0 ** -24                                        # half a step of binary32
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
DEV = "cuda"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


class Placed:
    """A matrix [rows, cols] with `gap` elements between rows, `off` elements into its buffer; the rest of the buffer is marked."""

    MARK = 12345.0

    def __init__(self, rows, cols, dtype, gap=0, off=0):
        self.ld, self.off, self.rows, self.cols = cols + gap, off, rows, cols
        self.buf = torch.full((off + max(rows, 1) * self.ld + 64,), self.MARK, dtype=torch.float32, device=DEV).to(dtype)
        self.t = self.buf[off:].as_strided((rows, cols), (self.ld, 1), off)
        self.mark = self.buf[-1].clone()

    def put(self, x):
        self.t.copy_(x)
        return self

    def intact(self):
        """Nothing outside the matrix was written."""
        other = torch.ones_like(self.buf, dtype=torch.bool)
        other[self.off:].as_strided((self.rows, self.cols), (self.ld, 1), self.off).fill_(False)
        return bool((self.buf[other] == self.mark).all())


def within(got, want, tol, what=""):
    """|got - want| <= tol element by element, in 64 bits; NaN and infinities have to agree."""
    got, want = got.double(), want.double()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=want.device).expand_as(want)
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~(same | ((got - want).abs() <= tol))
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d out, first at %s: got %.9g, want %.9g, tolerance %.3g" % (
            what, int(bad.sum()), bad.numel(), i, float(got[i]), float(want[i]), float(tol[i])))


def two_to(n):
    """2^n in 64 bits, exact."""
    return ((n.to(torch.int64) + 1023) << 52).view(torch.float64)


def saved64(x):
    """(q, e) of a checkpoint of x [rows, cols], from its definition, in 64 bits."""
    rows, cols = x.shape
    g = torch.cat([x.double(), torch.zeros(rows, -cols % 32, dtype=torch.float64, device=x.device)], 1).unflatten(1, (-1, 32))
    a = g.abs().amax(2)
    finite = torch.isfinite(g).all(2)
    power = torch.frexp(torch.where(finite & (a > 0), a, 2.0 ** -1000)).exponent - 1
    e = (power - 6 + 127).clamp(min=1)
    q = torch.where(finite[:, :, None], torch.round(g / two_to(e - 127)[:, :, None]).clamp(-127, 127), 0.0)
    return q.nan_to_num(0.0).to(torch.int8).flatten(1), torch.where(finite, e, 255).to(torch.uint8)


def stands_for(q, e, cols):
    """The values of a checkpoint in 64 bits."""
    step = two_to(e.to(torch.int64) - 127).masked_fill(e == 255, float("nan"))
    return (q.double() * step.repeat_interleave(32, 1))[:, :cols]
