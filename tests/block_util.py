"""Helpers for the tests of the feed-forward sublayer's operators: inputs between guards, and bounds on rounding.

Inputs are cut out of buffers of NaN, so that a read outside of one shows in the results, and outputs out of buffers of a marker that has to
be there afterwards.  `offset` elements put a tensor off its 16-byte boundary.
"""
import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half the distance of neighbouring numbers at 1, and what a rounding may lose at zero at the most
UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -133}
SUM = 2.0 ** -24                                                    # of one 32-bit operation
_GUARD = 64


class Guarded:
    """Tensors in device memory with guards on both sides."""

    def __init__(self):
        self._outs = []

    @staticmethod
    def _cut(buf, shape, offset):
        n = 1
        for s in shape:
            n *= s
        return buf[_GUARD + offset:_GUARD + offset + n].view(shape)

    def put(self, t, offset=0):
        buf = torch.full((t.numel() + 2 * _GUARD + offset,), float("nan"), dtype=t.dtype, device="cuda")
        v = self._cut(buf, t.shape, offset)
        v.copy_(t)
        return v

    def out(self, shape, dtype, offset=0):
        n = 1
        for s in shape:
            n *= s
        buf = torch.full((n + 2 * _GUARD + offset,), 77.0, dtype=dtype, device="cuda")
        v = self._cut(buf, tuple(shape), offset)
        v.fill_(float("nan"))
        self._outs.append((buf, n, offset))
        return v

    def check(self):
        for buf, n, offset in self._outs:
            assert bool((buf[:_GUARD + offset] == 77.0).all()) and bool((buf[_GUARD + offset + n:] == 77.0).all()), "written outside of an output"


def within(got, want, bound, what):
    """|got - want| <= bound, element by element; `want` and `bound` in 64 bits on the host."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    off = (got - want).abs()
    ok = (off <= bound) | (torch.isnan(got) & torch.isnan(want)) | (got == want)
    if not bool(ok.all()):
        worst = torch.where(ok, torch.zeros_like(off), torch.nan_to_num(off / bound.clamp_min(1e-300), nan=1e300, posinf=1e300))
        i = int(worst.argmax())
        raise AssertionError("%s: element %d of %s is %r, not %r (bound %r; %d outside)" % (
            what, i, tuple(got.shape), got.flatten()[i].item(), want.flatten()[i].item(), bound.flatten()[i].item(), int((~ok).sum())))


def rounded(want, dtype, before):
    """The bound on a result that is off by `before` before it is rounded to `dtype`."""
    return before + UNIT[dtype] * (want.abs() + before) + TINY[dtype]
