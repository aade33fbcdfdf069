"""The experts' products where workgroups of the largest tiles take several, and where few rows take the weights straight to registers: sizes that the library's rules are asked about, so that a case cannot leave the
kernel that it is for.

Bounds as in test_gpu_experts; the definitions in 64 bits on the device, for the sizes that several tiles a workgroup need."""
import pytest
import torch

from tests.block_util import DTYPES, SUM, UNIT, TINY
from tests.expert_util import BACK, BACK_PAIR, LARGE, PAIR, PLAIN, takes_few_rows, tiles_of
from tests.test_gpu_experts import Case, _check_gated_forward, _check_linear_forward, _gated_backward, _gated_forward, _linear_backward, _linear_forward, _zeros, experts  # noqa: F401
from tests.test_gpu_gated import _act, _activation_error

pytestmark = pytest.mark.gpu


def _near(got, want, before, dtype, what):
    """got is `want`, off by `before`, rounded to `dtype`."""
    off = (got.double() - want).abs()
    bad = ~(off <= before + UNIT[dtype] * (want.abs() + before) + TINY[dtype])
    assert not bool(bad.any()), "%s: %d of %s, the first at %s" % (what, int(bad.sum()), tuple(got.shape), torch.nonzero(bad)[0].tolist())


class Device:
    """A case's tensors on the device, and an expert's part of them in 64 bits."""

    def __init__(self, c):
        self.c, self.x, self.grad, self.wg, self.wu, self.source = c, c.x.cuda(), c.grad.cuda(), c.wg.cuda(), c.wu.cuda(), c.source.cuda().long()

    def experts(self):
        for e, a, b in self.c.groups:
            x = self.x[a:b] if self.c.ordered else self.x[self.source[a:b]]
            yield e, a, b, x.double(), self.grad[a:b].double(), self.wg[e].double(), self.wu[e].double()


def _check_grad_x(d, got, parts):
    c = d.c
    want = torch.zeros(d.x.shape, dtype=torch.float64, device="cuda")
    off, size = torch.zeros_like(want), torch.zeros_like(want)
    for (e, a, b), (w, o) in zip(c.groups, parts):
        if c.ordered:
            want[a:b], off[a:b] = w, o
        else:                                                # (a token is there once)
            at = d.source[a:b]
            want[at] += w
            off[at] += o
            size[at] += w.abs() + o
    _near(got, want, off if c.ordered else off + c.chosen * SUM * size, c.dtype, "grad_x")
    if c.ordered:
        _zeros(got, c.used)


def _check_gated(d, h, gate, up, grads):
    """SiLU: forward and, from the gate and up that it left, backward."""
    c, few, parts = d.c, _activation_error(d.c.dtype), []
    gamma = (c.d + 1) * SUM
    for e, a, b, x, dh, wg, wu in d.experts():
        g, u = x @ wg.t(), x @ wu.t()
        eg, eu = gamma * (x.abs() @ wg.abs().t()), gamma * (x.abs() @ wu.abs().t())
        v = _act("silu", g)[0]
        ev = 1.13 * eg + few * (v.abs() + 1.13 * eg)
        _near(h[a:b], v * u, ev * (u.abs() + eu) + v.abs() * eu + SUM * v.abs() * u.abs(), c.dtype, "h of expert %d" % e)
        _near(gate[a:b], g, eg, c.dtype, "gate of expert %d" % e)
        _near(up[a:b], u, eu, c.dtype, "up of expert %d" % e)
        g, u = gate[a:b].double(), up[a:b].double()
        v, slope = _act("silu", g)
        dg, du = dh * u * slope, dh * v
        rounded = lambda t, before: before + UNIT[c.dtype] * (t.abs() + before) + TINY[c.dtype]  # noqa: E731
        eg, eu = rounded(dg, few * 2 * (dh * u).abs()), rounded(du, few * du.abs())
        size, off = dg.abs() @ wg.abs() + du.abs() @ wu.abs(), eg @ wg.abs() + eu @ wu.abs()
        parts.append((dg @ wg + du @ wu, off + (2 * c.f + 2) * SUM * (size + off)))
        for t, err, got, name in ((dg, eg, grads[1], "grad_w_gate"), (du, eu, grads[2], "grad_w_up")):
            off = err.t() @ x.abs()
            _near(got[e], t.t() @ x, off + (b - a + 1) * SUM * (t.abs().t() @ x.abs() + off), c.dtype, "%s of expert %d" % (name, e))
    for t in (h, gate, up):
        _zeros(t, c.used)
    _check_grad_x(d, grads[0], parts)


def _check_linear(d, y, grad_x, grad_w):
    c, parts = d.c, []
    for e, a, b, x, gy, w, _ in d.experts():
        _near(y[a:b], x @ w.t(), (c.d + 1) * SUM * (x.abs() @ w.abs().t()), c.dtype, "y of expert %d" % e)
        parts.append((gy @ w, (c.f + 1) * SUM * (gy.abs() @ w.abs())))
        _near(grad_w[e], gy.t() @ x, (b - a + 1) * SUM * (gy.abs().t() @ x.abs()), c.dtype, "grad_w of expert %d" % e)
    _zeros(y, c.used)
    _check_grad_x(d, grad_x, parts)


# for which products the largest tiles are more than two to a workgroup (or whole rounds of them and then parts): rows of outputs on 64-byte boundaries and off them, summed indices with a rest and without, more
# experts than a wave has lanes
@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype,size,several,in_parts", [
    ("bf16", (4224, 2, 2, 264, 4352), (PAIR, PLAIN), ()), ("f16", (4224, 3, 2, 272, 4360), (PAIR, PLAIN), ()),
    ("bf16", (4224, 2, 2, 4352, 264), (BACK, BACK_PAIR), ()), ("f16", (4224, 3, 2, 4360, 272), (BACK, BACK_PAIR), ()),
    ("f16", (2600, 2, 2, 2056, 4088), (), (PLAIN,)), ("bf16", (2600, 2, 2, 4096, 2048), (), (PAIR, BACK, BACK_PAIR)), ("f16", (2600, 2, 2, 4088, 2040), (), (PAIR, BACK, BACK_PAIR)),
    ("bf16", (10500, 70, 2, 264, 1544), (PAIR, PLAIN), ()), ("f16", (10500, 66, 2, 1544, 200), (BACK, BACK_PAIR), ())], ids=str)
def test_several_tiles_to_a_workgroup(experts, dtype, size, several, in_parts, ordered):  # noqa: F811
    c = Case(experts, size, DTYPES[dtype], 19, how="holes" if ordered else "some", ordered=ordered)
    for kind in several + in_parts:
        tiles, count, full, splits = tiles_of(kind, c.groups, c.rows, c.n, c.d, c.f, 2)
        assert tiles == LARGE and (count > 2 * 256 if kind in several else full >= 256 and splits > 1), (kind, tiles, count, full, splits)
    d = Device(c)
    h, gate, up = _gated_forward(experts, c, "silu")
    assert torch.equal(_gated_forward(experts, c, "silu", keep=False)[0], h)
    grads = _gated_backward(experts, c, "silu", gate, up)
    _check_gated(d, h, gate, up, grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, _gated_backward(experts, c, "silu", gate, up)))
    y, both = _linear_forward(experts, c), _linear_backward(experts, c)
    _check_linear(d, y, *both)
    assert torch.equal(y, _linear_forward(experts, c)) and all(torch.equal(a, b) for a, b in zip(both, _linear_backward(experts, c)))


# (tokens, experts, chosen, d, f): a decode step's sums, long and short, four units of 128 bytes for each of eight waves and more, with and without a rest; an odd number of 16-bit elements, so that rows begin off 4-byte
# boundaries in turn; more experts than a wave has lanes
FEW = [("f16", (8, 8, 2, 4101, 50), (PAIR, PLAIN)), ("bf16", (16, 16, 2, 4097, 72), (PAIR, PLAIN)), ("bf16", (5, 3, 1, 8191, 33), (PAIR, PLAIN)), ("f16", (4, 4, 2, 2049, 40), (PAIR, PLAIN)),
       ("bf16", (6, 4, 2, 1701, 65), (PAIR, PLAIN)), ("f16", (24, 70, 2, 1751, 30), (PAIR, PLAIN)), ("bf16", (70, 70, 2, 4099, 20), (PAIR, PLAIN)), ("f16", (40, 20, 3, 4104, 24), (PLAIN,)),
       ("f16", (8, 4, 1, 4096, 96), (PAIR, PLAIN)), ("bf16", (9, 4, 2, 6000, 17), (PLAIN,)), ("f32", (6, 6, 2, 2050, 40), (PAIR, PLAIN)), ("f32", (4, 4, 2, 4099, 36), (PAIR, PLAIN)),
       ("f32", (12, 6, 2, 1027, 25), (PAIR, PLAIN)), ("f32", (80, 70, 2, 1301, 9), (PAIR, PLAIN))]


@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype,size,kinds", FEW, ids=str)
def test_few_rows_take_the_weights_straight(experts, dtype, size, kinds, ordered):  # noqa: F811
    t, (tokens, n, chosen, d, f) = DTYPES[dtype], size
    for kind in kinds:
        assert takes_few_rows(kind, tokens * chosen, n, d, f, t.itemsize)
    for i, how in enumerate(("some", "one", "holes", "first")):
        for offset in (0, 1, 2):                             # (1: off the 4-byte boundaries that odd rows are read by)
            c = Case(experts, size, t, 60 + i, how=how, ordered=ordered)
            if PAIR in kinds:
                kept = _gated_forward(experts, c, "silu", offset=offset)
                _check_gated_forward(c, "silu", *kept)
                assert torch.equal(_gated_forward(experts, c, "silu", keep=False, offset=offset)[0], kept[0])
            _check_linear_forward(c, _linear_forward(experts, c, offset))


@pytest.mark.parametrize("way", ["tiles", "any"])
def test_more_tiles_than_a_launch_takes(experts, way):  # noqa: F811
    """Products whose tiles of 64 by 64 (of both projections 64 by 32) are more than 2^22 go in several launches: fetched straight to LDS, and at any alignment; every element looked at."""
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GiB")
    tokens, n, d = (1 << 20) + 77, 3, 8
    t, f = (torch.float32, 8200) if way == "tiles" else (torch.bfloat16, 16400)
    g = torch.Generator(device="cuda").manual_seed(70)
    x = torch.randn(tokens * d + 1, generator=g, device="cuda").to(t)[1 if way == "any" else 0:][:tokens * d].view(tokens, d)      # (off a 16-byte boundary, or on it)
    wg, wu = ((torch.randn(n, f, d, generator=g, device="cuda") / d ** 0.5).to(t) for _ in range(2))
    plan = experts.plan_of((torch.arange(tokens, device="cuda") * 7 % 10 % 4 - 1)[:, None], n)
    cols = 32 if way == "tiles" else 64
    o = plan.offsets.tolist()
    assert sum(-(-(b - a) // 64) for a, b in zip(o, o[1:] + [tokens])) * -(-f // cols) > 1 << 22
    out = torch.full((plan.rows, f), float("nan"), dtype=t, device="cuda")
    if way == "tiles":
        experts.bt_expert_gated_forward(x, plan, wg, wu, "relu", out, None, None, experts.new_gated_workspace(plan, d, f, t))
    else:
        experts.bt_expert_linear_forward(x, plan, wg, out, experts.new_linear_workspace(plan, d, f, t, ordered=False), ordered=False)
    gamma = (d + 1) * SUM
    for e in range(n):
        for a in range(o[e], o[e + 1], 1 << 16):
            b = min(a + (1 << 16), o[e + 1])
            v = x[plan.source[a:b].long()].double()
            want, off = v @ wg[e].double().t(), gamma * (v.abs() @ wg[e].double().abs().t())
            if way == "tiles":
                u, eu = v @ wu[e].double().t(), gamma * (v.abs() @ wu[e].double().abs().t())
                want.clamp_(min=0)
                off = off * (u.abs() + eu) + want * eu + SUM * (want * u).abs()
                want = want * u
            _near(out[a:b], want, off, t, "rows from %d on" % a)
            del want, off
    assert o[n] < tokens
    for a in range(o[n], tokens, 1 << 16):
        assert not bool(out[a:a + (1 << 16)].any())
