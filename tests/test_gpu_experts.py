"""The experts' products and their gradients against their definitions in 64 bits, expert by expert.

Bounds, as for the dense projections: a sum of n products in 32 bits is off by at most (n + 1) 2^-24 of the sum of their magnitudes (any order); activations as there; a
token's rows of the gradient of x are added up in 32 bits, each addition off by 2^-24 of what has been added up; factors that are rounded to the type,
and results, are off by half a unit."""
import pytest
import torch

from tests.block_util import DTYPES, SUM, Guarded, rounded, within
from tests.expert_util import choices, plan_on_device
from tests.test_gpu_gated import _act, _activation_error, _check_forward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def experts():
    from paper_2110_15362_amd import experts
    experts.lib()
    return experts


def _weights(n, f, d, dtype, g):
    return (torch.randn(n, f, d, generator=g) / max(d, 1) ** 0.5).to(dtype)


class Case:
    """Inputs, plan and groups of (tokens, experts, chosen, d, f)."""

    def __init__(self, experts, size, dtype, seed, how="some", ordered=False):
        self.tokens, self.n, self.chosen, self.d, self.f = size
        g = torch.Generator().manual_seed(seed)
        self.ordered, self.dtype, self.rows = ordered, dtype, self.tokens * self.chosen
        self.x = torch.randn(self.rows if ordered else self.tokens, self.d, generator=g).to(dtype)
        self.wg, self.wu = _weights(self.n, self.f, self.d, dtype, g), _weights(self.n, self.f, self.d, dtype, g)
        self.grad = torch.randn(self.rows, self.f, generator=g).to(dtype)
        self.plan, self.groups, self.source = plan_on_device(experts, choices(self.tokens, self.n, self.chosen, seed + 1, how), self.n)
        self.used = self.groups[-1][2]
        # rows of no expert may hold anything
        self.grad[self.used:] = float("nan")
        if ordered:
            self.x[self.used:] = float("nan")

    def of(self, first, end):
        return self.x[first:end] if self.ordered else self.x[self.source[first:end].long()]


def _filled(ws):
    if ws is not None:
        ws.fill_(0xFF)                                       # NaNs: nothing may rest on what a workspace holds
    return ws


def _zeros(t, first):
    assert not bool(t[first:].cpu().view(torch.int16 if t.element_size() == 2 else torch.int32).any()), "rows of no expert"


# ---- the gated projections

def _gated_forward(experts, c, activation, keep=True, offset=0):
    m = Guarded()
    h = m.out((c.rows, c.f), c.dtype, offset)
    gate, up = (m.out(h.shape, c.dtype, offset), m.out(h.shape, c.dtype, offset)) if keep else (None, None)
    ws = _filled(experts.new_gated_workspace(c.plan, c.d, c.f, c.dtype, c.ordered))
    experts.bt_expert_gated_forward(m.put(c.x, offset), c.plan, m.put(c.wg, offset), m.put(c.wu, offset), activation, h, gate, up, ws, c.ordered)
    torch.cuda.synchronize()
    m.check()
    return h, gate, up


def _check_gated_forward(c, activation, h, gate=None, up=None):
    for e, a, b in c.groups:
        if b > a:
            _check_forward(c.of(a, b), c.wg[e], c.wu[e], activation, h[a:b], None if gate is None else gate[a:b], None if up is None else up[a:b])
    for t in (h, gate, up):
        if t is not None:
            _zeros(t, c.used)


def _gated_backward(experts, c, activation, gate, up, which=(True, True), offset=0):
    m = Guarded()
    grad_x = m.out(c.x.shape, c.dtype, offset) if which[0] else None
    grads = (m.out(c.wg.shape, c.dtype, offset), m.out(c.wu.shape, c.dtype, offset)) if which[1] else (None, None)
    ws = _filled(experts.new_gated_workspace(c.plan, c.d, c.f, c.dtype, c.ordered, backward=True))
    put = lambda t: m.put(t, offset)  # noqa: E731
    experts.bt_expert_gated_backward(put(c.grad), put(c.x), c.plan, put(c.wg), put(c.wu), put(gate.cpu()), put(up.cpu()), activation, grad_x, *grads, ws, c.ordered)
    torch.cuda.synchronize()
    m.check()
    return (grad_x,) + grads


def _check_grad_x(c, got, parts):
    """parts: of each group (want, bound, size of the sum) of its rows before they are added up and rounded."""
    want = torch.zeros(c.x.shape, dtype=torch.float64)
    off, size = torch.zeros_like(want), torch.zeros_like(want)
    for (e, a, b), (w, o) in zip(c.groups, parts):
        if b == a:
            continue
        if c.ordered:
            want[a:b], off[a:b] = w, o
        else:
            at = c.source[a:b].long()
            want[at] += w
            off[at] += o
            size[at] += w.abs() + o
    if not c.ordered:
        off = off + c.chosen * SUM * size
    within(got, want, rounded(want, c.dtype, off), "grad_x")
    if c.ordered:
        _zeros(got, c.used)


def _check_gated_backward(c, activation, gate, up, grads):
    few, parts = _activation_error(c.dtype), []
    for e, first, end in c.groups:
        dh, x, wg, wu, g, u = (t.double() for t in (c.grad[first:end], c.of(first, end), c.wg[e], c.wu[e], gate[first:end].cpu(), up[first:end].cpu()))
        a, slope = _act(activation, g)
        if activation == "relu":
            slope = (g > 0).double()
        dg, du = dh * u * slope, dh * a
        eg, eu = rounded(dg, c.dtype, few * 2 * (dh * u).abs()), rounded(du, c.dtype, few * du.abs())
        size, off = dg.abs() @ wg.abs() + du.abs() @ wu.abs(), eg @ wg.abs() + eu @ wu.abs()
        parts.append((dg @ wg + du @ wu, off + (2 * c.f + 2) * SUM * (size + off)))
        for d, err, got, name in ((dg, eg, grads[1], "grad_w_gate"), (du, eu, grads[2], "grad_w_up")):
            if got is not None:
                want, off = d.t() @ x, err.t() @ x.abs()
                within(got[e], want, rounded(want, c.dtype, off + (len(d) + 1) * SUM * (d.abs().t() @ x.abs() + off)), "%s of expert %d" % (name, e))
    if grads[0] is not None:
        _check_grad_x(c, grads[0], parts)


# tokens, experts, chosen, d, f: one token and many, one expert and many, experts without rows, tiles that end inside, rows of less than a vector and off the boundaries
SIZES = [(1, 1, 1, 1, 1), (1, 2, 1, 8, 8), (1, 4, 2, 64, 72), (2, 3, 3, 7, 5), (3, 64, 8, 96, 40), (5, 5, 2, 33, 129), (8, 16, 2, 256, 512), (16, 8, 1, 40, 16), (17, 7, 3, 65, 100),
         (33, 4, 2, 128, 257), (64, 2, 2, 200, 8), (65, 9, 4, 1001, 66), (100, 3, 2, 31, 333), (128, 300, 4, 64, 64), (129, 6, 2, 72, 136), (250, 5, 2, 264, 264),
         (300, 2, 1, 1000, 344), (513, 3, 2, 136, 520)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gated_forward(experts, dtype, size):
    for i, activation in enumerate(("relu", "silu", "gelu_tanh")):
        c = Case(experts, size, DTYPES[dtype], 10 * sum(size) + i, how=("some", "holes", "first")[i], ordered=i == 1)
        kept = _gated_forward(experts, c, activation)
        _check_gated_forward(c, activation, *kept)
        assert torch.equal(_gated_forward(experts, c, activation, keep=False)[0], kept[0])


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gated_backward(experts, dtype, size):
    for i, activation in enumerate(("relu", "silu", "gelu_tanh")):
        c = Case(experts, size, DTYPES[dtype], 10 * sum(size) + i, how=("some", "holes", "first")[i], ordered=i == 1)
        _, gate, up = _gated_forward(experts, c, activation)
        _check_gated_backward(c, activation, gate, up, _gated_backward(experts, c, activation, gate, up))


# ---- the product

def _linear_forward(experts, c, offset=0):
    m = Guarded()
    y = m.out((c.rows, c.f), c.dtype, offset)
    ws = _filled(experts.new_linear_workspace(c.plan, c.d, c.f, c.dtype, c.ordered))
    experts.bt_expert_linear_forward(m.put(c.x, offset), c.plan, m.put(c.wg, offset), y, ws, c.ordered)
    torch.cuda.synchronize()
    m.check()
    return y


def _check_linear_forward(c, y):
    for e, a, b in c.groups:
        x, w = c.of(a, b).double(), c.wg[e].double()
        within(y[a:b], x @ w.t(), rounded(x @ w.t(), c.dtype, (c.d + 1) * SUM * (x.abs() @ w.abs().t())), "y of expert %d" % e)
    _zeros(y, c.used)


def _linear_backward(experts, c, which=(True, True), offset=0):
    m = Guarded()
    grad_x, grad_w = m.out(c.x.shape, c.dtype, offset) if which[0] else None, m.out(c.wg.shape, c.dtype, offset) if which[1] else None
    ws = _filled(experts.new_linear_workspace(c.plan, c.d, c.f, c.dtype, c.ordered, backward=True))
    experts.bt_expert_linear_backward(m.put(c.grad, offset), m.put(c.x, offset), c.plan, m.put(c.wg, offset), grad_x, grad_w, ws, c.ordered)
    torch.cuda.synchronize()
    m.check()
    return grad_x, grad_w


def _check_linear_backward(c, grad_x, grad_w):
    parts = []
    for e, a, b in c.groups:
        gy, x, w = c.grad[a:b].double(), c.of(a, b).double(), c.wg[e].double()
        parts.append((gy @ w, (c.f + 1) * SUM * (gy.abs() @ w.abs())))
        if grad_w is not None:
            want = gy.t() @ x
            within(grad_w[e], want, rounded(want, c.dtype, (b - a + 1) * SUM * (gy.abs().t() @ x.abs())), "grad_w of expert %d" % e)
    if grad_x is not None:
        _check_grad_x(c, grad_x, parts)


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_linear(experts, dtype, size):
    for i, how in enumerate(("some", "holes", "first")):
        c = Case(experts, size, DTYPES[dtype], 10 * sum(size) + i, how=how, ordered=i != 1)
        _check_linear_forward(c, _linear_forward(experts, c))
        _check_linear_backward(c, *_linear_backward(experts, c))


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("size", [(1, 4, 2, 64, 72), (20, 3, 2, 128, 96), (140, 2, 1, 264, 200), (300, 2, 2, 1001, 65)], ids=str)
def test_tensors_off_a_16_byte_boundary(experts, dtype, size, offset):
    c = Case(experts, size, DTYPES[dtype], 5, how="holes")
    kept = _gated_forward(experts, c, "silu", offset=offset)
    _check_gated_forward(c, "silu", *kept)
    _check_gated_backward(c, "silu", *kept[1:], _gated_backward(experts, c, "silu", *kept[1:], offset=offset))
    _check_linear_forward(c, _linear_forward(experts, c, offset))
    _check_linear_backward(c, *_linear_backward(experts, c, offset=offset))


@pytest.mark.parametrize("how", ["one", "none", "even"])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("size", [(9, 5, 2, 72, 40), (200, 8, 2, 136, 72), (1100, 4, 2, 136, 264)], ids=str)
def test_all_rows_at_few_experts_and_none(experts, dtype, size, how):
    c = Case(experts, size, DTYPES[dtype], 6, how=how)
    kept = _gated_forward(experts, c, "gelu_tanh")
    _check_gated_forward(c, "gelu_tanh", *kept)
    _check_gated_backward(c, "gelu_tanh", *kept[1:], _gated_backward(experts, c, "gelu_tanh", *kept[1:]))
    _check_linear_forward(c, _linear_forward(experts, c))
    _check_linear_backward(c, *_linear_backward(experts, c))


@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gradients_that_are_not_wanted(experts, dtype, ordered):
    c = Case(experts, (70, 4, 2, 136, 88), DTYPES[dtype], 6, ordered=ordered)
    _, gate, up = _gated_forward(experts, c, "gelu_tanh")
    both, only_x, only_w = (_gated_backward(experts, c, "gelu_tanh", gate, up, which=w) for w in ((True, True), (True, False), (False, True)))
    assert torch.equal(both[0], only_x[0]) and torch.equal(both[1], only_w[1]) and torch.equal(both[2], only_w[2])
    both, only_x, only_w = (_linear_backward(experts, c, which=w) for w in ((True, True), (True, False), (False, True)))
    assert torch.equal(both[0], only_x[0]) and torch.equal(both[1], only_w[1])


@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_empty_sizes(experts, dtype, ordered):
    for size in ((0, 3, 2, 16, 24), (5, 3, 2, 0, 24), (5, 3, 2, 16, 0), (0, 3, 1, 0, 0), (70, 3, 2, 0, 24), (300, 3, 2, 0, 40), (300, 3, 2, 16, 0)):
        c = Case(experts, size, DTYPES[dtype], 7, ordered=ordered)
        h, gate, up = _gated_forward(experts, c, "relu")
        for t in (h, _linear_forward(experts, c)):
            assert t.shape == (c.rows, c.f) and not bool(t.any())
        for got, like in zip(_gated_backward(experts, c, "relu", gate, up) + _linear_backward(experts, c), (c.x, c.wg, c.wu, c.x, c.wg)):
            assert got.shape == like.shape and not bool(got.any()) and not bool(torch.isnan(got).any())


def test_one_expert_is_the_dense_projection(experts):
    """With one expert that all tokens use, forward and gradients are those of the dense operator within the roundings of either, the order of the rows that of the tokens."""
    from paper_2110_15362_amd import block
    for dtype in (torch.float32, torch.bfloat16):
        c = Case(experts, (200, 1, 1, 136, 264), dtype, 8)
        x, wg, wu = (t.cuda().requires_grad_() for t in (c.x, c.wg, c.wu))
        h = experts.gated_linear(x, c.plan, wg, wu, "silu")
        grads = torch.autograd.grad(h, (x, wg, wu), c.grad.cuda())
        dense = block.gated_linear(x, wg[0], wu[0], "silu")
        want = torch.autograd.grad(dense, (x, wg, wu), c.grad.cuda())
        for a, b in zip((h,) + grads, (dense,) + want):
            within(a, b.detach().cpu().double(), 4 * rounded(b.detach().cpu().double(), dtype, 300 * SUM * b.detach().abs().max().cpu().double()), "one expert")


def test_results_do_not_change_from_call_to_call(experts):
    c = Case(experts, (300, 5, 2, 520, 696), torch.bfloat16, 14)
    first = None
    for _ in range(3):
        kept = _gated_forward(experts, c, "silu")
        got = [t.cpu() for t in kept + _gated_backward(experts, c, "silu", *kept[1:]) + (_linear_forward(experts, c),) + _linear_backward(experts, c)]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


# the larger tiles, several of the largest to a workgroup, whole ones and ragged ones, summed indices with and without a rest, copies to 16-byte boundaries
@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype,size", [("bf16", (2100, 3, 2, 264, 2056)), ("f16", (4096, 2, 1, 1024, 2048)), ("bf16", (4500, 4, 2, 520, 1032)), ("f16", (1500, 8, 2, 1001, 1003)),
                                        ("f32", (700, 4, 2, 264, 520)), ("bf16", (1024, 2, 2, 2048, 4100))], ids=str)
def test_larger_tiles(experts, dtype, size, ordered):
    c = Case(experts, size, DTYPES[dtype], 18, how="holes" if ordered else "some", ordered=ordered)
    kept = _gated_forward(experts, c, "silu")
    _check_gated_forward(c, "silu", *kept)
    assert torch.equal(_gated_forward(experts, c, "silu", keep=False)[0], kept[0])
    grads = _gated_backward(experts, c, "silu", *kept[1:])
    _check_gated_backward(c, "silu", *kept[1:], grads)
    assert all(torch.equal(a, b) for a, b in zip(grads, _gated_backward(experts, c, "silu", *kept[1:])))
    _check_linear_forward(c, _linear_forward(experts, c))
    _check_linear_backward(c, *_linear_backward(experts, c))
