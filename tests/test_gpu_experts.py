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


# ---- which kernel

@pytest.mark.parametrize("dtype,size", [("bf16", (4, 16, 2, 4104, 72)), ("f16", (40, 8, 2, 4101, 50)), ("f32", (30, 6, 2, 2050, 40)), ("bf16", (2, 64, 8, 33, 4100)), ("bf16", (24, 4, 1, 4096, 300))], ids=str)
def test_few_rows(experts, dtype, size):
    """Weights straight to registers, an expert's rows in several sixteens; rows of an odd number of 16-bit elements."""
    for how in ("some", "one", "holes"):
        for offset in (0, 1, 2):
            c = Case(experts, size, DTYPES[dtype], 30 + offset, how=how)
            _check_gated_forward(c, "silu", *_gated_forward(experts, c, "silu", offset=offset))
            _check_linear_forward(c, _linear_forward(experts, c, offset))


@pytest.mark.parametrize("ordered", [False, True])
@pytest.mark.parametrize("dtype,size", [("bf16", (300, 2, 1, 4096, 264)), ("f16", (260, 3, 2, 2056, 200)), ("f32", (200, 2, 2, 1024, 136)), ("bf16", (700, 2, 2, 1032, 4104)), ("bf16", (4200, 2, 1, 2048, 520))], ids=str)
def test_tiles_in_parts(experts, dtype, size, ordered):
    """Long sums and few tiles, or few beyond whole rounds of them: parts of a tile's sum, joined."""
    c = Case(experts, size, DTYPES[dtype], 31, how="holes", ordered=ordered)
    kept = _gated_forward(experts, c, "gelu_tanh")
    _check_gated_forward(c, "gelu_tanh", *kept)
    grads = _gated_backward(experts, c, "gelu_tanh", *kept[1:])
    _check_gated_backward(c, "gelu_tanh", *kept[1:], grads)
    _check_linear_forward(c, _linear_forward(experts, c))
    both = _linear_backward(experts, c)
    _check_linear_backward(c, *both)
    for a, b in zip(grads + both, _gated_backward(experts, c, "gelu_tanh", *kept[1:]) + _linear_backward(experts, c)):
        assert torch.equal(a, b)


def test_infinities_and_nans_stay_in_their_rows(experts):
    """Rows of no expert that hold NaNs are not read, and what one row or one expert holds does not reach another's results."""
    t = torch.bfloat16
    for size in ((9, 5, 2, 72, 40), (300, 6, 2, 264, 200), (700, 4, 2, 520, 264)):
        c = Case(experts, size, t, 32, how="holes", ordered=True)
        e, first, end = max(c.groups, key=lambda g: g[2] - g[1])
        clean = _gated_forward(experts, c, "silu") + (_linear_forward(experts, c),)
        grads = _gated_backward(experts, c, "silu", *clean[1:3]) + _linear_backward(experts, c)
        c.x[first] = float("nan")
        c.x[end - 1] = float("inf")
        c.grad[first] = float("inf")
        other = torch.ones(c.rows, dtype=torch.bool)
        other[[first, end - 1]] = False
        got = _gated_forward(experts, c, "silu") + (_linear_forward(experts, c),)
        for a, b in zip(clean, got):
            assert torch.equal(a[other], b[other]) and not bool(torch.isfinite(b[first].float()).all())
        rest = torch.arange(c.n) != e
        got = _gated_backward(experts, c, "silu", *clean[1:3]) + _linear_backward(experts, c)
        for a, b, of_x in zip(grads, got, (True, False, False, True, False)):
            assert torch.equal(a[other], b[other]) if of_x else torch.equal(a[rest], b[rest])


def test_tables_that_reach_beyond_are_cut(experts):
    """Offsets and tokens outside of their ranges: results without meaning, inside of their tensors."""
    c = Case(experts, (40, 4, 2, 72, 40), torch.bfloat16, 33)
    for name, value in (("offsets", 1 << 30), ("offsets", -5), ("source", 1 << 30), ("source", -7), ("slots", 1 << 30), ("slots", -9)):
        plan, _, _ = plan_on_device(experts, choices(40, 4, 2, 34), 4)
        table = getattr(plan, name)
        table.view(-1)[1::2] = value
        c.plan = plan
        _, gate, up = _gated_forward(experts, c, "silu")
        _linear_forward(experts, c)
        gate, up = torch.zeros_like(gate), torch.zeros_like(up)
        _gated_backward(experts, c, "silu", gate, up)
        _linear_backward(experts, c)
        out = torch.empty(40, 40, dtype=torch.bfloat16, device="cuda")
        m = Guarded()
        y = m.put(c.grad)
        weights, grad_y, grad_w = torch.rand(40, 2, device="cuda"), m.out(c.grad.shape, torch.bfloat16), m.out((40, 2), torch.float32)
        experts.bt_combine_forward(y, plan, weights, out)
        experts.bt_combine_backward(out, y, plan, weights, grad_y, grad_w)
        torch.cuda.synchronize()
        m.check()


# ---- with autograd

def _sublayer(experts, x, w_router, wg, wu, wd, chosen, activation="silu", normalise=True):
    weights, plan = experts.route(x @ w_router.t(), chosen, normalise)
    return experts.combine(experts.linear(experts.gated_linear(x, plan, wg, wu, activation), plan, wd), plan, weights), plan


def _reference(x, w_router, wg, wu, wd, index, activation="silu", normalise=True):
    """The sublayer with given choices, in 64 bits, one expert after the other."""
    logits = x @ w_router.t()
    p = torch.softmax(torch.gather(logits, 1, index) if normalise else logits, dim=1)
    weights = p if normalise else torch.gather(p, 1, index)
    out = torch.zeros_like(x)
    for e in range(len(wg)):
        token, j = torch.nonzero(index == e, as_tuple=True)
        h = _act(activation, x[token] @ wg[e].t())[0] * (x[token] @ wu[e].t())
        out = out.index_add(0, token, (h @ wd[e].t()) * weights[token, j, None])
    return out


def _sublayer_inputs(tokens, n, d, f, seed):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(tokens, d, generator=g), torch.randn(n, d, generator=g) / d ** 0.5, torch.randn(n, f, d, generator=g) / d ** 0.5, torch.randn(n, f, d, generator=g) / d ** 0.5,
            torch.randn(n, d, f, generator=g) / f ** 0.5), torch.randn(tokens, d, generator=g)


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("activation", ["relu", "silu", "gelu_tanh"])
def test_a_sublayer_and_its_gradients(experts, activation, normalise):
    """Choice, gated projections, product back and sum together, in single precision: the output and every gradient within 1e-4 of its norm of the definition's by differentiation in 64 bits (a few
    thousand 32-bit operations lie between), and along a direction the difference of the definition's values."""
    inputs, v = _sublayer_inputs(90, 7, 72, 40, 40)
    dev = [t.cuda().requires_grad_() for t in inputs]
    out, plan = _sublayer(experts, *dev, 3, activation, normalise)
    out.backward(v.cuda())
    ref = [t.double().requires_grad_() for t in inputs]
    index = plan.index.cpu().long()
    want = _reference(*ref, index, activation, normalise)
    want.backward(v.double())
    assert float((out.detach().cpu().double() - want.detach()).norm()) <= 1e-4 * float(want.detach().norm())
    gen = torch.Generator().manual_seed(41)
    for i, (got, r) in enumerate(zip(dev, ref)):
        assert float((got.grad.cpu().double() - r.grad).norm()) <= 1e-4 * float(r.grad.norm()), i
        if activation == "relu":
            continue                                         # (whose gradient jumps)
        way = torch.randn(r.shape, generator=gen, dtype=torch.float64) / r.numel() ** 0.5

        def value(step):
            a = [t.double() for t in inputs]
            a[i] = a[i] + step * way
            return float((_reference(*a, index, activation, normalise) * v.double()).sum())
        slope = (value(1e-4) - value(-1e-4)) / 2e-4
        size = float((got.grad.cpu().double() * way).abs().sum())
        assert abs(float((got.grad.cpu().double() * way).sum()) - slope) <= 1e-5 * size + 1e-6 * max(1.0, abs(slope)), i


def test_strides_streams_and_frozen_weights(experts):
    """Transposed and expanded inputs and gradients, another stream, weights and inputs that need no gradient, no_grad."""
    inputs, v = _sublayer_inputs(60, 4, 48, 64, 42)
    x = inputs[0].t().contiguous().cuda().t().requires_grad_()
    wg = inputs[2].transpose(1, 2).contiguous().cuda().transpose(1, 2).requires_grad_()
    rest = [t.cuda().requires_grad_() for t in (inputs[1], inputs[3], inputs[4])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, plan = _sublayer(experts, x, rest[0], wg, rest[1], rest[2], 2)
        out.sum().backward()                                 # (a gradient of strides 0)
    torch.cuda.current_stream().wait_stream(side)
    ref = [t.double().requires_grad_() for t in inputs]
    _reference(*ref, plan.index.cpu().long()).sum().backward()
    for got, r in zip((x, rest[0], wg, rest[1], rest[2]), ref):
        assert float((got.grad.cpu().double() - r.grad).norm()) <= 1e-4 * float(r.grad.norm())
    frozen = [t.detach() for t in (rest[0], wg, rest[1], rest[2])]
    out, _ = _sublayer(experts, x, *frozen, 2)
    grad_x, = torch.autograd.grad(out.sum(), x)
    assert float((grad_x.cpu().double() - ref[0].grad).norm()) <= 1e-4 * float(ref[0].grad.norm())
    out, _ = _sublayer(experts, x.detach(), frozen[0], wg, *frozen[2:], 2)
    grad_w, = torch.autograd.grad(out.sum(), wg)
    assert torch.equal(grad_w, wg.grad)
    h = experts.linear(x, plan, wg, ordered=False)
    y = torch.cat([x.detach()[plan.source[a:b].long()] @ wg.detach()[e].t() for e, (a, b) in enumerate(zip(plan.offsets.tolist(), plan.offsets.tolist()[1:]))])
    assert torch.allclose(h, y, rtol=1e-4, atol=1e-4)
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            assert _sublayer(experts, x, rest[0], wg, rest[1], rest[2], 2)[0].grad_fn is None


def test_padding_tokens(experts):
    """Tokens whose logits are all -infinity have no expert: outputs of zero and no gradient, and the others' results are those without them."""
    inputs, v = _sublayer_inputs(50, 5, 40, 24, 43)
    x, wr, wg, wu, wd = (t.cuda() for t in inputs)
    real = torch.arange(50) % 10 < 7
    logits = (x @ wr.t()).masked_fill(~real.cuda()[:, None], float("-inf")).requires_grad_()
    x.requires_grad_()
    weights, plan = experts.route(logits, 2)
    out = experts.combine(experts.linear(experts.gated_linear(x, plan, wg, wu, "silu"), plan, wd), plan, weights)
    out.backward(v.cuda())
    for t in (out.detach(), x.grad, logits.grad, weights.detach()):
        assert not bool(t[~real.cuda()].any()) and bool(torch.isfinite(t).all())
    alone, plan2 = _sublayer(experts, x.detach()[real.cuda()], wr, wg, wu, wd, 2)
    assert torch.equal(alone, out.detach()[real.cuda()]) and plan2.rows == 70 and int(plan.offsets[-1]) == 70


def test_a_stash_keeps_what_relu_gates_save_compressed(experts):
    from paper_2110_15362_amd import autograd as ag
    inputs, v = _sublayer_inputs(512, 4, 128, 512, 44)
    dev = [t.cuda().requires_grad_() for t in inputs]

    def step():
        grads = torch.autograd.grad(_sublayer(experts, *dev, 2, "relu")[0].square().mean(), dev)
        return [g.clone() for g in grads]
    plain = step()
    stash = ag.BitmapStash(min_numel=4096)
    with stash:
        out = _sublayer(experts, *dev, 2, "relu")[0].square().mean()
    kept = torch.autograd.grad(out, dev)
    assert all(torch.equal(a, b) for a, b in zip(plain, kept))
    assert stash.stats["compressed"] >= 3 and stash.stats["stored_bytes"] < 0.9 * stash.stats["dense_bytes"]


def test_graph_replays(experts):
    """The calls of a sublayer and of its gradients recorded into a graph, replayed on other tokens, that go to other experts, with other work between the replays."""
    t, (tokens, n, chosen, d, f) = torch.bfloat16, (96, 5, 2, 264, 200)
    inputs, v = _sublayer_inputs(tokens, n, d, f, 45)
    x, wr, wg, wu, wd = (s.cuda().to(t) for s in inputs)
    go = v.cuda().to(t)
    plan = experts.new_plan(tokens, n, chosen)
    empty = lambda *s, dtype=t: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
    logits, weights, grad_weights, grad_logits = empty(tokens, n), empty(tokens, chosen, dtype=torch.float32), empty(tokens, chosen, dtype=torch.float32), empty(tokens, n)
    h, gate, up, grad_h = (empty(plan.rows, f) for _ in range(4))
    y, grad_y, out, grad_x = empty(plan.rows, d), empty(plan.rows, d), empty(tokens, d), empty(tokens, d)
    grads = torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)
    ws = [experts.new_route_workspace(tokens, n, chosen), experts.new_gated_workspace(plan, d, f, t, backward=True), experts.new_linear_workspace(plan, f, d, t, backward=True)]

    def calls():
        torch.mm(x, wr.t(), out=logits)
        experts.bt_route_forward(logits, plan, weights, ws[0])
        experts.bt_expert_gated_forward(x, plan, wg, wu, "silu", h, gate, up, ws[1])
        experts.bt_expert_linear_forward(h, plan, wd, y, ws[2])
        experts.bt_combine_forward(y, plan, weights, out)
        experts.bt_combine_backward(go, y, plan, weights, grad_y, grad_weights)
        experts.bt_expert_linear_backward(grad_y, h, plan, wd, grad_h, grads[2], ws[2])
        experts.bt_expert_gated_backward(grad_h, x, plan, wg, wu, gate, up, "silu", grad_x, grads[0], grads[1], ws[1])
        experts.bt_route_backward(grad_weights, logits, plan, weights, grad_logits)
    results = (weights, plan.index, plan.slots, plan.source, plan.offsets, h, y, out, grad_y, grad_weights, grad_h, grad_x, grad_logits) + grads
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        x.copy_(torch.randn(tokens, d, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        got = [s.clone() for s in results]
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, results)), i


def test_two_streams_with_workspaces_of_their_own(experts):
    """Calls on two streams at once, each with its workspace, have the results of calls one after the other."""
    cases = [Case(experts, (700, 4, 2, 520, 264), torch.bfloat16, 50 + i) for i in range(2)]
    put = [[t.cuda() for t in (c.x, c.wg, c.wu)] for c in cases]
    outs = [[torch.empty(c.rows, c.f, dtype=c.dtype, device="cuda") for _ in range(2)] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        experts.bt_expert_gated_forward(put[i][0], c.plan, *put[i][1:], "silu", outs[i][0], None, None, experts.new_gated_workspace(c.plan, c.d, c.f, c.dtype))
    torch.cuda.synchronize()
    spaces = [experts.new_gated_workspace(c.plan, c.d, c.f, c.dtype) for c in cases]
    for _ in range(5):
        for i, c in enumerate(cases):
            experts.bt_expert_gated_forward(put[i][0], c.plan, *put[i][1:], "silu", outs[i][1], None, None, spaces[i], stream=streams[i])
    torch.cuda.synchronize()
    for a, b in outs:
        assert torch.equal(a, b)


def test_no_tokens(experts):
    """A batch without tokens goes through a whole sublayer and back: empty outputs, zeros for the weights' gradients."""
    inputs, _ = _sublayer_inputs(3, 4, 24, 16, 60)
    dev = [inputs[0][:0].cuda().requires_grad_()] + [t.cuda().requires_grad_() for t in inputs[1:]]
    out, plan = _sublayer(experts, *dev, 2)
    assert out.shape == (0, 24) and plan.rows == 0 and plan.offsets.tolist() == [0] * 5
    out.sum().backward()
    assert dev[0].grad.shape == (0, 24) and not any(bool(t.grad.any()) for t in dev[1:])
    assert experts.plan_of(torch.empty(0, 2, dtype=torch.int64, device="cuda"), 4).offsets.tolist() == [0] * 5


@pytest.mark.parametrize("dtype,tokens,chosen,d,f", [("bf16", 70001, 2, 64, 16400), ("f32", 40000, 2, 33, 27000)], ids=str)
def test_outputs_beyond_2_to_the_31_elements(experts, dtype, tokens, chosen, d, f):
    """Element offsets that pass 32 bits, in forward outputs, factors and gradients, aligned and through the kernel for any alignment; rows of every expert looked at."""
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GiB")
    t, n = DTYPES[dtype], 3
    g = torch.Generator(device="cuda").manual_seed(61)
    x = torch.randn(tokens, d, generator=g, device="cuda").to(t)
    w = (torch.randn(n, f, d, generator=g, device="cuda") / d ** 0.5).to(t)
    index = torch.stack([torch.arange(tokens) % n, (torch.arange(tokens) + 1) % n], dim=1).int().cuda()
    plan = experts.plan_of(index, n)
    assert plan.rows * f > 1 << 31
    y = torch.full((plan.rows, f), float("nan"), dtype=t, device="cuda")
    ws = experts.new_linear_workspace(plan, d, f, t, ordered=False, backward=True)
    experts.bt_expert_linear_forward(x, plan, w, y, ws, ordered=False)
    o = plan.offsets.tolist()
    for e in range(n):
        for row in (o[e], (o[e] + o[e + 1]) // 2, o[e + 1] - 1):
            v, m = x[plan.source[row]].double(), w[e].double()
            within(y[row], (m @ v).cpu(), rounded((m @ v).cpu(), t, (d + 1) * SUM * (m.abs() @ v.abs()).cpu()), "row %d" % row)
    grad_x, grad_w = torch.empty_like(x), torch.empty_like(w)
    experts.bt_expert_linear_backward(y, x, plan, w, grad_x, grad_w, ws, ordered=False)
    for token in (0, tokens // 2, tokens - 1):
        want, off = torch.zeros(d, dtype=torch.float64), torch.zeros(d, dtype=torch.float64)
        for j in range(chosen):
            e, gy = int(index[token, j]), y[plan.slots[token, j]].double()
            want += (gy @ w[e].double()).cpu()
            off += (f + 3) * SUM * (gy.abs() @ w[e].double().abs()).cpu()
        within(grad_x[token], want, rounded(want, t, off), "grad_x of token %d" % token)
    for e in range(n):
        gy, v = y[o[e]:o[e + 1], f - 8:].double(), x[plan.source[o[e]:o[e + 1]].long()].double()
        within(grad_w[e, f - 8:], (gy.t() @ v).cpu(), rounded((gy.t() @ v).cpu(), t, (len(v) + 1) * SUM * (gy.abs().t() @ v.abs()).cpu()), "grad_w of expert %d" % e)


def test_gathered_tokens_beyond_2_gib(experts):
    """x of more bytes than a descriptor's offsets reach: gathered by 64-bit addresses."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    t, tokens, d, f, n = torch.bfloat16, 600000, 2048, 64, 4
    g = torch.Generator(device="cuda").manual_seed(62)
    x = torch.randn(tokens, d, generator=g, device="cuda", dtype=t)
    w = (torch.randn(n, f, d, generator=g, device="cuda") / d ** 0.5).to(t)
    index = (torch.arange(tokens, device="cuda") * 7 % 5 - 1).int()[:, None]          # (one in five has none)
    plan = experts.plan_of(index, n)
    y = experts.linear(x, plan, w, ordered=False)
    o = plan.offsets.tolist()
    assert o[n] == tokens * 4 // 5 and not bool(y[o[n]:].any())
    for e in range(n):
        at = plan.source[o[e]:o[e + 1]].long()
        assert bool((index[at, 0] == e).all())
        for part in (slice(0, 100), slice(-100, None)):
            v, m = x[at[part]].double(), w[e].double()
            within(y[o[e]:o[e + 1]][part], (v @ m.t()).cpu(), rounded((v @ m.t()).cpu(), t, (d + 1) * SUM * (v.abs() @ m.abs().t()).cpu()), "expert %d" % e)
