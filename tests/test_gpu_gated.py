"""The gated projections and their gradients against their definitions in 64 bits.

Bounds: a sum of n products in 32 bits is off by at most (n + 1) 2^-24 of the sum of their magnitudes (any order); the activations and
their slopes are off by a factor of at most 2^-18 (16-bit types: one 2^x and one 1/x instruction, the exponent's argument rounded) or 2^-20 and
follow an error of their argument with a slope of at most 1.13; factors that are rounded to the type, and results, are off by half a unit."""
import math

import pytest
import torch

from tests.block_util import DTYPES, UNIT, SUM, Guarded, rounded, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def block():
    from paper_2110_15362_amd import block
    block.lib()
    return block


def _act(name, g):
    """act(g) and act'(g)."""
    if name == "relu":
        return torch.where(g <= 0, torch.zeros_like(g), g), (g > 0).to(g.dtype)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 2 * c * (1 + 3 * 0.044715 * g * g)


def _activation_error(dtype):
    return 2.0 ** -20 if dtype == torch.float32 else 2.0 ** -18


def _inputs(rows, d, f, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, d, generator=g).to(dtype)
    wg = (torch.randn(f, d, generator=g) / max(d, 1) ** 0.5).to(dtype)
    wu = (torch.randn(f, d, generator=g) / max(d, 1) ** 0.5).to(dtype)
    return x, wg, wu, torch.randn(rows, f, generator=g).to(dtype)


def _products(x, wg, wu):
    """g and u and the bounds on their errors."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    gamma = (x.shape[1] + 1) * SUM
    return x @ wg.t(), x @ wu.t(), gamma * (x.abs() @ wg.abs().t()), gamma * (x.abs() @ wu.abs().t())


def _check_forward(x, wg, wu, activation, h, gate=None, up=None):
    dtype = x.dtype
    g, u, eg, eu = _products(x, wg, wu)
    a, _ = _act(activation, g)
    ea = 1.13 * eg + _activation_error(dtype) * (a.abs() + 1.13 * eg)
    within(h, a * u, rounded(a * u, dtype, ea * (u.abs() + eu) + a.abs() * eu + SUM * a.abs() * u.abs()), "h")
    if gate is None:
        return
    if activation == "relu":
        within(gate, a, rounded(a, dtype, eg), "gate")
        sure = g.abs() > eg                                  # which side of 0 it is on
        kept = torch.where(g > 0, u, torch.zeros_like(u))
        within(torch.where(sure, up.cpu().double(), kept), kept, rounded(kept, dtype, eu), "up")
        closed = gate.cpu() == 0
        for t in (h, gate, up):                              # zero as a bit pattern, together
            assert not bool(t.cpu()[closed].view(torch.int16 if t.element_size() == 2 else torch.int32).any())
    else:
        within(gate, g, rounded(g, dtype, eg), "gate")
        within(up, u, rounded(u, dtype, eu), "up")


def _forward(block, x, wg, wu, activation, keep=True, offset=0):
    m, (f, d), dtype = Guarded(), wg.shape, x.dtype
    h = m.out((x.shape[0], f), dtype, offset)
    gate, up = (m.out(h.shape, dtype, offset), m.out(h.shape, dtype, offset)) if keep else (None, None)
    block.bt_gated_forward(m.put(x, offset), m.put(wg, offset), m.put(wu, offset), activation, h, gate, up, block.new_gated_workspace(x.shape[0], d, f, dtype))
    torch.cuda.synchronize()
    m.check()
    return h, gate, up


def _check_backward(grad_h, x, wg, wu, gate, up, activation, grads):
    dtype = x.dtype
    dh, x, wg, wu, g, u = (t.double() for t in (grad_h, x, wg, wu, gate, up))
    a, slope = _act(activation, g)
    if activation == "relu":
        slope = (g > 0).double()
    dg, du = dh * u * slope, dh * a
    # the slope of an activation is a sum that may cancel: its error is that of its terms, of at most 1 + |g| / 4 + ...: 2 at the most
    few = _activation_error(dtype)
    eg, eu = rounded(dg, dtype, few * 2 * (dh * u).abs()), rounded(du, dtype, few * du.abs())
    if grads[0] is not None:
        gamma, want = (2 * dg.shape[1] + 2) * SUM, dg @ wg + du @ wu
        size = dg.abs() @ wg.abs() + du.abs() @ wu.abs()
        off = eg @ wg.abs() + eu @ wu.abs()
        within(grads[0], want, rounded(want, dtype, off + gamma * (size + off)), "grad_x")
    for d, e, got, name in ((dg, eg, grads[1], "grad_w_gate"), (du, eu, grads[2], "grad_w_up")):
        if got is not None:
            gamma, want = (d.shape[0] + 1) * SUM, d.t() @ x
            off = e.t() @ x.abs()
            within(got, want, rounded(want, dtype, off + gamma * (d.abs().t() @ x.abs() + off)), name)


def _backward(block, grad_h, x, wg, wu, gate, up, activation, which=(True, True), offset=0):
    m, dtype = Guarded(), x.dtype
    grad_x = m.out(x.shape, dtype, offset) if which[0] else None
    grad_wg, grad_wu = (m.out(wg.shape, dtype, offset), m.out(wu.shape, dtype, offset)) if which[1] else (None, None)
    ws = block.new_gated_workspace(x.shape[0], x.shape[1], wg.shape[0], dtype, backward=True)
    if ws is not None:
        ws.fill_(0xFF)                                       # NaNs: nothing may rest on what a workspace holds
    block.bt_gated_backward(*(m.put(t, offset) for t in (grad_h, x, wg, wu, gate, up)), activation, grad_x, grad_wg, grad_wu, ws)
    torch.cuda.synchronize()
    m.check()
    return grad_x, grad_wg, grad_wu


# one row and many, less than a step of the summed index and several tiles, tiles that end inside
SIZES = [(1, 1, 1), (1, 8, 8), (1, 64, 64), (1, 1024, 300), (2, 7, 5), (3, 96, 40), (5, 33, 129), (8, 256, 512), (16, 40, 16), (17, 65, 100), (31, 520, 72),
         (33, 128, 257), (64, 200, 8), (65, 1001, 66), (100, 31, 999), (128, 64, 128), (129, 72, 136), (130, 129, 131), (250, 256, 264), (257, 320, 640),
         (300, 1000, 344), (513, 136, 1032)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_forward(block, dtype, size):
    for i, activation in enumerate(("relu", "silu", "gelu_tanh")):
        x, wg, wu, _ = _inputs(*size, DTYPES[dtype], 10 * sum(size) + i)
        kept = _forward(block, x, wg, wu, activation, keep=True)
        _check_forward(x, wg, wu, activation, *kept)
        alone = _forward(block, x, wg, wu, activation, keep=False)[0]
        assert torch.equal(alone, kept[0])


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_backward(block, dtype, size):
    for i, activation in enumerate(("relu", "silu", "gelu_tanh")):
        x, wg, wu, grad_h = _inputs(*size, DTYPES[dtype], 10 * sum(size) + i)
        _, gate, up = _forward(block, x, wg, wu, activation)
        grads = _backward(block, grad_h, x, wg, wu, gate.cpu(), up.cpu(), activation)
        _check_backward(grad_h, x, wg, wu, gate.cpu(), up.cpu(), activation, grads)


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("size", [(1, 64, 72), (20, 128, 96), (140, 264, 200)], ids=str)
def test_tensors_off_a_16_byte_boundary(block, dtype, size, offset):
    x, wg, wu, grad_h = _inputs(*size, DTYPES[dtype], 5)
    kept = _forward(block, x, wg, wu, "silu", offset=offset)
    _check_forward(x, wg, wu, "silu", *kept)
    gate, up = kept[1].cpu(), kept[2].cpu()
    _check_backward(grad_h, x, wg, wu, gate, up, "silu", _backward(block, grad_h, x, wg, wu, gate, up, "silu", offset=offset))


# rows of an odd number of elements, or of less than a vector, none on a 16-byte boundary but the first: through registers, several tiles on their way
@pytest.mark.parametrize("offset", [0, 1, 2])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("size", [(1, 515, 100), (16, 1031, 50), (20, 129, 33), (32, 1001, 72), (40, 1001, 333), (64, 3, 40), (90, 9, 7), (100, 2003, 70), (127, 291, 601)], ids=str)
def test_rows_off_the_boundaries(block, dtype, size, offset):
    x, wg, wu, grad_h = _inputs(*size, DTYPES[dtype], 11 + offset)
    kept = _forward(block, x, wg, wu, "gelu_tanh", offset=offset)
    _check_forward(x, wg, wu, "gelu_tanh", *kept)
    gate, up = kept[1].cpu(), kept[2].cpu()
    _check_backward(grad_h, x, wg, wu, gate, up, "gelu_tanh", _backward(block, grad_h, x, wg, wu, gate, up, "gelu_tanh", offset=offset))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gradients_that_are_not_wanted(block, dtype):
    x, wg, wu, grad_h = _inputs(70, 136, 88, DTYPES[dtype], 6)
    _, gate, up = _forward(block, x, wg, wu, "gelu_tanh")
    args = grad_h, x, wg, wu, gate.cpu(), up.cpu(), "gelu_tanh"
    both, only_x, only_w = (_backward(block, *args, which=w) for w in ((True, True), (True, False), (False, True)))
    assert torch.equal(both[0], only_x[0]) and torch.equal(both[1], only_w[1]) and torch.equal(both[2], only_w[2])


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_empty_sizes(block, dtype):
    t = DTYPES[dtype]
    for rows, d, f in ((0, 16, 24), (5, 0, 24), (5, 16, 0), (0, 0, 0), (70, 0, 24), (300, 0, 40), (300, 16, 0)):
        x, wg, wu, grad_h = _inputs(rows, d, f, t, 7)
        h, gate, up = _forward(block, x, wg, wu, "relu")
        assert h.shape == (rows, f) and not bool(h.any())
        for got, like in zip(_backward(block, grad_h, x, wg, wu, gate.cpu(), up.cpu(), "relu"), (x, wg, wu)):
            assert got.shape == like.shape and not bool(got.any()) and not bool(torch.isnan(got).any())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_a_closed_relu_gate_selects(block, dtype):
    """Where the gate is closed nothing of the other factor comes through, not as a NaN or a negative zero; a NaN gate is one in the output."""
    t = DTYPES[dtype]
    x = torch.eye(4, dtype=t)
    inf, nan = float("inf"), float("nan")
    wg = torch.tensor([[-1.0, 1.0, 0.0, nan]], dtype=t).repeat(3, 1)
    wu = torch.tensor([[-2.0, -2.0, -2.0, -2.0], [inf, 2.0, -inf, 2.0], [nan, 3.0, nan, 3.0]], dtype=t)
    # (a row of x with one 1 leaves the others as 0 * w: rows of the identity need finite weights elsewhere)
    for row in range(4):
        one = torch.zeros(1, 1, dtype=t) + 1
        h, gate, up = _forward(block, one, wg[:, row:row + 1].contiguous(), wu[:, row:row + 1].contiguous(), "relu")
        g = wg[:, row].float()
        want = torch.where(g <= 0, torch.zeros_like(g), g * wu[:, row].float())
        got = h[0].cpu().float()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(5.0), want.nan_to_num(5.0)), (row, got, want)
        if row in (0, 2):
            for v in (h, gate, up):
                assert not bool(v.cpu().view(torch.int16 if v.element_size() == 2 else torch.int32).any())
            grads = _backward(block, torch.tensor([[inf, nan, 1.0]], dtype=t), one, wg[:, row:row + 1].contiguous(), wu[:, 1:2].contiguous(), gate.cpu(), up.cpu(), "relu")
            assert not any(bool(v.any()) for v in grads)


@pytest.mark.parametrize("size", [(1, 8, 16), (20, 9, 40), (40, 11, 7), (64, 4096, 72), (200, 40, 136)], ids=str)
def test_a_relu_gate_that_f16_does_not_hold_stays_open(block, size):
    """A pre-activation of 2^-26, which f16 rounds to 0: the gate is open, and its gradient is grad_h * u."""
    rows, d, f = size
    x, wg, wu = (torch.zeros(s, dtype=torch.float16) for s in ((rows, d), (f, d), (f, d)))
    x[:, 0], wg[:, 0], wu[:, 0] = 2.0 ** -13, 2.0 ** -13, 2.0 ** 13
    wg[1::2, 0] = -(2.0 ** -13)                              # (every other one is closed)
    h, gate, up = _forward(block, x, wg, wu, "relu")
    open_ = (torch.arange(f) % 2 == 0).expand(rows, f)
    assert not bool(h.any()) and torch.equal(gate.cpu() > 0, open_) and torch.equal(up.cpu(), open_.half())
    assert bool((gate.cpu().double() <= 2.0 ** -24).all())   # the smallest number that is not 0
    grads = _backward(block, torch.ones(rows, f, dtype=torch.float16), x, wg, wu, gate.cpu(), up.cpu(), "relu")
    want = torch.zeros(f, d, dtype=torch.float64)
    want[::2, 0] = rows * 2.0 ** -13
    within(grads[1], want, rounded(want, torch.float16, (rows + 1) * SUM * want), "grad_w_gate")


def test_values_at_the_ends_of_the_range(block):
    """Pre-activations that exp takes to infinity or 0: the activations are 0 or the argument itself there."""
    for dtype in (torch.float32, torch.bfloat16):
        g = torch.tensor([-3e38, -1e30, -2e4, -500.0, -89.0, 0.0, 89.0, 500.0, 2e4, 1e30], dtype=dtype)
        x = torch.ones(1, 1, dtype=dtype)
        for activation in ("silu", "gelu_tanh"):
            if activation == "gelu_tanh":
                g = g.clamp(-1e12, 1e12)                     # (its cube is finite)
            h, gate, up = _forward(block, x, g[:, None].contiguous(), torch.ones(len(g), 1, dtype=dtype), activation)
            want = torch.where(g > 50, g.double(), torch.zeros(len(g), dtype=torch.float64))
            within(h[0], want, 2.0 ** -7 * want.abs() + 1e-30, activation)
            grads = _backward(block, torch.ones(1, len(g), dtype=dtype), x, g[:, None].contiguous(), torch.ones(len(g), 1, dtype=dtype), gate.cpu(), up.cpu(), activation)
            slope = torch.where(g > 50, 1.0, torch.where(g == 0, 0.5, 0.0)).double()
            within(grads[1][:, 0], slope, torch.full_like(slope, 1e-6), "slope")


@pytest.mark.parametrize("activation", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_slopes_where_an_activation_is_done(block, dtype, activation):
    """Gates from where the activation is 0 or the gate itself to the ends of the type's range, and those that its rounding takes to an infinity: slopes of 0 and 1,
    not products with infinities.  (2 |g| is finite in 32 bits; the gate is kept in the type.)"""
    t = DTYPES[dtype]
    size = torch.tensor([200.0, 3e4, 65504.0] if dtype == "f16" else [200.0, 1e7, 1e13, 1e16, 1.8e19, 6e19, 1e25, 1e30, 1.6e38]).to(t)
    for sign in (-1.0, 1.0):
        wg = (sign * size)[:, None].repeat(1, 2).contiguous()
        x, wu = torch.ones(1, 2, dtype=t), torch.full((len(size), 2), 0.5, dtype=t)
        for terms in (1, 2):                                 # g = +-size and twice that: an infinity in f16
            x[0, 1] = terms - 1
            h, gate, up = _forward(block, x, wg, wu, activation)
            value = terms * size.double() * (sign > 0)
            want = value * terms / 2
            want[want > torch.finfo(t).max] = float("inf")
            within(h[0], want, rounded(want, t, 2.0 ** -17 * value), "h")
            grads = _backward(block, torch.ones(1, len(size), dtype=t), x, wg, wu, gate.cpu(), up.cpu(), activation)
            slope = torch.full((len(size), 1), float(sign > 0), dtype=torch.float64) * terms / 2
            within(grads[1][:, :1], slope, rounded(slope, t, 2.0 ** -17 * slope), "grad_w_gate")
            kept = torch.where(gate[0].cpu().double() > 0, gate[0].cpu().double(), 0.0)[:, None]
            within(grads[2][:, :1], kept, rounded(kept, t, 2.0 ** -17 * kept), "grad_w_up")


@pytest.mark.parametrize("activation", ["relu", "silu", "gelu_tanh"])
def test_autograd_against_differences(block, activation):
    """The directional derivative of a weighted sum of the definition, in 64 bits by central differences, and by the gradients.  (A difference over
    2e is off by e^2 / 6 of a third derivative; with ReLU the inputs are such that no gate changes sides.)"""
    rows, d, f = 37, 72, 40
    x, wg, wu, v = _inputs(rows, d, f, torch.float32, 11)
    if activation == "relu":
        wg = wg + 0.3 * torch.sign(wg)
        while True:                                          # no pre-activation near 0
            bad = (x.double() @ wg.double().t()).abs() < 1e-2
            if not bool(bad.any()):
                break
            x = torch.where(bad.any(dim=1, keepdim=True), torch.randn(rows, d, generator=torch.Generator().manual_seed(int(bad.sum()) + 100)), x)
    dev = [t.cuda().requires_grad_() for t in (x, wg, wu)]
    block.gated_linear(*dev, activation).backward(v.cuda())
    gen = torch.Generator().manual_seed(12)
    for i, t in enumerate((x, wg, wu)):
        way = torch.randn(t.shape, generator=gen, dtype=torch.float64) / t.numel() ** 0.5

        def value(step):
            a = [s.double() for s in (x, wg, wu)]
            a[i] = a[i] + step * way
            return float((_act(activation, a[0] @ a[1].t())[0] * (a[0] @ a[2].t()) * v.double()).sum())
        e = 1e-4
        slope = (value(e) - value(-e)) / (2 * e)
        got = float((dev[i].grad.cpu().double() * way).sum())
        # 32-bit gradients: 1e-5 of the magnitudes in the sum; the differences: 1e-6
        size = float((dev[i].grad.cpu().double() * way).abs().sum())
        assert abs(got - slope) <= 1e-5 * size + 1e-6 * max(1.0, abs(slope)), (i, got, slope)


def test_autograd_shapes_strides_and_streams(block):
    """Leading dimensions, transposed and negated inputs, an expanded gradient; on another stream; weights that need no gradient."""
    g = torch.Generator().manual_seed(13)
    x = torch.randn(3, 64, 10, generator=g).cuda().transpose(1, 2).requires_grad_()
    wg = torch.randn(64, 48, generator=g).cuda().t().mul(0.1).requires_grad_()
    wu = (torch.randn(48, 64, generator=g).cuda() * 0.1).requires_grad_()
    ref = [t.detach().double().requires_grad_() for t in (x, wg, wu)]
    (torch.relu(ref[0] @ ref[1].t()) * (ref[0] @ ref[2].t())).sum().backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        h = block.gated_linear(x, wg, wu, "relu")
        assert h.shape == (3, 10, 48)
        h.sum().backward()
    torch.cuda.current_stream().wait_stream(side)
    for t, r in zip((x, wg, wu), ref):
        assert torch.allclose(t.grad.double(), r.grad, rtol=1e-4, atol=1e-4)
    frozen = block.gated_linear(x, wg.detach(), wu.detach(), "silu")
    grad_x, = torch.autograd.grad(frozen.sum(), x)
    assert grad_x.shape == x.shape
    with torch.no_grad():
        assert block.gated_linear(x, wg, wu, "silu").grad_fn is None


def test_results_do_not_change_from_call_to_call(block):
    """Equal inputs, equal bits: nothing is added up in an order that the hardware chooses."""
    x, wg, wu, grad_h = _inputs(300, 520, 696, torch.bfloat16, 14)
    first = None
    for _ in range(3):
        kept = _forward(block, x, wg, wu, "silu")
        grads = _backward(block, grad_h, x, wg, wu, kept[1].cpu(), kept[2].cpu(), "silu")
        got = [t.cpu() for t in kept + grads]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got))
        first = got


def test_graph_replays(block):
    """The calls recorded into a graph, replayed on new values with other work between the replays."""
    t = torch.bfloat16
    x, wg, wu, grad_h = (v.cuda() for v in _inputs(96, 264, 200, t, 15))
    h, gate, up = (torch.empty(96, 200, dtype=t, device="cuda") for _ in range(3))
    grads = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    ws = block.new_gated_workspace(96, 264, 200, t, backward=True)

    def calls():
        block.bt_gated_forward(x, wg, wu, "silu", h, gate, up, ws)
        block.bt_gated_backward(grad_h, x, wg, wu, gate, up, "silu", *grads, ws)
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        x.copy_(torch.randn(96, 264, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        got = [v.clone() for v in (h, gate, up) + grads]
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (h, gate, up) + grads)), i


def test_a_stash_keeps_what_relu_gates_save_compressed(block):
    """gate, up and h are zero in the same places, and a BitmapStash gives back their bits."""
    from paper_2110_15362_amd import autograd as ag
    g = torch.Generator().manual_seed(16)
    x = torch.randn(512, 256, generator=g).cuda().requires_grad_()
    ws = [(torch.randn(1024, 256, generator=g) * 0.06).cuda().requires_grad_() for _ in range(2)]
    down = (torch.randn(256, 1024, generator=g) * 0.03).cuda().requires_grad_()

    def step():
        torch.nn.functional.linear(block.gated_linear(x, *ws, "relu"), down).square().mean().backward()
        grads = [t.grad for t in (x, *ws, down)]
        for t in (x, *ws, down):
            t.grad = None
        return grads
    plain = step()
    stash = ag.BitmapStash(min_numel=4096)
    with stash:
        kept = step()
    assert all(torch.equal(a, b) for a, b in zip(plain, kept))
    assert stash.stats["compressed"] >= 3 and stash.stats["stored_bytes"] < 0.8 * stash.stats["dense_bytes"]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(4099, 264, 4104), (4100, 4104, 264), (300, 4104, 4100), (4097, 1000, 4100)], ids=str)
def test_more_of_the_largest_tiles_than_compute_units(block, dtype, size):
    """Workgroups that take several tiles, whole ones and ragged ones, in each product; a summed index with and without a rest."""
    x, wg, wu, grad_h = _inputs(*size, DTYPES[dtype], 18)
    kept = _forward(block, x, wg, wu, "silu")
    _check_forward(x, wg, wu, "silu", *kept)
    alone = _forward(block, x, wg, wu, "silu", keep=False)[0]
    assert torch.equal(alone, kept[0])
    gate, up = kept[1].cpu(), kept[2].cpu()
    _check_backward(grad_h, x, wg, wu, gate, up, "silu", _backward(block, grad_h, x, wg, wu, gate, up, "silu"))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(6144, 4096, 160), (6200, 4128, 296), (288, 4096, 4352), (300, 4096, 4100), (512, 4128, 4112)], ids=str)
def test_several_of_the_largest_tiles_with_results_written_together(block, dtype, size):
    """Rows that begin on 64-byte boundaries, where a lane writes the results of two fragments at once: grad_x (the first two sizes) and the weights' gradients
    (the others) in more than 256 of the largest tiles, whole ones and ragged ones, each with several steps of the summed index.  Equal bits
    the second time."""
    x, wg, wu, grad_h = _inputs(*size, DTYPES[dtype], 19)
    kept = _forward(block, x, wg, wu, "silu")
    _check_forward(x, wg, wu, "silu", *kept)
    gate, up = kept[1].cpu(), kept[2].cpu()
    grads = _backward(block, grad_h, x, wg, wu, gate, up, "silu")
    _check_backward(grad_h, x, wg, wu, gate, up, "silu", grads)
    again = _backward(block, grad_h, x, wg, wu, gate, up, "silu")
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dtype,offset", [("f32", 0), ("bf16", 1)])
def test_outputs_of_more_tiles_than_a_launch_takes(block, dtype, offset):
    """2^23 tiles of 64 by 32 and more, of aligned tensors and, through the kernel for any alignment, of others: the last rows are another launch's."""
    t, rows, d, f = DTYPES[dtype], (1 << 20) + 70, 24, 1 << 14
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GiB")
    g = torch.Generator(device="cuda").manual_seed(20)
    x = torch.randn(rows * d + offset, generator=g, device="cuda").to(t)[offset:].view(rows, d)
    wg, wu = (torch.randn(f, d, generator=g, device="cuda").to(t) for _ in range(2))
    h = torch.empty(rows, f, dtype=t, device="cuda")
    block.bt_gated_forward(x, wg, wu, "relu", h, None, None, block.new_gated_workspace(rows, d, f, t))
    for at in (0, (1 << 19) - 2, (1 << 19) + 62, 1 << 20, rows - 3):
        _check_forward(x[at:at + 3].cpu(), wg.cpu(), wu.cpu(), "relu", h[at:at + 3])


def test_addresses_beyond_32_bits(block):
    """h of more than 2^32 bytes and of more than 2^31 elements: the last rows are where they belong."""
    t, rows, d, f = torch.bfloat16, 70000, 8, 32768
    free, _ = torch.cuda.mem_get_info()
    if free < 24 << 30:
        pytest.skip("needs 24 GiB")
    g = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(rows, d, generator=g, device="cuda").to(t)
    wg, wu = (torch.randn(f, d, generator=g, device="cuda").to(t) for _ in range(2))
    h = torch.empty(rows, f, dtype=t, device="cuda")
    block.bt_gated_forward(x, wg, wu, "relu", h, None, None, block.new_gated_workspace(rows, d, f, t))
    for at in (0, 32767, 65535, 65536, rows - 3):
        _check_forward(x[at:at + 3].cpu(), wg.cpu(), wu.cpu(), "relu", h[at:at + 3])
    # and the sums over all rows of a gradient that is 1 in the last row only
    grad_h = torch.zeros_like(h)
    grad_h[-1] = 1.0
    gate = torch.ones_like(h)
    up = h
    grads = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    block.bt_gated_backward(grad_h, x, wg, wu, gate, up, "relu", *grads, block.new_gated_workspace(rows, d, f, t, backward=True))
    assert torch.equal(grads[2], x[-1].expand(f, d)) and not bool(grads[0][:-1].any()) and bool(grads[0][-1].any())
