"""The norms around a block against their definition in 64 bits, gradients by differentiation of that definition and by differences.

Bounds: the root mean square of a row comes from a 32-bit sum over its columns, off by at most (cols + 8) 2^-24 relative (all terms are
positive), and each of the few operations behind it by 2^-24.  A mean over a row of products of both signs is off by (cols + 16) 2^-24 of
the mean of their magnitudes; a sum over rows likewise with the number of rows.  Where the backward pass reads a tensor that was rounded
(out), the reference reads the same one."""
import pytest
import torch

from tests.block_util import DTYPES, SUM, Guarded, rounded, within

pytestmark = pytest.mark.gpu
EPS, SCALE, KEEP = 1e-5, 0.5, 0.875


@pytest.fixture(scope="module")
def block():
    from paper_2110_15362_amd import block
    block.lib()
    return block


def _inputs(rows, cols, gate_rows, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return {"x": r(rows, cols).to(dtype), "block": (2 * r(rows, cols)).to(dtype), "post_weight": (1 + 0.3 * r(cols)).to(dtype),
            "gate": (0.7 * r(gate_rows, cols)).to(dtype) if gate_rows else None, "pre_weight": (1 + 0.3 * r(cols)).to(dtype),
            "grad_out": r(rows, cols).to(dtype), "grad_y": r(rows, cols).to(dtype)}


def _wide(t):
    return None if t is None else t.double()


def _spread(gate, rows):
    return 1.0 if gate is None else gate.double().repeat_interleave(rows // gate.shape[0], dim=0)


def _forward(block, s, post=True, pre=True, with_block=True, offset=0, stats=True):
    m, dtype, (rows, cols) = Guarded(), s["x"].dtype, s["x"].shape
    put = lambda k, there=True: m.put(s[k], offset) if there and s[k] is not None else None  # noqa: E731
    out = m.out((rows, cols), dtype, offset) if with_block else None
    y = m.out((rows, cols), dtype, offset) if pre else None
    st = m.out((2, rows), torch.float32) if stats else None
    block.bt_residual_norm_forward(put("x"), put("block", with_block), put("post_weight", post and with_block), put("gate", with_block),
                                   put("pre_weight", pre), out, y, st, EPS, SCALE, KEEP)
    torch.cuda.synchronize()
    m.check()
    return out, y, st


def _check_forward(s, out, y, stats, post=True):
    dtype, (rows, cols) = s["x"].dtype, s["x"].shape
    x, b = s["x"].double(), s["block"].double()
    few = (cols + 16) * SUM
    with_block = out is not None
    if with_block:
        rb = ((b * b).mean(dim=1, keepdim=True) + EPS).rsqrt() if post else torch.ones(rows, 1, dtype=torch.float64)
        branch = SCALE * b * rb * (s["post_weight"].double() if post else 1.0) * _spread(s["gate"], rows)
        want = KEEP * x + branch
        off = few * (branch.abs() + x.abs())
        within(out, want, rounded(want, dtype, off), "out")
    else:
        want, off, rb = x, torch.zeros_like(x), torch.ones(rows, 1, dtype=torch.float64)
    ro = ((want * want).mean(dim=1, keepdim=True) + EPS).rsqrt()
    # an error of the row enters its root mean square by at most its own root mean square
    off_ro = ro * (few + ro * (off * off).mean(dim=1, keepdim=True).sqrt())
    if y is not None:
        wn = s["pre_weight"].double()
        within(y, want * ro * wn, rounded(want * ro * wn, dtype, (off * ro + want.abs() * off_ro) * wn.abs() + few * (want * ro * wn).abs()), "y")
    if stats is not None:
        within(stats[0], rb[:, 0], few * rb[:, 0], "stats of block")
        if y is not None:
            within(stats[1], ro[:, 0], off_ro[:, 0] + few * ro[:, 0], "stats of out")


SHAPES = [(1, 1, 1), (1, 4096, 1), (2, 7, 2), (3, 64, 1), (5, 1000, 5), (7, 129, 1), (8, 256, 4), (9, 513, 3), (6, 1024, 0), (33, 1999, 33), (12, 2048, 2),
          (30, 4096, 5), (10, 5001, 1), (4, 8192, 4), (6, 8200, 3), (5, 16384, 1), (3, 16383, 0), (2100, 72, 700), (3000, 40, 8), (1500, 250, 1500),
          (1100, 136, 1), (4097, 8, 0), (2049, 24, 683), (6000, 40, 3000), (5001, 24, 1667), (4200, 600, 2100)]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_forward(block, dtype, shape):
    s = _inputs(*shape, DTYPES[dtype], sum(shape))
    _check_forward(s, *_forward(block, s))
    _check_forward(s, *_forward(block, s, post=False), post=False)
    out, y, _ = _forward(block, s, pre=False, stats=False)
    _check_forward(s, out, None, None)
    _check_forward(s, *_forward(block, s, with_block=False))


def _backward(block, s, out, stats, post=True, with_block=True, grad_out=True, grad_y=True, offset=0, want=(1, 1, 1, 1, 1)):
    m, dtype, (rows, cols) = Guarded(), s["x"].dtype, s["x"].shape
    put = lambda k, there=True: m.put(s[k], offset) if there and s[k] is not None else None  # noqa: E731
    gate = s["gate"] if with_block else None
    ws = block.new_residual_norm_workspace(rows, cols, 0 if gate is None else gate.shape[0], dtype)
    ws.fill_(0xFF)
    there = (True, with_block, post and with_block, gate is not None, grad_y)
    shapes = ((rows, cols), (rows, cols), (cols,), None if gate is None else gate.shape, (cols,))
    grads = [m.out(sh, dtype, offset) if t and w else None for t, w, sh in zip(there, want, shapes)]
    block.bt_residual_norm_backward(put("grad_out", grad_out), put("grad_y", grad_y), m.put(out, offset), put("block", with_block),
                                    put("post_weight", post and with_block), m.put(gate, offset) if gate is not None else None, put("pre_weight", grad_y),
                                    stats, *grads, ws, SCALE, KEEP)
    torch.cuda.synchronize()
    m.check()
    return grads


def _check_backward(s, out, grads, post=True, with_block=True, grad_out=True, grad_y=True):
    """By differentiation in 64 bits of norm(out) * pre_weight at the `out` that the backward pass reads (and the statistics of the forward
    pass belong to, up to its rounding), then of out itself."""
    dtype, (rows, cols) = s["x"].dtype, s["x"].shape
    few, col = (cols + 16) * SUM, (rows + 16) * SUM
    zero = torch.zeros(rows, cols, dtype=torch.float64)
    o = out.double()
    go = s["grad_out"].double() if grad_out else zero
    total, off = go, SUM * go.abs()
    # the statistics are those of out before it was rounded: off from the rounded one's by half a unit at the most, and much less on the average
    from tests.block_util import UNIT
    stat = UNIT[dtype] if with_block and dtype != torch.float32 else few
    if grad_y:
        gy, wn = s["grad_y"].double(), s["pre_weight"].double()
        ro = ((o * o).mean(dim=1, keepdim=True) + EPS).rsqrt()
        v, gv = o * ro, gy * wn
        mean, size = (gv * v).mean(dim=1, keepdim=True), (gv * v).abs().mean(dim=1, keepdim=True)
        total = total + ro * (gv - v * mean)
        parts = ro * (gv.abs() + v.abs() * size)
        off = off + (3 * stat + 2 * few) * parts
        if grads[4] is not None:
            want = (gy * v).sum(dim=0)
            within(grads[4], want, rounded(want, dtype, (stat + few + col) * (gy * v).abs().sum(dim=0)), "grad_pre_weight")
    keep = KEEP if with_block else 1.0
    if grads[0] is not None:
        within(grads[0], keep * total, rounded(keep * total, dtype, keep * off + SUM * total.abs()), "grad_x")
    if not with_block:
        return
    b = s["block"].double()
    rb = ((b * b).mean(dim=1, keepdim=True) + EPS).rsqrt() if post else torch.ones(rows, 1, dtype=torch.float64)
    z, wp, gate = b * rb, s["post_weight"].double() if post else torch.ones(cols, dtype=torch.float64), _spread(s["gate"], rows)
    branch, off_branch = SCALE * total, SCALE * off + 2 * SUM * total.abs()
    if grads[3] is not None:
        groups = s["gate"].shape[0]
        sums = lambda t: t.reshape(groups, rows // groups, cols).sum(dim=1)  # noqa: E731
        want = sums(branch * z * wp)
        within(grads[3], want, rounded(want, dtype, sums((off_branch + (few + col) * branch.abs()) * (z * wp).abs())), "grad_gate")
    dn = branch * gate
    off_dn = (off_branch + SUM * branch.abs()) * (gate.abs() if s["gate"] is not None else 1.0)
    if grads[2] is not None:
        want = (dn * z).sum(dim=0)
        within(grads[2], want, rounded(want, dtype, ((off_dn + (few + col) * dn.abs()) * z.abs()).sum(dim=0)), "grad_post_weight")
    if grads[1] is not None:
        dz, off_dz = dn * wp, off_dn * wp.abs()
        if post:
            mean, size = (dz * z).mean(dim=1, keepdim=True), (dz * z).abs().mean(dim=1, keepdim=True)
            off_mean = (off_dz * z.abs()).mean(dim=1, keepdim=True)
            want = rb * (dz - z * mean)
            bound = rb * (off_dz + z.abs() * off_mean + 3 * few * (dz.abs() + z.abs() * size))
        else:
            want, bound = dz, off_dz
        within(grads[1], want, rounded(want, dtype, bound), "grad_block")


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_backward(block, dtype, shape):
    s = _inputs(*shape, DTYPES[dtype], sum(shape) + 1)
    for post in (True, False):
        out, _, stats = _forward(block, s, post=post)
        _check_backward(s, out.cpu(), _backward(block, s, out.cpu(), stats, post=post), post=post)
    out, _, stats = _forward(block, s)
    _check_backward(s, out.cpu(), _backward(block, s, out.cpu(), stats, grad_out=False), grad_out=False)
    _check_backward(s, out.cpu(), _backward(block, s, out.cpu(), stats, grad_y=False), grad_y=False)
    _, _, stats = _forward(block, s, with_block=False)
    _check_backward(s, s["x"], _backward(block, s, s["x"], stats, with_block=False), with_block=False)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_each_gradient_alone(block, dtype):
    """A gradient does not depend on which others are wanted."""
    for shape in ((40, 264, 4), (1400, 72, 2), (5, 16384, 1)):
        s = _inputs(*shape, DTYPES[dtype], 3)
        out, _, stats = _forward(block, s)
        every = _backward(block, s, out.cpu(), stats)
        for i in range(5):
            one = _backward(block, s, out.cpu(), stats, want=[i == k for k in range(5)])
            assert torch.equal(one[i], every[i])


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_tensors_off_a_16_byte_boundary(block, dtype, offset):
    for shape in ((3, 64, 1), (9, 1024, 3), (4, 4097, 0)):
        s = _inputs(*shape, DTYPES[dtype], 4)
        out, y, stats = _forward(block, s, offset=offset)
        _check_forward(s, out, y, stats)
        _check_backward(s, out.cpu(), _backward(block, s, out.cpu(), stats, offset=offset))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_in_place(block, dtype):
    """out over x or over block; grad_x over grad_out and grad_block over block or over grad_y."""
    for shape in ((70, 264, 7), (4, 8192, 1), (3, 16384, 1)):
        s = _inputs(*shape, DTYPES[dtype], 5)
        out, y, stats = _forward(block, s)
        grads = _backward(block, s, out.cpu(), stats)
        d = {k: v.cuda() for k, v in s.items()}
        y2 = torch.empty_like(d["x"])
        for over in ("x", "block"):
            c = {k: v.clone() for k, v in d.items()}
            block.bt_residual_norm_forward(c["x"], c["block"], c["post_weight"], c["gate"], c["pre_weight"], c[over], y2, None, EPS, SCALE, KEEP)
            assert torch.equal(c[over], out) and torch.equal(y2, y)
        ws = block.new_residual_norm_workspace(*shape, DTYPES[dtype])
        for over in ("block", "grad_y"):
            c = {k: v.clone() for k, v in d.items()}
            gp, gg, gn = torch.empty_like(c["post_weight"]), torch.empty_like(c["gate"]), torch.empty_like(c["pre_weight"])
            block.bt_residual_norm_backward(c["grad_out"], c["grad_y"], out, c["block"], c["post_weight"], c["gate"], c["pre_weight"], stats,
                                            c["grad_out"], c[over], gp, gg, gn, ws, SCALE, KEEP)
            for a, b in zip(grads, (c["grad_out"], c[over], gp, gg, gn)):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_no_rows_and_no_columns(block, dtype):
    for rows, cols in ((0, 64), (5, 0)):
        s = _inputs(rows, cols, 0, DTYPES[dtype], 6)
        out, y, stats = _forward(block, s)
        for g in _backward(block, s, out.cpu(), stats):
            assert g is None or (not bool(g.any()) and not bool(torch.isnan(g).any()))


def test_rows_of_zeros_and_of_infinities(block):
    """A row of zeros stays one (eps keeps the quotient finite); a row with an infinity or a NaN is one of NaNs, and no other row is."""
    for dtype in DTYPES.values():
        s = _inputs(6, 300, 0, dtype, 7)
        s["x"][1] = 0
        s["block"][1] = 0
        s["block"][3, 17] = float("inf")
        s["block"][4, 299] = float("nan")
        out, y, stats = _forward(block, s)
        assert not bool(out[1].any()) and not bool(y[1].any())
        assert bool(torch.isnan(y[3]).any()) and bool(torch.isnan(out[3, 17])) and bool(torch.isnan(y[4]).all())
        clean = [0, 1, 2, 5]
        for t in (out, y):
            assert not bool(torch.isnan(t[clean]).any())
        grads = _backward(block, s, out.cpu(), stats)
        assert not bool(torch.isnan(grads[0][clean]).any()) and not bool(torch.isnan(grads[1][clean]).any())
        _check_forward({k: (v[clean] if v is not None and v.dim() == 2 else v) for k, v in s.items()}, out[clean], y[clean], None)


def test_large_values(block):
    """fp16 values whose squares its own range does not hold."""
    s = _inputs(4, 512, 0, torch.float16, 8)
    s["block"] = s["block"] * 5000
    s["x"] = s["x"] * 3000
    _check_forward(s, *_forward(block, s))


@pytest.mark.parametrize("gate_shape", [None, (48,), (3, 48), (3, 1, 48), (3, 7, 48)], ids=str)
def test_autograd(block, gate_shape):
    """Both outputs, one alone, and a gate in each of its shapes, against the definition differentiated in 64 bits."""
    g = torch.Generator().manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    leaves = [r(3, 7, 48), r(3, 7, 48), r(48), r(48)] + ([r(*gate_shape)] if gate_shape else [])
    dev = [t.cuda().requires_grad_() for t in leaves]
    ref = [t.double().requires_grad_() for t in leaves]
    norm = lambda t: t * (t.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()  # noqa: E731
    gate = 1.0 if gate_shape is None else ref[4]
    if gate_shape == (3, 48):
        gate = ref[4][:, None]
    want_out = KEEP * ref[0] + SCALE * gate * norm(ref[1]) * ref[2]
    want_y = norm(want_out) * ref[3]
    a, b = r(3, 7, 48), r(3, 7, 48)
    for wo, wy in ((a, b), (a, None), (None, b)):
        out, y = block.residual_norm(dev[0], dev[1], dev[2], dev[4] if gate_shape else None, dev[3], EPS, SCALE, KEEP)
        roots = [(t, w.cuda()) for t, w in ((out, wo), (y, wy)) if w is not None]
        got = torch.autograd.grad([t for t, _ in roots], dev, [w for _, w in roots], allow_unused=True)
        roots = [(t, w.double()) for t, w in ((want_out, wo), (want_y, wy)) if w is not None]
        want = torch.autograd.grad([t for t, _ in roots], ref, [w for _, w in roots], retain_graph=True, allow_unused=True)
        for p, q in zip(got, want):
            q = torch.zeros_like(p).cpu().double() if q is None else q
            assert torch.allclose(p.cpu().double() if p is not None else torch.zeros_like(q), q, rtol=2e-5, atol=2e-5)
    first = block.rms_norm(dev[0], dev[3], EPS)
    got = torch.autograd.grad(first, (dev[0], dev[3]), b.cuda())
    want = torch.autograd.grad(norm(ref[0]) * ref[3], (ref[0], ref[3]), b.double())
    assert all(torch.allclose(p.cpu().double(), q, rtol=2e-5, atol=2e-5) for p, q in zip(got, want))


def test_a_gate_for_each_position(block):
    """[T, cols] and [1, T, cols] for several sequences: refused as they are, right when expanded to the shape of x, their gradients sums over the sequences."""
    g = torch.Generator().manual_seed(15)
    x, b, gate, v = (torch.randn(*s, generator=g) for s in ((4, 6, 48), (4, 6, 48), (1, 6, 48), (4, 6, 48)))
    dev, ref = [[t.to(d, k).requires_grad_() for t in (x, b, gate)] for d, k in (("cuda", torch.float32), ("cpu", torch.float64))]
    for bad in (dev[2], dev[2][0]):
        with pytest.raises(ValueError, match="expand it to the shape of x"):
            block.residual_norm(dev[0], dev[1], None, bad)
    out, _ = block.residual_norm(dev[0], dev[1], None, dev[2].expand(x.shape))
    want = ref[0] + ref[2] * ref[1]
    assert torch.allclose(out.cpu().double(), want, rtol=1e-6, atol=1e-6)
    for p, q in zip(torch.autograd.grad(out, dev, v.cuda()), torch.autograd.grad(want, ref, v.double())):
        assert p.shape == q.shape and torch.allclose(p.cpu().double(), q, rtol=1e-5, atol=1e-5)


def test_gradients_against_differences(block):
    """The slope of a weighted sum of both outputs along a direction: central differences of the definition in 64 bits."""
    s = _inputs(24, 100, 4, torch.float32, 10)
    out, _, stats = _forward(block, s)
    grads = _backward(block, s, out.cpu(), stats)
    norm = lambda t: t * (t.square().mean(dim=1, keepdim=True) + EPS).rsqrt()  # noqa: E731
    names = ("x", "block", "post_weight", "gate", "pre_weight")
    gen = torch.Generator().manual_seed(11)
    for name, grad in zip(names, grads):
        way = torch.randn(s[name].shape, generator=gen, dtype=torch.float64)

        def value(step):
            v = {k: t.double() for k, t in s.items()}
            v[name] = v[name] + step * way
            o = KEEP * v["x"] + SCALE * _spread(v["gate"], 24) * norm(v["block"]) * v["post_weight"]
            return float((o * v["grad_out"]).sum() + (norm(o) * v["pre_weight"] * v["grad_y"]).sum())
        e = 1e-5
        slope, got = (value(e) - value(-e)) / (2 * e), grad.cpu().double() * way
        # 32-bit gradients: 1e-5 of the magnitudes in the sum; differences: cancellation of 64-bit sums over 2e, 1e-6
        assert abs(float(got.sum()) - slope) <= 1e-5 * float(got.abs().sum()) + 1e-6 * max(1.0, abs(slope)), name


def test_results_do_not_change_and_graphs_replay(block):
    s = {k: v.cuda() for k, v in _inputs(1300, 264, 13, torch.bfloat16, 12).items()}
    out, y = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    stats = torch.empty(2, 1300, device="cuda")
    grads = [torch.empty_like(s[k]) for k in ("x", "block", "post_weight", "gate", "pre_weight")]
    ws = block.new_residual_norm_workspace(1300, 264, 13, torch.bfloat16)

    def calls():
        block.bt_residual_norm_forward(s["x"], s["block"], s["post_weight"], s["gate"], s["pre_weight"], out, y, stats, EPS, SCALE, KEEP)
        block.bt_residual_norm_backward(s["grad_out"], s["grad_y"], out, s["block"], s["post_weight"], s["gate"], s["pre_weight"], stats, *grads, ws, SCALE, KEEP)
    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        s["x"].copy_(torch.randn(1300, 264, generator=torch.Generator().manual_seed(i)))
        graph.replay()
        got = [t.clone() for t in [out, y] + grads]
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [out, y] + grads)), i


def test_more_rows_than_a_launch_takes(block):
    """2^23 + 3 short rows: the last ones are another launch's, and take their own gate rows."""
    rows, cols, t = (1 << 23) + 4, 8, torch.bfloat16
    if torch.cuda.mem_get_info()[0] < 4 << 30:
        pytest.skip("needs 4 GiB")
    g = torch.Generator(device="cuda").manual_seed(14)
    x, b = (torch.randn(rows, cols, generator=g, device="cuda").to(t) for _ in range(2))
    w, gate = torch.ones(cols, dtype=t, device="cuda"), torch.tensor([[1.0], [-2.0]], device="cuda").repeat(1, cols).to(t)
    out, y = torch.empty_like(x), torch.empty_like(x)
    block.bt_residual_norm_forward(x, b, w, gate, w, out, y, None, EPS, SCALE, KEEP)
    for at in (0, rows // 2 - 2, rows // 2, rows - 4):
        s = {"x": x[at:at + 2].cpu(), "block": b[at:at + 2].cpu(), "post_weight": w.cpu(), "gate": gate[at * 2 // rows:at * 2 // rows + 1].cpu(), "pre_weight": w.cpu()}
        _check_forward(s, out[at:at + 2], y[at:at + 2], None)


def test_addresses_beyond_32_bits(block):
    """More than 2^31 elements: the last rows are where they belong."""
    rows, cols, t = 140000, 16384, torch.bfloat16
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GiB")
    g = torch.Generator(device="cuda").manual_seed(13)
    x = torch.randn(1, cols, generator=g, device="cuda").to(t).expand(rows, cols).contiguous()
    b = x.clone()
    for at in (0, 131071, rows - 1):
        x[at].mul_(2.0)
    w = torch.ones(cols, dtype=t, device="cuda")
    out, y, stats = torch.empty_like(x), torch.empty_like(x), torch.empty(2, rows, device="cuda")
    block.bt_residual_norm_forward(x, b, w, None, w, out, y, stats, EPS, SCALE, KEEP)
    for at in (0, 131071, 131072, rows - 1):
        s = {"x": x[at:at + 1].cpu(), "block": b[at:at + 1].cpu(), "post_weight": w.cpu(), "gate": None, "pre_weight": w.cpu()}
        _check_forward(s, out[at:at + 1], y[at:at + 1], stats[:, at:at + 1])
