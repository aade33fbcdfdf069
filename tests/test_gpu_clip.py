"""The norm of many gradients and their clipping, against sums in 64 bits.

Bounds: the sum of squares is one of doubles, whose error does not show in the norm's 24 bits: half a unit of those, and a few of the sum's
2^-53.  A clipped element is off by the rounding of the factor (from 64 bits to 32), of the product and of the result."""
import math

import pytest
import torch

from tests.block_util import DTYPES, SUM, Guarded, rounded, within

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def block():
    from paper_2110_15362_amd import block
    block.lib()
    return block


def _grads(sizes, dtypes, seed, std=0.1):
    g = torch.Generator().manual_seed(seed)
    return [(std * torch.randn(n, generator=g)).to(dtypes[i % len(dtypes)]) for i, n in enumerate(sizes)]


def _norm(grads):
    return math.sqrt(math.fsum(float(t.double().square().sum()) for t in grads))


def _check(block, grads, max_norm, in_place=False, offset=0):
    m = Guarded()
    dev = [m.put(t, offset) for t in grads]
    outs = dev if in_place else [m.out(t.shape, t.dtype, offset) for t in grads]
    norm = m.out((1,), torch.float32)
    ws = block.new_clip_workspace(grads)
    ws.fill_(0xFF)
    block.bt_clip_grads(dev, outs, max_norm, norm, ws, EPS)
    alone = m.out((1,), torch.float32)
    keep = None if in_place else [t.clone() for t in dev]
    if not in_place:
        block.bt_grad_norm(dev, alone, ws)
    torch.cuda.synchronize()
    m.check()
    want = _norm(grads)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    if not in_place:
        assert float(alone) == float(norm) and all(torch.equal(a, b) for a, b in zip(keep, dev))
    factor = min(1.0, max_norm / (want + EPS))
    for i, (t, o) in enumerate(zip(grads, outs)):
        exact = t.double() * factor
        within(o, exact, rounded(exact, t.dtype, 3 * SUM * exact.abs() + 2.0 ** -149), "gradient %d" % i)
        if factor == 1.0:
            assert torch.equal(o.cpu(), t)
    return outs


SETS = [[1], [5], [64, 1, 0, 3], [8192], [8193, 16384, 16385], [100000, 7, 7, 0, 40001], [1 << 20, 333], list(range(0, 127)), list(range(1, 129)),
        [3] * 129, [50 + 7 * i for i in range(300)], [1 << 22, 1 << 20, 4097] * 3, [0, 0]]


@pytest.mark.parametrize("which", range(len(SETS)))
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16", "mixed"])
def test_clip(block, dtype, which):
    dtypes = list(DTYPES.values()) if dtype == "mixed" else [DTYPES[dtype]]
    grads = _grads(SETS[which], dtypes, which)
    for max_norm in (0.01, 1e6, float("inf"), 0.0):
        _check(block, grads, max_norm)
        _check(block, grads, max_norm, in_place=True)


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_tensors_off_a_16_byte_boundary(block, dtype, offset):
    grads = _grads([9, 20000, 33000], [DTYPES[dtype]], 40)
    _check(block, grads, 0.5, offset=offset)
    _check(block, grads, 0.5, in_place=True, offset=offset)


def test_no_gradients_at_all(block):
    norm = torch.full((1,), -1.0, device="cuda")
    ws = block.new_clip_workspace([])
    block.bt_clip_grads([], [], 1.0, norm, ws)
    assert float(norm) == 0.0
    norm.fill_(-1.0)
    block.bt_grad_norm([], norm, ws)
    assert float(norm) == 0.0


def test_values_whose_squares_no_float_holds(block):
    """1e30 and 1e-30: the sum is taken in 64 bits."""
    for v in (1e30, 1e-30):
        g = torch.full((100000,), v, device="cuda")
        norm, ws = torch.empty(1, device="cuda"), block.new_clip_workspace([g])
        out = torch.empty_like(g)
        block.bt_clip_grads([g], [out], 1.0, norm, ws, 0.0)
        want = float(g[0].double()) * math.sqrt(100000)
        assert abs(float(norm) - want) <= 2.0 ** -22 * want
        assert torch.allclose(out, torch.full_like(out, min(v, 1.0 / math.sqrt(100000))), rtol=1e-6)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_infinities_and_nans_are_told(block, dtype):
    t = DTYPES[dtype]
    for bad in (float("inf"), float("-inf"), float("nan")):
        grads = [torch.ones(50000, dtype=t, device="cuda"), torch.ones(11, dtype=t, device="cuda")]
        grads[0][49999] = bad
        norm, ws = torch.empty(1, device="cuda"), block.new_clip_workspace(grads)
        outs = [torch.empty_like(g) for g in grads]
        block.bt_clip_grads(grads, outs, 1.0, norm, ws)
        if math.isnan(bad):
            assert math.isnan(float(norm)) and all(bool(torch.isnan(o).all()) for o in outs)
        else:                                                # the factor is 0: 0 * infinity is a NaN
            assert float(norm) == float("inf") and bool(torch.isnan(outs[0][49999])) and not bool(outs[0][:49999].any()) and not bool(outs[1].any())


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_no_clipping_whatever_the_norm(block, dtype):
    """An infinite max_norm leaves gradients as they are, also where one of them is an infinity or a NaN; one of 0 leaves zeros zeros without an eps."""
    t = DTYPES[dtype]
    for bad in (float("inf"), float("-inf"), float("nan"), 0.0):
        grads = [torch.full((50000,), 0.5 if bad else 0.0, dtype=t, device="cuda"), torch.full((11,), bad, dtype=t, device="cuda")]
        norm, ws = torch.empty(1, device="cuda"), block.new_clip_workspace(grads)
        for eps in (0.0, EPS):
            outs = [torch.full_like(g, 3.0) for g in grads]
            block.bt_clip_grads(grads, outs, float("inf") if bad else 0.0, norm, ws, eps)
            assert all(torch.equal(o, g) or (math.isnan(bad) and i == 1 and bool(torch.isnan(o).all())) for i, (o, g) in enumerate(zip(outs, grads)))
            assert float(norm) == abs(bad) or (math.isnan(bad) and math.isnan(float(norm)))


def test_results_do_not_change_and_graphs_replay(block):
    grads = [g.cuda() for g in _grads([70000 + 13 * i for i in range(150)], list(DTYPES.values()), 41)]
    outs = [torch.empty_like(g) for g in grads]
    norm, ws = torch.empty(1, device="cuda"), block.new_clip_workspace(grads)
    block.bt_clip_grads(grads, outs, 1.0, norm, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.bt_clip_grads(grads, outs, 1.0, norm, ws)
    for i in range(4):
        grads[3].fill_(0.1 * i)
        graph.replay()
        got = [t.clone() for t in outs + [norm]]
        torch.cuda.synchronize()
        block.bt_clip_grads(grads, outs, 1.0, norm, ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs + [norm])), i


def test_clip_grad_norm(block):
    """The call on parameters: in place, those without a gradient left out, transposed gradients too; against torch's own."""
    g = torch.Generator().manual_seed(42)
    params = [torch.nn.Parameter(torch.zeros(s, device="cuda")) for s in ((64, 32), (7,), (128, 5), (3,))]
    ref = [torch.nn.Parameter(torch.zeros_like(p)) for p in params]
    for p, r in zip(params[:3], ref):
        p.grad = torch.randn(p.shape, generator=g).cuda()
        r.grad = p.grad.clone()
    params[2].grad = params[2].grad.t().contiguous().t()
    want = torch.nn.utils.clip_grad_norm_(ref, 0.7)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm = block.clip_grad_norm_(params, 0.7)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.allclose(norm[0], want, rtol=1e-6) and params[3].grad is None
    for p, r in zip(params[:3], ref):
        assert torch.allclose(p.grad, r.grad, rtol=1e-5, atol=0)
    before = [p.grad.clone() for p in params[:3]]
    again = block.clip_grad_norm_([params[0], params[1], params[2], params[0]], 0.35)      # a parameter twice
    assert torch.allclose(again, torch.full_like(again, 0.7), rtol=1e-5)
    for p, b in zip(params[:3], before):
        assert torch.allclose(p.grad, b * 0.5, rtol=1e-5, atol=0)
    with pytest.raises(ValueError, match="no parameter"):
        block.clip_grad_norm_([params[3]], 1.0)


def test_a_gradient_that_two_parameters_share(block):
    """One tensor as the gradient of two parameters: counted once and scaled once."""
    g = torch.Generator().manual_seed(43)
    params = [torch.nn.Parameter(torch.zeros(300000, device="cuda")) for _ in range(3)]
    shared, alone = (torch.randn(300000, generator=g) for _ in range(2))
    params[0].grad = params[2].grad = shared.cuda()
    params[1].grad = alone.cuda()
    want = _norm([shared, alone])
    norm = block.clip_grad_norm_(params, 1.0)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for p, t in ((params[0], shared), (params[1], alone)):
        exact = t.double() / (want + EPS)
        within(p.grad, exact, rounded(exact, t.dtype, 3 * SUM * exact.abs()), "gradient")


def test_a_tensor_of_more_than_32_bits(block):
    n = (1 << 32) + 5
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[0], g[-1], g[1 << 31] = 3.0, 4.0, 12.0
    norm, ws = torch.empty(1, device="cuda"), block.new_clip_workspace([g])
    block.bt_clip_grads([g], [g], 1.0, norm, ws)
    assert float(norm) == 13.0
    for i, v in ((0, 3.0), (-1, 4.0), (1 << 31, 12.0)):
        assert abs(float(g[i]) - v / 13.0) < 2.0 ** -8 * v / 13.0
