"""The choice of experts, the order of the rows and the sums of a token's rows against their definitions.

Tables are whole numbers and have to be equal.  Bounds on weights: exp in 32 bits is off by 2^-22, its argument, a difference, by 2^-24 of itself, a sum of n positive terms by n
2^-24, a quotient by 2^-24.  Sums over columns: (n + 1) 2^-24 of the magnitudes."""
import pytest
import torch

from tests.block_util import DTYPES, SUM, Guarded, rounded, within
from tests.expert_util import choices, plan_on_device, tables

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def experts():
    from paper_2110_15362_amd import experts
    experts.lib()
    return experts


def _chosen(logits, chosen):
    """The definition, one token at a time: NaN above all, equal ones by number, -infinity never."""
    rows = []
    for row in logits.tolist():
        key = [(-INF if v != v else -v, e) for e, v in enumerate(row)]
        # (a NaN is above +infinity)
        order = sorted(range(len(row)), key=lambda e: (0 if row[e] != row[e] else 1, key[e]))
        order = [e for e in order if row[e] != -INF][:chosen]
        rows.append(order + [-1] * (chosen - len(order)))
    return torch.tensor(rows, dtype=torch.int32).view(len(rows), chosen)


def _weights(logits, index, normalise):
    """The softmax in 64 bits and the bound on it."""
    v = logits.double()
    there = index >= 0
    top = v.amax(dim=1, keepdim=True).nan_to_num(0.0, posinf=INF, neginf=0.0) if len(v) else v[:, :1]
    nan = torch.isnan(v).any(dim=1, keepdim=True)
    e = torch.exp(v - top)
    mine = torch.gather(e, 1, index.clamp(min=0).long()) * there
    total = mine.sum(dim=1, keepdim=True) if normalise else e.sum(dim=1, keepdim=True)
    w = torch.where(there, mine / total, torch.zeros_like(mine))
    w = torch.where(nan & there, torch.full_like(w, NAN), w)
    spread = torch.where(torch.isinf(v), torch.zeros_like(v), (v - top).abs()).nan_to_num(0.0).amax(dim=1, keepdim=True)
    spread = spread.clamp(max=120.0)                         # (beyond it exp is 0 in 32 bits)
    off = (2.0 ** -22 * 2 + 2 * SUM * spread + (v.shape[1] + 2) * SUM) * w.abs() + 2.0 ** -126
    return w, off


def _route(experts, logits, chosen, normalise, offset=0):
    m = Guarded()
    tokens, n = logits.shape
    x = m.put(logits, offset)
    plan = experts.new_plan(tokens, n, chosen)
    for t in (plan.index, plan.slots, plan.source, plan.offsets):
        t.fill_(-7)
    weights = m.out((tokens, chosen), torch.float32)
    ws = experts.new_route_workspace(tokens, n, chosen)
    if ws is not None:
        ws.fill_(0xFF)
    experts.bt_route_forward(x, plan, weights, ws, normalise)
    torch.cuda.synchronize()
    m.check()
    return plan, weights


def _check_tables(plan, index):
    slots, source, offsets = tables(index, plan.experts)
    for got, want, name in ((plan.index, index, "index"), (plan.offsets, offsets, "offsets"), (plan.slots, slots, "slots"), (plan.source, source, "source")):
        assert torch.equal(got.cpu(), want), name


SIZES = [(1, 1, 1), (1, 2, 2), (1, 64, 8), (2, 3, 1), (7, 8, 2), (16, 64, 4), (33, 65, 7), (63, 128, 8), (64, 129, 3), (65, 7, 7), (100, 256, 32), (129, 257, 5), (300, 16, 2), (513, 512, 4),
         (700, 61, 3), (1025, 9, 2), (2049, 1, 1), (40, 513, 32), (1500, 1000, 2), (17, 1024, 1), (5000, 128, 8), (16385, 8, 2)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_choice_and_order(experts, dtype, size):
    tokens, n, chosen = size
    g = torch.Generator().manual_seed(sum(size))
    logits = (torch.randn(tokens, n, generator=g) * 2).to(DTYPES[dtype])
    logits[tokens // 3: tokens // 2] = -INF                  # padding
    index = _chosen(logits, chosen)
    for normalise in (True, False):
        plan, weights = _route(experts, logits, chosen, normalise)
        _check_tables(plan, index)
        within(weights, *_weights(logits, index, normalise), "weights")


@pytest.mark.parametrize("n,chosen,tokens", [(64, 8, (64, 128, 129)), (64, 7, (146, 147)), (65, 1, (64, 65)), (128, 16, (63, 64, 65)), (129, 1, (32, 33, 65)), (256, 32, (31, 32, 33)),
                                              (257, 2, (15, 16, 17, 33)), (1024, 1, (16, 17, 1024, 1025, 4096, 4097)), (600, 32, (32, 33))], ids=str)
def test_numbers_of_tokens_between_the_ways(experts, n, chosen, tokens):
    """Tokens and choices around which one workgroup makes way for several, and more tokens a workgroup than it takes at once; the order alone has bounds of its own."""
    for count in tokens:
        logits = torch.randn(count, n, generator=torch.Generator().manual_seed(count))
        index = _chosen(logits, chosen)
        plan, weights = _route(experts, logits, chosen, True)
        _check_tables(plan, index)
        within(weights, *_weights(logits, index, True), "weights")
        again = experts.new_plan(count, n, chosen)
        again.index.copy_(index)
        for t in (again.slots, again.source, again.offsets):
            t.fill_(-7)
        size = experts.lib().bt_route_workspace_bytes(count, n, chosen)
        ws = torch.full((size + 128,), 0xFF, dtype=torch.uint8, device="cuda")
        experts.bt_route_order(again, ws[:size] if size else None)
        _check_tables(again, index)
        assert bool((ws[size:] == 0xFF).all())


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("n", [5, 8, 61, 128, 300])
def test_logits_off_a_16_byte_boundary(experts, dtype, n, offset):
    logits = torch.randn(200, n, generator=torch.Generator().manual_seed(n)).to(DTYPES[dtype])
    index = _chosen(logits, min(n, 4))
    plan, weights = _route(experts, logits, min(n, 4), True, offset)
    _check_tables(plan, index)
    within(weights, *_weights(logits, index, True), "weights")


@pytest.mark.parametrize("n", [4, 16, 100, 200, 400, 1000])
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_equal_logits_masks_infinities_and_nans(experts, dtype, n):
    """Rows of equal logits, of both zeros, of few values, of the type's lowest value, masked but for some and altogether, with a NaN, with an infinity; the largest logits there are."""
    t = DTYPES[dtype]
    low = torch.finfo(t).min
    g = torch.Generator().manual_seed(n)
    rows = [torch.full((n,), 3.0), torch.zeros(n) * torch.where(torch.arange(n) % 2 == 0, 1.0, -1.0), torch.randint(0, 3, (n,), generator=g).float(), torch.full((n,), low),
            torch.full((n,), -INF), torch.where(torch.arange(n) == n - 1, 0.5, -INF), torch.where(torch.arange(n) < 2, 0.5, low), torch.where(torch.arange(n) == 1, NAN, 0.0),
            torch.full((n,), NAN), torch.where(torch.arange(n) == 2, INF, 1.0), torch.where(torch.arange(n) % 2 == 0, -low, low), torch.randint(0, 2, (n,), generator=g).float() * -low]
    logits = torch.stack(rows).to(t)
    chosen = min(n, 4)
    index = _chosen(logits, chosen)
    for normalise in (True, False):
        plan, weights = _route(experts, logits, chosen, normalise)
        _check_tables(plan, index)
        want, off = _weights(logits, index, normalise)
        want[9] = NAN                                        # infinity - infinity
        within(weights, want, off, "weights")


@pytest.mark.parametrize("how", ["some", "one", "first", "holes", "none"])
@pytest.mark.parametrize("size", [(1, 1, 1), (9, 5, 3), (300, 70, 6), (700, 8, 4), (3000, 1024, 3), (70000, 40, 2), (5, 33, 32)], ids=str)
def test_order_of_given_choices(experts, size, how):
    tokens, n, chosen = size
    index = choices(tokens, n, chosen, 3, how)
    given = torch.where(index < 0, torch.tensor(-5 if how == "holes" else n + 3, dtype=torch.int32), index)      # (any number that is no expert's)
    plan = experts.new_plan(tokens, n, chosen)
    plan.index.copy_(given)
    experts.bt_route_order(plan, experts.new_route_workspace(tokens, n, chosen))
    for got, want in zip((plan.slots, plan.source, plan.offsets), tables(index, n)):
        assert torch.equal(got.cpu(), want)
    made = experts.plan_of(given.long().cuda(), n)
    assert torch.equal(made.index.cpu(), torch.where(index < 0, torch.tensor(-1, dtype=torch.int32), index)) and torch.equal(made.slots, plan.slots)


@pytest.mark.parametrize("size", [(1, 1, 1), (1, 64, 8), (7, 8, 2), (33, 65, 7), (100, 256, 32), (300, 16, 2), (513, 512, 4), (40, 1000, 5), (3000, 128, 8)], ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_gradient_of_the_logits(experts, dtype, size):
    tokens, n, chosen = size
    t, g = DTYPES[dtype], torch.Generator().manual_seed(sum(size))
    logits = torch.randn(tokens, n, generator=g).to(t)
    logits[tokens // 3: tokens // 2] = -INF
    if n > 4:
        logits[tokens // 2:, 2] = -INF
    grad_weights = torch.randn(tokens, chosen, generator=g)
    index = _chosen(logits, chosen)
    there = index >= 0
    grad_weights[~there] = NAN                               # not looked at
    for normalise in (True, False):
        plan, weights = _route(experts, logits, chosen, normalise)
        m = Guarded()
        grad = m.out((tokens, n), t)
        experts.bt_route_backward(m.put(grad_weights), None if normalise else m.put(logits), plan, weights, grad, normalise)
        torch.cuda.synchronize()
        m.check()
        w, off = _weights(logits, index, normalise)
        gw = torch.where(there, grad_weights, 0.0).double()
        mean, size_of = (w * gw).sum(dim=1, keepdim=True), (w * gw.abs()).sum(dim=1, keepdim=True)
        at = index.clamp(min=0).long()
        rel = (off / w.clamp_min(1e-30)).where(w > 1e-30, torch.zeros_like(w)).amax(dim=1, keepdim=True)      # of all weights of the token
        p = torch.zeros(tokens, n, dtype=torch.float64)
        if not normalise:
            v = logits.double()
            some = there[:, :1]
            p = torch.where(some, torch.softmax(torch.where(some, v, torch.zeros_like(v)), dim=1), p)
        want, scale = -p * mean, p * size_of
        mine, sizes = torch.where(there, w * gw, 0.0), torch.where(there, w * (gw.abs() + size_of), 0.0)
        want, scale = want.scatter_add(1, at, mine - torch.where(there, w * mean, 0.0) if normalise else mine), scale.scatter_add(1, at, sizes)
        before = (2 * rel + (chosen + 6) * SUM) * scale + 2.0 ** -120
        within(grad, want, rounded(want, t, before), "grad_logits, normalise %s" % normalise)


# ---- a token's rows

def _combine_inputs(experts, size, dtype, how, seed=4):
    tokens, n, chosen, cols = size
    g = torch.Generator().manual_seed(seed)
    plan, groups, source = plan_on_device(experts, choices(tokens, n, chosen, seed, how), n)
    y = torch.randn(tokens * chosen, cols, generator=g).to(dtype)
    y[groups[-1][2]:] = NAN
    weights = torch.rand(tokens, chosen, generator=g)
    slots = plan.slots.cpu()
    weights[slots < 0] = NAN                                 # not looked at
    return plan, y, weights, slots, torch.randn(tokens, cols, generator=g).to(dtype)


def _rows_of(y, slots):
    """[tokens, chosen, cols] in 64 bits, zeros where there is no row."""
    return torch.where((slots >= 0)[:, :, None], y.double()[slots.clamp(min=0).long()], 0.0)


@pytest.mark.parametrize("how", ["some", "first", "holes", "none"])
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (1, 4, 2, 8), (2, 3, 3, 7), (9, 64, 8, 130), (33, 40, 32, 65), (64, 5, 5, 1999), (65, 4, 1, 4096), (100, 9, 6, 2049), (700, 16, 2, 520)], ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_combine(experts, dtype, size, how):
    t, (tokens, n, chosen, cols) = DTYPES[dtype], size
    plan, y, weights, slots, grad_out = _combine_inputs(experts, size, t, how)
    rows, there = _rows_of(y, slots), slots >= 0
    for offset in (0, 1):
        for w in (weights, None):
            m = Guarded()
            out, grad_y, grad_w = m.out((tokens, cols), t, offset), m.out(y.shape, t, offset), m.out(weights.shape, torch.float32)
            dw, dy, dg = None if w is None else m.put(w), m.put(y, offset), m.put(grad_out, offset)
            experts.bt_combine_forward(dy, plan, dw, out)
            experts.bt_combine_backward(dg, dy, plan, dw, grad_y, grad_w)
            torch.cuda.synchronize()
            m.check()
            v = torch.where(there, weights.double() if w is not None else torch.ones(tokens, chosen, dtype=torch.float64), 0.0)
            want = (v[:, :, None] * rows).sum(dim=1)
            within(out, want, rounded(want, t, (chosen + 1) * SUM * (v[:, :, None] * rows).abs().sum(dim=1)), "out")
            want = torch.zeros(y.shape, dtype=torch.float64)
            want[slots[there].long()] = (v[:, :, None] * grad_out.double()[:, None, :])[there]
            within(grad_y, want, rounded(want, t, SUM * want.abs()), "grad_y")
            products = rows * grad_out.double()[:, None, :]
            want = products.sum(dim=2)
            within(grad_w, want, (cols + 1) * SUM * products.abs().sum(dim=2) + 2.0 ** -140, "grad_weights")
    for which in ((True, False), (False, True)):
        one, two = (torch.full(s.shape, 5.0, dtype=s.dtype, device="cuda") if k else None for s, k in zip((y, weights), which))
        experts.bt_combine_backward(grad_out.cuda(), y.cuda(), plan, weights.cuda(), one, two)
        if which[0]:
            again = torch.empty_like(one)
            experts.bt_combine_backward(grad_out.cuda(), y.cuda(), plan, weights.cuda(), again, torch.empty_like(weights, device="cuda"))
            assert torch.equal(one, again) and not bool((one == 5.0).all(dim=1).any())


@pytest.mark.parametrize("how", ["some", "holes", "none"])
@pytest.mark.parametrize("size", [(1, 40, 32, 16383), (1, 1, 1, 9000), (2, 8, 8, 8192), (7, 6, 5, 4097), (130, 12, 12, 1030), (513, 9, 9, 264), (1025, 4, 3, 1025)], ids=str)
@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_few_tokens_in_pieces(experts, dtype, size, how):
    """A token's columns, and backward its choices, in several workgroups; pieces that the last column or choice ends in."""
    test_combine(experts, dtype, size, how)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_combine_of_nothing(experts, dtype):
    t = DTYPES[dtype]
    for tokens, cols in ((0, 8), (3, 0)):
        plan, *_ = plan_on_device(experts, choices(tokens, 4, 2, 1), 4)
        out, grad_w = torch.empty(tokens, cols, dtype=t, device="cuda"), torch.full((tokens, 2), 5.0, device="cuda")
        y = torch.empty(2 * tokens, cols, dtype=t, device="cuda")
        experts.bt_combine_forward(y, plan, None, out)
        experts.bt_combine_backward(out, y, plan, None, torch.empty_like(y), grad_w)
        assert not bool(grad_w.any())


@pytest.mark.parametrize("dtype,n", [(torch.uint8, 256), (torch.uint8, 300), (torch.uint8, 50), (torch.int8, 128), (torch.int8, 200), (torch.int16, 1024), (torch.uint16, 40)], ids=str)
def test_given_choices_in_few_bits(experts, dtype, n):
    """Integers that hold neither the number of experts nor -1; some numbers that are no expert's."""
    info = torch.iinfo(dtype)
    index = torch.stack([torch.randperm(min(n, info.max + 1), generator=torch.Generator().manual_seed(i))[:3] for i in range(90)])
    index[::7, 1] = info.max if info.max >= n else info.min
    want = torch.where((index >= 0) & (index < n), index, -1).int()
    plan = experts.plan_of(index.to(dtype).cuda(), n)
    _check_tables(plan, want)


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("n", [5, 70, 1000])
def test_gradient_where_index_is_no_expert(experts, n, normalise):
    """A number beyond the experts counts as none, as -1 does: neither its weight nor the gradient of it is looked at."""
    g = torch.Generator().manual_seed(n)
    logits = torch.randn(40, n, generator=g)
    logits[::3, 2:] = -INF                                   # two experts, for three choices
    logits[1::3] = -INF
    plan, weights = _route(experts, logits, 3, normalise)
    none = plan.index < 0
    grad_weights = torch.randn(40, 3, generator=g).cuda()
    grad_weights[none] = NAN
    want = torch.empty(40, n, device="cuda")
    experts.bt_route_backward(grad_weights, logits.cuda(), plan, weights, want, normalise)
    assert bool(torch.isfinite(want).all())
    for number in (n, n + 1, 1 << 30, -9):
        plan.index[none] = number
        got = torch.empty_like(want)
        experts.bt_route_backward(grad_weights, logits.cuda(), plan, weights, got, normalise)
        assert torch.equal(got, want), number


def test_given_choices_stay_as_they_are(experts):
    """The plan's index is its own: strides of any kind, and what is written to it later does not reach the caller's tensor, nor the other way round."""
    for dtype in (torch.int32, torch.int64, torch.uint8):
        given = choices(60, 9, 3, 8).t().contiguous().to(dtype).cuda().t()
        before = given.clone()
        plan = experts.plan_of(given, 9)
        _check_tables(plan, before.cpu().int())
        plan.index.fill_(0)
        assert torch.equal(given, before)
        given.fill_(5)
        assert not bool(plan.index.any())
