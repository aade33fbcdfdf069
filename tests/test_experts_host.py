"""What the experts' calls refuse, on the host: through the C ABI with made-up addresses, which nothing dereferences, and through the binding with tensors that do not
fit.  No GPU."""
import ctypes
import os

import pytest
import torch

from tests.expert_util import choices, tables
from tests.test_block_host import ALIGN, ARGUMENT, BF16, DTYPE, F16, F32, F64, NULL, SIZE, WORKSPACE, A, _Fake

vp, u64, sz, ci = ctypes.c_void_p, ctypes.c_uint64, ctypes.c_size_t, ctypes.c_int


class _Plan(ctypes.Structure):
    _fields_ = [("tokens", u64), ("experts", u64), ("chosen", u64), ("d_index", vp), ("d_slots", vp), ("d_source", vp), ("d_offsets", vp)]


def plan(tokens=6, n=4, chosen=2, index=A, slots=A, source=A, offsets=A):
    return ctypes.byref(_Plan(tokens, n, chosen, index, slots, source, offsets))


@pytest.fixture(scope="module")
def experts():
    import paper_2110_15362_amd.bittrain as bt
    if not os.path.exists(bt.LIB_PATH):
        from paper_2110_15362_amd import build
        build.build()
    from paper_2110_15362_amd import experts
    experts.lib()
    return experts


@pytest.fixture(scope="module")
def L(experts):
    from paper_2110_15362_amd import block
    raw = ctypes.CDLL(block._LIB_PATH)
    raw.bt_route_workspace_bytes.restype, raw.bt_route_workspace_bytes.argtypes = sz, [u64, u64, u64]
    raw.bt_route_forward.argtypes = [vp, ci, ci, vp, vp, vp, sz, vp]
    raw.bt_route_order.argtypes = [vp, vp, sz, vp]
    raw.bt_route_backward.argtypes = [vp, vp, ci, ci, vp, vp, vp, vp]
    for name in ("gated", "linear"):
        f = getattr(raw, "bt_expert_%s_workspace_bytes" % name)
        f.restype, f.argtypes = sz, [vp, u64, u64, ci, ci, ci]
    raw.bt_expert_gated_forward.argtypes = [vp] * 4 + [u64] * 2 + [ci] * 3 + [vp] * 4 + [sz, vp]
    raw.bt_expert_gated_backward.argtypes = [vp] * 7 + [u64] * 2 + [ci] * 3 + [vp] * 4 + [sz, vp]
    raw.bt_expert_linear_forward.argtypes = [vp] * 3 + [u64] * 2 + [ci] * 2 + [vp] * 2 + [sz, vp]
    raw.bt_expert_linear_backward.argtypes = [vp] * 4 + [u64] * 2 + [ci] * 2 + [vp] * 3 + [sz, vp]
    raw.bt_combine_forward.argtypes = [vp, vp, vp, u64, ci, vp, vp]
    raw.bt_combine_backward.argtypes = [vp, vp, vp, vp, u64, ci, vp, vp, vp]
    return raw


# numbers that every call refuses
BAD_PLANS = [dict(n=0), dict(n=1025), dict(chosen=0), dict(chosen=5), dict(n=64, chosen=33), dict(tokens=1 << 30), dict(tokens=(1 << 63) + 1)]


def test_route_errors(L):
    def forward(logits=A, dt=BF16, p=plan(), weights=A, ws=A, wsb=1 << 30):
        return L.bt_route_forward(logits, dt, 1, p, weights, ws, wsb, None)

    def backward(gw=A, logits=A, dt=BF16, normalise=0, p=plan(), weights=A, gl=A):
        return L.bt_route_backward(gw, logits, dt, normalise, p, weights, gl, None)
    for bad in BAD_PLANS:
        assert forward(p=plan(**bad)) == L.bt_route_order(plan(**bad), A, 1 << 30, None) == backward(p=plan(**bad)) == SIZE
    assert forward(dt=F64) == backward(dt=F64) == forward(dt=9) == DTYPE
    assert forward(p=None) == L.bt_route_order(None, A, 1 << 30, None) == backward(p=None) == forward(logits=None) == forward(weights=None) == NULL
    assert backward(gw=None) == backward(logits=None) == backward(weights=None) == backward(gl=None) == backward(p=plan(index=None)) == NULL
    for name in ("index", "slots", "source", "offsets"):
        assert forward(p=plan(**{name: None})) == L.bt_route_order(plan(**{name: None}), A, 1 << 30, None) == NULL
        assert forward(p=plan(**{name: A + 2})) == L.bt_route_order(plan(**{name: A + 2}), A, 1 << 30, None) == ALIGN
    assert forward(logits=A + 1) == forward(logits=A + 2, dt=F32) == forward(weights=A + 2) == forward(ws=A + 64) == ALIGN
    assert backward(gw=A + 2) == backward(logits=A + 1) == backward(weights=A + 1) == backward(gl=A + 1) == backward(p=plan(index=A + 1)) == ALIGN
    assert backward(p=plan(tokens=0), gw=None, gl=None) == 0
    need = L.bt_route_workspace_bytes(5000, 64, 2)
    big = plan(tokens=5000, n=64)
    assert need > 0 == L.bt_route_workspace_bytes(6, 4, 2) and forward(p=big, ws=None) == NULL and forward(p=big, wsb=need - 1) == WORKSPACE
    assert L.bt_route_order(big, None, 0, None) == NULL and L.bt_route_order(big, A, need - 1, None) == WORKSPACE
    for bad in BAD_PLANS:
        a = dict(tokens=6, n=4, chosen=2) | bad
        assert L.bt_route_workspace_bytes(a["tokens"], a["n"], a["chosen"]) == 0


def test_gated_errors(L):
    def forward(x=A, wg=A, wu=A, p=plan(), d=16, f=24, dt=BF16, act=1, ordered=0, h=A, gate=A, up=A, ws=A, wsb=1 << 40):
        return L.bt_expert_gated_forward(x, wg, wu, p, d, f, dt, act, ordered, h, gate, up, ws, wsb, None)
    need = {o: L.bt_expert_gated_workspace_bytes(plan(), 16, 24, BF16, o, 1) for o in (0, 1)}

    def backward(gh=A, x=A, wg=A, wu=A, gate=A, up=A, p=plan(), d=16, f=24, dt=BF16, act=1, ordered=0, gx=A, gwg=A, gwu=A, ws=A, wsb=need[0]):
        return L.bt_expert_gated_backward(gh, x, wg, wu, gate, up, p, d, f, dt, act, ordered, gx, gwg, gwu, ws, wsb, None)
    for bad in BAD_PLANS:
        assert forward(p=plan(**bad)) == backward(p=plan(**bad)) == SIZE
        assert L.bt_expert_gated_workspace_bytes(plan(**bad), 16, 24, BF16, 0, 1) == 0
    assert forward(dt=F64) == backward(dt=F64) == DTYPE and forward(d=(1 << 24) + 1) == backward(f=(1 << 24) + 1) == SIZE
    assert forward(act=3) == forward(act=-1) == forward(gate=None) == forward(up=None) == backward(act=7) == backward(gwg=None) == backward(gwu=None) == ARGUMENT
    for name in ("x", "wg", "wu", "h", "p"):
        assert forward(**{name: None}) == NULL
    for name in ("gh", "x", "wg", "wu", "gate", "up", "p", "ws"):
        assert backward(**{name: None}) == NULL
    assert forward(p=plan(offsets=None)) == forward(p=plan(source=None)) == backward(p=plan(offsets=None)) == backward(p=plan(source=None)) == backward(p=plan(slots=None)) == NULL
    assert forward(p=plan(offsets=A + 1)) == forward(p=plan(source=A + 2)) == backward(p=plan(slots=A + 2)) == ALIGN
    for name in ("x", "wg", "wu", "h", "gate", "up"):
        assert forward(**{name: A + 1}) == ALIGN and forward(dt=F32, **{name: A + 2}) == ALIGN
    for name in ("gh", "x", "wg", "wu", "gate", "up", "gx", "gwg", "gwu"):
        assert backward(**{name: A + 1}) == ALIGN
    assert forward(ws=A + 64) == backward(ws=A + 32) == ALIGN and backward(wsb=need[0] - 1) == WORKSPACE
    assert need[0] > need[1] > 0
    assert forward(p=plan(tokens=0), x=None, h=None, gate=None, up=None) == forward(f=0, h=None, gate=None, up=None) == 0
    assert backward(gx=None, gwg=None, gwu=None) == backward(d=0) == 0
    # rows off the 16-byte boundaries are copied where there are many
    many = plan(tokens=4000)
    copies = L.bt_expert_gated_workspace_bytes(many, 1001, 24, BF16, 0, 0)
    assert copies >= 2 * (4000 * 1001 + 2 * 4 * 24 * 1001) and forward(p=many, d=1001, ws=None) == NULL and forward(p=many, d=1001, wsb=copies - 1) == WORKSPACE


def test_linear_errors(L):
    def forward(x=A, w=A, p=plan(), a=16, b=24, dt=F16, ordered=1, y=A, ws=A, wsb=1 << 40):
        return L.bt_expert_linear_forward(x, w, p, a, b, dt, ordered, y, ws, wsb, None)

    def backward(gy=A, x=A, w=A, p=plan(), a=16, b=24, dt=F16, ordered=0, gx=A, gw=A, ws=A, wsb=1 << 40):
        return L.bt_expert_linear_backward(gy, x, w, p, a, b, dt, ordered, gx, gw, ws, wsb, None)
    for bad in BAD_PLANS:
        assert forward(p=plan(**bad)) == backward(p=plan(**bad)) == SIZE
        assert L.bt_expert_linear_workspace_bytes(plan(**bad), 16, 24, F16, 0, 1) == 0
    assert forward(dt=F64) == backward(dt=F64) == DTYPE and forward(a=(1 << 24) + 1) == backward(b=(1 << 24) + 1) == SIZE
    for name in ("x", "w", "y", "p"):
        assert forward(**{name: None}) == NULL
    for name in ("gy", "x", "w", "p", "ws"):
        assert backward(**{name: None}) == NULL
    # ordered: the tokens' tables are not looked at; what belongs to a gradient that is not wanted neither
    assert forward(p=plan(offsets=None)) == forward(ordered=0, p=plan(source=None)) == backward(p=plan(source=None)) == backward(p=plan(slots=None)) == NULL
    assert forward(p=plan(tokens=0), x=None, y=None) == forward(b=0, y=None) == backward(gx=None, gw=None) == backward(a=0) == 0
    for name in ("x", "w", "y"):
        assert forward(**{name: A + 1}) == ALIGN
    for name in ("gy", "x", "w", "gx", "gw"):
        assert backward(**{name: A + 1}) == ALIGN
    need = L.bt_expert_linear_workspace_bytes(plan(), 16, 24, F16, 0, 1)
    assert need >= 12 * 16 * 4 and backward(wsb=need - 1) == WORKSPACE


def test_combine_errors(L):
    def forward(y=A, p=plan(), w=A, cols=16, dt=BF16, out=A):
        return L.bt_combine_forward(y, p, w, cols, dt, out, None)

    def backward(go=A, y=A, p=plan(), w=A, cols=16, dt=BF16, gy=A, gw=A):
        return L.bt_combine_backward(go, y, p, w, cols, dt, gy, gw, None)
    for bad in BAD_PLANS:
        assert forward(p=plan(**bad)) == backward(p=plan(**bad)) == SIZE
    assert forward(cols=(1 << 24) + 1) == backward(cols=(1 << 24) + 1) == SIZE and forward(dt=F64) == backward(dt=F64) == DTYPE
    assert forward(y=None) == forward(p=None) == forward(out=None) == forward(p=plan(slots=None)) == NULL
    assert backward(go=None) == backward(y=None) == backward(p=None) == backward(p=plan(slots=None)) == backward(p=plan(offsets=None)) == NULL
    assert forward(y=A + 1) == forward(w=A + 2) == forward(out=A + 1) == forward(p=plan(slots=A + 2)) == ALIGN
    assert backward(go=A + 1) == backward(y=A + 1) == backward(w=A + 1) == backward(gy=A + 1) == backward(gw=A + 2) == backward(p=plan(offsets=A + 1)) == ALIGN
    assert forward(p=plan(tokens=0), y=None, out=None) == forward(cols=0, y=None, out=None) == backward(gy=None, gw=None) == backward(cols=0, gw=None) == 0


def _int(*shape, **k):
    return _Fake(*shape, dtype=torch.int32, **k)


class _Tables:
    """Stands for a plan whose tables are made up."""

    def __init__(self, index=_int(6, 2), slots=_int(6, 2), source=_int(12), offsets=_int(5)):
        self.tables = index, slots, source, offsets

    def _tables(self):
        return self.tables


def test_binding_refuses_what_does_not_fit(experts):
    f32 = dict(dtype=torch.float32)
    bad_plans = [_Tables(index=_Fake(6, 2)), _Tables(slots=_int(6, 1)), _Tables(source=_int(11)), _Tables(offsets=_int(1)), _Tables(offsets=_int(5, is_cuda=False)),
                 _Tables(source=_int(12, contiguous=False)), _Tables(index=_Fake(6, 2, dtype=torch.int64))]

    def gated(x=_Fake(6, 16), p=_Tables(), wg=_Fake(4, 24, 16), wu=_Fake(4, 24, 16), act="silu", h=_Fake(12, 24), gate=None, up=None, ordered=False):
        experts.bt_expert_gated_forward(x, p, wg, wu, act, h, gate, up, None, ordered, 0)

    def linear(x=_Fake(12, 16), p=_Tables(), w=_Fake(4, 24, 16), y=_Fake(12, 24), ordered=True):
        experts.bt_expert_linear_forward(x, p, w, y, None, ordered, 0)

    def route(logits=_Fake(6, 4), p=_Tables(), weights=_Fake(6, 2, **f32)):
        experts.bt_route_forward(logits, p, weights, None, True, 0)

    def combine(y=_Fake(12, 16), p=_Tables(), weights=_Fake(6, 2, **f32), out=_Fake(6, 16)):
        experts.bt_combine_forward(y, p, weights, out, 0)

    def back(gy=_Fake(12, 24), x=_Fake(12, 16), p=_Tables(), w=_Fake(4, 24, 16), gx=_Fake(12, 16), gw=_Fake(4, 24, 16)):
        experts.bt_expert_linear_backward(gy, x, p, w, gx, gw, None, True, 0)
    for call in (gated, linear, route, combine, back):
        for p in bad_plans:
            with pytest.raises(ValueError):
                call(p=p)
    for call, bad in ((gated, dict(x=_Fake(12, 16))), (gated, dict(x=_Fake(6, 15))), (gated, dict(ordered=True)), (gated, dict(wg=_Fake(3, 24, 16))), (gated, dict(wg=_Fake(96, 16))),
                      (gated, dict(wu=_Fake(4, 24, 15))), (gated, dict(h=_Fake(6, 24))), (gated, dict(gate=_Fake(12, 23), up=_Fake(12, 24))), (gated, dict(act="tanh")),
                      (linear, dict(x=_Fake(6, 16))), (linear, dict(w=_Fake(5, 24, 16))), (linear, dict(y=_Fake(12, 25))), (route, dict(logits=_Fake(6, 5))),
                      (route, dict(logits=_Fake(5, 4))), (route, dict(weights=_Fake(6, 2))), (route, dict(weights=_Fake(6, 1, **f32))), (combine, dict(y=_Fake(6, 16))),
                      (combine, dict(weights=_Fake(6, 2))), (combine, dict(weights=_Fake(12, 2, **f32))), (combine, dict(out=_Fake(6, 15))), (back, dict(gy=_Fake(12, 23))),
                      (back, dict(gx=_Fake(6, 16))), (back, dict(gw=_Fake(4, 16, 24, 2))), (back, dict(w=_Fake(24, 16)))):
        with pytest.raises(ValueError):
            call(**bad)
    for call, bad in ((gated, dict(x=None)), (gated, dict(h=None)), (gated, dict(wu=_Fake(4, 24, 16, dtype=torch.float16))), (linear, dict(w=None)), (route, dict(weights=None)),
                      (combine, dict(y=None)), (combine, dict(out=_Fake(6, 16, **f32))), (back, dict(x=None)), (back, dict(gx=_Fake(12, 16, dtype=torch.float16)))):
        with pytest.raises(TypeError):
            call(**bad)
    from paper_2110_15362_amd.bittrain import BitTrainError
    with pytest.raises(BitTrainError, match="BT_ERR_DTYPE"):
        linear(x=_Fake(12, 16, dtype=torch.float64), w=_Fake(4, 24, 16, dtype=torch.float64), y=_Fake(12, 24, dtype=torch.float64))
    with pytest.raises(BitTrainError, match="bt_expert_gated_forward failed: BT_ERR_ARGUMENT"):
        gated(gate=_Fake(12, 24))
    with pytest.raises(BitTrainError, match="BT_ERR_SIZE"):
        linear(p=_Tables(index=_int(6, 2), offsets=_int(2)), w=_Fake(1, 24, 16))          # two of one expert


def test_functions_refuse_on_the_host(experts):
    index = choices(6, 4, 2, 1)
    p = experts.Plan(index, *tables(index, 4))
    assert (p.tokens, p.chosen, p.experts, p.rows) == (6, 2, 4, 12)
    x, w = torch.zeros(6, 8), torch.zeros(4, 5, 8)
    for call in (lambda: experts.route(torch.zeros(6, 4), 2), lambda: experts.plan_of(index, 4), lambda: experts.gated_linear(x, p, w, w), lambda: experts.linear(x, p, w),
                 lambda: experts.combine(torch.zeros(12, 8), p)):
        with pytest.raises(ValueError, match="device memory"):
            call()
    with pytest.raises(ValueError, match="activation"):
        experts.gated_linear(x, p, w, w, "swish")
    with pytest.raises(TypeError, match="must be a Plan"):
        experts.linear(x, index, w)
    with pytest.raises(ValueError, match="tokens, experts"):
        experts.route(torch.zeros(2, 3, 4), 2)
    for chosen, n in ((0, 4), (5, 4), (33, 64), (1, 0), (1, 1025)):
        with pytest.raises(ValueError):
            experts.new_plan(6, n, chosen, device="cpu")
    with pytest.raises(ValueError, match="2\\^31"):
        experts.new_plan(1 << 30, 4, 2, device="meta")
    with pytest.raises(TypeError, match="32-bit"):
        experts.Plan(index.long(), *tables(index, 4))
    with pytest.raises(ValueError):
        experts.Plan(index, *tables(index[:5], 4))
    with pytest.raises(ValueError):
        experts.plan_of(torch.zeros(6, 2), 4)
    with pytest.raises(TypeError, match="float32, float16 and bfloat16"):
        experts.new_linear_workspace(p, 8, 8, torch.float64)


def test_tables_of_the_definition():
    """The order that the GPU tests compare with, against a hand-made one."""
    index = torch.tensor([[2, 0], [-1, 2], [1, 2], [0, 7]], dtype=torch.int32)
    slots, source, offsets = tables(index, 4)
    assert offsets.tolist() == [0, 2, 3, 6, 6]
    assert slots.tolist() == [[3, 0], [-1, 4], [2, 5], [1, -1]]
    assert source.tolist() == [0, 3, 2, 0, 1, 2, -1, -1]


@pytest.mark.parametrize("dtype,n", [(torch.uint8, 7), (torch.uint8, 256), (torch.uint8, 300), (torch.int8, 100), (torch.int8, 128), (torch.int8, 200), (torch.int16, 1000), (torch.uint16, 7),
                                     (torch.int32, 7), (torch.int64, 300)], ids=str)
def test_given_choices_of_any_integer_type(experts, dtype, n):
    """Numbers that are no expert's are -1, whatever the type that they come in can hold."""
    info = torch.iinfo(dtype)
    numbers = sorted({v for v in (0, 1, 5, 6, 7, n - 1, n, 127, 128, 255, -1, -7, info.min, info.max) if info.min <= v <= info.max})
    got = experts._numbers(torch.tensor([numbers, numbers[::-1]], dtype=torch.int64).to(dtype), n)
    want = [v if 0 <= v < n else -1 for v in numbers]
    assert got.dtype == torch.int32 and got.tolist() == [want, want[::-1]]


def test_both_weights_have_one_shape(experts):
    """As many elements in another order are not the same weight."""
    x, wg, wu = _Fake(6, 16), _Fake(4, 24, 16), _Fake(4, 16, 24)
    kept = _Fake(12, 24)
    for up in (wu, _Fake(24, 4, 16), _Fake(96, 16), _Fake(4, 384)):
        with pytest.raises(ValueError, match="w_up"):
            experts.bt_expert_gated_forward(x, _Tables(), wg, up, "silu", kept, None, None, None, False, 0)
        with pytest.raises(ValueError, match="w_up"):
            experts.bt_expert_gated_backward(kept, x, _Tables(), wg, up, kept, kept, "silu", x, wg, wg, None, False, 0)


def test_combine_refuses_weights_of_another_shape(experts, monkeypatch):
    """[chosen, tokens] has as many elements as [tokens, chosen]."""
    index = choices(6, 4, 2, 1)
    p = experts.Plan(index, *tables(index, 4))
    monkeypatch.setattr(experts, "_check_plan", lambda *a: None)      # (the tensors are on the host)
    for shape in ((2, 6), (1, 12), (6, 2, 1), (4, 3)):
        with pytest.raises(ValueError, match="weights"):
            experts.combine(torch.zeros(12, 8), p, torch.zeros(shape))
