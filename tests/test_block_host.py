"""What the feed-forward sublayer's calls refuse, on the host: through the C ABI with made-up addresses, which nothing dereferences, and through the
binding with tensors that do not fit.  No GPU."""
import ctypes
import os

import pytest
import torch

from tests.test_abi_host import _FakeTensor as _Flat

NULL, DTYPE, ALIGN, WORKSPACE, SIZE, ARGUMENT = 1, 2, 3, 4, 6, 8
A = 0x10000
F32, F16, BF16, F64 = 0, 1, 2, 3


@pytest.fixture(scope="module")
def block():
    import paper_2110_15362_amd.bittrain as bt
    if not os.path.exists(bt.LIB_PATH):
        from paper_2110_15362_amd import build
        build.build()
    from paper_2110_15362_amd import block
    block.lib()
    return block


@pytest.fixture(scope="module")
def L(block):
    raw = ctypes.CDLL(block._LIB_PATH)
    u64, sz, vp, ci, d = ctypes.c_uint64, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int, ctypes.c_double
    raw.bt_gated_workspace_bytes.restype, raw.bt_gated_workspace_bytes.argtypes = sz, [u64, u64, u64, ci, ci]
    raw.bt_gated_forward.argtypes = [vp] * 3 + [u64] * 3 + [ci, ci] + [vp] * 4 + [sz, vp]
    raw.bt_gated_backward.argtypes = [vp] * 6 + [u64] * 3 + [ci, ci] + [vp] * 4 + [sz, vp]
    raw.bt_residual_norm_workspace_bytes.restype, raw.bt_residual_norm_workspace_bytes.argtypes = sz, [u64, u64, u64, ci]
    raw.bt_residual_norm_forward.argtypes = [vp] * 5 + [u64] * 3 + [ci] + [d] * 3 + [vp] * 4
    raw.bt_residual_norm_backward.argtypes = [vp] * 8 + [u64] * 3 + [ci] + [d] * 2 + [vp] * 6 + [sz, vp]
    raw.bt_clip_workspace_bytes.restype, raw.bt_clip_workspace_bytes.argtypes = sz, [sz]
    raw.bt_grad_norm.argtypes = [vp, sz, vp, vp, sz, vp]
    raw.bt_clip_grads.argtypes = [vp, sz, d, d, vp, vp, sz, vp]
    return raw


def test_gated_errors(L):
    def forward(x=A, wg=A, wu=A, rows=3, d=16, f=24, dt=BF16, act=1, h=A, gate=A, up=A, ws=A, wsb=1 << 30):
        return L.bt_gated_forward(x, wg, wu, rows, d, f, dt, act, h, gate, up, ws, wsb, None)
    assert forward(dt=F64) == forward(dt=9) == DTYPE
    assert forward(rows=1 << 31) == forward(d=(1 << 24) + 1) == forward(f=(1 << 24) + 1) == SIZE
    assert forward(act=3) == forward(act=-1) == forward(gate=None) == forward(up=None) == ARGUMENT
    assert forward(x=None) == forward(wg=None) == forward(wu=None) == forward(h=None) == NULL
    for name in ("x", "wg", "wu", "h", "gate", "up"):
        assert forward(**{name: A + 1}) == ALIGN and forward(dt=F32, **{name: A + 2}) == ALIGN
    assert forward(ws=A + 64) == ALIGN
    assert forward(rows=0, x=None, h=None, gate=None, up=None) == forward(f=0, wg=None, wu=None, h=None, gate=None, up=None) == 0
    need = L.bt_gated_workspace_bytes(3, 16, 24, BF16, 0)
    if need:
        assert forward(ws=None) == NULL and forward(wsb=need - 1) == WORKSPACE

    need = L.bt_gated_workspace_bytes(3, 16, 24, BF16, 1)

    def backward(gh=A, x=A, wg=A, wu=A, gate=A, up=A, rows=3, d=16, f=24, dt=BF16, act=1, gx=A, gwg=A, gwu=A, ws=A, wsb=need):
        return L.bt_gated_backward(gh, x, wg, wu, gate, up, rows, d, f, dt, act, gx, gwg, gwu, ws, wsb, None)
    assert backward(dt=F64) == DTYPE and backward(rows=1 << 31) == SIZE
    assert backward(act=7) == backward(gwg=None) == backward(gwu=None) == ARGUMENT
    for name in ("gh", "gate", "up", "x", "wg", "wu", "ws"):
        assert backward(**{name: None}) == NULL
    for name in ("gh", "x", "wg", "wu", "gate", "up", "gx", "gwg", "gwu"):
        assert backward(**{name: A + 1}) == ALIGN
    assert backward(ws=A + 32) == ALIGN and backward(wsb=need - 1) == WORKSPACE
    assert backward(gx=None, gwg=None, gwu=None) == 0                 # nothing is wanted
    assert backward(d=0) == 0
    assert need > 0 and L.bt_gated_workspace_bytes(3, 16, 24, F64, 1) == 0 and L.bt_gated_workspace_bytes(1 << 31, 16, 24, F32, 1) == 0
    assert L.bt_gated_workspace_bytes(0, 16, 24, F32, 1) == L.bt_gated_workspace_bytes(4, 16, 0, F32, 1) == 0


def test_residual_norm_errors(L):
    inf, nan = float("inf"), float("nan")

    def forward(x=A, b=A, wp=A, gate=A, wn=A, rows=6, cols=16, gate_rows=3, dt=F16, eps=1e-6, scale=1.0, keep=1.0, out=A, y=A, stats=A):
        return L.bt_residual_norm_forward(x, b, wp, gate, wn, rows, cols, gate_rows, dt, eps, scale, keep, out, y, stats, None)
    assert forward(dt=F64) == DTYPE and forward(rows=1 << 31) == forward(cols=16385) == SIZE
    assert forward(eps=-1e-9) == forward(eps=nan) == forward(eps=inf) == forward(scale=nan) == forward(keep=inf) == ARGUMENT
    assert forward(gate_rows=4) == forward(gate_rows=0) == forward(gate_rows=12) == ARGUMENT
    assert forward(wn=None) == forward(y=None) == forward(b=None) == ARGUMENT
    assert forward(b=None, out=None, wp=None) == forward(b=None, out=None, gate=None) == forward(b=None, wp=None, gate=None) == ARGUMENT
    assert forward(x=None) == forward(out=None) == NULL
    for name in ("x", "b", "wp", "gate", "wn", "out", "y"):
        assert forward(**{name: A + 1}) == ALIGN
    assert forward(stats=A + 2) == ALIGN
    assert forward(rows=0, x=None, out=None, y=None) == forward(cols=0) == 0

    need = L.bt_residual_norm_workspace_bytes(6, 16, 3, F16)
    assert need > L.bt_residual_norm_workspace_bytes(6, 16, 0, F16) == L.bt_residual_norm_workspace_bytes(6, 16, 6, F16) > 0
    assert L.bt_residual_norm_workspace_bytes(6, 16, 3, F64) == L.bt_residual_norm_workspace_bytes(6, 16385, 3, F16) == 0

    def backward(go=A, gy=A, out=A, b=A, wp=A, gate=A, wn=A, stats=A, rows=6, cols=16, gate_rows=3, dt=F16, scale=1.0, keep=1.0, gx=A, gb=A, gwp=A, gg=A,
                 gwn=A, ws=A, wsb=need):
        return L.bt_residual_norm_backward(go, gy, out, b, wp, gate, wn, stats, rows, cols, gate_rows, dt, scale, keep, gx, gb, gwp, gg, gwn, ws, wsb, None)
    assert backward(dt=F64) == DTYPE and backward(cols=16385) == SIZE and backward(scale=inf) == backward(keep=nan) == ARGUMENT
    assert backward(gy=None) == backward(wn=None) == backward(wp=None) == backward(gate=None) == backward(b=None) == backward(gate_rows=5) == ARGUMENT
    assert backward(out=None) == backward(stats=None) == backward(ws=None) == NULL
    assert backward(wsb=need - 1) == WORKSPACE and backward(ws=A + 64) == ALIGN and backward(stats=A + 1) == ALIGN
    for name in ("go", "gy", "out", "b", "wp", "gate", "wn", "gx", "gb", "gwp", "gg", "gwn"):
        assert backward(**{name: A + 1}) == ALIGN
    assert backward(cols=0) == 0


def test_clip_errors(L):
    class Item(ctypes.Structure):
        _fields_ = [("d_in", ctypes.c_void_p), ("d_out", ctypes.c_void_p), ("n", ctypes.c_uint64), ("dtype", ctypes.c_int)]

    def clip(d_in=A, d_out=A, n=100, dt=BF16, max_norm=1.0, eps=0.0, norm=A, ws=A, wsb=1 << 20, count=2, call=None):
        items = (Item * 2)(Item(A, A, 10, F32), Item(d_in, d_out, n, dt))
        if call == "norm":
            return L.bt_grad_norm(items, count, norm, ws, wsb, None)
        return L.bt_clip_grads(items if count else None, count, max_norm, eps, norm, ws, wsb, None)
    nan = float("nan")
    assert clip(max_norm=-1.0) == clip(max_norm=nan) == clip(eps=-1.0) == clip(eps=nan) == ARGUMENT
    for call in (None, "norm"):
        assert clip(dt=F64, call=call) == clip(dt=-1, call=call) == DTYPE
        assert clip(n=(1 << 37) + 1, call=call) == SIZE
        assert clip(d_in=None, call=call) == clip(norm=None, call=call) == clip(ws=None, call=call) == NULL
        assert clip(d_in=A + 1, call=call) == clip(norm=A + 2, call=call) == clip(ws=A + 8, call=call) == ALIGN
        assert clip(wsb=L.bt_clip_workspace_bytes(2) - 1, call=call) == WORKSPACE
    assert clip(d_out=None) == NULL and clip(d_out=A + 1) == ALIGN
    assert L.bt_clip_grads(None, 1, 1.0, 0.0, A, A, 1 << 20, None) == NULL
    assert 0 < L.bt_clip_workspace_bytes(0) <= L.bt_clip_workspace_bytes(128) < L.bt_clip_workspace_bytes(1000)


class _Fake(_Flat):
    def __init__(self, *shape, dtype=torch.bfloat16, is_cuda=True, contiguous=True, ptr=0x10000):
        n = 1
        for s in shape:
            n *= s
        super().__init__(n, dtype, is_cuda, contiguous, ptr)
        self.shape = shape


def test_binding_refuses_what_does_not_fit(block):
    def gated(x=_Fake(2, 3, 16), wg=_Fake(24, 16), wu=_Fake(24, 16), act="silu", h=_Fake(2, 3, 24), gate=None, up=None):
        block.bt_gated_forward(x, wg, wu, act, h, gate, up, None, 0)
    for bad in ({"x": _Fake(2, 3, 17)}, {"wu": _Fake(24, 15)}, {"wu": _Fake(23, 16)}, {"h": _Fake(2, 3, 25)}, {"gate": _Fake(1), "up": _Fake(6, 24)},
                {"x": _Fake(2, 3, 16, is_cuda=False)}, {"wg": _Fake(24, 16, contiguous=False)}, {"act": "tanh"}, {"act": 1}, {"x": _Fake()}):
        with pytest.raises(ValueError):
            gated(**bad)
    for bad in ({"wg": _Fake(24, 16, dtype=torch.float16)}, {"h": _Fake(2, 3, 24, dtype=torch.float32)}, {"x": None}, {"h": None},
                {k: _Fake(*s, dtype=torch.int32) for k, s in (("x", (6, 16)), ("wg", (24, 16)), ("wu", (24, 16)), ("h", (6, 24)))}):
        with pytest.raises(TypeError):
            gated(**bad)
    double = {k: _Fake(*s, dtype=torch.float64) for k, s in (("x", (6, 16)), ("wg", (24, 16)), ("wu", (24, 16)), ("h", (6, 24)))}
    with pytest.raises(block.bt.BitTrainError, match="BT_ERR_DTYPE"):
        gated(**double)
    with pytest.raises(block.bt.BitTrainError, match="bt_gated_forward failed: BT_ERR_ARGUMENT"):
        gated(gate=_Fake(6, 24))
    with pytest.raises(ValueError):
        block.bt_gated_backward(_Fake(6, 24), _Fake(6, 16), _Fake(24, 16), _Fake(24, 16), _Fake(6, 24), _Fake(6, 24), "relu", _Fake(6, 15), None, None, _Fake(8), 0)
    with pytest.raises(TypeError):
        block.bt_gated_backward(None, _Fake(6, 16), _Fake(24, 16), _Fake(24, 16), _Fake(6, 24), _Fake(6, 24), "relu", None, None, None, None, 0)

    def norm(x=_Fake(6, 16), b=_Fake(6, 16), wp=_Fake(16), gate=_Fake(3, 16), wn=_Fake(16), out=_Fake(6, 16), y=_Fake(6, 16), stats=_Fake(2, 6, dtype=torch.float32),
             eps=1e-6):
        block.bt_residual_norm_forward(x, b, wp, gate, wn, out, y, stats, eps, stream=0)
    for bad in ({"b": _Fake(5, 16)}, {"wp": _Fake(15)}, {"gate": _Fake(4, 16)}, {"gate": _Fake(3, 15)}, {"wn": _Fake(1)}, {"out": _Fake(7, 16)}, {"y": _Fake(16)},
                {"stats": _Fake(6, dtype=torch.float32)}, {"stats": _Fake(2, 6, dtype=torch.float16)}, {"gate": _Fake(0, 16)}):
        with pytest.raises(ValueError):
            norm(**bad)
    for bad in ({"b": _Fake(6, 16, dtype=torch.float16)}, {"x": None}, {"eps": "small"}, {"wn": _Fake(16, dtype=torch.float32)}):
        with pytest.raises(TypeError):
            norm(**bad)
    with pytest.raises(block.bt.BitTrainError, match="BT_ERR_ARGUMENT"):
        norm(eps=-1.0)

    one = _Fake(1, dtype=torch.float32)
    ws = _Fake(1 << 16, dtype=torch.uint8)
    for grads, outs, error in (([_Fake(5)], [_Fake(6)], TypeError), ([_Fake(5)], [_Fake(5, dtype=torch.float16)], TypeError), ([_Fake(5)], [], ValueError),
                               (_Fake(5), [_Fake(5)], TypeError), ([_Fake(5)], None, TypeError), ([_Fake(5, is_cuda=False)], [_Fake(5)], ValueError),
                               ([_Fake(5, dtype=torch.int64)], [_Fake(5, dtype=torch.int64)], TypeError)):
        with pytest.raises(error):
            block.bt_clip_grads(grads, outs, 1.0, one, ws, stream=0)
    with pytest.raises(ValueError):
        block.bt_grad_norm([_Fake(5)], _Fake(1, dtype=torch.float64), ws, stream=0)
    with pytest.raises(block.bt.BitTrainError, match="BT_ERR_DTYPE"):
        block.bt_grad_norm([_Fake(5, dtype=torch.float64)], one, ws, stream=0)
    with pytest.raises(block.bt.BitTrainError, match="BT_ERR_ARGUMENT"):
        block.bt_clip_grads([_Fake(5)], [_Fake(5)], -1.0, one, ws, stream=0)


def test_functions_refuse_on_the_host(block):
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError, match="device memory"):
        block.gated_linear(x, w, w)
    with pytest.raises(ValueError, match="activation"):
        block.gated_linear(x, w, w, "swish")
    with pytest.raises(ValueError, match="device memory"):
        block.residual_norm(x, x)
    with pytest.raises(ValueError, match="device memory"):
        block.rms_norm(x, torch.ones(8))
    p = torch.nn.Parameter(torch.zeros(3))
    with pytest.raises(ValueError, match="no parameter has a gradient"):
        block.clip_grad_norm_([p], 1.0)
    p.grad = torch.zeros(3)
    with pytest.raises(ValueError, match="device memory"):
        block.clip_grad_norm_([p], 1.0)
    with pytest.raises(TypeError, match="float32, float16 and bfloat16"):
        block.new_gated_workspace(1, 8, 8, torch.float64)


def test_what_the_norms_cannot_do_without(block):
    with pytest.raises(TypeError, match="needs a weight"):
        block.rms_norm(torch.zeros(4, 8), None)
    with pytest.raises(TypeError, match="needs a block"):
        block.residual_norm(torch.zeros(4, 8), None)


def test_a_gate_that_broadcasting_reads_in_another_way_is_refused(block):
    """A gate is taken by rows of x in their order: one that lacks leading dimensions of x, which broadcasting repeats, is not that."""
    def matrix(gate, shape):
        return block._gate_matrix(gate, torch.Size(shape))
    x = (4, 6, 8)
    for shape, rows in (((8,), 1), ((1, 8), 1), ((1, 1, 8), 1), ((4, 8), 4), ((4, 1, 8), 4), ((4, 6, 8), 24), ((24, 8), 24), ((12, 8), 12), ((3, 8), 3), ((2, 2, 8), 4)):
        gate = torch.arange(float(torch.Size(shape).numel())).view(shape)
        assert torch.equal(matrix(gate, x), gate.view(rows, 8)), shape
        if gate.dim() == 3 and shape != (2, 2, 8):           # as broadcasting has it
            assert torch.equal(gate.expand(x).reshape(24, 8), gate.view(rows, 8).repeat_interleave(24 // rows, 0))
    for shape in ((6, 8), (1, 6, 8)):
        with pytest.raises(ValueError, match="expand it to the shape of x"):
            matrix(torch.zeros(shape), x)
        assert matrix(torch.zeros(shape).expand(x), x).shape == (24, 8)
    with pytest.raises(ValueError, match="expand it to the shape of x"):
        matrix(torch.zeros(2, 1, 5, 8), (2, 3, 5, 8))
    assert matrix(torch.zeros(2, 3, 1, 8), (2, 3, 5, 8)).shape == (6, 8)
    for shape, of in (((6, 8), (1, 6, 8)), ((1, 6, 8), (1, 6, 8)), ((5, 8), (15, 8)), ((15, 8), (15, 8)), ((4, 8), (4, 4, 8))):
        assert matrix(torch.zeros(shape), of).shape[0] == shape[-2]
    assert matrix(torch.zeros(3, 0), (3, 5, 0)).shape == (3, 0) and matrix(None, x) is None


def test_constants_are_the_headers(block):
    import re
    text = open(os.path.join(os.path.dirname(__file__), "..", "include", "bittrain.h")).read()
    for name, code in block.ACTIVATIONS.items():
        assert int(re.search(r"BT_ACT_%s = (\d+)" % name.upper(), text).group(1)) == code
    assert int(re.search(r"#define BT_MAX_NORM_COLS (\d+)", text).group(1)) == block.BT_MAX_NORM_COLS
