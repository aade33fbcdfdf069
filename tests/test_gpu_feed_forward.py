"""The operators of a feed-forward sublayer together, as examples/feed_forward.py uses them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("feed_forward_example", os.path.join(ROOT, "examples", "feed_forward.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _reference(model, x, condition):
    """The model's forward pass in plain torch, in 64 bits; returns the output and the parameters that it used."""
    p = {k: v.detach().double().requires_grad_() for k, v in model.named_parameters()}
    f = torch.nn.functional
    norm = lambda t: t * (t.square().mean(dim=-1, keepdim=True) + 1e-6).rsqrt()  # noqa: E731
    x, condition = x.double(), condition.double()
    y = norm(x) * p["first_norm"]
    for i in range(len(model.w_gate)):
        g = f.linear(y, p["w_gate.%d" % i])
        a = f.relu(g) if model.activation == "relu" else f.silu(g)
        b = f.linear(a * f.linear(y, p["w_up.%d" % i]), p["w_down.%d" % i])
        gate = f.linear(condition, p["w_condition.%d" % i])[:, None]
        x = x + model.scale * gate * norm(b) * p["post_norm.%d" % i]
        y = norm(x) * p["pre_norm.%d" % i]
    return y, p


def test_gradients_of_the_whole_stack(example):
    """Single precision against 64 bits: a few thousand 32-bit operations lie between, so 1e-4 of each gradient's norm; SiLU, whose gradient does not
    jump."""
    g = torch.Generator().manual_seed(3)
    model = example.FeedForwardStack(3, 72, 136, 8, activation="silu", dtype=torch.float32)
    x, target = (torch.randn(4, 9, 72, generator=g).cuda() for _ in range(2))
    condition = torch.randn(4, 8, generator=g).cuda()
    (model(x, condition) - target).square().mean().backward()
    y, params = _reference(model, x, condition)
    grads = torch.autograd.grad((y - target.double()).square().mean(), list(params.values()))
    for (name, _), want in zip(params.items(), grads):
        got = model.get_parameter(name).grad.double()
        assert float((got - want).norm()) <= 1e-4 * float(want.norm()), name


@pytest.mark.parametrize("deferred", [False, True])
def test_the_stash_changes_nothing_but_the_memory(example, deferred):
    """Equal losses and gradients bit for bit with saved tensors compressed, at less stored than dense."""
    from paper_2110_15362_amd import autograd
    g = torch.Generator().manual_seed(4)
    x, target = (torch.randn(8, 128, 256, generator=g).cuda().bfloat16() for _ in range(2))
    condition = torch.randn(8, 16, generator=g).cuda().bfloat16()
    results = []
    for stash in (None, autograd.BitmapStash(min_numel=4096, deferred=deferred)):
        model = example.FeedForwardStack(2, 256, 1024, 16)
        loss, norm = example.step(model, x, condition, target, stash, 1.0, 0.1)
        results.append([loss, norm] + [p.grad for p in model.parameters()] + [p.detach() for p in model.parameters()])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert stash.stats["compressed"] >= 6 and stash.stats["stored_bytes"] < 0.9 * stash.stats["dense_bytes"]


def test_nothing_is_kept_where_no_gradient_can_be_asked_for(monkeypatch):
    """Weights that are parameters, under no_grad and inference_mode: the calls get no place for what backward would need; with gradients they do.  Equal results."""
    from paper_2110_15362_amd import block
    kept = []

    def watch(name, places):
        call = getattr(block, name)

        def watched(*args):
            kept.append([args[i] is not None for i in places])
            return call(*args)
        monkeypatch.setattr(block, name, watched)
    watch("bt_gated_forward", (5, 6))                        # gate, up
    watch("bt_residual_norm_forward", (7,))                  # stats
    g = torch.Generator().manual_seed(5)
    x, w_gate, w_up, w_down, one, two = (torch.nn.Parameter(torch.randn(*s, generator=g).cuda()) for s in ((9, 16), (24, 16), (24, 16), (16, 24), (16,), (16,)))

    def sublayer():
        y = block.rms_norm(x, one)
        return block.residual_norm(x, block.gated_linear(y, w_gate, w_up) @ w_down.t(), one, two, two)
    want = sublayer()
    assert kept == [[True], [True, True], [True]] and want[0].requires_grad and want[1].requires_grad
    for mode in (torch.no_grad, torch.inference_mode):
        del kept[:]
        with mode():
            got = sublayer()
        assert kept == [[False], [False, False], [False]]
        assert all(torch.equal(a, b) and not a.requires_grad for a, b in zip(got, want))


def test_the_command_trains(example, capsys):
    losses = example.main(["--layers", "2", "--features", "256", "--hidden", "512", "--rows", "512", "--steps", "6", "--stash"])
    assert len(losses) == 6 and losses[-1] < losses[0]
    out = capsys.readouterr().out
    assert "tensors compressed" in out and "peak memory" in out
