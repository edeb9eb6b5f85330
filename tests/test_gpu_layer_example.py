"""The example layer: its gradients, its training and its 8-bit form.

Errors are compared as vectors.  A rounding to bf16 moves a vector by at most u16 = 2^-8 of its size; forward there are four
(x, the products of gate and up, a row's result, the sum), and the gradients pass through as many again.  The router's gradient
is what is left when softmax has taken the mean off, so that twice as much is allowed there.
"""
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16 = 2.0 ** -8


@pytest.fixture(scope="module")
def example(lib):
    import importlib.util

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")
    spec = importlib.util.spec_from_file_location("moe_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain(h, y, gain, router, blobs, ids):
    """The layer in 64 bits, with the experts that were chosen."""
    s = h if y is None else h + y
    x = s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain
    weight = torch.softmax(x @ router.t(), 1).gather(1, ids.long())
    out = torch.zeros_like(x)
    for e in range(blobs.shape[0]):
        gate, up, down = blobs[e].unbind(1)
        t, place = (ids == e).nonzero(as_tuple=True)
        out = out.index_add(0, t, weight[t, place, None] * ((torch.nn.functional.silu(x[t] @ gate.t()) * (x[t] @ up.t())) @ down))
    return s, out


def off(got, want):
    got, want = got.detach().double(), want.detach().double()
    return float((got - want).norm() / want.norm())


@pytest.mark.parametrize("tokens,added", [(1, True), (77, False), (600, True)])
def test_gradients(example, tokens, added):
    torch.manual_seed(tokens)
    layer = example.MoELayer(512, 200, 6, 2)
    h = torch.randn(tokens, 512, device=DEV, requires_grad=True)
    y = torch.randn(tokens, 512, device=DEV).bfloat16().requires_grad_() if added else None
    s, out = layer(h, y)
    ids, _ = layer.choose(example.moe.norm_rows(s.detach(), None, layer.gain.detach()).x)
    to_s, to_out = torch.randn_like(s), torch.randn_like(out)
    leaves = [h] + ([y] if added else []) + [layer.gain, layer.router, layer.blobs]
    got = torch.autograd.grad((s * to_s).sum() + (out.float() * to_out.float()).sum(), leaves)

    wide = [t.detach().double().requires_grad_() for t in leaves]
    ws, wout = plain(wide[0], wide[1] if added else None, *wide[-3:], ids)
    want = torch.autograd.grad((ws * to_s).sum() + (wout * to_out).sum(), wide)
    assert off(s, ws) <= 2.0 ** -22 and off(out, wout) <= 4 * U16
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.dtype == leaves[i].dtype
        assert off(a, b) <= (16 if leaves[i] is layer.router else 8) * U16, i


def test_training_and_8_bit_form(example):
    torch.manual_seed(1)
    teacher, layer = (example.MoELayer(1024, 128, 8, 2) for _ in range(2))
    h = torch.randn(400, 1024, device=DEV)
    with torch.no_grad():
        layer.router.copy_(teacher.router)
        target = teacher(h)[1]
    losses = example.train(layer, h, target, 40)
    assert losses[-1] < 0.5 * losses[0]
    with torch.no_grad():
        want = layer(h)[1]
    # codes are off by half a step of 1/127 of the largest value at most: of rows of 1024 normal values about 0.7 % of their size,
    # rows and weights of the first products and weights of the last, each twice over allowed
    served = example.ServedLayer(layer)
    few = [served(h[i:i + 1])[1] for i in range(8)]
    same = [i for i in range(8) if torch.equal(layer.choose(example.moe.norm_rows(h[i:i + 1], None, layer.gain.detach()).x)[0],
                                               served.choose(dequant(example, served, h[i:i + 1]))[0])]
    assert len(same) >= 4
    for i in same:
        assert off(few[i], want[i:i + 1]) <= 0.06


def dequant(example, served, h):
    n = example.moe.norm_rows(h, None, served.gain, out=torch.int8)
    return n.x.float() * n.scale[:, None]
