"""The example decoder layer: its gradients, and tokens one by one against whole sequences.

Errors are compared as vectors.  A rounding to bf16 moves a vector by at most u16 = 2^-8 of its size.  Forward there are eight on the
way (x, its projection, the exponentials, y, the output projection, and the experts' norm, products and sums count four more times
with two each); gradients pass through as many again, and what the softmax takes off is added for q and k.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U16 = 2.0 ** -8


@pytest.fixture(scope="module")
def example(lib):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def off(got, want):
    got, want = got.detach().double(), want.detach().double()
    return float((got - want).norm() / want.norm())


def plain(layer, leaves, offsets, ids):
    """The layer in 64 bits, with the experts that were chosen."""
    h, gain, to_qkv, to_out, gain2, router, blobs = leaves
    x = h * (h.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain
    qkv = (x @ to_qkv.t()).view(-1, layer.heads + 2 * layer.kv_heads, layer.dim)
    ys = []
    window, sinks = layer.sees["window"], layer.sees["sinks"]
    for a, b in zip(offsets, offsets[1:]):
        p, j = torch.arange(b - a, device=DEV)[:, None], torch.arange(b - a, device=DEV)[None]
        ok = (j <= p) & ((j > p - window) | (j < sinks)) if window else j <= p
        heads = []
        for i in range(layer.heads):
            kv = layer.heads + i // (layer.heads // layer.kv_heads)
            z = (qkv[a:b, i] @ qkv[a:b, kv].t()) * layer.dim ** -0.5
            heads.append(torch.softmax(z.masked_fill(~ok, float("-inf")), 1) @ qkv[a:b, kv + layer.kv_heads])
        ys.append(torch.cat(heads, 1))
    s = h + torch.cat(ys) @ to_out.t()
    x = s * (s.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gain2
    weight = torch.softmax(x @ router.t(), 1).gather(1, ids.long())
    out = torch.zeros_like(x)
    for e in range(blobs.shape[0]):
        gate, up, down = blobs[e].unbind(1)
        t, place = (ids == e).nonzero(as_tuple=True)
        out = out.index_add(0, t, weight[t, place, None] * ((torch.nn.functional.silu(x[t] @ gate.t()) * (x[t] @ up.t())) @ down))
    return s, out


@pytest.mark.parametrize("offsets,window,sinks", [([0, 1], 0, 0), ([0, 50, 77], 0, 0), ([0, 200, 203, 420], 60, 3)])
def test_gradients(example, offsets, window, sinks):
    torch.manual_seed(offsets[-1])
    layer = example.DecoderLayer(512, 4, 2, 64, 64, 4, 2, window, sinks)
    h = torch.randn(offsets[-1], 512, device=DEV, requires_grad=True)
    chosen = []
    choose = layer.experts.choose
    layer.experts.choose = lambda x: chosen.append(choose(x)) or chosen[-1]
    s, out = layer(h, torch.tensor(offsets, dtype=torch.int32, device=DEV))
    to_s, to_out = torch.randn_like(s), torch.randn_like(out)
    leaves = [h, layer.gain, layer.to_qkv, layer.to_out, layer.experts.gain, layer.experts.router, layer.experts.blobs]
    got = torch.autograd.grad((s * to_s).sum() + (out.float() * to_out.float()).sum(), leaves)
    wide = [t.detach().double().requires_grad_() for t in leaves]
    ws, wout = plain(layer, wide, offsets, chosen[0][0])
    want = torch.autograd.grad((ws * to_s).sum() + (wout * to_out).sum(), wide)
    assert off(s, ws) <= 5 * U16 and off(out, wout) <= 8 * U16
    for i, (a, b) in enumerate(zip(got, want)):
        assert a.dtype == leaves[i].dtype
        assert off(a, b) <= 16 * U16, i


@pytest.mark.parametrize("cache,most", [(torch.bfloat16, 10 * U16), (torch.int8, 0.08)])
def test_tokens_one_by_one(example, cache, most):
    torch.manual_seed(3)
    layer = example.DecoderLayer(512, 4, 2, 64, 64, 4, 4, 30, 2)  # (all experts: none is chosen otherwise after a rounding)
    n, new = [70, 1, 33], 12
    hs = [torch.randn(m + new, 512, device=DEV) for m in n]
    with torch.no_grad():
        offsets = torch.tensor([0, n[0] + new, n[0] + n[1] + 2 * new, sum(n) + 3 * new], dtype=torch.int32, device=DEV)
        s, out = layer(torch.cat(hs), offsets)
        want = (s + out.float()).split([m + new for m in n])
    served = example.Served(layer, 3, 100, cache=cache)
    s, out = served.prompts(torch.cat([h[:m] for h, m in zip(hs, n)]), torch.tensor(n, dtype=torch.int32, device=DEV))
    for got, w, m in zip((s + out.float()).split(n), want, n):
        assert off(got, w[:m]) <= 10 * U16
    for t in range(new):
        s, out = served.token(torch.stack([h[m + t] for h, m in zip(hs, n)]))
        assert off(s + out.float(), torch.stack([w[m + t] for w, m in zip(want, n)])) <= most


def test_it_runs(example):
    assert len(example.main(hidden=512, heads=4, tokens=300, steps=3, window=50)) == 3
