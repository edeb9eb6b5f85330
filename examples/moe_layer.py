"""A mixture-of-experts layer on many rows, trained and then served with 8-bit experts.

    python examples/moe_layer.py

h + y -> norm -> router -> rows sorted by expert -> SwiGLU experts -> weighted sum, forward and backward on the library's
operators; the router's small product and the optimiser are PyTorch's.  The weights of the experts are one tensor in the layout
that the kernels stream ([experts, inter, 3, hidden]: gate row, up row, column of down), and so are their gradients.
"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2412_00099_amd as moe  # noqa: E402
from paper_2412_00099_amd import binding  # noqa: E402


class AddNorm(torch.autograd.Function):
    """(h + y, its norm in bf16)"""

    @staticmethod
    def forward(ctx, h, y, gain):
        n = moe.norm_rows(h, y, gain)
        ctx.save_for_backward(n.h, gain, n.rstd)
        ctx.y_type = None if y is None else y.dtype
        return n.h, n.x

    @staticmethod
    def backward(ctx, dh, dx):
        d, dgain = moe.norm_rows_backward(*ctx.saved_tensors, dx.contiguous(), dh.contiguous())
        return d, None if ctx.y_type is None else d.to(ctx.y_type), dgain


class Experts(torch.autograd.Function):
    """y = sum over a token's experts of weight * expert(x)"""

    @staticmethod
    def forward(ctx, x, ids, weight, blobs):
        order = moe.sort_tokens(ids, blobs.shape[0])
        xs, _ = moe.gather_rows(x, order)
        ys, kept = moe.experts_rows("bf16", blobs, blobs.shape[1], xs, order.offsets, keep=True)
        ctx.save_for_backward(weight, blobs, xs, ys, *kept, *order)
        return moe.combine_rows(ys, order, weight)

    @staticmethod
    def backward(ctx, dy):
        weight, blobs, xs, ys, h, gu, *order = ctx.saved_tensors
        order = moe.TokenOrder(*order)
        dys, dweight = moe.combine_rows_backward(dy.contiguous(), ys, order, weight)
        dxs, dblobs = moe.experts_rows_backward("bf16", blobs, blobs.shape[1], xs, order.offsets, moe.KeptExperts(h, gu), dys)
        return moe.combine_rows(dxs, order), None, dweight, dblobs


class MoELayer(torch.nn.Module):
    def __init__(self, hidden, inter, experts, top_k, device="cuda"):
        super().__init__()
        self.top_k = top_k
        self.gain = torch.nn.Parameter(torch.ones(hidden, device=device))
        self.router = torch.nn.Parameter(torch.randn(experts, hidden, device=device) * hidden ** -0.5)
        self.blobs = torch.nn.Parameter((torch.randn(experts, inter, 3, hidden, device=device) * hidden ** -0.5).bfloat16())

    def choose(self, x):
        """(ids, softmax weights) of a token's experts, strongest first"""
        p = torch.softmax(x.float() @ self.router.t(), 1)
        weight, ids = p.topk(self.top_k, 1)
        return ids.int(), weight

    def forward(self, h, y=None):
        """(h + y, the experts' output on it): the next layer adds them"""
        h, x = AddNorm.apply(h, y, self.gain)
        ids, weight = self.choose(x)
        return h, Experts.apply(x, ids, weight, self.blobs)


class ServedLayer:
    """The layer with 8-bit experts and 8-bit rows."""

    @torch.no_grad()
    def __init__(self, layer):
        self.choose, self.gain = layer.choose, layer.gain.detach()
        e, self.inter, _, d = layer.blobs.shape
        self.blobs = torch.zeros(e, binding.moe_blob_bytes(binding.MOE_W_INT8_PC, d, self.inter), dtype=torch.uint8, device=layer.blobs.device)
        stream = torch.cuda.current_stream().cuda_stream
        for i in range(e):
            gate, up, columns = layer.blobs[i].float().unbind(1)
            parts = [self.codes(w.contiguous()) for w in (gate, up, columns.t())]
            binding.moe_pack_expert(binding.MOE_W_INT8_PC, d, self.inter, *(q.data_ptr() for q, _ in parts),
                                    *(s.data_ptr() for _, s in parts), self.blobs[i].data_ptr(), stream)

    @staticmethod
    def codes(w):
        """8-bit codes of the rows of w and their scales"""
        scale = (w.abs().amax(1) / 127).clamp_min(1e-6).half()
        return (w / scale.float()[:, None]).round().clamp(-127, 127).to(torch.int8), scale

    @torch.no_grad()
    def __call__(self, h, y=None):
        n = moe.norm_rows(h, y, self.gain, out=torch.int8)
        ids, weight = self.choose(n.x.float() * n.scale[:, None])
        order = moe.sort_tokens(ids, self.blobs.shape[0])
        xs, scale = moe.gather_rows(n.x, order, n.scale)
        ys = moe.experts_rows("int8", self.blobs, self.inter, xs, order.offsets, scale=scale)
        return n.h, moe.combine_rows(ys, order, weight)


def train(layer, h, target, steps, rate=2e-3):
    """Fit the layer's output on h to target; the share of target's square that is missed, before each step."""
    blobs = layer.blobs.detach().float()  # (the optimiser's steps are smaller than the roundings of bf16)
    adam = torch.optim.Adam([layer.gain, layer.router, blobs], lr=rate)
    size, losses = target.float().square().mean(), []
    for _ in range(steps):
        _, y = layer(h)
        loss = (y.float() - target.float()).square().mean() / size
        loss.backward()
        blobs.grad, layer.blobs.grad = layer.blobs.grad.float(), None
        adam.step()
        adam.zero_grad()
        with torch.no_grad():
            layer.blobs.copy_(blobs)
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


def main(hidden=1024, inter=512, experts=16, top_k=4, tokens=2000, steps=60):
    torch.manual_seed(0)
    teacher, layer = (MoELayer(hidden, inter, experts, top_k) for _ in range(2))
    with torch.no_grad():
        layer.router.copy_(teacher.router)
        h = torch.randn(tokens, hidden, device="cuda")
        target = teacher(h)[1]
    losses = train(layer, h, target, steps)
    print(f"{tokens} tokens, {experts} experts of {hidden} x {inter}, {top_k} a token: loss {losses[0]:.3f} -> {losses[-1]:.3f} in {steps} steps")
    served = ServedLayer(layer)
    with torch.no_grad():
        want = layer(h)[1].float()
    prompt = served(h)[1].float()
    single = torch.cat([served(h[i:i + 1])[1] for i in range(16)]).float()
    print(f"8-bit experts: a prompt differs from bf16 by {(prompt - want).norm() / want.norm():.4f} of its size, "
          f"single tokens by {(single - want[:16]).norm() / want[:16].norm():.4f}")
    return losses


if __name__ == "__main__":
    main()
