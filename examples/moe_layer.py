"""A mixture-of-experts layer from the library's operators: trained for a few steps,
then served token by token from 4-bit matrices.

    python examples/moe_layer.py

    logits = x Wr                          sgemm
    ids, weights, order = route(logits)    moe_route
    h = W1[expert] x                       grouped_gemm, rows gathered through the order
    z = W2[expert] silu(h)                 grouped_gemm
    y = sum of weights z                   moe_combine

The matrices of the experts are stored E x out x in (transb 'T'), as q4_pack wants
them.  Everything is ordered on torch's current stream and nothing waits for the
device: how many rows an expert has is known there only.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2609_04663_amd as emu  # noqa: E402


class MoE(torch.autograd.Function):
    """y of tokens x (T x D) for the router Wr (D x E, float32) and the experts'
    W1 (E x H x D) and W2 (E x D x H), k experts a token."""

    @staticmethod
    def forward(ctx, x, Wr, W1, W2, k, scope):
        logits = emu.sgemm(x.float(), Wr)
        r = emu.moe_route(logits, k, scope)
        h = emu.grouped_gemm(x, W1, r.offsets, transb="T", rows=r.rows)
        a = torch.nn.functional.silu(h)
        z = emu.grouped_gemm(a, W2, r.offsets, transb="T")
        ctx.save_for_backward(x, Wr, W1, W2, logits, h, a, z, *r)
        ctx.scope = scope
        return emu.moe_combine(z, r.slots, r.weights)

    @staticmethod
    def backward(ctx, dy):
        x, Wr, W1, W2, logits, h, a, z, *r = ctx.saved_tensors
        r = emu.Routing(*r)
        dz, dweights = emu.moe_combine_grad(dy.contiguous(), z, r.slots, r.weights, r.rows)
        dW2 = emu.grouped_wgrad(a, dz, r.offsets, transb="T")
        da = emu.grouped_gemm(dz, W2, r.offsets)
        s = torch.sigmoid(h.float())
        dh = (da.float() * s * (1 + h.float() * (1 - s))).to(h.dtype)
        dW1 = emu.grouped_wgrad(x, dh, r.offsets, transb="T", rows=r.rows)
        dx = emu.moe_combine(emu.grouped_gemm(dh, W1, r.offsets), r.slots)     # each token's rows
        dlogits = emu.moe_route_grad(logits, r.ids, r.weights, dweights, ctx.scope)
        dWr = emu.sgemm_ex(x.float(), dlogits, transa="T")
        dx = dx + emu.sgemm_ex(dlogits, Wr, transb="T").to(dx.dtype)
        return dx, dWr, dW1, dW2, None, None


def moe(x, Wr, W1, W2, k, scope="chosen"):
    return MoE.apply(x, Wr, W1, W2, k, scope)


class Served:
    """The layer with the experts' matrices in 4 bits, for a few tokens at a time."""

    def __init__(self, Wr, W1, W2, k, scope="chosen", group=64):
        self.Wr, self.k, self.scope = Wr, k, scope
        self.W1, self.W2 = emu.q4_pack(W1, group), emu.q4_pack(W2, group)

    def __call__(self, x):
        r = emu.moe_route(emu.sgemm(x.float(), self.Wr), self.k, self.scope)
        h = emu.q4_gemm(x, *self.W1, offsets=r.offsets, rows=r.rows)
        z = emu.q4_gemm(torch.nn.functional.silu(h), *self.W2, offsets=r.offsets)
        return emu.moe_combine(z, r.slots, r.weights)


def main(T=4096, D=1024, H=512, E=32, k=4, steps=20, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape, scale=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * scale

    x = randn(T, D).to(dtype)
    target = torch.tanh(x.float() @ randn(D, D, scale=D ** -0.5))
    Wr, W1, W2 = randn(D, E, scale=D ** -0.5), randn(E, H, D, scale=D ** -0.5), randn(E, D, H, scale=H ** -0.5)
    masters = [w.requires_grad_() for w in (Wr, W1, W2)]
    opt = torch.optim.Adam(masters, lr=2e-3)
    for step in range(steps):
        y = moe(x, Wr, W1.to(dtype), W2.to(dtype), k)
        loss = ((y.float() - target) ** 2).mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        if step % 5 == 0 or step == steps - 1:
            print(f"step {step:3d}  loss {loss.item():.4f}", flush=True)
    with torch.no_grad():
        W1, W2 = W1.to(dtype), W2.to(dtype)
        served = Served(Wr, W1, W2, k)
        exact = moe(x[:16], Wr, W1, W2, k).float()
        off = torch.cat([served(x[t:t + 1]).float() for t in range(16)]) - exact
        print(f"served from 4 bits, token by token: relative difference {(off.norm() / exact.norm()).item():.3f}")
    return loss.item()


if __name__ == "__main__":
    main()
