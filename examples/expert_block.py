"""Trains a block of experts (layer norm with its residual sum, router with a bias for
balance, 4-bit experts, a shared 8-bit MLP) to imitate a fixed function, then serves
single tokens from its codes.

    python examples/expert_block.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2411_10948_amd.experts import ExpertBlock  # noqa: E402


def run(steps=200, tokens=1024, dim=512, hidden=256, experts=16, top_k=2, shared=256, lr=0.05, log=print):
    """(loss of each step, the last step's gradients, how far a token served alone is from the same one in a batch)"""
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    rule = dict(score="sigmoid", renormalize=True)
    layer = ExpertBlock(tokens, dim, hidden, experts, top_k, shared, **rule)
    names = ("gamma", "beta", "router", "w1", "w2", "s1", "s2")
    master = dict(zip(names, (torch.ones(dim, device="cuda"), torch.zeros(dim, device="cuda"), r(experts, dim) / dim ** 0.5,
                              r(experts, 2 * hidden, dim) / dim ** 0.5, r(experts, dim, hidden) / hidden ** 0.5,
                              r(2 * shared, dim) / dim ** 0.5, r(dim, shared) / shared ** 0.5)))
    bias = torch.zeros(experts, device="cuda")
    target = r(dim, dim) / dim ** 0.5

    def weights():
        return [master[n] if n in ("gamma", "beta", "router") else master[n].bfloat16() for n in names] + [bias]
    losses, grads = [], {}
    for step in range(steps):
        layer.set_weights(*weights())
        x, residual = r(tokens, dim).bfloat16(), r(tokens, dim).bfloat16()
        out, h = layer.forward(x, residual)
        err = out.float() - torch.tanh(h.float() @ target)
        losses.append(float((err * err).mean()))
        grads = layer.backward((2 * err / tokens).bfloat16())
        for n in names:
            master[n] -= lr * grads[n]
        rows = layer.router.offsets.diff().float()      # towards an even load
        bias += 0.01 * torch.sign(rows.mean() - rows)
        if step % 50 == 0 or step == steps - 1:
            log(f"step {step}: loss {losses[-1]:.4f}, rows of an expert {int(rows.min())} to {int(rows.max())}")
    batch = ExpertBlock(8, dim, hidden, experts, top_k, shared, train=False, **rule)
    one = ExpertBlock(1, dim, hidden, experts, top_k, shared, train=False, **rule)
    for served in (batch, one):
        served.set_weights(*weights())
    x, residual = r(8, dim).bfloat16(), r(8, dim).bfloat16()
    want = batch.forward(x, residual)[0].float().clone()
    got = torch.cat([one.forward(x[i:i + 1], residual[i:i + 1])[0].float().clone() for i in range(8)])
    far = float((got - want).norm() / want.norm())
    log(f"eight tokens served one by one: {far:.2e} from the same ones together")
    return losses, grads, far


if __name__ == "__main__":
    run()
