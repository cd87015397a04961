"""Train a small layer of experts with 4-bit products and an 8-bit activation
copy, then serve single tokens from its 4-bit weights.

    python examples/expert_mlp.py [--steps 60] [--tokens 512] [--dim 256] [--hidden 384] [--experts 8] [--top-k 2]

The target is a fixed random layer of the same shape computed in fp32; the data
are synthetic and seeded.  Prints the loss as it falls, the bytes of the codes
that the backward pass reads in place of tensors and of all the layer's buffers,
and how far the served tokens are from the trained layer's own forward.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2411_10948_amd.experts import ExpertMLP  # noqa: E402


def target(x, router, w1, w2, top_k):
    """The layer in fp32, every expert on every token."""
    g, u = torch.matmul(x, w1.transpose(1, 2).contiguous()).chunk(2, -1)
    y = torch.matmul(torch.nn.functional.silu(g) * u, w2.transpose(1, 2).contiguous()).transpose(0, 1)
    share, chosen = torch.softmax(x @ router.t(), -1).topk(top_k, -1)
    return (y.gather(1, chosen.unsqueeze(-1).expand(-1, -1, x.shape[1])) * share.unsqueeze(-1)).sum(1)


def run(steps=60, tokens=512, dim=256, hidden=384, experts=8, top_k=2, lr=2e-3, log=print):
    """(first loss, last loss, relative distance of served tokens)"""
    gen = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    shapes = {"router": (experts, dim), "w1": (experts, 2 * hidden, dim), "w2": (experts, dim, hidden)}
    goal = {k: rand(*s) / s[-1] ** 0.5 for k, s in shapes.items()}
    weights = {k: v + 0.3 * rand(*v.shape) / v.shape[-1] ** 0.5 for k, v in goal.items()}
    moments = {k: (torch.zeros_like(v), torch.zeros_like(v)) for k, v in weights.items()}

    held = torch.cuda.memory_allocated()
    layer = ExpertMLP(tokens, dim, hidden, experts, top_k)
    held = torch.cuda.memory_allocated() - held
    first = last = None
    for step in range(1, steps + 1):
        x = rand(tokens, dim)
        want = target(x, goal["router"], goal["w1"], goal["w2"], top_k)
        layer.set_weights(weights["w1"].bfloat16(), weights["w2"].bfloat16())
        diff = layer.forward(x.bfloat16(), weights["router"]).float() - want
        grads = layer.backward((2 * diff / diff.numel()).bfloat16())
        for k, (m, v) in moments.items():      # Adam
            m.lerp_(grads[k], 0.1)
            v.lerp_(grads[k].square(), 0.01)
            weights[k] -= lr * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.99 ** step)).sqrt() + 1e-12)
        last = diff.square().mean().item()
        first = last if first is None else first
        if step == 1 or step % 20 == 0:
            log(f"step {step:3d}  loss {last:.5f}", flush=True)
    kept = sum(t.numel() for t in (layer.up.x_t.codes, layer.up.x_t.scales, layer.down.x_t.codes, layer.down.x_t.scales,
                                   layer.act.codes, layer.act.scales))
    log(f"codes that the backward pass reads: {kept / 1e6:.2f} MB (segments of 512 rows an expert included); the same "
        f"tensors in bf16: {2 * tokens * top_k * (dim + 3 * hidden) / 1e6:.2f} MB; all of the layer's buffers, weights' codes, "
        f"outputs and gradients among them: {held / 1e6:.2f} MB")

    one = ExpertMLP(1, dim, hidden, experts, top_k, train=False)
    w = weights["w1"].bfloat16(), weights["w2"].bfloat16()
    one.set_weights(*w)
    layer.set_weights(*w)
    x = rand(tokens, dim).bfloat16()
    whole = layer.forward(x, weights["router"]).float()
    served = torch.cat([one.forward(x[i:i + 1], weights["router"]).float() for i in range(16)])
    far = ((served - whole[:16]).norm() / whole[:16].norm()).item()
    log(f"16 tokens served one at a time: {far:.1e} from the batch's")
    return first, last, far


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, default in (("steps", 60), ("tokens", 512), ("dim", 256), ("hidden", 384), ("experts", 8), ("top-k", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    run(**{k: v for k, v in vars(ap.parse_args()).items()})
