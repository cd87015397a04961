"""A feed-forward layer of experts on the microscaled 4-bit products: every token
goes to ``top_k`` of E experts, each a gated MLP y = W2 (silu(g) u), (g, u) = W1 x,
and its outputs are added up by the router's weights.

Forward and backward use, in order: the products by expert (``LinearPlan`` with
``experts``), the gated activation with its 8-bit copy (``ActPlan``) and the
products by expert again.  The backward pass reads the 4-bit codes of both
products' inputs, 33/32 bytes an element of the activation's input, and, for the
router's gradient, x and the chosen experts' outputs [tokens, top_k, dim].  What is
allocated is more: the plans hold their outputs and gradients in full as long as
the layer lives.  In serving the activation writes its copy too, which nothing
reads then.  Routing (softmax, top-k, a stable sort) is torch's.
"""
from __future__ import annotations

from typing import Dict, Optional

import torch

from . import mx


class ExpertMLP:
    """``tokens`` rows of ``dim`` through ``experts`` gated MLPs of ``hidden`` units.
    Training (``train=True``): ``set_weights``, ``forward``, ``backward``; serving: ``set_weights``
    once, ``forward`` for any inputs of ``tokens`` rows (one token: single launches that read the
    chosen experts' weights once)."""

    def __init__(self, tokens: int, dim: int, hidden: int, experts: int, top_k: int, dtype=torch.bfloat16,
                 train: bool = True, device="cuda"):
        self.tokens, self.dim, self.hidden, self.experts, self.top_k, self.train = tokens, dim, hidden, experts, top_k, train
        rows = tokens * top_k
        self.up = mx.LinearPlan(rows, dim, 2 * hidden, dtype=dtype, experts=experts, train=train, device=device)
        self.act = mx.ActPlan(rows, hidden, "silu", gated=True, dtype=dtype, device=device)
        self.down = mx.LinearPlan(rows, hidden, dim, dtype=dtype, experts=experts, train=train, device=device)
        self._codes = None
        self._saved: Optional[tuple] = None

    def set_weights(self, w1: torch.Tensor, w2: torch.Tensor) -> None:
        """W1 [experts, 2 hidden, dim] (gate rows first) and W2 [experts, dim, hidden], in the layer's type: after every
        update of the weights."""
        if self.train:
            self.up.quantize_weight(w1)
            self.down.quantize_weight(w2)
        else:
            self._codes = mx.quantize(w1)[0], mx.quantize(w2)[0]

    def _route(self, x: torch.Tensor, router: torch.Tensor):
        """(router probabilities, chosen experts' share [tokens, top_k], row order, its inverse, offsets)"""
        probs = torch.softmax(x.float() @ router.float().t(), -1)
        share, chosen = probs.topk(self.top_k, -1)
        flat = chosen.reshape(-1)
        order = torch.argsort(flat, stable=True)
        inverse = torch.empty_like(order)
        inverse[order] = torch.arange(order.numel(), device=order.device)
        ends = torch.searchsorted(flat[order], torch.arange(self.experts, device=flat.device), right=True)
        offsets = torch.cat([ends.new_zeros(1), ends]).to(torch.int32)
        return probs, share, chosen, order, inverse, offsets

    def forward(self, x: torch.Tensor, router: torch.Tensor) -> torch.Tensor:
        """x [tokens, dim], router [experts, dim] -> [tokens, dim]"""
        probs, share, chosen, order, inverse, offsets = self._route(x, router)
        rows = x[order // self.top_k]
        w1, w2 = self._codes if self._codes else (None, None)
        h = self.act.forward(self.up.forward(rows, w1, offsets))
        y = self.down.forward(h, w2, offsets)
        y = y[inverse].view(self.tokens, self.top_k, self.dim)
        if self.train:
            self._saved = x, router, probs, share, chosen, order, inverse, y
        return (y.float() * share.unsqueeze(-1)).sum(1).to(x.dtype)

    def backward(self, dout: torch.Tensor) -> Dict[str, torch.Tensor]:
        """Gradients of the last forward: x, router, w1 and w2 (the last two in float32, the layer's buffers)."""
        if self._saved is None:
            raise ValueError("backward needs a forward of a layer with train=True")
        x, router, probs, share, chosen, order, inverse, y = self._saved
        d = dout.float().unsqueeze(1)
        dy = (d * share.unsqueeze(-1)).to(x.dtype).reshape(-1, self.dim)[order]
        dh, dw2 = self.down.backward(dy)
        drows, dw1 = self.up.backward(self.act.backward(dh))
        dx = drows[inverse].view(self.tokens, self.top_k, self.dim).float().sum(1)
        # the shares are the chosen entries of a softmax
        dprobs = torch.zeros_like(probs).scatter_(1, chosen, (d * y.float()).sum(-1))
        dlogits = probs * (dprobs - (dprobs * probs).sum(-1, keepdim=True))
        dx = dx + dlogits @ router.float()
        return {"x": dx.to(x.dtype), "router": dlogits.t() @ x.float(), "w1": dw1, "w2": dw2}
