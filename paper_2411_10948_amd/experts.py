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

from typing import Dict, Optional, Tuple

import torch

from . import f8, mx, norm, route


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


class ExpertBlock:
    """h = x + residual, y = norm(h), out = shared MLP(y) + sum over the chosen experts of share MLP_e(y),
    for ``tokens`` rows of ``dim``: ``experts`` gated MLPs of ``hidden`` units in microscaled 4 bits, ``top_k``
    of them a token, and one of ``shared`` units in 8 bits (0: none).  The router takes y in float32; its
    rule (``score``, ``groups``, ``top_groups``, ``renormalize``, ``scale``) is ``RouterPlan``'s.  A token whose
    shares are NaN (NaN among its logits, +Inf under softmax) has NaN in all of its out.

    Training (``train=True``): ``set_weights``, ``forward``, ``backward``; serving: ``set_weights`` once, ``forward``
    for any inputs of ``tokens`` rows.  Results are the layer's buffers, overwritten by its next call; no step
    needs the host, so both can be captured into a graph."""

    def __init__(self, tokens: int, dim: int, hidden: int, experts: int, top_k: int, shared: int = 0, eps: float = 1e-5,
                 score: str = "softmax", groups: int = 1, top_groups: Optional[int] = None, renormalize: bool = True,
                 scale: float = 1.0, dtype=torch.bfloat16, train: bool = True, device="cuda"):
        rows, kw = tokens * top_k, dict(dtype=dtype, device=device)
        self.tokens, self.dim, self.hidden, self.experts, self.top_k, self.shared = tokens, dim, hidden, experts, top_k, shared
        self.dtype, self.train = dtype, train
        self.norm = norm.NormPlan(tokens, dim, eps, residual=True, train=train, **kw)
        self.router = route.RouterPlan(tokens, experts, top_k, score, groups, top_groups, renormalize, scale, dtype=torch.float32,
                                       device=device)
        self.exchange = route.ExchangePlan(tokens, top_k, dim, train=train, **kw)
        self.up = mx.LinearPlan(rows, dim, 2 * hidden, experts=experts, train=train, **kw)
        self.act = mx.ActPlan(rows, hidden, "silu", gated=True, **kw)
        self.down = mx.LinearPlan(rows, hidden, dim, experts=experts, train=train, **kw)
        if shared:
            self.shared_up = f8.LinearPlan(tokens, dim, 2 * shared, train=train, **kw)
            self.shared_act = mx.ActPlan(tokens, shared, "silu", gated=True, **kw)
            self.shared_down = f8.LinearPlan(tokens, shared, dim, train=train, **kw)
        self._zero = torch.zeros(1, device=device)
        self._codes: tuple = (None, None, None, None)
        self._weights: Optional[tuple] = None
        self._saved: Optional[tuple] = None

    def set_weights(self, gamma: torch.Tensor, beta: torch.Tensor, router: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor,
                    s1: Optional[torch.Tensor] = None, s2: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None) -> None:
        """The norm's weights [dim], the router [experts, dim] and its bias [experts] (what moves the choice alone), all float32;
        W1 [experts, 2 hidden, dim] (gate rows first) and W2 [experts, dim, hidden], the shared MLP's [2 shared, dim] and
        [dim, shared], in the layer's type: after every update of the weights.  The first four are kept, not copied."""
        if (s1 is None or s2 is None) == bool(self.shared):
            raise ValueError("s1, s2: expected for a layer with shared > 0, and for no other")
        if router.shape != (self.experts, self.dim) or router.dtype != torch.float32:
            raise ValueError(f"router: expected float32 values of shape {(self.experts, self.dim)}")
        self._weights = gamma, beta, router, bias
        if self.train:
            self.up.quantize_weight(w1)
            self.down.quantize_weight(w2)
            if self.shared:
                self.shared_up.quantize_weight(s1)
                self.shared_down.quantize_weight(s2)
        else:
            dense = (f8.quantize(s1, square=True)[0], f8.quantize(s2, square=True)[0]) if self.shared else (None, None)
            self._codes = (mx.quantize(w1)[0], mx.quantize(w2)[0], *dense)

    def forward(self, x: torch.Tensor, residual: torch.Tensor) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out, h) [tokens, dim]; the backward pass reads h, so it is not written to before that"""
        if self._weights is None:
            raise ValueError("forward needs set_weights before it")
        gamma, beta, router, bias = self._weights
        w1, w2, s1, s2 = self._codes
        y = self.norm.forward(x, gamma, beta, residual)
        logits = y.float() @ router.t()
        share, _ = self.router.forward(logits, bias)
        place, offsets = self.router.place, self.router.offsets
        rows = self.exchange.dispatch(y, place)
        z = self.down.forward(self.act.forward(self.up.forward(rows, w1, offsets)), w2, offsets)
        dense = None
        if self.shared:
            dense = self.shared_down.forward(self.shared_act.forward(self.shared_up.forward(y, s1)), s2)
        if self.train:
            self._saved = y, logits, share, place, z
        # such a token has no rows to bring its NaN back: share 0 adds it, and nothing to the others
        return self.exchange.combine(z, place, share, dense).addcmul_(share[:, :1], self._zero), self.norm.H

    def backward(self, dout: torch.Tensor, dh: Optional[torch.Tensor] = None) -> Dict[str, torch.Tensor]:
        """Gradients of the last forward, dh that of h: x (the residual's too), gamma, beta, router, w1, w2 and, with a shared
        MLP, s1 and s2; x in the layer's type, the others in float32."""
        if self._saved is None:
            raise ValueError("backward needs a forward of a layer with train=True")
        gamma, _, router, _ = self._weights
        y, logits, share, place, z = self._saved
        dz, dshare = self.exchange.combine_backward(dout, z, place, share)
        dlogits = self.router.backward(dshare, logits)
        da, dw2 = self.down.backward(dz)
        drows, dw1 = self.up.backward(self.act.backward(da))
        dy, grads = dlogits @ router, {"w1": dw1, "w2": dw2}
        if self.shared:
            da, grads["s2"] = self.shared_down.backward(dout)
            dense, grads["s1"] = self.shared_up.backward(self.shared_act.backward(da))
            dy = dy + dense.float()
        # In bf16 the addend is rounded before the experts' part is added in fp32 and the sum is rounded once more: the exchange
        # adds rows of its own type, and half a step of the addend is what the experts' and the shared MLP's parts are off anyway.
        dy = self.exchange.dispatch_backward(drows, place, dy.to(self.dtype))
        grads["x"], grads["gamma"], grads["beta"] = self.norm.backward(dy, self.norm.H, gamma, dh)
        grads["router"] = dlogits.t() @ y.float()
        return grads
