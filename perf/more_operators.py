"""What stands around the products of an expert layer, as cases to be timed: a
layer norm, the router, the exchange of rows between tokens and experts, and dense
layers in 8-bit floating point.

``norm``      y = layer norm of x, or of h = x + residual (h rounded to the type), with
              ``train`` the gradients of x, of the weight and of the bias too.
``route``     the top_k of E experts for each token by softmax or sigmoid scores (a bias
              that moves the choice alone, groups of which the best are kept, shares
              renormalised), every (token, slot)'s place among the rows sorted by
              expert, the experts' offsets; with ``train`` the logits' gradient.
``exchange``  rows[place] = x[token], out[token] = sum of share y[place]; with ``train``
              the gradients of y, share and x.
``f8``        Y = X W^T with X quantized on the way and W's codes at hand; with ``train``
              a whole step: W and X quantized, Y, dY quantized, dX = dY W and dW = dY^T X.

8 bits: E4M3, one power-of-two scale (E8M0) for 128 consecutive elements of a
product's inner axis (X and dY) or for 128 x 128 elements (W): 2^(s - 127) with s the
smallest that leaves no element more than half a step off, max |x| / scale <= 464;
element = x / scale rounded to the nearest, ties to the even code.

Routing: an expert whose logit is -inf is never chosen, a slot without an expert has
chosen = place = -1 and share 0.  Without a bias experts are ordered by their logits,
with one by score + bias; a group counts as the sum of its two highest; ties go to the
lowest index.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

MOST_FLOPS = 6 * 8192 * 4096 * 11008.0      # of the largest listed case
MOST_BYTES = 1.2e9
EPS = 1e-5


def listed():
    return [
        # one token on its way into the next layer of a 4096-wide model: residual sum and norm
        {"name": "norm_token", "kind": "norm", "dtype": "bf16", "param": "bf16", "M": 1, "C": 4096, "residual": True,
         "train": False},
        # 16 sequences of 197 tokens, fp32, forward and backward: an odd row count
        {"name": "norm_train_197", "kind": "norm", "dtype": "f32", "param": "f32", "M": 16 * 197, "C": 768,
         "residual": False, "train": True},
        # a training batch of a 4096-wide model with its residual stream
        {"name": "norm_train_large", "kind": "norm", "dtype": "bf16", "param": "f32", "M": 16384, "C": 4096,
         "residual": True, "train": True},
        # one token's experts: 8 of 64
        {"name": "route_token", "kind": "route", "dtype": "f32", "T": 1, "E": 64, "k": 8, "score": "softmax",
         "renorm": True, "groups": 1, "top_groups": 1, "bias": False, "scale": 1.0, "pad": 0.0, "train": False},
        # a small training batch with padded tokens on few experts: 2 of 12, shares as they come
        {"name": "route_train_padded", "kind": "route", "dtype": "f32", "T": 1187, "E": 12, "k": 2, "score": "softmax",
         "renorm": False, "groups": 1, "top_groups": 1, "bias": False, "scale": 1.0, "pad": 0.1, "train": True},
        # a training batch: 8 of 256 experts from the best 4 of 8 groups, by sigmoid scores and a bias for balance
        {"name": "route_train_groups", "kind": "route", "dtype": "f32", "T": 16384, "E": 256, "k": 8, "score": "sigmoid",
         "renorm": True, "groups": 8, "top_groups": 4, "bias": True, "scale": 2.5, "pad": 0.0, "train": True},
        # one token out to 8 experts and back
        {"name": "exchange_token", "kind": "exchange", "dtype": "bf16", "T": 1, "E": 64, "k": 8, "D": 2048, "skew": 0.3,
         "train": False},
        # a small training batch in fp32, an odd token count and a width that no power of two divides
        {"name": "exchange_train_uneven", "kind": "exchange", "dtype": "f32", "T": 1187, "E": 12, "k": 2, "D": 1000,
         "skew": 1.5, "train": True},
        # 4096 tokens to 8 of 64 experts each and back, forward and backward
        {"name": "exchange_train_large", "kind": "exchange", "dtype": "bf16", "T": 4096, "E": 64, "k": 8, "D": 2048,
         "skew": 0.5, "train": True},
        # one token through a projection of a 4096-wide model: the weights are all there is to read
        {"name": "f8_token", "kind": "f8", "dtype": "bf16", "M": 1, "K": 4096, "N": 4096, "train": False},
        # an attention projection over 16 sequences of 197 tokens, fp32, trained
        {"name": "f8_train_197", "kind": "f8", "dtype": "f32", "M": 16 * 197, "K": 768, "N": 768, "train": True},
        # the training step of the large linear layer, the benchmark's sizes
        {"name": "f8_train_large", "kind": "f8", "dtype": "bf16", "M": 8192, "K": 4096, "N": 11008, "train": True},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        c = {"kind": rng.choice(["norm", "route", "exchange", "f8"]), "dtype": rng.choice(["bf16", "bf16", "f32"]),
             "train": rng.random() < 0.6}
        if c["kind"] == "norm":
            c |= {"param": rng.choice(["bf16", "f32"]), "M": _log_int(rng, 1, 32768), "C": _log_int(rng, 32, 16384),
                  "residual": rng.random() < 0.5}
            if rng.random() < 0.5:
                c["C"] = -(-c["C"] // 64) * 64
        elif c["kind"] == "route":
            groups = rng.choice([1, 1, 4, 8])
            e = groups * _log_int(rng, 4, 512 // groups)
            top = groups if groups == 1 else rng.randint(1, groups)
            c |= {"T": _log_int(rng, 1, 32768), "E": e, "k": min(_log_int(rng, 1, 16), e // groups * top),
                  "score": rng.choice(["softmax", "sigmoid"]), "renorm": rng.random() < 0.5, "groups": groups,
                  "top_groups": top, "bias": rng.random() < 0.5, "scale": rng.choice([1.0, 2.5]),
                  "pad": rng.choice([0.0, 0.0, 0.2])}
        elif c["kind"] == "exchange":
            e = _log_int(rng, 2, 256)
            c |= {"T": _log_int(rng, 1, 16384), "E": e, "k": min(_log_int(rng, 1, 8), e), "D": _log_int(rng, 64, 8192),
                  "skew": round(rng.uniform(0.0, 1.5), 2)}
        else:
            c |= {"M": _log_int(rng, 1, 16384), "K": _log_int(rng, 64, 8192), "N": _log_int(rng, 32, 11008)}
            if rng.random() < 0.5:      # widths that are not odd by design: multiples of 64
                c["K"], c["N"] = -(-c["K"] // 64) * 64, -(-c["N"] // 64) * 64
        w = work(c)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return c


def work(case):
    s = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "norm":
        m, c, r = case["M"], case["C"], case["residual"]
        n = 2 + 2 * r + (3 + r) * case["train"]     # x, y (residual, h); dy, x or h, dx (the residual's gradient)
        return {"bytes": float(n * m * c * s), "flops": float((8 + 14 * case["train"]) * m * c)}
    if case["kind"] == "route":
        t, e, k = case["T"], case["E"], case["k"]
        # logits; share, chosen, place; again the logits and their gradient, share's gradient
        return {"bytes": float(t * e * s + 12 * t * k + case["train"] * (2 * t * e * s + 4 * t * k)),
                "flops": float((10 + 8 * case["train"]) * t * e)}
    if case["kind"] == "exchange":
        t, k, d = case["T"], case["k"], case["D"]
        n = 2 * (1 + k) + case["train"] * (2 + 3 * k)
        return {"bytes": float(n * t * d * s), "flops": float((2 + 4 * case["train"]) * t * k * d)}
    m, k, n = case["M"], case["K"], case["N"]
    if not case["train"]:
        return {"bytes": m * k * s + n * k * 129 / 128 + m * n * s, "flops": 2.0 * m * n * k}
    # x, dy, W once; y, dx in their type and dW in 32 bits once
    return {"bytes": float(2 * m * (k + n) * s + n * k * (s + 4)), "flops": 6.0 * m * n * k}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEVICE)


def _spread(g, rows, cols, sigma):
    """Normal values, each channel with a log-normal size of its own."""
    return _normal(g, rows, cols) * torch.exp(sigma * _normal(g, cols))


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "norm":
        m, c = case["M"], case["C"]
        st["x"] = (_spread(g, m, c, 0.5) + 0.3 * _normal(g, c)).to(dt)
        st["gamma"] = (1 + 0.2 * _normal(g, c)).to(DTYPES[case["param"]])
        st["beta"] = (0.1 * _normal(g, c)).to(DTYPES[case["param"]])
        if case["residual"]:
            st["residual"] = (2 * _spread(g, m, c, 0.5)).to(dt)
        if case["train"]:
            st["dy"] = (0.01 * _spread(g, m, c, 0.5)).to(dt)
            if case["residual"]:
                st["dh"] = (0.01 * _normal(g, m, c)).to(dt)
    elif case["kind"] == "route":
        t, e, k = case["T"], case["E"], case["k"]
        st["logits"] = (1.5 * _normal(g, t, e) + 0.5 * _normal(g, e)).to(dt)
        padded = int(case["pad"] * t)
        if padded:
            st["logits"][t - padded:] = -math.inf
        if case["bias"]:
            st["bias"] = 0.05 * _normal(g, e)
        if case["train"]:
            st["dshare"] = 0.1 * _normal(g, t, k)
    elif case["kind"] == "exchange":
        t, e, k, d = case["T"], case["E"], case["k"], case["D"]
        logits = _normal(g, t, e) + case["skew"] * _normal(g, e)
        top = torch.sort(logits, dim=1, descending=True, stable=True)
        chosen = top.indices[:, :k].reshape(-1)
        st["share"] = torch.softmax(top.values[:, :k], 1).contiguous()
        place = torch.empty(t * k, dtype=torch.int32, device=DEVICE)
        place[torch.argsort(chosen, stable=True)] = torch.arange(t * k, dtype=torch.int32, device=DEVICE)
        st["place"] = place.view(t, k)
        st["x"] = _spread(g, t, d, 0.5).to(dt)
        st["y"] = _spread(g, t * k, d, 0.5).to(dt)
        if case["train"]:
            st["dout"] = (0.01 * _spread(g, t, d, 0.5)).to(dt)
            st["drows"] = (0.01 * _spread(g, t * k, d, 0.5)).to(dt)
    else:
        m, k, n = case["M"], case["K"], case["N"]
        st["x"] = _spread(g, m, k, 0.5).to(dt)
        w = (0.02 * _normal(g, n, k)).to(dt)
        if case["train"]:
            st["w"] = w
            st["dy"] = (0.001 * _spread(g, m, n, 1.0)).to(dt)
        else:
            st["w_codes"], st["w_scales"] = _packed(w)
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _plain_norm(st):
    case, dt = st["case"], st["x"].dtype
    h = (st["x"].float() + st["residual"].float()).to(dt) if case["residual"] else st["x"]
    v = h.float()
    mean = v.mean(1, keepdim=True)
    c = v - mean
    rstd = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
    xh = c * rstd
    y = (xh * st["gamma"].float() + st["beta"].float()).to(dt)
    out = (y, h) if case["residual"] else (y,)
    if not case["train"]:
        return out
    dy = st["dy"].float()
    q = dy * st["gamma"].float()
    dx = rstd * (q - q.mean(1, keepdim=True) - xh * (q * xh).mean(1, keepdim=True))
    if case["residual"]:
        dx = dx + st["dh"].float()
    return out + (dx.to(dt), (dy.double() * xh).sum(0).float(), dy.double().sum(0).float())


def _chosen(st):
    """(scores in 64 bits, experts of every token's slots, -1 for none)"""
    case, logits = st["case"], st["logits"].double()
    t, e = logits.shape
    live = logits > -math.inf
    if case["score"] == "softmax":
        top = logits.amax(1, keepdim=True)
        x = torch.exp(logits - torch.where(top > -math.inf, top, 0.0))
        s = x / torch.clamp(x.sum(1, keepdim=True), min=1e-300)
    else:
        s = 1 / (1 + torch.exp(-logits))
    value = s + st["bias"].double() if case["bias"] else s
    key = torch.where(live, value if case["bias"] else logits, -math.inf)
    if case["groups"] > 1:
        by_group = torch.where(live, value, -math.inf).view(t, case["groups"], -1)
        two = torch.sort(by_group, dim=2, descending=True).values[:, :, :2]
        total = torch.where(two > -math.inf, two, 0.0).sum(2)
        total = torch.where(two[:, :, 0] > -math.inf, total, -math.inf)
        best = torch.sort(total, dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        kept = torch.zeros(t, case["groups"], dtype=torch.bool, device=logits.device).scatter_(1, best, True)
        key = torch.where(kept.repeat_interleave(e // case["groups"], 1), key, -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True)
    k = case["k"]
    return s, torch.where(order.values[:, :k] > -math.inf, order.indices[:, :k], -1)


def _plain_route(st):
    case = st["case"]
    s, chosen = _chosen(st)
    t, e = s.shape
    some = chosen >= 0
    got = torch.where(some, s.gather(1, chosen.clamp(min=0)), 0.0)
    total = torch.clamp(got.sum(1, keepdim=True), min=1e-300)
    share = case["scale"] * (got / total if case["renorm"] else got)
    flat = torch.where(some, chosen, e).reshape(-1)
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(flat.numel(), device=flat.device)
    place = torch.where(some, place.view(t, -1), -1)
    ends = torch.searchsorted(flat[order], torch.arange(e, device=flat.device), right=True)
    offsets = torch.cat([ends.new_zeros(1), ends])
    out = share.float(), chosen.to(torch.int32), place.to(torch.int32), offsets.to(torch.int32)
    if not case["train"]:
        return out
    dw = torch.where(some, st["dshare"].double(), 0.0)
    at = chosen.clamp(min=0)
    if case["score"] == "softmax" and not case["renorm"]:
        ds = torch.zeros_like(s).scatter_add_(1, at, case["scale"] * dw)
        dl = s * (ds - (ds * s).sum(1, keepdim=True))
    else:
        if case["renorm"]:
            r = got / total
            d = case["scale"] * (dw - (dw * r).sum(1, keepdim=True))
            d = d * r if case["score"] == "softmax" else d * r * (1 - got)
        else:
            d = case["scale"] * dw * got * (1 - got)
        dl = torch.zeros_like(s).scatter_add_(1, at, torch.where(some, d, 0.0))
    return out + (dl.to(st["logits"].dtype),)


def _plain_exchange(st):
    x, y, place, share = st["x"], st["y"].float(), st["place"].long(), st["share"]
    dt, (t, k) = x.dtype, place.shape
    flat = place.reshape(-1)

    def sorted_rows(v):
        out = torch.empty_like(v)
        out[flat] = v
        return out.to(dt)
    rows = sorted_rows(x.repeat_interleave(k, 0))
    mine = y[flat].view(t, k, -1)
    out = (mine * share.unsqueeze(2)).sum(1).to(dt)
    if not st["case"]["train"]:
        return rows, out
    d = st["dout"].float().unsqueeze(1)
    dy = sorted_rows((d * share.unsqueeze(2)).view(t * k, -1))
    dshare = (d * mine).sum(2)
    return rows, out, dy, dshare, st["drows"].float()[flat].view(t, k, -1).sum(1).to(dt)


def _scale(s):
    return torch.clamp(s << 23, min=1 << 22).view(torch.float32)    # 2^(s - 127), 2^-127 for s = 0


def _rounded8(v):
    """The nearest E4M3 value: steps of 2^-9 up to 2^-6, then eight to a binade."""
    e = torch.clamp(((v.abs().view(torch.int32) >> 23) - 127), min=-6) - 3
    step = ((e + 127) << 23).view(torch.float32)
    return torch.clamp(torch.round(v / step) * step, min=-448.0, max=448.0)


def _codes8(x, square):
    """(E4M3 values, exponents of the scales) of x [rows, cols] in blocks of 128 along its rows' elements, or of 128 x
    128, padded to whole blocks."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -cols % 128, 0, -rows % 128 if square else 0))
    v = v.view(-1, 128 if square else 1, v.shape[1] // 128, 128)
    bits = v.abs().amax((1, 3), keepdim=True).view(torch.int32)
    s = torch.clamp(((bits + 0x17FFFF) >> 23) - 8, min=0)
    q = _rounded8(v * ((254 - s) << 23).view(torch.float32))
    return q, s


def _f8(x, square=False):
    """The values that the 8-bit codes of x stand for."""
    q, s = _codes8(x, square)
    v = q * _scale(s)
    return v.reshape(-1, v.shape[2] * 128)[:x.shape[0], :x.shape[1]]


def _packed(w):
    """A matrix as E4M3 codes in 128 x 128 blocks, in the layout of the matrix products: tiles of 16 rows x 128
    elements, in them [16 elements][row][16 bytes]; scales by 16 rows x 512 elements, in them [row][tile]."""
    rows, cols = w.shape
    q, s = _codes8(torch.nn.functional.pad(w, (0, -cols % 512)), True)
    k = q.shape[2]
    q = q.view(-1, k * 128)[:-(-rows // 16) * 16]
    a = q.abs()
    e = torch.clamp((a.view(torch.int32) >> 23) - 127, min=-6)
    m = torch.round(a / ((e + 124) << 23).view(torch.float32)).to(torch.int32)      # 8..15, below 2^-6 0..7
    c = torch.where(m >= 8, ((e + 7) << 3) + m - 8, m) | (torch.signbit(q).to(torch.int32) << 7)
    codes = c.to(torch.uint8).view(-1, 16, k, 8, 16).permute(0, 2, 3, 1, 4).contiguous()
    s = s.to(torch.uint8).view(-1, 1, k).expand(-1, 128, k).reshape(-1, k)[:q.shape[0]]
    scales = s.view(-1, 16, k // 4, 4).permute(0, 2, 1, 3).contiguous()
    return codes.view(-1), scales.view(-1)


def _unpacked(codes, scales, rows, cols):
    n = -(-rows // 16)
    b = codes.view(n, -1, 8, 16, 16).permute(0, 3, 1, 2, 4).reshape(n * 16, -1, 128).to(torch.int32)
    e, m = (b >> 3) & 15, b & 7
    v = torch.where(e > 0, (8 + m).float() * ((e + 117) << 23).view(torch.float32), m.float() * 2.0 ** -9)
    v = torch.where(b >= 128, -v, v)
    s = scales.view(n, -1, 16, 4).permute(0, 2, 1, 3).reshape(n * 16, -1, 1).to(torch.int32)
    return (v * _scale(s)).reshape(n * 16, -1)[:rows, :cols]


def _plain_f8(st):
    case, x = st["case"], st["x"]
    dt = x.dtype
    if not case["train"]:
        return (_f8(x) @ _unpacked(st["w_codes"], st["w_scales"], case["N"], case["K"]).T).to(dt)
    w, dy = _f8(st["w"], True), st["dy"]
    return (_f8(x) @ w.T).to(dt), (_f8(dy) @ w).to(dt), _f8(dy.T) @ _f8(x.T).T


_PLAIN = {"norm": _plain_norm, "route": _plain_route, "exchange": _plain_exchange, "f8": _plain_f8}


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own_norm(st):
    from paper_2411_10948_amd import norm

    case, x = st["case"], st["x"]
    plan = st.get("plan")
    if plan is None:
        plan = st["plan"] = norm.NormPlan(case["M"], case["C"], eps=EPS, dtype=x.dtype, param_dtype=st["gamma"].dtype,
                                          residual=case["residual"], train=case["train"])
    y = plan.forward(x, st["gamma"], st["beta"], st.get("residual"))
    out = (y, plan.H) if case["residual"] else (y,)
    if not case["train"]:
        return out
    return out + plan.backward(st["dy"], plan.H if case["residual"] else x, st["gamma"], st.get("dh"))


def _own_route(st):
    from paper_2411_10948_amd import route

    case, logits = st["case"], st["logits"]
    plan = st.get("plan")
    if plan is None:
        plan = st["plan"] = route.RouterPlan(case["T"], case["E"], case["k"], score=case["score"], groups=case["groups"],
                                             top_groups=case["top_groups"], renormalize=case["renorm"],
                                             scale=case["scale"], dtype=logits.dtype)
    share, chosen = plan.forward(logits, st.get("bias"))
    out = share, chosen, plan.place, plan.offsets
    return out + (plan.backward(st["dshare"], logits),) if case["train"] else out


def _own_exchange(st):
    from paper_2411_10948_amd import route

    case, x = st["case"], st["x"]
    plan = st.get("plan")
    if plan is None:
        plan = st["plan"] = route.ExchangePlan(case["T"], case["k"], case["D"], dtype=x.dtype, train=case["train"])
    rows = plan.dispatch(x, st["place"])
    out = plan.combine(st["y"], st["place"], st["share"])
    if not case["train"]:
        return rows, out
    dy, dshare = plan.combine_backward(st["dout"], st["y"], st["place"], st["share"])
    return rows, out, dy, dshare, plan.dispatch_backward(st["drows"], st["place"])


def _own_f8(st):
    from paper_2411_10948_amd import f8

    case, x = st["case"], st["x"]
    plan = st.get("plan")
    if plan is None:
        plan = st["plan"] = f8.LinearPlan(case["M"], case["K"], case["N"], dtype=x.dtype, train=case["train"])
    if not case["train"]:
        w = st.get("weight")
        if w is None:
            w = st["weight"] = f8.F8Matrix(st["w_codes"], st["w_scales"], case["N"], case["K"])
        return plan.forward(x, w)
    plan.quantize_weight(st["w"])
    y = plan.forward(x)
    dx, dw = plan.backward(st["dy"])
    return y, dx, dw


_OWN = {"norm": _own_norm, "route": _own_route, "exchange": _own_exchange, "f8": _own_f8}


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_norm(case, st):
    x = st["x"].double()
    h = None
    if case["residual"]:
        h = (x + st["residual"].double()).float().to(st["x"].dtype)
        x = h.double()
    var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
    sd = torch.sqrt(var + EPS)
    xh = (x - mean) / sd
    gamma = st["gamma"].double()
    y = torch.addcmul(st["beta"].double(), xh, gamma)
    out = (y, None) if case["residual"] else (y,)
    if not case["train"]:
        return out
    dy = st["dy"].double()
    q = dy * gamma
    n = x.shape[1]
    # the Jacobian (I - 1 1^T / n - xh xh^T / n) / sd, a projection applied twice
    p = q - xh * (q * xh).sum(1, keepdim=True) / n
    dx = (p - q.sum(1, keepdim=True) / n) / sd
    if case["residual"]:
        dx = dx + st["dh"].double()
    return out + (dx, torch.einsum("mc,mc->c", dy, xh), torch.ones(1, dy.shape[0], dtype=dy.dtype, device=dy.device).mm(dy)[0])


def _exact_route(case, st):
    leaf = st["logits"].double().detach().requires_grad_(True)
    t, e = leaf.shape
    k, groups = case["k"], case["groups"]
    dead = torch.isneginf(leaf.detach())
    empty = dead.all(1, keepdim=True)
    if case["score"] == "softmax":
        s = torch.softmax(torch.where(empty, torch.zeros_like(leaf), leaf), 1).masked_fill(dead, 0.0)
    else:
        s = torch.sigmoid(leaf)
    value = s.detach() + (st["bias"].double() if case["bias"] else 0.0)
    key = value if case["bias"] else leaf.detach()
    # rank of an expert: how many come before it, by key and then by index
    step = max(1, 2 ** 24 // (e * e))
    index = torch.arange(e, device=leaf.device)
    if groups > 1:
        per = e // groups
        v = value.masked_fill(dead, -math.inf).view(t, groups, per)
        first = v.amax(2)
        rest = v.scatter(2, v.argmax(2, keepdim=True), -math.inf).amax(2) if per > 1 else torch.full_like(first, -math.inf)
        total = torch.where(torch.isneginf(rest), first, first + rest)
        gi = torch.arange(groups, device=leaf.device)
        before = (total.unsqueeze(1) > total.unsqueeze(2)) | ((total.unsqueeze(1) == total.unsqueeze(2)) & (gi.view(1, 1, -1) < gi.view(1, -1, 1)))
        dropped = (before.sum(2) >= case["top_groups"]).repeat_interleave(per, 1)
        out_of_it = dead | dropped
    else:
        out_of_it = dead
    key = key.masked_fill(out_of_it, -math.inf)
    ranks = []
    for lo in range(0, t, step):
        a = key[lo:lo + step]
        before = (a.unsqueeze(1) > a.unsqueeze(2)) | ((a.unsqueeze(1) == a.unsqueeze(2)) & (index.view(1, 1, -1) < index.view(1, -1, 1)))
        ranks.append(before.sum(2))
    rank = torch.cat(ranks)
    taken = (rank < k) & ~out_of_it
    kept = torch.where(taken, s, torch.zeros_like(s))
    if case["renorm"]:
        kept = kept / kept.sum(1, keepdim=True).clamp(min=1e-300)
    kept = kept * case["scale"]
    slot = torch.where(taken, rank, k)
    share = torch.zeros(t, k + 1, dtype=torch.float64, device=leaf.device).scatter_add(1, slot, kept)[:, :k]
    if not case["train"]:
        return share.detach(), None, None, None
    grad, = torch.autograd.grad(share, leaf, st["dshare"].double())
    return share.detach(), None, None, None, torch.where(dead, 0.0, grad)


def _exact_exchange(case, st):
    t, k, d = case["T"], case["k"], case["D"]
    place, share = st["place"].long(), st["share"].double()
    rows = torch.zeros(t * k, d, dtype=torch.float64, device=share.device)
    out = torch.zeros(t, d, dtype=torch.float64, device=share.device)
    for j in range(k):
        rows.index_copy_(0, place[:, j], st["x"].double())
        out.addcmul_(st["y"][place[:, j]].double(), share[:, j:j + 1])
    if not case["train"]:
        return rows, out
    dy, dx, dshare = torch.zeros_like(rows), torch.zeros_like(out), torch.zeros_like(share)
    dout = st["dout"].double()
    for j in range(k):
        dy.index_copy_(0, place[:, j], dout * share[:, j:j + 1])
        dshare[:, j] = torch.linalg.vecdot(dout, st["y"][place[:, j]].double())
        dx += st["drows"][place[:, j]].double()
    return rows, out, dy, dshare, dx


def _f8_64(x, square=False):
    rows, cols = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -cols % 128, 0, -rows % 128 if square else 0))
    b = v.unflatten(1, (-1, 128))
    most = b.abs().amax(2, keepdim=True)
    if square:
        most = most.unflatten(0, (-1, 128)).amax(1, keepdim=True).expand(-1, 128, -1, -1).flatten(0, 1)
    e = torch.ceil(torch.log2(torch.clamp(most, min=2.0 ** -140) / 464))
    e = torch.where(most / torch.exp2(e - 1) <= 464, e - 1, e)      # log2 may be off by an ulp either way
    e = torch.where(most / torch.exp2(e) > 464, e + 1, e)
    scale = torch.exp2(torch.clamp(e, min=-127.0))
    b = b / scale
    _, p = torch.frexp(b)                       # b = f 2^p, f in [0.5, 1): four bits of it
    step = torch.exp2(torch.clamp(p.double() - 4, min=-9.0))
    q = torch.clamp(torch.round(b / step) * step, min=-448.0, max=448.0)
    return (q * scale).flatten(1)[:rows, :cols]


def _exact_f8(case, st):
    x = _f8_64(st["x"])
    if not case["train"]:
        return x @ _unpacked(st["w_codes"], st["w_scales"], case["N"], case["K"]).double().T
    w, dy = _f8_64(st["w"], True), st["dy"]
    return x @ w.T, _f8_64(dy) @ w, _f8_64(dy.T) @ _f8_64(st["x"].T).T


_EXACT = {"norm": _exact_norm, "route": _exact_route, "exchange": _exact_exchange, "f8": _exact_f8}


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))
